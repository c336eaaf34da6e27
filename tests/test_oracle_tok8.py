"""Pins of the oracle's 8-bit products with token and channel scales and of its AdamW with moments in 8 bits: brute force, 64-bit references with bounds
(u = 2^-24, half a step of binary32 relative to the value; a bf16 output adds 2^-8 of it), hand-worked cases, gradients against differences."""
import numpy as np
import pytest

import oracle as O
import synth

U, UBF = 2.0 ** -24, 2.0 ** -8
F = np.float32


def wide(x):
    return (synth.from_bf16(x) if x.dtype == np.uint16 else x).astype(np.float64)


def rows(M, K, seed, std=1.0):
    return synth.to_bf16((synth.normal_f32((M, K), std, seed=seed, tid=1) * np.exp(0.7 * synth.normal_f32((K,), 1.0, seed=seed, tid=2))).astype(F))


def test_codes_by_hand():
    bf = lambda *v: synth.to_bf16(np.array([v], F))
    q, s = O.tok8_quant(bf(127.0, -127.0, 0.5, 1.5, 2.5, -3.0, 0.0))              # scale 1: ties go to the even code
    assert s[0] == 1.0 and q.tolist() == [[127, -127, 0, 2, 2, -3, 0]]
    q, s = O.tok8_quant(bf(0.0, 0.0, -0.0))
    assert s[0] == 0.0 and not q.any()
    for bad in (np.inf, -np.inf, np.nan):
        q, s = O.tok8_quant(bf(1.0, bad, 2.0))
        assert np.isnan(s[0]) and not q.any()
    q, s = O.tok8_quant(bf(1.2e-38, 0.0))                                          # a 127th of it is flushed
    assert s[0] == 0.0 and not q.any()
    q, s = O.tok8_quant(bf(2.0, 1.0), row_factor=[3.0], col_factor=[1.0, 4.0])     # 6, 12
    assert s[0] == F(12) / F(127) and q.tolist() == [[64, 127]]                    # 6 / 12 of 127 is 63.5
    q, s = O.tok8_quant(synth.to_bf16(np.array([[1, 4], [2, -8]], F)), by_col=True)
    assert q.tolist() == [[64, 127], [64, -127]] and s.tolist() == [F(2) / F(127), F(8) / F(127)]


@pytest.mark.parametrize("M,K", [(1, 1), (7, 33), (40, 500)])
def test_codes_in_64_bits(M, K):
    """The largest value of a row has a code of 127 and no value is off by more than half a scale: |v - q s| <= s (1/2 + 127 * 3 u), three roundings on the
    way to the code and the scale's own."""
    x = rows(M, K, 3)
    q, s = O.tok8_quant(x)
    v = wide(x)
    assert (np.abs(q).max(1) == 127).all()
    assert np.abs(s - np.abs(v).max(1) / 127).max() <= U * s.max()
    assert (np.abs(v - q * s.astype(np.float64)[:, None]) <= s[:, None] * (0.5 + 127 * 4 * U)).all()


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (5, 9, 40), (33, 20, 300)])
def test_products_by_brute_force(M, N, K):
    """The products are exact integers, and each output three roundings (conversion, product of the scales, product) and the last one from them."""
    x, w, dy = rows(M, K, 1), synth.normal_bf16((N, K), 0.02, seed=2), rows(M, N, 3, 0.01)
    Y, qX, sX, qW, sW = O.tok8_linear_fwd(x, w)
    acc = qX.astype(np.int64) @ qW.astype(np.int64).T
    want = acc * (sX.astype(np.float64)[:, None] * sW.astype(np.float64))
    assert (np.abs(wide(Y) - want) <= np.abs(want) * (UBF + 4 * U)).all()
    dX, dW = O.tok8_linear_bwd(dy, x, w)
    qA, sA = O.tok8_quant(dy, col_factor=sW)
    qG, sG = O.tok8_quant(dy, row_factor=sX, by_col=True)
    want = (qA.astype(np.int64) @ qW.astype(np.int64)) * sA.astype(np.float64)[:, None]
    assert (np.abs(wide(dX) - want) <= np.abs(want) * (UBF + 3 * U)).all()
    want = (qG.astype(np.int64) @ qX.astype(np.int64)) * sG.astype(np.float64)[:, None]
    assert (np.abs(dW - want) <= np.abs(want) * 3 * U).all()


def _products_off(A, B, S):
    """How far the product over S of codes of A (scaled by the row) and of B's codes (times B's scale, which is in A) may be from A B's: half a code of either,
    sum |A - s q||q'| + |A||B - q'| <= S amax (127/2/127 + 1/2), with four roundings of the scales."""
    return S * np.abs(A).max(1)[:, None] * (1 + 508 * U) * np.ones(B.shape[1])


def test_linear_against_64_bits():
    """What the codes leave of the mathematics, element by element."""
    M, N, K = 40, 30, 256
    x, w, dy = rows(M, K, 4), synth.normal_bf16((N, K), 0.02, seed=5), rows(M, N, 6, 0.01)
    Y = wide(O.tok8_linear_fwd(x, w)[0])
    X, W, D = wide(x), wide(w), wide(dy)
    ax, aw = np.abs(X).max(1)[:, None], np.abs(W).max(1)[None, :]
    # half a code of either operand: ax/254 aw + ax aw/254 + both for each of K terms
    assert (np.abs(Y - X @ W.T) <= K * ax * aw / 127 * (1 + 1 / 508 + 508 * U) + UBF * np.abs(Y)).all()
    dX, dW = O.tok8_linear_bwd(dy, x, w)
    sX, sW = np.abs(X).max(1) / 127, np.abs(W).max(1) / 127
    assert (np.abs(wide(dX) - D @ W) <= _products_off(D * sW, W, N) + UBF * np.abs(wide(dX))).all()
    assert (np.abs(dW - D.T @ X) <= _products_off((D * sX[:, None]).T, X, M) + 4 * U * np.abs(dW)).all()


def test_exact_where_nothing_is_rounded():
    """Values that are codes times a power of two come out as the plain product, forward and backward."""
    rng = np.random.default_rng(1)
    code = lambda r, c, e: synth.to_bf16((np.concatenate([rng.integers(-60, 61, (r, c - 1)), np.full((r, 1), 127)], 1) * 2.0 ** e).astype(F))
    x, w = code(6, 20, -3), code(8, 20, -9)
    want = wide(x) @ wide(w).T
    assert np.array_equal(O.tok8_linear_fwd(x, w)[0], synth.to_bf16(want.astype(F)))
    one = np.zeros((6, 8), F)
    one[2, 5] = 127 * 2.0 ** -4                                                    # one entry of the gradient: its codes are 127 on either side
    dX, dW = O.tok8_linear_bwd(synth.to_bf16(one), x, w)
    s = F(127 * 2.0 ** -4) * F(2.0 ** -9)
    assert np.array_equal(dX[2], synth.to_bf16((F(127) * wide(w)[5].astype(F) / F(2.0 ** -9)) * (s / F(127)))) and not dX[[0, 1, 3, 4, 5]].any()
    assert np.allclose(dW[5], 127 * 2.0 ** -4 * wide(x)[2], rtol=4 * U, atol=0) and not dW[[0, 1, 2, 3, 4, 6, 7]].any()


def test_rows_are_on_their_own():
    x, w = rows(9, 64, 7), synth.normal_bf16((5, 64), 0.02, seed=8)
    whole = O.tok8_linear_fwd(x, w)[0]
    assert np.array_equal(np.concatenate([O.tok8_linear_fwd(x[i:i + 1], w)[0] for i in range(9)]), whole)


def test_gated_block_against_formula_and_differences():
    """The gradient of sum(h c) at the block's own gate and up: the oracle's within what bf16 (a half step of dgu, which goes into N or M products) and the
    codes leave of the formula's in 64 bits, and the formula's against central differences (third derivatives of silu times up are below 1, so the
    quotient is off by e^2/6 of a sum of |c| (1 + |u|) |d gu|^3, and by 2^-52 of the loss over e)."""
    M, Fh, K = 12, 10, 64
    x, w, c = rows(M, K, 1, 0.5), synth.normal_bf16((2 * Fh, K), 0.1, seed=2), rows(M, Fh, 3)
    X, W, C = wide(x), wide(w), wide(c)
    gu = O.tok8_linear_fwd(x, w)[0]
    g, u = wide(gu)[:, :Fh], wide(gu)[:, Fh:]
    f = 1 / (1 + np.exp(-g))
    dgu = np.concatenate([C * u * f * (1 + g * (1 - f)), C * g * f], 1)
    dX, dW = O.tok8_linear_bwd(O.swiglu_bwd(c, gu), x, w)
    # swiglu_bwd: a dozen roundings of terms up to |c u f| (1 + |g|), then bf16
    off = UBF * np.abs(dgu) + 40 * U * np.concatenate([np.abs(C * u) * f * (1 + np.abs(g)), np.abs(C * g) * f], 1)
    sX, sW = np.abs(X).max(1) / 127, np.abs(W).max(1) / 127
    big = np.abs(dgu) + off
    assert (np.abs(wide(dX) - dgu @ W) <= off @ np.abs(W) + _products_off(big * sW, W, 2 * Fh) + UBF * np.abs(wide(dX))).all()
    assert (np.abs(dW - dgu.T @ X) <= off.T @ np.abs(X) + _products_off((big * sX[:, None]).T, X, M) + 4 * U * np.abs(dW)).all()

    def loss(gu):
        return ((gu[:, :Fh] / (1 + np.exp(-gu[:, :Fh]))) * gu[:, Fh:] * C).sum()
    rng, e = np.random.default_rng(3), 1e-4
    for _ in range(20):
        dx, dw = rng.standard_normal(X.shape) / K, rng.standard_normal(W.shape) / K
        d = dx @ W.T + X @ dw.T
        slope = (loss(wide(gu) + e * d) - loss(wide(gu) - e * d)) / (2 * e)
        size = (np.abs(C) * (1 + np.abs(u)) * (np.abs(d[:, :Fh]) + np.abs(d[:, Fh:])) ** 3).sum()
        assert abs(slope - ((dgu @ W) * dx).sum() - ((dgu.T @ X) * dw).sum()) <= e * e * size + 1e-11 * (np.abs(C * g * u).sum() + 1) / e * 1e-3


def test_moment_codes_by_hand():
    m = np.zeros(256, F)
    m[:5] = [1.0, -0.25, 0.0625, 1e-6, -1e-9]
    v = np.zeros(256, F)
    v[:4] = [16.0, 1.0, 1e-20, 1e-40]
    m8, v8, s = O.adamw8_pack(m, v)
    assert s.tolist() == [[1.0, 4.0]]
    # root of the share, of 127: 127, 63.5 and 31.75; 0.127 is nothing.  Of 255: r = 4, 1, 1e-10: 255, 127.5 and at least 1; a subnormal is zero
    assert m8[:5].tolist() == [127, -64, 32, 0, 0] and not m8[5:].any()
    assert v8[:4].tolist() == [255, 128, 1, 0] and not v8[4:].any()
    bm, bv = O.adamw8_unpack(m8, v8, s)
    assert np.allclose(bm[:3], [1, -(64 / 127) ** 2, (32 / 127) ** 2], rtol=6 * U) and np.allclose(bv[:2], [16, 16 * (128 / 255) ** 4], rtol=12 * U)
    z = O.adamw8_pack(np.zeros(300, F), np.zeros(300, F))
    assert not z[0].any() and not z[1].any() and not z[2].any() and z[2].shape == (2, 2)
    for at, bad in ((0, np.nan), (1, np.inf)):
        arr = [np.ones(300, F), np.ones(300, F)]
        arr[at][299] = bad
        m8, v8, s = O.adamw8_pack(*arr)
        assert np.isnan(s[1, at]) and not (m8, v8)[at][256:].any() and np.isfinite(s[0]).all() and np.isfinite(s[1, 1 - at])


@pytest.mark.parametrize("n", [1, 255, 256, 257, 5000])
def test_moment_codes_in_64_bits(n):
    """A code is the root of the share, off by half a part and a few roundings: |sqrt(|m|/sm) - c/127| <= (1/2 + 127 * 3 u)/127."""
    m = (synth.normal_f32((n,), 1.0, seed=1) * np.exp(2 * synth.normal_f32((n,), 1.0, seed=2))).astype(F)
    v = (synth.normal_f32((n,), 1.0, seed=3) ** 2 * np.exp(2 * synth.normal_f32((n,), 1.0, seed=4))).astype(F)
    m8, v8, s = O.adamw8_pack(m, v)
    sm, sr = (np.repeat(s[:, k].astype(np.float64), 256)[:n] for k in (0, 1))
    assert (np.abs(np.sqrt(np.abs(m) / sm) * 127 - np.abs(m8)) <= 0.5 + 127 * 4 * U).all()
    assert (np.abs(np.sqrt(np.sqrt(v.astype(np.float64)) / sr) * 255 - v8) <= 0.5 + 255 * 5 * U + (v8 == 1)).all()
    assert ((np.sign(m8) == np.sign(m)) | (m8 == 0)).all()
    bm, bv = O.adamw8_unpack(m8, v8, s)
    assert (np.abs(bm - np.sign(m8) * sm * (m8 / 127.0) ** 2) <= 6 * U * np.abs(bm)).all() and (np.abs(bv - (sr * (v8 / 255.0) ** 2) ** 2) <= 12 * U * bv).all()


def test_updates_against_32_bits():
    """One step from zero moments is the step of 32 bits.  In the second one the moments are off by what their codes leave: with t = sqrt(share) and half a
    part e, |m^ - m| <= sm e (2 t + e), e = 1/2/127, and r likewise with 255, or a whole part where the code is held at 1; four roundings each besides.  The step
    grows with m and falls with r, so it lies between those of the corners, and its dozen roundings are relative to it and to the terms of m."""
    n, h = 3000, (1e-3, 0.9, 0.95, 1e-8, 0.1)
    lr, b1, b2, eps, wd = (float(F(x)) for x in h)
    p = synth.normal_f32((n,), 0.02, seed=1)
    st8, st = (p, np.zeros(n, np.int8), np.zeros(n, np.uint8), np.zeros((12, 2), F)), (p, np.zeros(n, F), np.zeros(n, F))
    size = np.exp(2 * synth.normal_f32((n,), 1.0, seed=9) - 6)
    g = [(synth.normal_f32((n,), 1.0, seed=100 + t) * size).astype(F) for t in (1, 2)]
    st8, st = O.adamw8(st8[0], g[0], *st8[1:], *h, 1), O.adamw(st[0], g[0], *st[1:], *h, 1)
    assert np.array_equal(st8[0], st[0])
    m, r = st[1].astype(np.float64), np.sqrt(st[2].astype(np.float64))
    sm, sr = (np.repeat(st8[3][:, k].astype(np.float64), 256)[:n] for k in (0, 1))
    tm, tr = np.sqrt(np.abs(m) / sm), np.sqrt(r / sr)
    em, er = (0.5 + 127 * 4 * U) / 127, np.where(st8[2] == 1, 1.0, 0.5 + 255 * 5 * U) / 255
    dm, dr = sm * em * (2 * tm + em) + 4 * U * np.abs(m), sr * er * (2 * tr + er) + 4 * U * r
    st8 = O.adamw8(st8[0], g[1], *st8[1:], *h, 2)
    g2 = g[1].astype(np.float64)

    def step(m, r):
        return lr * (b1 * m + (1 - b1) * g2) / (1 - 0.9 ** 2) / (np.sqrt((b2 * r * r + (1 - b2) * g2 * g2) / (1 - 0.95 ** 2)) + eps)
    corners = np.stack([step(m + a * dm, np.maximum(r + b * dr, 0)) for a in (-1, 1) for b in (-1, 1)])
    terms = lr * (b1 * (np.abs(m) + dm) + np.abs(g2)) / (1 - 0.9 ** 2) / (np.sqrt((b2 * np.maximum(r - dr, 0) ** 2 + (1 - b2) * g2 * g2) / (1 - 0.95 ** 2)) + eps)
    moved = st[0].astype(np.float64) * (1 - lr * wd) - st8[0]
    slack = 3 * U * np.abs(st[0]) + 20 * U * (np.abs(corners).max(0) + terms)
    assert (moved >= corners.min(0) - slack).all() and (moved <= corners.max(0) + slack).all()


def test_update_in_64_bits():
    """p against the formulas in 64 bits from the same codes: m, v and r have six to twelve roundings each, the step as many more."""
    n, (lr, b1, b2, eps, wd), t = 700, (3e-4, 0.9, 0.95, 1e-8, 0.1), 7
    p = synth.normal_f32((n,), 0.02, seed=1)
    g = synth.normal_f32((n,), 1e-3, seed=2)
    m8, v8, s = O.adamw8_pack(synth.normal_f32((n,), 1e-3, seed=3), synth.normal_f32((n,), 1e-3, seed=4) ** 2)
    m, v = (x.astype(np.float64) for x in O.adamw8_unpack(m8, v8, s))
    q, _, _, s2 = O.adamw8(p, g, m8, v8, s, lr, b1, b2, eps, wd, t)
    fb1, fb2 = float(F(b1)), float(F(b2))
    m, v = fb1 * m + (1 - fb1) * g.astype(np.float64), fb2 * v + (1 - fb2) * g.astype(np.float64) ** 2
    step = lr * (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    # m is a sum of terms that may cancel: its error is relative to them
    scale = lr * (fb1 * np.abs(m) + np.abs(g)) / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    assert (np.abs(q - (p * (1 - lr * wd) - step)) <= 3 * U * np.abs(p) + 20 * U * (np.abs(step) + scale)).all()
    assert np.allclose(s2[:, 1], [np.sqrt(v[i:i + 256]).max() for i in range(0, n, 256)], rtol=12 * U)


def test_step_learns_from_every_parameter():
    """No gradient of the block is lost: every parameter of a step with these linears moves, and so with moments in 8 bits."""
    from oracle import step as ostep
    cfg = dict(n_layers=2, d_model=128, n_heads=1, ffn=96, vocab=128, seq=64, micro_batch=1, mesh=(1, 1, 1), linear="token", state8=True, act8=True, recurrent=(1,),
               lr=1e-2)
    params = synth.model_params(cfg, seed=5)
    first = ostep.run_step(cfg, params, synth.model_tokens(cfg, 1, seed=5))
    for name, p in first["params"].items():
        assert not np.array_equal(p, params[name]), name
    assert np.isfinite(first["loss"]) and abs(first["loss"] - np.log(128)) < 0.5 and not any(n.endswith("s_x") for n in params)
