"""Pins of the oracle's layer norm, 8-bit checkpoints and gated linear recurrence: 64-bit references, differences, hand-worked cases,
and the properties the definitions promise."""
import numpy as np
import pytest

import blockref as R
import oracle
import synth

F = np.float32


def _rows(shape, seed, bf, mean=0.0, scale=1.0):
    x = synth.normal_f32(shape, scale, mean=mean, seed=seed, tid=1)
    return synth.to_bf16(x) if bf else x


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("rows,D,mean", [(5, 1, 0.0), (3, 2, 1.0), (7, 8, 0.0), (33, 257, 3.0), (16, 1003, 0.0), (4, 2048, -50.0), (1, 4097, 0.5)])
def test_layernorm_against_64_bits(bf, rows, D, mean):
    x = _rows((rows, D), 3, bf, mean)
    g, b = _rows(D, 4, bf, 1.0, 0.1), _rows(D, 5, bf, 0.0, 0.3)
    dy, res = _rows((rows, D), 6, bf), _rows((rows, D), 7, bf)
    for gain, shift in ((g, b), (None, None), (g, None)):
        y, mu, rs = oracle.layernorm_fwd(x, gain, shift, 1e-6, bf=bf)
        w = R.layernorm(x, gain, shift, 1e-6)
        R.close(mu, w["mean"], w["err_mean"], what="mean")
        if D > 2:                                    # of one or two values the variance is what rounding leaves of it
            R.close(rs, w["rstd"], w["err_rstd"], what="rstd")
            R.close(y, w["y"], w["err_y"], bf, "y")
        for other in (None, res):
            dx, dg, db = oracle.layernorm_bwd(dy, x, gain, mu, rs, other, bf=bf)
            w = R.layernorm_bwd(dy, x, gain, mu, rs, other)
            R.close(dx, w["dx"], w["err_dx"], bf, "dx")
            R.close(dg, w["dgamma"], w["err_dgamma"], what="dgamma")
            R.close(db, w["dbeta"], w["err_dbeta"], what="dbeta")


def test_layernorm_by_hand():
    # mean 3, differences -2 0 2 0, variance 2; eps 2: rstd = 1/2
    y, mu, rs = oracle.layernorm_fwd(np.array([[1, 3, 5, 3]], F), np.array([1, 1, 2, 1], F), np.array([0, 7, 1, -1], F), eps=2.0)
    assert mu[0] == 3 and rs[0] == 0.5 and y.tolist() == [[-1, 7, 3, -1]]


def test_layernorm_gradient_by_differences():
    rng = np.random.default_rng(1)
    x, g, b, dy = rng.normal(size=(3, 24)), 1 + 0.2 * rng.normal(size=24), rng.normal(size=24), rng.normal(size=(3, 24))

    def loss(x, g, b):
        d = x - x.mean(1, keepdims=True)
        return ((d / np.sqrt((d * d).mean(1, keepdims=True) + 1e-6) * g + b) * dy).sum()

    f32 = lambda a: a.astype(F)
    _, mu, rs = oracle.layernorm_fwd(f32(x), f32(g), f32(b))
    dx, dg, db = oracle.layernorm_bwd(f32(dy), f32(x), f32(g), mu, rs)
    h = 1e-6
    for a, got in ((x, dx), (g, dg), (b, db)):
        for i in range(0, a.size, 7):
            keep = a.flat[i]
            a.flat[i] = keep + h
            up = loss(x, g, b)
            a.flat[i] = keep - h
            down = loss(x, g, b)
            a.flat[i] = keep
            # second order h^2 f''' and the 64-bit roundings 1e-16 / h of the difference, binary32 roundings of the gradient
            assert abs((up - down) / (2 * h) - got.flat[i]) < 1e-5 * max(1.0, abs(got.flat[i]))


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("rows,D", [(1, 1), (3, 31), (4, 32), (5, 33), (9, 200), (2, 1000)])
def test_act8_against_64_bits(bf, rows, D):
    x = _rows((rows, D), 11, bf) if bf else synth.normal_f32((rows, D), 1.0, seed=11, tid=2) * np.exp(synth.normal_f32((rows, D), 3.0, seed=12, tid=3)).astype(F)
    q, e = oracle.act8_pack(x, bf)
    want, step = R.act8(x)
    got = oracle.act8_unpack(q, e, bf)
    assert np.array_equal(R.wide(got), want)                       # exact in either type
    assert (np.abs(R.wide(x) - want) <= step / 2).all()
    assert np.abs(q.astype(int)).max() <= 127
    assert np.array_equal(oracle.act8_unpack(q, e, True), synth.to_bf16(oracle.act8_unpack(q, e, False)))


def test_act8_ends():
    big = F(3.4028235e38)
    x = np.zeros((8, 40), F)
    x[0, :3] = 127.0, -126.5, 0.5                                  # step 1: ties to even
    x[1, :2] = 127.00001, 1.0                                      # just past 127: step 2
    x[2, :2] = big, -big
    x[3, :3] = 1e-40, 2.0 ** -126, -3 * 2.0 ** -126                # the smallest step; a subnormal is zero
    x[4, :4] = np.inf, -np.inf, np.nan, 5.0
    x[4, 35] = 2.0                                                 # the next group of the row is its own
    x[5, 39] = -127.5
    x[6] = -0.0
    q, e = oracle.act8_pack(x, False)
    assert q[0, :3].tolist() == [127, -126, 0] and e[0].tolist() == [127, 1]
    assert q[1, :2].tolist() == [64, 0] and e[1, 0] == 128
    assert q[2, :2].tolist() == [64, -64] and e[2, 0] == 249
    assert q[3, :3].tolist() == [0, 1, -3] and e[3, 0] == 1
    assert q[4, :4].tolist() == [127, -127, 0, 0] and e[4].tolist() == [255, 122]
    assert q[5, 39] == -64 and e[5, 1] == 128 and not q[6].any()
    y = oracle.act8_unpack(q, e, False)
    assert y[4, 0] == np.inf and y[4, 1] == -np.inf and np.isnan(y[4, 2:32]).all() and y[4, 35] == 2 and not y[4, 32]


def _gv(B, S, D, seed, gate=2.0):
    g = synth.normal_f32((B * S, D), 2.0, mean=gate, seed=seed, tid=1)
    return synth.to_bf16(np.concatenate([g, synth.normal_f32((B * S, D), 1.0, seed=seed, tid=2)], 1))


def _flags(B, S, every, seed):
    return (synth.randint((B, S), every, seed=seed, tid=9) == 0).astype(np.uint8) if every else None


@pytest.mark.parametrize("B,S,D,every,ends", [(1, 1, 2, 0, True), (2, 7, 4, 0, False), (1, 8, 2, 3, True), (1, 9, 2, 0, True), (2, 63, 6, 5, True),
                                              (1, 64, 2, 0, True), (3, 65, 4, 0, False), (1, 500, 10, 40, True), (1, 2000, 4, 0, True),
                                              (1, 130, 4, 1, True)])
def test_linrec_against_64_bits(B, S, D, every, ends):
    gv, fl = _gv(B, S, D, 21), _flags(B, S, every, 22)
    h0 = synth.normal_f32((B, D), 1.0, seed=23, tid=1) if ends else None
    dhT = synth.normal_f32((B, D), 1.0, seed=23, tid=2) if ends else None
    dy = synth.normal_bf16((B * S, D), 1.0, seed=24, tid=1)
    y, hT, states = oracle.linrec_fwd(gv, B, S, fl, h0)
    w = R.linrec(gv, B, S, fl, h0)
    R.close(y, w["h"], w["err_h"], True, "y")
    R.close(hT, w["hT"], w["err_hT"], what="hT")
    for k in range(1, states.shape[1]):
        R.close(states[:, k], w["h"].reshape(B, S, D)[:, 8 * k - 1], w["err_h"].reshape(B, S, D)[:, 8 * k - 1], what="states")
    dgv, dh0 = oracle.linrec_bwd(dy, gv, states, B, S, fl, dhT)
    w = R.linrec_bwd(dy, gv, B, S, fl, h0, dhT)
    R.close(np.ascontiguousarray(dgv[:, D:]), w["dv"], w["err_dv"], True, "dv")
    R.close(np.ascontiguousarray(dgv[:, :D]), w["dg"], w["err_dg"], True, "dg")
    R.close(dh0, w["dh0"], w["err_dh0"], what="dh0")


def test_linrec_gradient_by_differences():
    B, S, D = 1, 12, 2
    rng = np.random.default_rng(3)
    gv = synth.from_bf16(synth.to_bf16(rng.normal(size=(S, 2 * D)).astype(F))).astype(np.float64)
    h0, dhT = rng.normal(size=(B, D)), rng.normal(size=(B, D))
    dy = synth.from_bf16(synth.to_bf16(rng.normal(size=(S, D)).astype(F))).astype(np.float64)
    fl = np.zeros((B, S), np.uint8)
    fl[0, 5] = 1

    def loss(gv, h0):
        s, total = h0[0].copy(), 0.0
        for t in range(S):
            f = 1 / (1 + np.exp(-gv[t, :D]))
            s = (0 if fl[0, t] else f * s) + (1 - f) * gv[t, D:]
            total += (s * dy[t]).sum()
        return total + (s * dhT[0]).sum()

    bits = synth.to_bf16(gv.astype(F))
    _, _, states = oracle.linrec_fwd(bits, B, S, fl, h0.astype(F))
    dgv, dh0 = oracle.linrec_bwd(synth.to_bf16(dy.astype(F)), bits, states, B, S, fl, dhT.astype(F))
    h = 1e-6
    for a, got in ((gv, synth.from_bf16(dgv)), (h0, dh0)):
        for i in range(a.size):
            keep = a.flat[i]
            a.flat[i] = keep + h
            up = loss(gv, h0)
            a.flat[i] = keep - h
            down = loss(gv, h0)
            a.flat[i] = keep
            d = (up - down) / (2 * h)
            assert abs(d - got.flat[i]) <= R.UBF * abs(d) + 1e-7       # bf16 gradients; the difference is good to 1e-9


def test_linrec_in_pieces_of_whole_spans_is_the_same():
    """A sequence in pieces of whole spans (128 rows), each starting from what the one before left: every bit.  Backward the spans are counted from the
    end of the call."""
    S, D, cut = 256 + 130, 4, 128
    gv, dy = _gv(1, S, D, 31), synth.normal_bf16((S, D), 1.0, seed=32, tid=1)
    y, hT, st = oracle.linrec_fwd(gv, 1, S)
    y0, s, st0 = oracle.linrec_fwd(gv[:cut], 1, cut)
    y1, s, st1 = oracle.linrec_fwd(gv[cut:], 1, S - cut, h0=s)
    assert np.array_equal(y, np.concatenate([y0, y1])) and np.array_equal(hT, s) and np.array_equal(st, np.concatenate([st0, st1], 1))
    S = 256
    dgv, dh0 = oracle.linrec_bwd(dy[:S], gv[:S], st[:, :S // 8], 1, S)
    d1, c = oracle.linrec_bwd(dy[cut:S], gv[cut:S], st[:, cut // 8:S // 8], 1, S - cut)
    d0, c = oracle.linrec_bwd(dy[:cut], gv[:cut], st[:, :cut // 8], 1, cut, dhT=c)
    assert np.array_equal(dgv, np.concatenate([d0, d1])) and np.array_equal(dh0, c)


def test_linrec_cut_keeps_a_nan_on_its_side():
    """Rows of documents side by side: a NaN or an infinity in one reaches neither the others' outputs nor their gradients."""
    S, D = 200, 4
    gv, dy = _gv(1, S, D, 41), synth.normal_bf16((S, D), 1.0, seed=42, tid=1)
    fl = np.zeros((1, S), np.uint8)
    fl[0, [50, 131, 132]] = 1
    y, hT, st = oracle.linrec_fwd(gv, 1, S, fl)
    dgv, dh0 = oracle.linrec_bwd(dy, gv, st, 1, S, fl)
    bad, bdy = gv.copy(), dy.copy()
    bad[70, 0] = bad[90, D + 1] = 0x7FC0                            # a gate and a value
    bad[60, D + 2] = 0x7F80
    bdy[100, 3] = 0x7FC0
    y2, hT2, st2 = oracle.linrec_fwd(bad, 1, S, fl)
    dgv2, dh02 = oracle.linrec_bwd(bdy, bad, st2, 1, S, fl)
    out = np.r_[0:50, 131:200]
    assert np.array_equal(y[out], y2[out]) and np.array_equal(hT, hT2) and np.array_equal(dgv[out], dgv2[out]) and np.array_equal(dh0, dh02)
    assert np.isnan(synth.from_bf16(y2[70:131, 0])).all() and np.isnan(synth.from_bf16(y2[90:131, 1])).all()
    assert np.isinf(synth.from_bf16(y2[60, 2])) and np.isnan(synth.from_bf16(dgv2[50:101, D + 3])).all()


def test_linrec_saturated_gates():
    """f = 1 keeps the state to the bit, f = 0 takes the value; the complement keeps its digits where 1 - f would have none."""
    g = np.array([[200.0], [200.0], [-200.0], [20.0]], F).repeat(2, 1)
    v = np.array([[5.0], [7.0], [3.0], [1e6]], F).repeat(2, 1)
    y, hT, _ = oracle.linrec_fwd(synth.to_bf16(np.concatenate([g, v], 1)), 1, 4, h0=np.full((1, 2), 1.25, F))
    assert synth.from_bf16(y)[:3, 0].tolist() == [1.25, 1.25, 3.0]
    z = np.exp(-20.0) / (1 + np.exp(-20.0))
    # 16 u of each term, which are below 4
    assert abs(float(hT[0, 0]) - (3.0 * (1 - z) + float(synth.from_bf16(synth.to_bf16(np.array([1e6], F)))[0]) * z)) < 16 * R.U * 4
