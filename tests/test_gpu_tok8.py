"""8-bit products with token and channel scales and the gated block on them on the GPU against the oracle, bit for bit (the oracle's own pins against 64
bits are in test_oracle_tok8.py)."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import assert_same_bits, dev, empty, host, ws

pytestmark = pytest.mark.gpu
F = np.float32
GUARD = 0x5A


@pytest.fixture(scope="module")
def det():
    import paper_2609_17380_b200 as d
    d.load()
    return d


def _sync():
    import torch
    torch.cuda.synchronize()


def same(got, want, what):
    """Every bit; NaNs as NaNs (their payloads are not defined)."""
    wide = lambda x: synth.from_bf16(x) if x.dtype == np.uint16 else x
    want = np.ascontiguousarray(want)
    nan = np.isnan(wide(want)) if want.dtype in (np.uint16, np.float32) else np.zeros(want.shape, bool)
    if nan.any():
        assert np.array_equal(np.isnan(wide(got)), nan), what
        got, want = got[~nan], want[~nan]
    assert_same_bits(got, want, what)


def codes(q):
    """Codes as the library lays them out: rows 16-byte aligned, zeros behind their end."""
    return np.pad(q, ((0, 0), (0, -q.shape[1] % 16)))


def rows(M, K, seed, std=1.0):
    """Channels of different scale; some rows are zero, one is large, one so small that its scale is flushed."""
    x = synth.normal_f32((M, K), std, seed=seed, tid=1) * np.exp(0.7 * synth.normal_f32((K,), 1.0, seed=seed, tid=2))
    if M > 6:
        x[3] = 0
        x[5] *= F(1e30)
        x[6] = x[6] * F(1e-38)
    return synth.to_bf16(x.astype(F))


def strided(a, ld, fill=0xABAB):
    """The rows of a ld elements apart, and what lies between them."""
    out = np.full((a.shape[0], ld), fill, a.dtype)
    out[:, :a.shape[1]] = a
    return out


# one token, some, ragged tiles of every kind, odd widths and whole ones; contractions shorter than a stage, of one stage and of several
SIZES = [(1, 1, 1), (1, 64, 128), (2, 33, 7), (7, 130, 65), (16, 256, 256), (31, 100, 1000), (64, 257, 384), (129, 65, 129), (128, 128, 128), (130, 520, 264),
         (257, 200, 515), (300, 1003, 777), (256, 768, 256), (515, 384, 2056), (1000, 1040, 96), (9, 4104, 2048), (4, 40, 9000), (3, 24, 17000),
         # up to eight tokens by every number of channels a warp has at a time; tiles that two, four and eight CTAs share, ragged ones among them
         (1, 9500, 40), (2, 4800, 300), (1, 2048, 2048), (2, 130, 9000), (5, 9480, 72), (8, 4800, 528), (3, 9999, 17), (8, 500, 1000),
         (24, 136, 8192), (9, 70, 1024), (32, 4100, 600), (33, 257, 2050), (100, 90, 4096), (128, 500, 2000), (150, 40, 3000), (20, 9000, 520)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_codes_and_transpose(det, M, N, K):
    x = rows(M, K, 11)
    want, scale = oracle.tok8_quant(x)
    ld = det.det_tok8_ld(K)
    assert ld == -(-K // 16) * 16
    for pitch in {K, K + 3, -(-K // 8) * 8 + 8}:
        q, s = dev(np.full((M, ld), GUARD, np.int8)), empty((M,), F)
        det.det_tok8_quant(dev(strided(x, pitch)), pitch, M, K, q, s)
        _sync()
        same(host(s), scale, "scales")
        same(host(q), codes(want), "codes")
    t = dev(np.full((K, det.det_tok8_ld(M)), GUARD, np.int8))
    det.det_tok8_transpose(q, M, K, t)
    _sync()
    same(host(t), codes(np.ascontiguousarray(want.T)), "transposed")


@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear(det, M, N, K):
    x, w, dy = rows(M, K, 1), synth.normal_bf16((N, K), 0.02, seed=2), rows(M, N, 3, 0.01)
    if N > 4:
        w[2] = 0                                                      # a channel whose scale is zero
    Y, qX, sX, qW, sW = oracle.tok8_linear_fwd(x, w)
    wc, wt = dev(codes(qW)), dev(codes(np.ascontiguousarray(qW.T)))
    for ld in {N, N + 5, -(-N // 8) * 8}:
        y, q, s = dev(np.full((M, ld), 0xABAB, np.uint16)), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
        det.det_tok8_linear_fwd(dev(x), K, wc, dev(sW), M, N, K, y, ld, q, s)
        _sync()
        same(host(y, np.uint16), strided(Y, ld), "y")
        same(host(q), codes(qX), "codes")
        same(host(s), sX, "scales")
        y2 = dev(np.full((M, ld), 0xABAB, np.uint16))
        det.det_tok8_linear_fwd_q(q, s, wc, dev(sW), M, N, K, y2, ld)
        _sync()
        same(host(y2, np.uint16), strided(Y, ld), "y from codes")
    dX, dW = oracle.tok8_linear_bwd(dy, x, w)
    work = ws(det.det_tok8_linear_bwd_ws_bytes(M, N, K))
    work.fill_(GUARD)
    for ldx, ldy in ((K, N), (K + 3, N + 1), (-(-K // 8) * 8, -(-N // 8) * 8)):
        dx, dw = dev(np.full((M, ldx), 0xABAB, np.uint16)), empty((N, K), F)
        det.det_tok8_linear_bwd(dev(strided(dy, ldy)), ldy, q, s, wt, dev(sW), M, N, K, dx, ldx, dw, work)
        _sync()
        same(host(dx, np.uint16), strided(dX, ldx), "dx")
        same(host(dw), dW, "dw")
    dx, dw = empty((M, K), np.uint16), empty((N, K), F)
    det.det_tok8_linear_bwd(dev(dy), N, q, s, wt, dev(sW), M, N, K, dx, K, None, work)        # either gradient alone
    det.det_tok8_linear_bwd(dev(dy), N, q, s, wt, dev(sW), M, N, K, None, 0, dw, work)
    _sync()
    same(host(dx, np.uint16), dX, "dx alone")
    same(host(dw), dW, "dw alone")


# and with enough pairs that CTAs stay and look the sigmoids up
@pytest.mark.parametrize("M,Fh,K", SIZES + [(1201, 8104, 40), (1300, 8101, 24)])
def test_glu(det, M, Fh, K):
    x, w, dh = rows(M, K, 4), synth.normal_bf16((2 * Fh, K), 0.02, seed=5), rows(M, Fh, 6, 0.01)
    gu, qX, sX, qW, sW = oracle.tok8_linear_fwd(x, w)
    h = oracle.swiglu_fwd(gu)
    wc, wt = dev(codes(qW)), dev(codes(np.ascontiguousarray(qW.T)))
    q, s = empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
    for ldh, ldg in ((Fh, 2 * Fh), (Fh + 3, 2 * Fh + 1), (-(-Fh // 8) * 8, -(-2 * Fh // 8) * 8)):
        gh, gg = dev(np.full((M, ldh), 0xABAB, np.uint16)), dev(np.full((M, ldg), 0xABAB, np.uint16))
        det.det_tok8_glu_fwd(dev(x), K, wc, dev(sW), M, Fh, K, gh, ldh, gg, ldg, q, s)
        _sync()
        same(host(gh, np.uint16), strided(h, ldh), "h")
        same(host(gg, np.uint16), strided(gu, ldg), "gu")
        same(host(s), sX, "scales")
        gh = dev(np.full((M, ldh), 0xABAB, np.uint16))
        det.det_tok8_glu_fwd_q(q, s, wc, dev(sW), M, Fh, K, gh, ldh)                            # gate and up not kept
        _sync()
        same(host(gh, np.uint16), strided(h, ldh), "h alone")
    dX, dW = oracle.tok8_linear_bwd(oracle.swiglu_bwd(dh, gu), x, w)
    work = ws(det.det_tok8_glu_bwd_ws_bytes(M, Fh, K))
    work.fill_(GUARD)
    for ldx, ldh, ldg in ((K, Fh, 2 * Fh), (K + 1, Fh + 3, 2 * Fh + 1), (-(-K // 8) * 8, -(-Fh // 8) * 8, -(-2 * Fh // 8) * 8)):
        dx, dw = dev(np.full((M, ldx), 0xABAB, np.uint16)), empty((2 * Fh, K), F)
        det.det_tok8_glu_bwd(dev(strided(dh, ldh)), ldh, dev(strided(gu, ldg)), ldg, q, s, wt, dev(sW), M, Fh, K, dx, ldx, dw, work)
        _sync()
        same(host(dx, np.uint16), strided(dX, ldx), "dx")
        same(host(dw), dW, "dw")


@pytest.mark.parametrize("M,N,K", [(5, 40, 48), (150, 136, 264)])
def test_not_finite(det, M, N, K):
    """An infinity or a NaN in a token makes that token's output NaN and every weight gradient; in a channel that channel's; nothing else."""
    x, w, dy = rows(M, K, 1), synth.normal_bf16((N, K), 0.02, seed=2), rows(M, N, 3, 0.01)
    for place, value in (("x", 0x7F80), ("x", 0x7FC1), ("w", 0xFF80), ("dy", 0x7FC1)):
        a = dict(x=x.copy(), w=w.copy(), dy=dy.copy())
        a[place][2, 3] = value
        Y, qX, sX, qW, sW = oracle.tok8_linear_fwd(a["x"], a["w"])
        y, q, s = empty((M, N), np.uint16), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
        det.det_tok8_linear_fwd(dev(a["x"]), K, dev(codes(qW)), dev(sW), M, N, K, y, N, q, s)
        dx, dw = empty((M, K), np.uint16), empty((N, K), F)
        det.det_tok8_linear_bwd(dev(a["dy"]), N, q, s, dev(codes(np.ascontiguousarray(qW.T))), dev(sW), M, N, K, dx, K, dw,
                                ws(det.det_tok8_linear_bwd_ws_bytes(M, N, K)))
        _sync()
        same(host(y, np.uint16), Y, "y")
        nan = np.isnan(synth.from_bf16(Y))
        assert nan.sum() == dict(x=N, w=M, dy=0)[place] and (nan[2].all() if place == "x" else nan[:, 2].all() if place == "w" else True)
        dX, dW = oracle.tok8_linear_bwd(a["dy"], a["x"], a["w"])
        same(host(dx, np.uint16), dX, "dx")
        same(host(dw), dW, "dw")


def test_no_tokens(det):
    w = synth.normal_bf16((48, 32), 0.02, seed=2)
    qW, sW = oracle.tok8_quant(w)
    dw = dev(np.full((48, 32), 7, F))
    keep = dev(np.full((4, 48), 0xABAB, np.uint16))
    q, s = empty((4, 32), np.int8), empty((4,), F)
    det.det_tok8_linear_fwd(keep, 32, dev(codes(qW)), dev(sW), 0, 48, 32, keep, 48, q, s)
    det.det_tok8_linear_bwd(keep, 48, q, s, dev(codes(np.ascontiguousarray(qW.T))), dev(sW), 0, 48, 32, keep, 32, dw, None)
    _sync()
    assert (host(keep, np.uint16) == 0xABAB).all() and not host(dw).any()


@pytest.mark.parametrize("M", [1, 3, 40, 300])
def test_tokens_do_not_depend_on_each_other(det, M):
    """A token's output has the bits that it has alone."""
    N, K = 520, 1032
    x, w = rows(M, K, 8), synth.normal_bf16((N, K), 0.02, seed=9)
    qW, sW = oracle.tok8_quant(w)
    run = lambda a, m, y: det.det_tok8_linear_fwd(a, K, dev(codes(qW)), dev(sW), m, N, K, y, N, empty((m, det.det_tok8_ld(K)), np.int8), empty((m,), F))
    y, one = empty((M, N), np.uint16), empty((1, N), np.uint16)
    run(dev(x), M, y)
    run(dev(x[M - 1:]), 1, one)
    _sync()
    same(host(y, np.uint16)[M - 1:], host(one, np.uint16), "last token")


def test_graph_and_streams(det):
    """Captured and replayed on new inputs in the same buffers, two captures with a workspace each on two streams."""
    import torch
    M, Fh, K = 200, 136, 264
    w = synth.normal_bf16((2 * Fh, K), 0.02, seed=5)
    qW, sW = oracle.tok8_quant(w)
    wc, wt, sw = dev(codes(qW)), dev(codes(np.ascontiguousarray(qW.T))), dev(sW)
    sets, graphs = [], []
    for i in range(2):
        st = torch.cuda.Stream()
        b = dict(x=dev(rows(M, K, 4)), dh=dev(rows(M, Fh, 6, 0.01)), h=empty((M, Fh), np.uint16), gu=empty((M, 2 * Fh), np.uint16), dx=empty((M, K), np.uint16),
                 dw=empty((2 * Fh, K), F), q=empty((M, det.det_tok8_ld(K)), np.int8), s=empty((M,), F), ws=ws(det.det_tok8_glu_bwd_ws_bytes(M, Fh, K)))

        def both():
            det.det_tok8_glu_fwd(b["x"], K, wc, sw, M, Fh, K, b["h"], Fh, b["gu"], 2 * Fh, b["q"], b["s"])
            det.det_tok8_glu_bwd(b["dh"], Fh, b["gu"], 2 * Fh, b["q"], b["s"], wt, sw, M, Fh, K, b["dx"], K, b["dw"], b["ws"])
        with torch.cuda.stream(st):
            both()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            both()
        sets.append(b)
        graphs.append((g, st))
    for seed in (21, 22):
        want = []
        for i, b in enumerate(sets):
            x, dh = rows(M, K, seed + 10 * i), rows(M, Fh, seed + 10 * i + 5, 0.01)
            b["x"].copy_(dev(x))
            b["dh"].copy_(dev(dh))
            gu = oracle.tok8_linear_fwd(x, w)[0]
            want.append((oracle.swiglu_fwd(gu), *oracle.tok8_linear_bwd(oracle.swiglu_bwd(dh, gu), x, w)))
        torch.cuda.synchronize()
        for g, st in graphs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for b, (h, dX, dW) in zip(sets, want):
            same(host(b["h"], np.uint16), h, "h")
            same(host(b["dx"], np.uint16), dX, "dx")
            same(host(b["dw"]), dW, "dw")


# contractions near the limit, forward and backward
@pytest.mark.parametrize("M,N,K", [(2, 24, 131071), (1, 16, 40000), (70001, 24, 40), (24, 70001, 40)])
def test_long_contractions(det, M, N, K):
    x, w, dy = rows(M, K, 1), synth.normal_bf16((N, K), 0.02, seed=2), rows(M, N, 3, 0.01)
    Y, qX, sX, qW, sW = oracle.tok8_linear_fwd(x, w)
    y, q, s = empty((M, N), np.uint16), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
    det.det_tok8_linear_fwd(dev(x), K, dev(codes(qW)), dev(sW), M, N, K, y, N, q, s)
    dx, dw = empty((M, K), np.uint16), empty((N, K), F)
    det.det_tok8_linear_bwd(dev(dy), N, q, s, dev(codes(np.ascontiguousarray(qW.T))), dev(sW), M, N, K, dx, K, dw, ws(det.det_tok8_linear_bwd_ws_bytes(M, N, K)))
    _sync()
    dX, dW = oracle.tok8_linear_bwd(dy, x, w)
    same(host(y, np.uint16), Y, "y")
    same(host(dx, np.uint16), dX, "dx")
    same(host(dw), dW, "dw")


def test_extreme_codes(det):
    """The largest sum there is: 131071 products of 127 and -127."""
    K = 131071
    x = np.full((9, K), 0x3F80, np.uint16)
    w = np.full((70, K), 0xBF80, np.uint16)
    for M in (1, 9):
        Y, _, _, qW, sW = oracle.tok8_linear_fwd(x[:M], w)
        y = empty((M, 70), np.uint16)
        det.det_tok8_linear_fwd(dev(x[:M]), K, dev(codes(qW)), dev(sW), M, 70, K, y, 70, empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F))
        _sync()
        same(host(y, np.uint16), Y, "y")
        assert (synth.from_bf16(host(y, np.uint16)) == synth.from_bf16(synth.to_bf16(np.array([-K], F)))).all()


@pytest.mark.parametrize("M,Fh,K", [(1, 40, 48), (2, 33, 65), (5, 24, 40), (40, 72, 264), (130, 65, 129)])
def test_any_address(det, M, Fh, K):
    """Every matrix one element off an aligned address, and rows in front of and behind the outputs that stay."""
    import torch
    N = 2 * Fh
    x, w, dh = rows(M, K, 4), synth.normal_bf16((N, K), 0.02, seed=5), rows(M, Fh, 6, 0.01)
    gu, qX, sX, qW, sW = oracle.tok8_linear_fwd(x, w)
    hold = []

    def off(a, fill=0):
        """An array one element off, with room in front and behind; its address and how to read it back."""
        t = torch.full((a.size + 64,), fill, dtype={2: torch.int16, 4: torch.float32}[a.itemsize], device="cuda")
        t[1:1 + a.size] = dev(a).reshape(-1)
        hold.append(t)
        return t.data_ptr() + a.itemsize, t
    wc, wt = dev(codes(qW)), dev(codes(np.ascontiguousarray(qW.T)))
    px, ps = off(x)[0], off(sW)[0]
    ph, th = off(np.zeros((M, Fh), np.uint16), 77)
    pg, tg = off(np.zeros((M, N), np.uint16), 77)
    psx, tsx = off(np.zeros(M, F), 77)
    q = empty((M, det.det_tok8_ld(K)), np.int8)
    det.det_tok8_glu_fwd(px, K, wc, ps, M, Fh, K, ph, Fh, pg, N, q, psx)
    _sync()
    back = lambda t, a, dt: host(t, dt)[1:1 + a.size].reshape(a.shape)
    same(back(th, np.zeros((M, Fh)), np.uint16), oracle.swiglu_fwd(gu), "h")
    same(back(tg, gu, np.uint16), gu, "gu")
    same(back(tsx, sX, F), sX, "scales")
    pd = off(dh)[0]
    pdx, tdx = off(np.zeros((M, K), np.uint16), 77)
    pdw, tdw = off(np.zeros((N, K), F), 77)
    det.det_tok8_glu_bwd(pd, Fh, pg, N, q, psx, wt, ps, M, Fh, K, pdx, K, pdw, ws(det.det_tok8_glu_bwd_ws_bytes(M, Fh, K)))
    _sync()
    dX, dW = oracle.tok8_linear_bwd(oracle.swiglu_bwd(dh, gu), x, w)
    same(back(tdx, dX, np.uint16), dX, "dx")
    same(back(tdw, dW, F), dW, "dw")
    for t, n in ((th, M * Fh), (tg, M * N), (tsx, M), (tdx, M * K), (tdw, N * K)):
        assert t[0] == 77 and (t[1 + n:] == 77).all()


@pytest.mark.parametrize("M", [1, 2, 3, 12])
def test_few_tokens_that_are_zero_or_not_finite(det, M):
    N, K = 70, 264
    w = synth.normal_bf16((N, K), 0.02, seed=2)
    qW, sW = oracle.tok8_quant(w)
    for value in (0x0000, 0x8000, 0x7F80, 0x7FC1, 0x0001, 0x0080):                # zeros, an infinity, a NaN, a subnormal, the smallest normal
        x = rows(M, K, 1)
        x[M - 1] = value if value in (0x0000, 0x8000, 0x0001, 0x0080) else x[M - 1]
        x[M - 1, 5] = value
        Y, qX, sX, _, _ = oracle.tok8_linear_fwd(x, w)
        y, q, s = empty((M, N), np.uint16), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
        det.det_tok8_linear_fwd(dev(x), K, dev(codes(qW)), dev(sW), M, N, K, y, N, q, s)
        _sync()
        same(host(y, np.uint16), Y, "y")
        same(host(q), codes(qX), "codes")
        same(host(s), sX, "scales")


def test_two_calls_at_once(det):
    """Two streams with workspaces of their own, over and over, give what each gives alone."""
    import torch
    M, N, K = 700, 520, 392
    x, w, dy = rows(M, K, 1), synth.normal_bf16((N, K), 0.02, seed=2), rows(M, N, 3, 0.01)
    Y, qX, sX, qW, sW = oracle.tok8_linear_fwd(x, w)
    dX, dW = oracle.tok8_linear_bwd(dy, x, w)
    wc, wt, sw, gx, gy = dev(codes(qW)), dev(codes(np.ascontiguousarray(qW.T))), dev(sW), dev(x), dev(dy)
    torch.cuda.synchronize()
    sides = []
    for _ in range(2):
        sides.append(dict(st=torch.cuda.Stream(), y=empty((M, N), np.uint16), q=empty((M, det.det_tok8_ld(K)), np.int8), s=empty((M,), F),
                          dx=empty((M, K), np.uint16), dw=empty((N, K), F), ws=ws(det.det_tok8_linear_bwd_ws_bytes(M, N, K))))
    torch.cuda.synchronize()
    for _ in range(20):
        for b in sides:
            with torch.cuda.stream(b["st"]):
                det.det_tok8_linear_fwd(gx, K, wc, sw, M, N, K, b["y"], N, b["q"], b["s"])
                det.det_tok8_linear_bwd(gy, N, b["q"], b["s"], wt, sw, M, N, K, b["dx"], K, b["dw"], b["ws"])
    _sync()
    for b in sides:
        same(host(b["y"], np.uint16), Y, "y")
        same(host(b["dx"], np.uint16), dX, "dx")
        same(host(b["dw"]), dW, "dw")
