"""Layer norm, 8-bit checkpoints and the gated linear recurrence on the GPU against the oracle, bit for bit (the oracle's own pins against
64 bits are in test_oracle_blocks.py)."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import assert_same_bits, dev, empty, host, ws

pytestmark = pytest.mark.gpu
F = np.float32


@pytest.fixture(scope="module")
def det():
    import paper_2609_17380_b200 as d
    d.load()
    return d


def _sync():
    import torch
    torch.cuda.synchronize()


def _rows(shape, seed, bf, mean=0.0, scale=1.0):
    x = synth.normal_f32(shape, scale, mean=mean, seed=seed, tid=1)
    return synth.to_bf16(x) if bf else x


def _wide(x):
    return synth.from_bf16(x) if x.dtype == np.uint16 else x


def same(got, want, what):
    """Every bit; NaNs as NaNs (their payloads are not defined)."""
    g, w = _wide(got), _wide(np.asarray(want))
    if np.isnan(w).any():
        assert np.array_equal(np.isnan(g), np.isnan(w)), what
        got, want = got[~np.isnan(w)], np.asarray(want)[~np.isnan(w)]
    assert_same_bits(got, want, what)


LN_SIZES = [(1, 1), (3, 2), (5, 7), (33, 8), (128, 256), (17, 257), (40, 504), (31, 777), (64, 1000), (300, 1003), (19, 1024), (70, 2040),
            (1000, 2048), (9, 2049), (12, 4096), (5, 4097), (3, 8191), (26, 8192)]


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("rows,D", LN_SIZES)
def test_layernorm(det, bf, rows, D):
    dt = np.uint16 if bf else F
    x, dy = _rows((rows, D), 3, bf, 0.5), _rows((rows, D), 6, bf)
    g, b = _rows(D, 4, bf, 1.0, 0.1), _rows(D, 5, bf, 0.0, 0.3)
    w = ws(det.det_layernorm_bwd_ws_bytes(rows, D))
    for gain, shift in ((g, b), (None, b), (g, None)):
        dgain, dshift = dev(gain) if gain is not None else None, dev(shift) if shift is not None else None
        y, mean, rstd = empty((rows, D), dt), empty((rows,), F), empty((rows,), F)
        det.det_layernorm_fwd(int(bf), dev(x), dgain, dshift, rows, D, 1e-6, y, mean, rstd)
        _sync()
        oy, om, ors = oracle.layernorm_fwd(x, gain, shift, 1e-6, bf=bf)
        same(host(mean), om, "mean")
        same(host(rstd), ors, "rstd")
        same(host(y, dt), oy, "y")
        dx, dg, db = empty((rows, D), dt), empty((D,), F), empty((D,), F)
        det.det_layernorm_bwd(int(bf), dev(dy), dev(x), dgain, mean, rstd, rows, D, dx, dg, db, w)
        _sync()
        odx, odg, odb = oracle.layernorm_bwd(dy, x, gain, om, ors, bf=bf)
        same(host(dx, dt), odx, "dx")
        same(host(dg), odg, "dgamma")
        same(host(db), odb, "dbeta")
    for dg, db in ((None, empty((D,), F)), (empty((D,), F), None), (None, None)):    # each gradient alone, and none without a workspace
        dx = empty((rows, D), dt)
        det.det_layernorm_bwd(int(bf), dev(dy), dev(x), dgain, mean, rstd, rows, D, dx, dg, db, w if dg is not None or db is not None else None)
        _sync()
        same(host(dx, dt), odx, "dx")
        if dg is not None:
            same(host(dg), odg, "dgamma")
        if db is not None:
            same(host(db), odb, "dbeta")


@pytest.mark.parametrize("rows,D", [(30000, 64), (15001, 256), (9000, 768), (29000, 512), (7300, 2048), (3700, 4096), (2000, 8192), (8001, 2041), (150001, 8)])
def test_layernorm_many_rows(det, rows, D):
    """Rows enough for every number of passes a group of warps makes."""
    x, dy, g = _rows((rows, D), 13, True), _rows((rows, D), 16, True), _rows(D, 14, True, 1.0, 0.1)
    mean, rstd = synth.normal_f32(rows, 0.1, seed=17, tid=1), np.abs(synth.normal_f32(rows, 1.0, seed=17, tid=2)) + F(0.5)
    dx, dg, db = empty((rows, D), np.uint16), empty((D,), F), empty((D,), F)
    det.det_layernorm_bwd(det.DET_BF16, dev(dy), dev(x), dev(g), dev(mean), dev(rstd), rows, D, dx, dg, db, ws(det.det_layernorm_bwd_ws_bytes(rows, D)))
    _sync()
    odx, odg, odb = oracle.layernorm_bwd(dy, x, g, mean, rstd, bf=True)
    same(host(dx, np.uint16), odx, "dx")
    same(host(dg), odg, "dgamma")
    same(host(db), odb, "dbeta")


@pytest.mark.parametrize("rows,D", [(1, 64), (4, 2048), (3, 1003), (2, 4096), (1, 8192)])
def test_layernorm_few_rows(det, rows, D):
    """One block of rows: gain and shift come from the first kernel, or from the second where their place is not aligned; a row alone is flushed."""
    x, dy, g = _rows((rows, D), 33, True), _rows((rows, D), 36, True), _rows(D, 34, True, 1.0, 0.1)
    dy[0, :D // 2] = 0x0003                                         # subnormal
    mean, rstd = synth.normal_f32(rows, 0.1, seed=37, tid=1), np.abs(synth.normal_f32(rows, 1.0, seed=37, tid=2)) + F(0.5)
    odx, odg, odb = oracle.layernorm_bwd(dy, x, g, mean, rstd, bf=True)
    for off in (0, 1):
        for which in ((1, 1), (1, 0), (0, 1)):
            dx, buf = empty((rows, D), np.uint16), [dev(np.full(D + 2, 7.0, F)) for _ in range(2)]
            dg, db = (b[off:off + D] if w else None for b, w in zip(buf, which))
            det.det_layernorm_bwd(det.DET_BF16, dev(dy), dev(x), dev(g), dev(mean), dev(rstd), rows, D, dx, dg, db, ws(det.det_layernorm_bwd_ws_bytes(rows, D)))
            _sync()
            same(host(dx, np.uint16), odx, "dx")
            for b, w, want, what in zip(buf, which, (odg, odb), ("dgamma", "dbeta")):
                if w:
                    same(host(b[off:off + D]), want, what)
                assert (b[:off] == 7).all() and (b[off + D * w:] == 7).all()


@pytest.mark.parametrize("rows,D", [(113001, 8), (15001, 200), (5001, 1024), (2399, 2056)])
def test_layernorm_many_rows_binary32(det, rows, D):
    x, dy, g = _rows((rows, D), 23, False), _rows((rows, D), 26, False), _rows(D, 24, False, 1.0, 0.1)
    mean, rstd = synth.normal_f32(rows, 0.1, seed=27, tid=1), np.abs(synth.normal_f32(rows, 1.0, seed=27, tid=2)) + F(0.5)
    dx, dg, db = empty((rows, D), F), empty((D,), F), empty((D,), F)
    det.det_layernorm_bwd(det.DET_F32, dev(dy), dev(x), dev(g), dev(mean), dev(rstd), rows, D, dx, dg, db, ws(det.det_layernorm_bwd_ws_bytes(rows, D)))
    _sync()
    odx, odg, odb = oracle.layernorm_bwd(dy, x, g, mean, rstd, bf=False)
    same(host(dx), odx, "dx")
    same(host(dg), odg, "dgamma")
    same(host(db), odb, "dbeta")


@pytest.mark.parametrize("rows,D", [(1, 8), (37, 200), (264, 512), (65, 1000), (130, 2048), (11, 4096), (5, 8184), (40, 333)])
def test_layernorm_with_the_residual_stream(det, rows, D):
    """The sum in front of the norm, the codes of the next linear, the checkpoint beside it; the gradient from x and from its checkpoint,
    added to the one that bypasses the norm, in place too."""
    a, b = _rows((rows, D), 43, True), _rows((rows, D), 44, True)
    g, s = _rows(D, 45, True, 1.0, 0.1), _rows(D, 46, True, 0.0, 0.2)
    dy, res = _rows((rows, D), 47, True), _rows((rows, D), 48, True)
    sq = np.array([0.021], F)
    osum = oracle.residual_add(a, b)
    oy, om, ors = oracle.layernorm_fwd(osum, g, s, 1e-6, bf=True)
    oq, oe = oracle.act8_pack(osum)
    ng = (D + 31) // 32
    full = D % 8 == 0
    total, y, mean, rstd = empty((rows, D), np.uint16), empty((rows, D), np.uint16), empty((rows,), F), empty((rows,), F)
    qy, q8, e8 = empty((rows, D), np.int8), empty((rows, D), np.int8), empty((rows, ng), np.uint8)
    det.det_residual_layernorm_fwd(dev(a), dev(b), dev(g), dev(s), rows, D, 1e-6, total, y, mean, rstd, *((dev(sq), qy, q8, e8) if full else ()))
    _sync()
    same(host(total, np.uint16), osum, "sum")
    same(host(y, np.uint16), oy, "y")
    same(host(mean), om, "mean")
    same(host(rstd), ors, "rstd")
    if full:
        same(host(qy), oracle.lsq_quantize(oy, sq, False), "codes of y")
        same(host(q8), oq, "checkpoint codes")
        same(host(e8), oe, "checkpoint steps")
        y2 = empty((rows, D), np.uint16)
        det.det_residual_layernorm_fwd(total, None, dev(g), dev(s), rows, D, 1e-6, None, y2, mean, rstd)     # without a second summand
        _sync()
        same(host(y2, np.uint16), oy, "y of the sum")
    w = ws(det.det_layernorm_bwd_ws_bytes(rows, D))
    dx, dg, db = dev(res), empty((D,), F), empty((D,), F)
    det.det_layernorm_bwd_residual(dev(dy), total, dev(g), mean, rstd, rows, D, dx, dx, dg, db, w)
    _sync()
    odx, odg, odb = oracle.layernorm_bwd(dy, osum, g, om, ors, res, bf=True)
    same(host(dx, np.uint16), odx, "dx")
    same(host(dg), odg, "dgamma")
    same(host(db), odb, "dbeta")
    kept = oracle.act8_unpack(oq, oe)
    for other in (res, None):
        dx = empty((rows, D), np.uint16)
        det.det_layernorm_bwd_act8(dev(dy), dev(oq), dev(oe), dev(g), mean, rstd, rows, D, dev(other) if other is not None else None, dx, dg, db, w)
        _sync()
        odx, odg, odb = oracle.layernorm_bwd(dy, kept, g, om, ors, other, bf=True)
        same(host(dx, np.uint16), odx, "dx from the checkpoint")
        same(host(dg), odg, "dgamma from the checkpoint")
        same(host(db), odb, "dbeta")


def test_layernorm_not_finite(det):
    """An infinity or a NaN stays in its row (and in its column's gradients)."""
    rows, D = 9, 264
    x, g, b = _rows((rows, D), 51, True), _rows(D, 52, True, 1.0), _rows(D, 53, True)
    x[2, 5], x[4, 263], x[5] = 0x7FC0, 0x7F80, 0x0000
    dy = _rows((rows, D), 54, True)
    dy[7, 9] = 0xFF80
    y, mean, rstd = empty((rows, D), np.uint16), empty((rows,), F), empty((rows,), F)
    det.det_layernorm_fwd(1, dev(x), dev(g), dev(b), rows, D, 1e-6, y, mean, rstd)
    dx, dg, db = empty((rows, D), np.uint16), empty((D,), F), empty((D,), F)
    det.det_layernorm_bwd(1, dev(dy), dev(x), dev(g), mean, rstd, rows, D, dx, dg, db, ws(det.det_layernorm_bwd_ws_bytes(rows, D)))
    _sync()
    oy, om, ors = oracle.layernorm_fwd(x, g, b, 1e-6, bf=True)
    odx, odg, odb = oracle.layernorm_bwd(dy, x, g, om, ors, bf=True)
    for got, want in ((host(y, np.uint16), oy), (host(mean), om), (host(rstd), ors), (host(dx, np.uint16), odx), (host(dg), odg), (host(db), odb)):
        same(got, want, "not finite")
    assert np.isfinite(synth.from_bf16(oy)[[0, 1, 3, 5, 6, 7, 8]]).all()


def test_layernorm_one_row_flushes(det):
    """The gradient of the shift of one row is that row, subnormals flushed."""
    dy = synth.to_bf16(np.array([[1e-39, -1e-39, 1.0, -0.0, 2.0 ** -126, 3.0, 0.0, 5.0]], F))
    x, one, zero = _rows((1, 8), 55, True), dev(np.ones(1, F)), dev(np.zeros(1, F))
    dx, db = empty((1, 8), np.uint16), empty((8,), F)
    det.det_layernorm_bwd(1, dev(dy), dev(x), None, zero, one, 1, 8, dx, None, db, ws(det.det_layernorm_bwd_ws_bytes(1, 8)))
    _sync()
    same(host(db), oracle.layernorm_bwd(dy, x, None, np.zeros(1, F), np.ones(1, F), bf=True)[2], "dbeta")


# ---- 8-bit checkpoints --------------------------------------------------------------------------------------
@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("rows,D,pad", [(1, 1, 0), (3, 31, 0), (7, 32, 0), (65, 40, 8), (9, 33, 3), (100, 264, 0), (33, 1000, 24), (501, 777, 0),
                                        (40, 2048, 2), (11, 4096, 0), (2, 100000, 0)])
def test_act8(det, bf, rows, D, pad):
    dt = np.uint16 if bf else F
    x = synth.normal_f32((rows, D + pad), 1.0, seed=61, tid=1) * np.exp(synth.normal_f32((rows, 1), 20.0, seed=62, tid=1)).astype(F)
    x[0, 0] = 1e-41
    x[rows // 2, D // 2] = np.nan
    x[rows - 1, D - 1] = -np.inf
    x = synth.to_bf16(x) if bf else x
    ng = (D + 31) // 32
    assert det.det_act8_exp_bytes(rows, D) == rows * ng
    q, e = empty((rows, D), np.int8), empty((rows, ng), np.uint8)
    det.det_act8_pack(int(bf), dev(x), D + pad, rows, D, q, e)
    y = dev(np.zeros_like(x))
    det.det_act8_unpack(int(bf), q, e, rows, D, y, D + pad)
    _sync()
    oq, oe = oracle.act8_pack(np.ascontiguousarray(x[:, :D]), bf)
    same(host(e), oe, "steps")
    same(host(q), oq, "codes")
    got = host(y, dt)
    same(np.ascontiguousarray(got[:, :D]), oracle.act8_unpack(oq, oe, bf), "values")
    assert not np.ascontiguousarray(got[:, D:]).view(np.uint8).any()          # what lies between the rows is left alone


def test_act8_at_odd_addresses(det):
    import torch
    rows, D = 21, 64
    x = _rows((rows, D), 63, True)
    room = torch.zeros(rows * D + 8, dtype=torch.int16, device="cuda")
    q8 = torch.zeros(rows * D + 8, dtype=torch.int8, device="cuda")
    oq, oe = oracle.act8_pack(x)
    for off, qoff in ((1, 0), (0, 1), (3, 5)):
        room[off:off + rows * D].copy_(dev(x).view(-1))
        e = empty((rows, 2), np.uint8)
        det.det_act8_pack(1, room.data_ptr() + 2 * off, D, rows, D, q8.data_ptr() + qoff, e)
        out = torch.zeros_like(room)
        det.det_act8_unpack(1, q8.data_ptr() + qoff, e, rows, D, out.data_ptr() + 2 * off, D)
        _sync()
        same(host(q8)[qoff:qoff + rows * D].reshape(rows, D), oq, "codes")
        same(host(e), oe, "steps")
        got = host(out, np.uint16)
        same(got[off:off + rows * D].reshape(rows, D), oracle.act8_unpack(oq, oe), "values")
        assert not got[:off].any() and not got[off + rows * D:].any()


@pytest.mark.parametrize("rows,Fd", [(1, 32), (37, 1024), (5, 96), (129, 512), (1000, 64), (3, 8192), (2000, 1056), (1300, 2112)])
def test_swiglu_from_checkpoint(det, rows, Fd):
    gu = synth.normal_bf16((rows, 2 * Fd), 2.0, seed=71, tid=1)
    gu[0, :4] = synth.to_bf16(np.array([-200.0, 200.0, 90.0, -90.0], F))
    dh = synth.normal_bf16((rows, Fd), 1.0, seed=71, tid=2)
    sq = np.array([0.021], F)
    h, q, e = empty((rows, Fd), np.uint16), empty((rows, 2 * Fd), np.int8), empty((rows, 2 * Fd // 32), np.uint8)
    qh = empty((rows, Fd), np.int8)
    det.det_swiglu_fwd_act8(dev(gu), rows, Fd, h, q, e, dev(sq), qh)
    again, qa, dgu = empty((rows, Fd), np.uint16), empty((rows, Fd), np.int8), empty((rows, 2 * Fd), np.uint16)
    det.det_swiglu_act8(q, e, rows, Fd, again, dev(sq), qa)
    det.det_swiglu_bwd_act8(dev(dh), q, e, rows, Fd, dgu)
    _sync()
    oq, oe = oracle.act8_pack(gu)
    kept = oracle.act8_unpack(oq, oe)
    same(host(q), oq, "codes")
    same(host(e), oe, "steps")
    same(host(h, np.uint16), oracle.swiglu_fwd(gu), "h")
    same(host(qh), oracle.lsq_quantize(oracle.swiglu_fwd(gu), sq, False), "codes of h")
    same(host(again, np.uint16), oracle.swiglu_fwd(kept), "h again")
    same(host(qa), oracle.lsq_quantize(oracle.swiglu_fwd(kept), sq, False), "codes of h again")
    same(host(dgu, np.uint16), oracle.swiglu_bwd(dh, kept), "dgu")


def test_swiglu_from_checkpoint_every_gate(det):
    """Every value a code and a step can stand for as the gate (infinities and NaNs among them)."""
    rows, Fd = 255, 256
    e = np.arange(1, 256, dtype=np.uint8)[:, None].repeat(2 * Fd // 32, 1).copy()
    e[249:254] = 127                                                        # fields that no group has
    e[:, Fd // 32:] = 122
    q = np.concatenate([np.arange(-128, 128).astype(np.int8)[None].repeat(rows, 0), synth.randint((rows, Fd), 255, seed=72, tid=1).astype(np.int8)], 1)
    q[q == -128] = -127
    dh = synth.normal_bf16((rows, Fd), 1.0, seed=73, tid=2)
    h, dgu = empty((rows, Fd), np.uint16), empty((rows, 2 * Fd), np.uint16)
    det.det_swiglu_act8(dev(q), dev(e), rows, Fd, h)
    det.det_swiglu_bwd_act8(dev(dh), dev(q), dev(e), rows, Fd, dgu)
    _sync()
    kept = oracle.act8_unpack(q, e)
    same(host(h, np.uint16), oracle.swiglu_fwd(kept), "h")
    same(host(dgu, np.uint16), oracle.swiglu_bwd(dh, kept), "dgu")


def test_swiglu_by_table_every_gate(det):
    """Rows enough for the table: every bf16 as the gate of the forward pass, every code and step as that of the others."""
    rows, Fd = 1300, 2112
    g = np.arange(rows * Fd, dtype=np.uint32).astype(np.uint16).reshape(rows, Fd)
    up, dh = synth.normal_bf16((rows, Fd), 1.0, seed=74, tid=1), synth.normal_bf16((rows, Fd), 1.0, seed=74, tid=2)
    gu = np.concatenate([g, up], 1)
    h, q, e = empty((rows, Fd), np.uint16), empty((rows, 2 * Fd), np.int8), empty((rows, 2 * Fd // 32), np.uint8)
    det.det_swiglu_fwd_act8(dev(gu), rows, Fd, h, q, e)
    _sync()
    oq, oe = oracle.act8_pack(gu)
    same(host(q), oq, "codes")
    same(host(e), oe, "steps")
    same(host(h, np.uint16), oracle.swiglu_fwd(gu), "h")
    n = Fd // 32
    codes = (np.arange(rows * Fd) % 255 - 127).astype(np.int8).reshape(rows, Fd)
    steps = (np.arange(rows * n) % 250).astype(np.uint8).reshape(rows, n)
    steps[steps == 0] = 255
    q8, e8 = np.concatenate([codes, oq[:, Fd:]], 1), np.concatenate([steps, oe[:, n:]], 1)
    again, dgu = empty((rows, Fd), np.uint16), empty((rows, 2 * Fd), np.uint16)
    det.det_swiglu_act8(dev(q8), dev(e8), rows, Fd, again)
    det.det_swiglu_bwd_act8(dev(dh), dev(q8), dev(e8), rows, Fd, dgu)
    _sync()
    kept = oracle.act8_unpack(q8, e8)
    same(host(again, np.uint16), oracle.swiglu_fwd(kept), "h again")
    same(host(dgu, np.uint16), oracle.swiglu_bwd(dh, kept), "dgu")


# ---- gated linear recurrence ----------------------------------------------------------------------------------
def _gv(B, S, D, seed, gate=2.0):
    g = synth.normal_f32((B * S, D), 2.0, mean=gate, seed=seed, tid=1)
    gv = synth.to_bf16(np.concatenate([g, synth.normal_f32((B * S, D), 1.0, seed=seed, tid=2)], 1))
    ends = synth.to_bf16(np.array([200.0, -200.0, 88.0, -87.5, 127.5, -128.0, 1e-9, -1e-30, 0.0, -0.0, 2.0 ** -26, 2.0 ** -27], F))
    gv[0, :min(ends.size, D)] = ends[:D]
    return gv


def _flags(B, S, every, seed):
    return (synth.randint((B, S), every, seed=seed, tid=9) == 0).astype(np.uint8) if every else None


def _linrec(det, gv, dy, B, S, fl, h0, dhT, pad=0):
    """Both passes on the GPU, operands inside wider rows where pad > 0."""
    D = gv.shape[1] // 2
    T, ld = B * S, 2 * D + pad
    wide = np.zeros((T, ld), np.uint16)
    wide[:, :2 * D] = gv
    dgv_in, ddy = dev(wide), dev(dy)
    opt = lambda a: dev(a) if a is not None else None
    y, hT, dh0 = dev(np.zeros((T, D + pad), np.uint16)), empty((B, D), F), empty((B, D), F)
    n = det.det_linrec_state_floats(B, S, D)
    assert n == B * ((S + 7) // 8) * D
    states, out = empty((n,), F), dev(np.zeros((T, ld), np.uint16))
    p = dgv_in.data_ptr()
    dfl, dh, ddhT = opt(fl), opt(h0), opt(dhT)
    det.det_linrec_fwd(p, p + 2 * D, ld, B, S, D, y, D + pad, flags=dfl, h0=dh, hT=hT, states=states)
    o = out.data_ptr()
    det.det_linrec_bwd(ddy, D, p, p + 2 * D, ld, B, S, D, states, o, o + 2 * D, ld, flags=dfl, dhT=ddhT, dh0=dh0)
    _sync()
    gy, gd = host(y, np.uint16), host(out, np.uint16)
    assert not gy[:, D:].any() and not gd[:, 2 * D:].any()
    c = np.ascontiguousarray
    return c(gy[:, :D]), host(hT), host(states).reshape(B, -1, D), c(gd[:, :2 * D]), host(dh0)


def _linrec_check(det, B, S, D, every=0, ends=True, pad=0, gv=None, dy=None, fl=None):
    gv = _gv(B, S, D, 81) if gv is None else gv
    fl = _flags(B, S, every, 82) if fl is None else fl
    h0 = synth.normal_f32((B, D), 1.0, seed=83, tid=1) if ends else None
    dhT = synth.normal_f32((B, D), 1.0, seed=83, tid=2) if ends else None
    dy = synth.normal_bf16((B * S, D), 1.0, seed=84, tid=1) if dy is None else dy
    got = _linrec(det, gv, dy, B, S, fl, h0, dhT, pad)
    oy, ohT, ost = oracle.linrec_fwd(gv, B, S, fl, h0)
    odgv, odh0 = oracle.linrec_bwd(dy, gv, ost, B, S, fl, dhT)
    for g, w, what in zip(got, (oy, ohT, ost, odgv, odh0), ("y", "hT", "states", "dgv", "dh0")):
        same(g, w, what)
    return got


@pytest.mark.parametrize("B,S,D,every,ends,pad", [
    (1, 1, 2, 0, True, 0), (3, 1, 64, 0, False, 0), (2, 7, 66, 0, True, 4), (1, 8, 128, 3, True, 0), (1, 9, 30, 0, False, 2), (2, 63, 130, 5, True, 0),
    (1, 64, 64, 0, True, 0), (3, 65, 34, 0, True, 0), (1, 128, 256, 0, True, 0), (2, 129, 70, 1, True, 2), (1, 500, 100, 40, True, 0),
    (2, 513, 64, 0, True, 0), (1, 1000, 200, 0, False, 0), (1, 4096, 64, 100, True, 0), (4, 333, 512, 0, True, 0), (1, 5000, 30, 0, True, 6), (2, 1025, 4, 0, True, 0), (1, 1024, 2, 0, True, 0), (1, 33000, 6, 300, True, 0), (2, 31, 18, 0, True, 0),
    (1, 96, 32, 0, True, 0), (3, 127, 16, 4, True, 0), (1, 2177, 512, 0, True, 0), (1, 700, 1500, 0, True, 0),
    (40, 300, 128, 0, True, 0), (130, 260, 64, 9, True, 0), (1, 20000, 16, 0, True, 0), (500, 70, 64, 0, False, 0),
    (400, 260, 32, 9, True, 0), (300, 140, 34, 5, True, 2), (310, 136, 40, 0, True, 0)])
def test_linrec(det, B, S, D, every, ends, pad):
    """Lengths around chunks, blocks and spans, every number of CTAs in a cluster, either number of warps along a sequence, cuts, strides."""
    _linrec_check(det, B, S, D, every, ends, pad)


def test_linrec_every_gate(det):
    """All 65536 bit patterns of a gate, by table and by formula."""
    g = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    for S, D in ((4096, 16), (16, 4096)):
        v = synth.normal_bf16((S, D), 1.0, seed=91, tid=1)
        gv = np.concatenate([g.reshape(S, D), v], 1)
        fl = np.ones((1, S), np.uint8)                                   # every row on its own, so that a NaN stays where it is
        _linrec_check(det, 1, S, D, gv=gv, fl=fl)


def test_linrec_cut_keeps_a_nan_on_its_side(det):
    S, D = 1000, 64
    gv, dy = _gv(1, S, D, 41), synth.normal_bf16((S, D), 1.0, seed=42, tid=1)
    fl = np.zeros((1, S), np.uint8)
    fl[0, [50, 131, 132, 640]] = 1
    clean = _linrec_check(det, 1, S, D, gv=gv, dy=dy, fl=fl)
    bad, bdy = gv.copy(), dy.copy()
    bad[70, 0] = bad[90, D + 1] = bad[700, 5] = 0x7FC0
    bad[60, D + 2] = 0x7F80
    bdy[100, 3] = bdy[999, 7] = 0x7FC0
    got = _linrec_check(det, 1, S, D, gv=bad, dy=bdy, fl=fl)
    out = np.r_[0:50, 131:640]
    assert np.array_equal(got[0][out], clean[0][out]) and np.array_equal(got[3][out], clean[3][out]) and np.array_equal(got[4], clean[4])


def test_linrec_one_row_at_a_time(det):
    """The state handed from call to call in place, a row each."""
    B, S, D = 2, 5, 66
    gv = _gv(B, S, D, 95)
    h = dev(np.zeros((B, D), F))
    want = np.zeros((B, D), F)
    x = dev(gv.reshape(B, S, 2 * D).transpose(1, 0, 2))
    for t in range(S):
        y = empty((B, D), np.uint16)
        p = x[t].data_ptr()
        det.det_linrec_fwd(p, p + 2 * D, 2 * D, B, 1, D, y, D, h0=h, hT=h)
        _sync()
        oy, want, _ = oracle.linrec_fwd(np.ascontiguousarray(gv.reshape(B, S, 2 * D)[:, t]), B, 1, h0=want)
        same(host(y, np.uint16), oy, "y")
        same(host(h), want, "state")


def test_linrec_state_in_place_over_a_long_sequence(det):
    S, D = 1500, 70
    gv = _gv(1, S, D, 99)
    h0, dhT = synth.normal_f32((1, D), 1.0, seed=83, tid=1), synth.normal_f32((1, D), 1.0, seed=83, tid=2)
    dy = synth.normal_bf16((S, D), 1.0, seed=84, tid=1)
    x, h, c = dev(gv), dev(h0), dev(dhT)
    y, st, out = empty((S, D), np.uint16), empty((det.det_linrec_state_floats(1, S, D),), F), empty((S, 2 * D), np.uint16)
    p, o = x.data_ptr(), out.data_ptr()
    det.det_linrec_fwd(p, p + 2 * D, 2 * D, 1, S, D, y, D, h0=h, hT=h, states=st)
    det.det_linrec_bwd(dev(dy), D, p, p + 2 * D, 2 * D, 1, S, D, st, o, o + 2 * D, 2 * D, dhT=c, dh0=c)
    _sync()
    oy, ohT, ost = oracle.linrec_fwd(gv, 1, S, None, h0)
    odgv, odh0 = oracle.linrec_bwd(dy, gv, ost, 1, S, None, dhT)
    same(host(h), ohT, "hT")
    same(host(out, np.uint16), odgv, "dgv")
    same(host(c), odh0, "dh0")


def test_linrec_rows_far_apart(det):
    """Offsets of rows that pass 2^32 bytes."""
    import torch
    S, D, ld = 70, 64, 1 << 25
    gv = _gv(1, S, D, 96)
    room = torch.empty(S * ld, dtype=torch.int16, device="cuda")
    room.view(S, ld)[:, :2 * D].copy_(dev(gv))
    y, hT = empty((S, D), np.uint16), empty((1, D), F)
    p = room.data_ptr()
    det.det_linrec_fwd(p, p + 2 * D, ld, 1, S, D, y, D, hT=hT)
    _sync()
    oy, ohT, _ = oracle.linrec_fwd(gv, 1, S)
    same(host(y, np.uint16), oy, "y")
    same(host(hT), ohT, "hT")


def test_linrec_results_do_not_depend_on_how_the_work_is_split(det):
    """A sequence among many (a CTA each) and alone (a cluster): the same bits."""
    S, D = 400, 64
    gv, dy = _gv(1, S, D, 97), synth.normal_bf16((S, D), 1.0, seed=98, tid=1)
    one = _linrec(det, gv, dy, 1, S, None, None, None)
    many = _linrec(det, np.tile(gv, (600, 1)), np.tile(dy, (600, 1)), 600, S, None, None, None)
    assert np.array_equal(one[0], many[0][-S:]) and np.array_equal(one[3], many[3][:S]) and np.array_equal(one[1][0], many[1][77])


# ---- how they are called -------------------------------------------------------------------------------------------
def test_nothing_to_do(det):
    """No rows: the tensors stay as they are, gradients of the parameters are zero, the state passes through."""
    x, s = dev(np.zeros((1, 8), np.uint16)), dev(np.zeros(8, F))
    dg, db = dev(np.ones(8, F)), dev(np.ones(8, F))
    det.det_layernorm_fwd(1, x, x, x, 0, 8, 1e-6, x, s, s)
    det.det_layernorm_bwd(1, x, x, x, s, s, 0, 8, x, dg, db, None)
    q = dev(np.zeros(64, np.int8))
    e = dev(np.zeros(8, np.uint8))
    det.det_act8_pack(1, x, 8, 0, 8, q, e)
    det.det_act8_unpack(1, q, e, 0, 8, x, 8)
    h0, hT, dh0 = dev(synth.normal_f32((2, 4), 1.0, seed=1, tid=1)), empty((2, 4), F), empty((2, 4), F)
    det.det_linrec_fwd(x, x, 8, 2, 0, 4, x, 4, h0=h0, hT=hT)
    det.det_linrec_bwd(x, 4, x, x, 8, 2, 0, 4, None, x, x, 8, dhT=None, dh0=dh0)
    _sync()
    assert not host(dg).any() and not host(db).any() and not host(dh0).any()
    assert_same_bits(host(hT), host(h0), "state")


def _chain(det, seed):
    """Norm with the residual stream, checkpoint and recurrence forward, recurrence and norm backward from the checkpoint, as a block runs them."""
    S, D = 700, 264
    a, b, g, s = _rows((S, D), seed, True), _rows((S, D), seed + 1, True), _rows(D, seed + 2, True, 1.0, 0.1), _rows(D, seed + 3, True, 0.0, 0.1)
    gate, dy, res = _rows((S, D), seed + 4, True, 2.0, 2.0), _rows((S, D), seed + 5, True), _rows((S, D), seed + 6, True)
    osum = oracle.residual_add(a, b)
    on, om, ors = oracle.layernorm_fwd(osum, g, s, 1e-6, bf=True)
    oq, oe = oracle.act8_pack(osum)
    ogv = np.concatenate([gate, on], 1)                        # the normalised stream is the value
    oy, ohT, ost = oracle.linrec_fwd(ogv, 1, S)
    odgv, odh0 = oracle.linrec_bwd(dy, ogv, ost, 1, S)
    odx, odg, odb = oracle.layernorm_bwd(np.ascontiguousarray(odgv[:, D:]), oracle.act8_unpack(oq, oe), g, om, ors, res, bf=True)
    t = dict(a=dev(a), b=dev(b), g=dev(g), s=dev(s), gate=dev(gate), dy=dev(dy), res=dev(res))
    e = dict(sum=empty((S, D), np.uint16), n=empty((S, D), np.uint16), mean=empty((S,), F), rstd=empty((S,), F), q=empty((S, D), np.int8),
             e=empty(oe.shape, np.uint8), y=empty((S, D), np.uint16), hT=empty((1, D), F), st=empty(ost.shape, F), dg=empty((S, D), np.uint16),
             dv=empty((S, D), np.uint16), dh0=empty((1, D), F), dx=empty((S, D), np.uint16), dgamma=empty((D,), F), dbeta=empty((D,), F))
    w = ws(det.det_layernorm_bwd_ws_bytes(S, D))
    want = dict(sum=osum, n=on, mean=om, rstd=ors, q=oq, e=oe, y=oy, hT=ohT, st=ost, dg=np.ascontiguousarray(odgv[:, :D]),
                dv=np.ascontiguousarray(odgv[:, D:]), dh0=odh0, dx=odx, dgamma=odg, dbeta=odb)

    def run():
        det.det_residual_layernorm_fwd(t["a"], t["b"], t["g"], t["s"], S, D, 1e-6, e["sum"], e["n"], e["mean"], e["rstd"], q8=e["q"], e8=e["e"])
        det.det_linrec_fwd(t["gate"], e["n"], D, 1, S, D, e["y"], D, hT=e["hT"], states=e["st"])
        det.det_linrec_bwd(t["dy"], D, t["gate"], e["n"], D, 1, S, D, e["st"], e["dg"], e["dv"], D, dh0=e["dh0"])
        det.det_layernorm_bwd_act8(e["dv"], e["q"], e["e"], t["g"], e["mean"], e["rstd"], S, D, t["res"], e["dx"], e["dgamma"], e["dbeta"], w)

    def check(out=None):
        for k, x in want.items():
            same(host((out or e)[k], x.dtype), x, k)
    return t, e, run, check


def test_a_run_of_them_on_two_streams_and_in_a_captured_graph(det):
    """The operators one after the other as a block uses them: on two streams at once with buffers of their own; captured, and replayed twice on
    inputs that changed after the capture."""
    import torch
    ta, ea, ra, ca = _chain(det, 101)
    tb, eb, rb, cb = _chain(det, 201)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    _sync()
    for _ in range(5):
        with torch.cuda.stream(s1):
            ra()
        with torch.cuda.stream(s2):
            rb()
    _sync()
    ca()
    cb()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ra()
    for k in ta:
        ta[k].copy_(tb[k])
    for _ in range(2):
        for v in ea.values():
            v.zero_()
        graph.replay()
        _sync()
        cb(ea)
