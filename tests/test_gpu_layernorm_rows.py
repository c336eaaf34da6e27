"""Layer norm of many rows on the GPU: more than 2^30 of them, and forward passes in which every CTA walks over several pieces of rows."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import dev, empty, host, ws
from test_gpu_blocks import _rows, _sync, same

pytestmark = pytest.mark.gpu
F = np.float32


@pytest.fixture(scope="module")
def det():
    import paper_2609_17380_b200 as d
    d.load()
    return d


def _periodic(base, rows):
    """`rows` rows on the GPU, those of base over and over."""
    import torch
    b = dev(base)
    x = torch.empty((rows,) + b.shape[1:], dtype=b.dtype, device="cuda")
    n = rows // b.shape[0]
    x[:n * b.shape[0]].view((n,) + b.shape).copy_(b.expand((n,) + b.shape))
    x[n * b.shape[0]:] = b[:rows - n * b.shape[0]]
    return x


def _is_periodic(x, base):
    import torch
    b = dev(base)
    P, bits = b.shape[0], {1: torch.int8, 2: torch.int16, 4: torch.int32}[b.element_size()]
    x, b = x.view(bits), b.view(bits)
    for lo in range(0, x.shape[0], P * 8192):
        part = x[lo:lo + P * 8192]
        n = part.shape[0] // P
        if not bool((part[:n * P].view((n,) + b.shape) == b).all()) or not torch.equal(part[n * P:], b[:part.shape[0] - n * P]):
            return False
    return True


@pytest.mark.parametrize("bf,D", [(True, 2), (False, 8)])
def test_more_rows_than_two_to_the_thirty(det, bf, D):
    """The rows repeat, so every result is one of those of the first 4099."""
    import torch
    rows, P, dt = 1100000001, 4099, np.uint16 if bf else F
    if torch.cuda.mem_get_info()[0] < rows * (2 * D * np.dtype(dt).itemsize + 8) + (4 << 30):
        pytest.skip("not enough memory on the GPU")
    base, g, b = _rows((P, D), 3, bf, 0.5), _rows(D, 4, bf, 1.0, 0.1), _rows(D, 5, bf, 0.0, 0.3)
    x = _periodic(base, rows)
    y, mean, rstd = torch.zeros_like(x), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    det.det_layernorm_fwd(int(bf), x, dev(g), dev(b), rows, D, 1e-6, y, mean, rstd)
    _sync()
    oy, om, ors = oracle.layernorm_fwd(base, g, b, 1e-6, bf=bf)
    assert _is_periodic(y, oy) and _is_periodic(mean, om) and _is_periodic(rstd, ors)


def test_backward_of_more_rows_than_two_to_the_thirty(det):
    import torch
    rows, P, D = 1100000001, 4099, 2
    if torch.cuda.mem_get_info()[0] < rows * (6 * D + 8) + (4 << 30):
        pytest.skip("not enough memory on the GPU")
    base, g = _rows((P, D), 3, True, 0.5), _rows(D, 4, True, 1.0, 0.1)
    mean, rstd = synth.normal_f32(P, 0.1, seed=17, tid=1), np.abs(synth.normal_f32(P, 1.0, seed=17, tid=2)) + F(0.5)
    dy = np.full((P, D), 0x3F80, np.uint16)
    x = _periodic(base, rows)
    gy, gm, gr = _periodic(dy, rows), _periodic(mean, rows), _periodic(rstd, rows)
    dx, dg, db = torch.zeros_like(x), empty((D,), F), empty((D,), F)
    det.det_layernorm_bwd(det.DET_BF16, gy, x, dev(g), gm, gr, rows, D, dx, dg, db, ws(det.det_layernorm_bwd_ws_bytes(rows, D)))
    _sync()
    assert _is_periodic(dx, oracle.layernorm_bwd(dy, base, g, mean, rstd, bf=True)[0])
    # the tree over ones: perfect subtrees are exact, those on the right are joined from the smallest up
    total = None
    for k in range(31):
        if rows >> k & 1:
            total = F(2.0 ** k) if total is None else F(2.0 ** k) + total
    assert host(db).tolist() == [total, total]
    assert np.isfinite(host(dg)).all()


# rows for more passes of a CTA than are on their way ahead, the last one ragged, for every number of warps a row
WALK = [(60001, 256), (60003, 40), (29001, 512), (15001, 1000), (8191, 2048), (3001, 4096), (1501, 8192), (1499, 8184)]


def _walks(det, rows, D):
    passes, most, _, _ = det.det_test_layernorm_walk(det.DET_BF16, rows, D, det.det_device_sm_count())
    return passes > 4 and most >= 5


@pytest.mark.parametrize("rows,D", WALK)
def test_forward_walk(det, rows, D):
    assert _walks(det, rows, D)
    x, g, b = _rows((rows, D), 3, True, 0.5), _rows(D, 4, True, 1.0, 0.1), _rows(D, 5, True, 0.0, 0.3)
    y, mean, rstd = dev(np.full((rows + 2, D), 0x7ABC, np.uint16)), dev(np.full(rows + 2, 7.0, F)), dev(np.full(rows + 2, 7.0, F))
    det.det_layernorm_fwd(det.DET_BF16, dev(x), dev(g), dev(b), rows, D, 1e-6, y, mean, rstd)
    _sync()
    oy, om, ors = oracle.layernorm_fwd(x, g, b, 1e-6, bf=True)
    same(host(mean)[:rows], om, "mean")
    same(host(rstd)[:rows], ors, "rstd")
    got = host(y, np.uint16)
    same(got[:rows], oy, "y")
    assert (got[rows:] == 0x7ABC).all() and (host(mean)[rows:] == 7).all() and (host(rstd)[rows:] == 7).all()      # behind the last row


@pytest.mark.parametrize("rows,D", WALK)
def test_forward_walk_with_the_residual_stream(det, rows, D):
    """The sum, the codes of the next linear and the checkpoint, with the sum and without a second summand."""
    assert _walks(det, rows, D)
    a, b = _rows((rows, D), 43, True), _rows((rows, D), 44, True)
    g, s = _rows(D, 45, True, 1.0, 0.1), _rows(D, 46, True, 0.0, 0.2)
    sq = np.array([0.021], F)
    for other in (b, None):
        osum = a if other is None else oracle.residual_add(a, other)
        oy, om, ors = oracle.layernorm_fwd(osum, g, s, 1e-6, bf=True)
        oq, oe = oracle.act8_pack(osum)
        total, y, mean, rstd = empty((rows, D), np.uint16), empty((rows, D), np.uint16), empty((rows,), F), empty((rows,), F)
        qy, q8, e8 = empty((rows, D), np.int8), empty((rows, D), np.int8), empty((rows, (D + 31) // 32), np.uint8)
        det.det_residual_layernorm_fwd(dev(a), None if other is None else dev(other), dev(g), dev(s), rows, D, 1e-6, total, y, mean, rstd, dev(sq), qy, q8, e8)
        _sync()
        if other is not None:
            same(host(total, np.uint16), osum, "sum")
        same(host(y, np.uint16), oy, "y")
        same(host(mean), om, "mean")
        same(host(rstd), ors, "rstd")
        same(host(qy), oracle.lsq_quantize(oy, sq, False), "codes of y")
        same(host(q8), oq, "checkpoint codes")
        same(host(e8), oe, "checkpoint steps")
