"""What is not finite stays in the recurrence's state until a cut, on the GPU as in the oracle, in every form of the kernels."""
import numpy as np
import pytest

import synth
from test_gpu_blocks import _linrec_check, det  # noqa: F401  (det is the fixture)
from test_oracle_linrec_not_finite import finite, inputs

pytestmark = pytest.mark.gpu


# one chunk; a lone CTA; clusters of 2 to 16, of several rounds, with odd lengths and widths; lone CTAs of several rounds and strips
@pytest.mark.parametrize("B,S,D", [(2, 7, 6), (1, 40, 64), (1, 200, 70), (1, 512, 32), (1, 1900, 64), (1, 5000, 34), (600, 300, 32)])
@pytest.mark.parametrize("gate", [-14.0, -100.0])
@pytest.mark.parametrize("flags", [False, True])
def test_it_stays_until_a_cut(det, B, S, D, gate, flags):  # noqa: F811
    gv, dy = (np.tile(a, (B, 1)) for a in inputs(S, D, gate))
    at, last = min(20, S // 2), max(S - 30, S // 2)
    gv[at, D + 1] = 0x7FC0
    gv[at + 1, D + 2] = 0x7F80
    dy[last, 3] = 0x7FC0
    fl = None
    if flags:
        fl = np.zeros((B, S), np.uint8)
        fl[:, S // 2 + 1] = 1
    y, hT, _, dgv, dh0 = _linrec_check(det, B, S, D, gv=gv, dy=dy, fl=fl)
    end = S // 2 + 1 if flags else S
    ends = {1: end, 2: end if at + 1 < end else S}       # of 7 rows the infinity is the cut row's own value, which no cut holds back
    ok = finite(y)[:S]
    for c in range(D):
        assert ok[:, c].all() if c not in ends else not ok[at + c - 1:ends[c], c].any() and ok[:at + c - 1, c].all() and ok[ends[c]:, c].all()
    assert finite(hT)[0].tolist() == [ends.get(c, 0) < S for c in range(D)]
    begin = S // 2 + 1 if flags and last > S // 2 else 0
    assert not finite(dgv)[begin:last + 1, D + 3].any() and finite(dgv)[:begin, D + 3].all()
    assert bool(finite(dh0)[0, 3]) == (begin > 0) and finite(hT)[1:].all()


def test_it_comes_in_with_the_state(det):  # noqa: F811
    import oracle
    from gpu_util import dev, empty, host
    from test_gpu_blocks import _sync, same
    F = np.float32
    for S in (5, 100, 700):
        D = 34
        gv, _ = inputs(S, D, -14.0)
        h0 = np.zeros((1, D), F)
        h0[0, 1], h0[0, 33] = np.nan, -np.inf
        y, hT, x = empty((S, D), np.uint16), empty((1, D), F), dev(gv)
        p = x.data_ptr()
        det.det_linrec_fwd(p, p + 2 * D, 2 * D, 1, S, D, y, D, h0=dev(h0), hT=hT)
        _sync()
        oy, ohT, _ = oracle.linrec_fwd(gv, 1, S, h0=h0)
        same(host(y, np.uint16), oy, "y")
        same(host(hT), ohT, "hT")
        assert not finite(host(hT))[0, [1, 33]].any() and not finite(host(y, np.uint16))[:, [1, 33]].any()
