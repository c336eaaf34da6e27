"""What SwiGLU refuses on the host (addresses are never followed, so this runs without a GPU)."""
import paper_2609_17380_b200 as det

ARG, SHAPE, ALIGN = -1, -2, -3
A = 4096


def test_swiglu_forward_refusals():
    call = lambda gu=A, rows=4, F=64, h=A: det.load().det_swiglu_fwd(gu, rows, F, h, None)
    for bad in (dict(gu=None), dict(h=None), dict(rows=-1), dict(F=0), dict(F=-8)):
        assert call(**bad) == ARG, bad
    for bad in (dict(gu=A + 2), dict(h=A + 8), dict(gu=A + 1, F=65), dict(h=A + 1, F=65)):
        assert call(**bad) == ALIGN, bad
    assert call(F=2 ** 31 - 1, rows=2 ** 31 - 1) == SHAPE
    assert call(rows=0) == 0 and call(rows=0, F=65, gu=A + 2) == 0
    lib = det.load()
    assert lib.det_swiglu_fwd_q(A, 4, 65, A, A, A, None) == SHAPE and lib.det_swiglu_bwd(A, A, 4, 65, A, None) == SHAPE
