"""What is not finite stays in the recurrence's state until a cut, however much the gates forget (oracle)."""
import numpy as np
import pytest

import oracle
import synth

F = np.float32


def inputs(S, D, gate, seed=51):
    """Gates near `gate`: at -14 the product of eight is below 2^-126."""
    g = synth.normal_f32((S, D), 0.5, mean=gate, seed=seed, tid=1)
    gv = synth.to_bf16(np.concatenate([g, synth.normal_f32((S, D), 1.0, seed=seed, tid=2)], 1))
    return gv, synth.normal_bf16((S, D), 1.0, seed=seed, tid=3)


def finite(x):
    return np.isfinite(synth.from_bf16(x) if x.dtype == np.uint16 else x)


@pytest.mark.parametrize("bad", [0x7FC0, 0x7F80, 0xFF80])
@pytest.mark.parametrize("gate", [-14.0, -6.0, -100.0, 2.0])
@pytest.mark.parametrize("S,row", [(7, 3), (40, 20), (512, 20), (512, 127), (512, 128), (700, 300)])
def test_it_stays(S, row, gate, bad):
    D = 6
    gv, dy = inputs(S, D, gate)
    gv[row, D + 2] = bad                                 # a value
    y, hT, st = oracle.linrec_fwd(gv, 1, S)
    ok = finite(y)
    assert ok[:row].all() and not ok[row:, 2].any() and ok[:, [0, 1, 3, 4, 5]].all()
    assert finite(hT)[0].tolist() == [c != 2 for c in range(D)]
    assert not finite(st)[0, (row + 8) // 8:, 2].any() and finite(st)[0, :(row + 7) // 8 if row % 8 else row // 8 + 1].all()
    gv, dy = inputs(S, D, gate)
    dy[row, 4] = bad                                     # a gradient goes on to the first row
    _, _, st = oracle.linrec_fwd(gv, 1, S)
    dgv, dh0 = oracle.linrec_bwd(dy, gv, st, 1, S)
    ok = finite(dgv[:, D:])
    assert ok[row + 1:].all() and not ok[:row + 1, 4].any() and ok[:, [0, 1, 2, 3, 5]].all()
    assert finite(dh0)[0].tolist() == [c != 4 for c in range(D)]


def test_it_comes_in_with_the_state():
    S, D = 600, 4
    gv, dy = inputs(S, D, -14.0)
    h0, dhT = np.zeros((1, D), F), np.zeros((1, D), F)
    h0[0, 1], dhT[0, 3] = np.nan, np.inf
    y, hT, st = oracle.linrec_fwd(gv, 1, S, h0=h0)
    assert finite(y).all(0).tolist() == [True, False, True, True] and not finite(y)[:, 1].any() and not finite(hT)[0, 1]
    dgv, dh0 = oracle.linrec_bwd(dy, gv, oracle.linrec_fwd(gv, 1, S)[2], 1, S, dhT=dhT)
    assert not finite(dgv[:, D + 3]).any() and not finite(dh0)[0, 3] and finite(dgv[:, D:D + 3]).all()


def test_a_cut_ends_it():
    """A cut, behind rows that forget everything too, and its sign through products that underflow behind it."""
    S, D = 400, 4
    gv, dy = inputs(S, D, -14.0)
    gv[20, D + 1] = 0x7FC0
    dy[390, 2] = 0x7FC0
    for cut in (21, 24, 127, 128, 131, 255, 256, 300):
        fl = np.zeros((1, S), np.uint8)
        fl[0, cut] = 1
        y, hT, st = oracle.linrec_fwd(gv, 1, S, fl)
        assert not finite(y)[20:cut, 1].any() and finite(y)[cut:].all() and finite(hT).all()
        dgv, dh0 = oracle.linrec_bwd(dy, gv, st, 1, S, fl)
        assert not finite(dgv)[cut:391, D + 2].any() and finite(dgv)[:cut, D + 2].all() and finite(dh0).all()


def test_finite_results_do_not_depend_on_underflow():
    """Against a walk over the rows in 64 bits, where the products of the gates underflow in every chunk."""
    S, D = 300, 4
    gv, _ = inputs(S, D, -14.0)
    x = synth.from_bf16(gv).astype(np.float64)
    h, f = np.full(D, 3.0), 1 / (1 + np.exp(-x[:, :D]))
    y, hT, _ = oracle.linrec_fwd(gv, 1, S, h0=np.full((1, D), 3.0, F))
    for t in range(S):
        h = f[t] * h + (1 - f[t]) * x[t, D:]
        # one rounding to bf16 and a few of binary32
        assert (np.abs(synth.from_bf16(y[t]) - h) <= (2.0 ** -8 + 2.0 ** -20) * (np.abs(h) + 1e-4)).all()
    assert (np.abs(hT[0] - h) <= 2.0 ** -20 * (np.abs(h) + 1e-4)).all()
