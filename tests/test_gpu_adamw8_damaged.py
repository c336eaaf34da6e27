"""AdamW over many tensors where a second moment in 32 bits is damaged: what det_adamw_batch and the oracle make of it."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import assert_same_bits, dev, host

pytestmark = pytest.mark.gpu
F = np.float32
H = (3e-4, 0.9, 0.95, 1e-8, 0.1, 3)


def same(got, want, what):
    wide = lambda x: synth.from_bf16(x) if x.dtype == np.uint16 else x
    nan = np.isnan(wide(want))
    assert np.array_equal(np.isnan(wide(got)), nan), what
    assert_same_bits(got[~nan], want[~nan], what)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("n", [7, 700])
def test_negative_second_moments(n, bf):
    """A root of a negative number is NaN and so is the parameter, however small the number; zeros, subnormals, infinities and NaN as ever."""
    import paper_2609_17380_b200 as det
    p, g = synth.normal_f32((n,), 0.02, seed=1), synth.normal_f32((n,), 1e-3, seed=2)
    p = synth.to_bf16(p) if bf else p
    m, v = synth.normal_f32((n,), 1e-3, seed=3), synth.normal_f32((n,), 1e-3, seed=4) ** 2
    g[:6] = 0
    for i, x in enumerate((-1e-4, -1e-30, 0.0, -0.0, -1e-42, np.nan)):
        v[i] = x
    v[6], m[2] = -np.inf, 0
    if n > 500:
        v[300], v[301], v[302], m[302] = -3e38, np.inf, -1e-12, 0
        g[302] = 0
    wp, wm, wv = oracle.adamw(p, g, m, v, *H)
    # the root's argument is b2 v + (1 - b2) g^2; where that stays negative nothing finite may come out
    wide = (lambda x: synth.from_bf16(x)) if bf else (lambda x: x)
    assert np.isnan(wide(wp)[[0, 1, 5, 6]]).all() and np.isfinite(wide(wp)[[3, 4]]).all()
    a, b = [[dev(x) for x in (p, g, m, v)] for _ in range(2)]
    desc, kind = det.det_adamw_desc(*H), det.DET_BF16 if bf else det.DET_F32
    det.det_adamw8_batch([desc], [kind], [a[0]], [a[1]], [a[2]], [a[3]], [None])
    det.det_adamw_batch([desc], [kind], [b[0]], [b[1]], [b[2]], [b[3]])
    for got, what in ((a, "together"), (b, "det_adamw_batch")):
        same(host(got[0], p.dtype), wp, "p, " + what)
        same(host(got[2]), wm, "m, " + what)
        same(host(got[3]), wv, "v, " + what)
