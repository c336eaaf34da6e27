"""Blocks whose largest moment is a subnormal number or -0: scale 0 and codes 0, as the oracle has them."""
import numpy as np
import pytest

import oracle
from gpu_util import assert_same_bits, dev, empty, host

pytestmark = pytest.mark.gpu
F = np.float32
LEAST = F(2.0 ** -126)                                                # the smallest normal number


@pytest.mark.parametrize("n", [300, 1024, 1500])
def test_scales_of_subnormal_blocks(n):
    import paper_2609_17380_b200 as det
    below = np.nextafter(LEAST, F(0), dtype=F)                        # the largest subnormal
    m, v = np.zeros(n, F), np.zeros(n, F)
    m[:256], v[:256] = -F(1e-40), F(1e-44)
    m[3], v[5], v[7] = below, below, -below
    m[256:300], v[256:300] = -0.0, -0.0
    if n > 1000:                                                      # beside ordinary numbers, and at the border
        m[512:768], v[512:768] = below, below
        m[600], v[601] = F(0.5), F(0.25)
        m[768:1024], v[768:1024] = LEAST, LEAST
    m8, v8, s = empty((n,), np.int8), empty((n,), np.uint8), empty((-(-n // 256), 2), F)
    det.det_adamw8_pack([dev(m)], [dev(v)], [m8], [v8], [s])
    om, ov, os_ = oracle.adamw8_pack(m, v)
    assert not os_[:2].any() and not om[:512].any() and not ov[:512].any()
    assert n < 1000 or (os_[2].tolist() == [0.5, 0.5] and os_[3, 0] == LEAST and os_[3, 1] == F(2.0 ** -63))
    assert_same_bits(host(s), np.abs(os_), "scales")                  # a block of -0 has the scale +0
    assert_same_bits(host(m8), om, "m")
    assert_same_bits(host(v8), ov, "v")
