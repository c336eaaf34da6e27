"""The rows that the CTAs of the layer norm's forward pass walk over, worked out on the host: up to the largest number that the call takes."""
import pytest

import paper_2609_17380_b200 as det

MOST = 2000000000                                        # rows of a call at most


@pytest.mark.parametrize("io,D", [(0, 8), (0, 2048), (0, 1003), (1, 1), (1, 8), (1, 1024), (1, 2048), (1, 4096), (1, 8192)])
@pytest.mark.parametrize("rows", [1, 37, 1 << 20, (1 << 30) - 3, 1100000001, MOST])
def test_every_pass_starts_inside(io, D, rows):
    """Each piece of rows is one pass of one CTA, and no pass starts before the first row or behind the last one."""
    passes, most, low, high = det.det_test_layernorm_walk(io, rows, D, 148)
    assert low == 0 and 0 <= high < rows
    # a piece is a power of two of rows, at most 8 groups of 4
    piece = next(p for p in (1, 2, 4, 8, 16, 32) if -(-rows // p) == passes)
    assert high == (passes - 1) * piece
    if io == 0 or D % 8:
        assert most == 1                                 # a CTA for every piece


def test_refusals():
    for bad in ((2, 8, 8, 148), (1, 0, 8, 148), (1, MOST + 1, 8, 148), (1, 8, 0, 148), (1, 8, 8193, 148), (1, 8, 8, 0)):
        with pytest.raises(det.DetError):
            det.det_test_layernorm_walk(*bad)
    assert det.load().det_layernorm_fwd(1, 4096, None, None, MOST + 1, 8, 1e-6, 4096, 4096, 4096, None) == -2
