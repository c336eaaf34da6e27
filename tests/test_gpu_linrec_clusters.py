"""The recurrence with every number of CTAs that a cluster can have, in one round and in two, where few strips leave the GPU room for any of them."""
import pytest

from test_gpu_blocks import _linrec_check, det  # noqa: F401  (det is the fixture)

pytestmark = pytest.mark.gpu


# so many spans of 128 rows are one round of a cluster of as many CTAs; the last span is ragged
@pytest.mark.parametrize("spans", range(2, 17))
def test_one_round(det, spans):  # noqa: F811
    _linrec_check(det, 1, 128 * spans - 5 * spans, 34, every=spans % 3 and 90)


# an odd number of rounds or CTAs: 2 rounds of 9 to 16, 3 of 11 to 16; the last round of some has fewer spans than CTAs
@pytest.mark.parametrize("spans", [17, 19, 21, 23, 25, 27, 29, 31, 33, 37, 43])
def test_several_rounds(det, spans):  # noqa: F811
    _linrec_check(det, 1, 128 * spans - 77, 34, every=0 if spans % 3 else 200)
