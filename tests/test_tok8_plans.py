"""The sizes that the parity tests of the 8-bit products run on the GPU reach every way a product is cut, so that a rule that is tuned anew cannot leave one
untested (worked out on the host, for the 148 SMs of a B200)."""
import pytest

import paper_2609_17380_b200 as det
from tok8_cases import BF16, F32, GATED, GLU, LINEAR, NARROW, PAIR, WIDE, products, rounds_and_steps

SMS = 148
ALL = [p for glu, cases in ((False, LINEAR), (True, GLU)) for c in cases for p in products(*c, glu)]


def plans():
    for p in ALL:
        yield p, det.det_test_tok8_plan(*p, SMS)


def test_every_plan_is_reached():
    seen = {(p[0], plan) for p, plan in plans()}
    want = {(kind, (tile, 1)) for kind in (BF16, F32, GATED) for tile in (PAIR, WIDE, NARROW)}
    want |= {(kind, (NARROW, parts)) for kind in (BF16, F32, GATED) for parts in (2, 4, 8)}
    assert {(k, (NARROW, plan[1]) if plan[1] > 1 else plan) for k, plan in seen} == want


@pytest.mark.parametrize("kind,tile", [(k, t) for k in (BF16, F32, GATED) for t in (PAIR, WIDE, NARROW)])
def test_rings_and_rounds_wrap(kind, tile):
    """More steps than the eight stages there are at most, and accumulators that are used again (three rounds for the pair); with ragged edges of rows, columns
    and contraction."""
    found = [(p, rounds_and_steps(plan, *p, SMS)) for p, plan in plans() if p[0] == kind and plan == (tile, 1)]
    need = 3 if tile == PAIR else 2
    assert any(r >= need and s > 8 for _, (r, s) in found), found
    assert any(p[1] % 128 and p[2] % 64 and p[3] % 16 for p, _ in found), found


def test_tiles_of_the_search_for_the_largest():
    """Whole tiles of 32, 64 and 128 rows, in the form with rows in whole pieces as well as in the other."""
    for cases in (LINEAR, GLU):
        seen = {(N % 8 == 0, det.det_test_tok8_tile_rows(M, N, int(N % 8 == 0), SMS)) for M, N, _ in cases if N >= 256}
        assert {(True, 32), (True, 64), (True, 128), (False, 128)} <= seen, seen
    assert any(M // 64 and N // 256 for M, N, _ in GLU)


def test_refusals():
    for bad in ((3, 1, 1, 1, 148), (-1, 1, 1, 1, 148), (0, 0, 1, 1, 148), (0, 1, 0, 1, 148), (0, 1, 1, 0, 148), (0, 1, 1, 1, 1)):
        with pytest.raises(Exception):
            det.det_test_tok8_plan(*bad)
    assert det.det_test_tok8_tile_rows(0, 1, 1, 148) == -1
