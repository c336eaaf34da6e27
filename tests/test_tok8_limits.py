"""The limits that the header states for the 8-bit linears are the ones that the calls have (refusals only: addresses are never followed)."""
import os
import re

import paper_2609_17380_b200 as det

SHAPE = -2
A = 4096
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "det.h")


def test_rows_of_the_transposition():
    text = open(HEADER).read()
    rows = re.search(r"det_tok8_transpose: codes .*?at most (\d+) \* (\d+) rows", text)
    most = int(rows.group(1)) * int(rows.group(2))
    for M in (most + 1, 1 << 24, 1 << 28):
        assert det.load().det_tok8_transpose(A, M, 64, A, None) == SHAPE, M
