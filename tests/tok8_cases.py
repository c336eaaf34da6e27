"""Sizes of the 8-bit linears and the gated block that between them take every way a product is cut (on 148 SMs), for each kind of output: [M, K] tokens
through [N, K] weights, of the gated block [2 N, K]."""

# the tile of 256 x 256 by two CTAs for all three products, several rounds of them and more steps of the contraction than there are stages: odd widths and whole
# pieces; the tile of 128 columns; of 64 in several rounds; tiles that two, four and eight CTAs share, of tokens and of weights' gradients; and gradients with
# tiles of 64 and 128 rows in the search for the largest magnitudes, in whole pieces and not
LINEAR = [(2701, 4205, 2903), (2704, 4200, 2896), (2104, 2104, 2104), (2101, 2109, 2103), (20001, 60, 1200), (1201, 20001, 40), (79, 4072, 4656), (379, 350, 5247), (713, 8, 5468), (4656, 79, 4072),
          (5247, 379, 350), (5468, 713, 8), (1800, 8200, 40), (3500, 8200, 40), (1800, 8201, 40), (3500, 8203, 24)]
GLU = [(2701, 2103, 2903), (2704, 2104, 2896), (2104, 2104, 2104), (2101, 2109, 2103), (20001, 24, 1201), (49, 1384, 5015), (379, 350, 5247), (17, 548, 2276), (1800, 8200, 40),
       (3500, 8200, 40), (3500, 8203, 24)]
BF16, F32, GATED = 0, 1, 2                  # kinds of output
PAIR, WIDE, NARROW = 0, 1, 2                # tiles: 256 x 256 by two CTAs, 128 columns, 64


def products(M, N, K, glu):
    """(kind of output, rows, columns, contraction) of the forward product and the two backward ones."""
    n = 2 * N if glu else N
    return [(GATED if glu else BF16, M, N, K), (BF16, M, K, n), (F32, n, K, M)]


def rounds_and_steps(plan, kind, I, J, K, sms):
    """Rounds of tiles over the SMs, and steps of the contraction, of a product without shared tiles."""
    rows, cols = ((256, 256), (128, 128), (128, 64))[plan[0]]
    tiles = -(-I // rows) * -(-J // (cols // 2 if kind == GATED else cols))
    return -(-tiles // (sms // 2 if plan[0] == PAIR else sms)), -(-K // 128)
