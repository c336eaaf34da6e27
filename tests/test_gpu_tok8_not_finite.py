"""The gated block where a token, a channel, a gradient or a kept gate or up is not finite, or gates are at the ends of the sigmoid: against the oracle, bit for
bit, NaN as NaN.  Sizes: few tokens, tiles that CTAs share, tiles of their own, and rows in whole pieces in the search for the largest magnitudes."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import assert_same_bits, dev, empty, host, ws

pytestmark = pytest.mark.gpu
F = np.float32


def same(got, want, what):
    wide = lambda x: synth.from_bf16(x) if x.dtype == np.uint16 else x
    nan = np.isnan(wide(want))
    assert np.array_equal(np.isnan(wide(got)), nan), what
    assert_same_bits(got[~nan], want[~nan], what)


def codes(q):
    return np.pad(q, ((0, 0), (0, -q.shape[1] % 16)))


@pytest.mark.parametrize("place", ["x", "w", "dh", "gu"])
@pytest.mark.parametrize("M,Fh,K", [(2, 40, 48), (4, 24, 40), (24, 136, 2056), (150, 136, 264), (257, 520, 72), (1300, 8104, 40)])
def test_gated_block(M, Fh, K, place):
    import torch

    import paper_2609_17380_b200 as det
    N = 2 * Fh
    x, w, dh = synth.normal_bf16((M, K), 1.0, seed=1), synth.normal_bf16((N, K), 0.02, seed=2), synth.normal_bf16((M, Fh), 0.01, seed=3)
    if place == "x":
        x[0, 1], x[M - 1, 3] = 0x7F80, 0xFFC1
    if place == "w":
        w[2, 3], w[Fh + 5, 1] = 0xFF80, 0x7FC1
    if place == "dh":
        dh[0, 1], dh[M - 1, 7] = 0xFF80, 0x7FC1
    (qX, sX), (qW, sW) = oracle.tok8_quant(x), oracle.tok8_quant(w)
    gu = oracle.tok8_product(qX, qW, sX, sW)
    h = oracle.swiglu_fwd(gu)
    wc, wt, sw = dev(codes(qW)), dev(codes(np.ascontiguousarray(qW.T))), dev(sW)
    gh, gg, q, s = empty((M, Fh), np.uint16), empty((M, N), np.uint16), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
    det.det_tok8_glu_fwd(dev(x), K, wc, sw, M, Fh, K, gh, Fh, gg, N, q, s)
    torch.cuda.synchronize()
    same(host(gg, np.uint16), gu, "gu")
    same(host(gh, np.uint16), h, "h")
    if place == "gu":                                                 # large gates of either sign, borders of the sigmoid's table, infinities and NaN in gates and ups
        ends = synth.to_bf16(np.array([88.0, -88.0, 88.5, -88.5, 89.0, -89.0, 127.0, -127.0, 128.0, -128.0, 3e38, -3e38, 2.0 ** -27, -2.0 ** -26, 1e-40, 0.0], F))
        gu[0, :16], gu[1, :16] = ends, ends[::-1]
        gu[M - 1, 3], gu[M - 1, Fh + 4] = 0x7F80, 0xFF80
        gu[M - 2, 5] = 0xFFC1
    dgu = oracle.swiglu_bwd(dh, gu)
    qA, sA = oracle.tok8_quant(dgu, col_factor=sW)
    qG, sG = oracle.tok8_quant(dgu, row_factor=sX, by_col=True)
    dX = oracle.tok8_product(qA, np.ascontiguousarray(qW.T), sA)
    dW = oracle.tok8_product(qG, np.ascontiguousarray(qX.T), sG, bf=False)
    dx, dw = empty((M, K), np.uint16), empty((N, K), F)
    det.det_tok8_glu_bwd(dev(dh), Fh, dev(gu), N, q, s, wt, sw, M, Fh, K, dx, K, dw, ws(det.det_tok8_glu_bwd_ws_bytes(M, Fh, K)))
    torch.cuda.synchronize()
    same(host(dx, np.uint16), dX, "dx")
    same(host(dw), dW, "dw")
    assert place != "gu" or (np.isnan(synth.from_bf16(dX)).any() and (M == 2 or not np.isnan(synth.from_bf16(dX)).all()))
