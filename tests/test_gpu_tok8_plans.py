"""The 8-bit linears and the gated block at sizes that take every way a product is cut (which that are is checked on the host), bit for bit: the codes are the oracle's, and the integer products are
summed in 64-bit floating point on the device, where they are exact (below 2^31), before the three roundings of an output."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import assert_same_bits, dev, empty, host, ws
from tok8_cases import GLU, LINEAR

pytestmark = pytest.mark.gpu
F = np.float32


@pytest.fixture(scope="module")
def det():
    import paper_2609_17380_b200 as d
    d.load()
    return d


def _values(M, K, std, seed):
    """Channels of different scale and a row of zeros; bf16 bits."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = std * torch.randn(M, K, generator=gen, device="cuda") * torch.exp(0.7 * torch.randn(K, generator=gen, device="cuda"))
    if M > 4:
        x[3] = 0
    return host(x.to(torch.bfloat16).view(torch.int16), np.uint16)


def _codes(q):
    return np.pad(q, ((0, 0), (0, -q.shape[1] % 16)))


def _product(a, b, si, sj=None):
    """float(sum_k a[i,k] b[j,k]) times the scales, in binary32."""
    acc = (dev(a).to(torch.float64) @ dev(b).to(torch.float64).T).to(torch.float32)
    si = dev(si)[:, None]
    return acc * (si * dev(sj) if sj is not None else si)


def _same(got, want, what):
    """Compared on the device; on the first difference the arrays are shown."""
    want = want.to(torch.bfloat16).view(torch.int16) if got.dtype == torch.int16 else want
    if not torch.equal(got.view(torch.uint8), want.contiguous().view(torch.uint8)):
        assert_same_bits(host(got), host(want), what)


def _backward(dy, qX, sX, qW, sW):
    qA, sA = oracle.tok8_quant(dy, col_factor=sW)
    qG, sG = oracle.tok8_quant(dy, row_factor=sX, by_col=True)
    t = lambda q: np.ascontiguousarray(q.T)
    return _product(qA, t(qW), sA), _product(qG, t(qX), sG)


@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear(det, M, N, K):
    x, w, dy = _values(M, K, 1.0, 1), _values(N, K, 0.02, 2), _values(M, N, 0.01, 3)
    (qX, sX), (qW, sW) = oracle.tok8_quant(x), oracle.tok8_quant(w)
    want = _product(qX, qW, sX, sW)
    wc, wt, sw, status = dev(_codes(qW)), dev(_codes(np.ascontiguousarray(qW.T))), dev(sW), torch.zeros(1, dtype=torch.int32, device="cuda")
    y, q, s = empty((M, N), np.uint16), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
    det.det_tok8_linear_fwd(dev(x), K, wc, sw, M, N, K, y, N, q, s, status)
    _same(q, dev(_codes(qX)), "codes")
    _same(s, dev(sX), "scales")
    _same(y, want, "y")
    dX, dW = _backward(dy, qX, sX, qW, sW)
    work = ws(det.det_tok8_linear_bwd_ws_bytes(M, N, K))
    work.fill_(0x5A)
    for both in (True, False):                                        # the products side by side or one behind the other, and each alone
        dx, dw = empty((M, K), np.uint16), empty((N, K), F)
        if both:
            det.det_tok8_linear_bwd(dev(dy), N, q, s, wt, sw, M, N, K, dx, K, dw, work, status)
        else:
            det.det_tok8_linear_bwd(dev(dy), N, q, s, wt, sw, M, N, K, dx, K, None, work, status)
            det.det_tok8_linear_bwd(dev(dy), N, q, s, wt, sw, M, N, K, None, 0, dw, work, status)
        _same(dx, dX, "dx")
        _same(dw, dW, "dw")
    assert not host(status).any()


@pytest.mark.parametrize("M,Fh,K", GLU)
def test_glu(det, M, Fh, K):
    N = 2 * Fh
    x, w, dh = _values(M, K, 1.0, 4), _values(N, K, 0.02, 5), _values(M, Fh, 0.01, 6)
    (qX, sX), (qW, sW) = oracle.tok8_quant(x), oracle.tok8_quant(w)
    gu = host(_product(qX, qW, sX, sW).to(torch.bfloat16).view(torch.int16), np.uint16)
    want = dev(oracle.swiglu_fwd(gu))
    wc, wt, sw, status = dev(_codes(qW)), dev(_codes(np.ascontiguousarray(qW.T))), dev(sW), torch.zeros(1, dtype=torch.int32, device="cuda")
    h, alone, got, q, s = empty((M, Fh), np.uint16), empty((M, Fh), np.uint16), empty((M, N), np.uint16), empty((M, det.det_tok8_ld(K)), np.int8), empty((M,), F)
    det.det_tok8_glu_fwd(dev(x), K, wc, sw, M, Fh, K, h, Fh, got, N, q, s, status)
    det.det_tok8_glu_fwd_q(q, s, wc, sw, M, Fh, K, alone, Fh, None, 0, status)
    _same(got.view(torch.uint8), dev(gu).view(torch.uint8), "gu")
    _same(h.view(torch.uint8), want.view(torch.uint8), "h")
    _same(alone.view(torch.uint8), want.view(torch.uint8), "h alone")
    dX, dW = _backward(oracle.swiglu_bwd(dh, gu), qX, sX, qW, sW)
    work = ws(det.det_tok8_glu_bwd_ws_bytes(M, Fh, K))
    work.fill_(0x5A)
    dx, dw = empty((M, K), np.uint16), empty((N, K), F)
    det.det_tok8_glu_bwd(dev(dh), Fh, got, N, q, s, wt, sw, M, Fh, K, dx, K, dw, work, status)
    _same(dx, dX, "dx")
    _same(dw, dW, "dw")
    assert not host(status).any()
