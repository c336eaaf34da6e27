"""The 8-bit linears and the gated block where an output, a gradient and their codes have more than 2^31 elements: the definition in elementary torch operations,
some rows at a time (products in 64-bit floating point, where they are exact)."""
import pytest
import torch

from gpu_util import ws

pytestmark = pytest.mark.gpu
F32, F64, BF = torch.float32, torch.float64, torch.bfloat16
M, N, K, STEP = 131071, 16400, 16, 8192


@pytest.fixture(scope="module")
def det():
    import paper_2609_17380_b200 as d
    d.load()
    return d


def _scale(a):
    s = a / torch.full_like(a, 127.0)
    return s, torch.where(s > 0, torch.ones_like(s) / s, torch.zeros_like(s))


def _codes(v, dim):
    s, inv = _scale(v.abs().amax(dim, keepdim=True))
    return torch.round(v * inv), s


def _inputs():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    r = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    x, w = r(M, K).to(BF), (0.02 * r(N, K)).to(BF)
    qW, sW = _codes(w.to(F32), 1)
    return gen, x, qW, sW


def _backward_matches(grad_of, x, qW, sW, dX, dW):
    """grad_of(rows): those rows of the gradient, in binary32."""
    sX = _codes(x.to(F32), 1)[1]
    cm, spans = torch.zeros(N, device="cuda"), [slice(i, min(i + STEP, M)) for i in range(0, M, STEP)]
    for r in spans:
        g = grad_of(r)
        qa, sa = _codes(g * sW.view(1, -1), 1)
        assert torch.equal(dX[r], ((qa.to(F64) @ qW.to(F64)).to(F32) * sa).to(BF)), r
        cm = torch.maximum(cm, (g * sX[r]).abs().amax(0))
    s, inv = _scale(cm)
    acc = torch.zeros(N, K, dtype=F64, device="cuda")
    for r in spans:
        acc += torch.round(grad_of(r) * sX[r] * inv).to(F64).T @ _codes(x[r].to(F32), 1)[0].to(F64)
    assert torch.equal(dW, acc.to(F32) * s.view(-1, 1))


def _laid_out(q):
    return torch.nn.functional.pad(q, (0, -q.shape[1] % 16)).to(torch.int8).contiguous()


def test_linear(det):
    gen, x, qW, sW = _inputs()
    y, q, s = torch.empty(M, N, dtype=BF, device="cuda"), torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    det.det_tok8_linear_fwd(x, K, _laid_out(qW), sW.view(-1), M, N, K, y, N, q, s)
    for i in range(0, M, STEP):
        r = slice(i, min(i + STEP, M))
        qx, sx = _codes(x[r].to(F32), 1)
        assert torch.equal(y[r], ((qx.to(F64) @ qW.to(F64).T).to(F32) * (sx * sW.view(1, -1))).to(BF)), i
    dy = y                                                            # any gradient will do
    dX, dW = torch.empty(M, K, dtype=BF, device="cuda"), torch.empty(N, K, device="cuda")
    det.det_tok8_linear_bwd(dy, N, q, s, _laid_out(qW.T), sW.view(-1), M, N, K, dX, K, dW, ws(det.det_tok8_linear_bwd_ws_bytes(M, N, K)))
    _backward_matches(lambda r: dy[r].to(F32), x, qW, sW, dX, dW)


def test_gated_block(det):
    """Its gradient is checked against the codes of the separate calls' gradient, det_swiglu_bwd's, which the gated block has bit for bit."""
    gen, x, qW, sW = _inputs()
    Fh = N // 2
    h, gu = torch.empty(M, Fh, dtype=BF, device="cuda"), torch.empty(M, N, dtype=BF, device="cuda")
    q, s = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    det.det_tok8_glu_fwd(x, K, _laid_out(qW), sW.view(-1), M, Fh, K, h, Fh, gu, N, q, s)
    want = torch.empty_like(h)
    det.det_swiglu_fwd(gu, M, Fh, want)
    assert torch.equal(h, want)
    for i in range(0, M, STEP):
        r = slice(i, min(i + STEP, M))
        qx, sx = _codes(x[r].to(F32), 1)
        assert torch.equal(gu[r], ((qx.to(F64) @ qW.to(F64).T).to(F32) * (sx * sW.view(1, -1))).to(BF)), i
    dX, dW = torch.empty(M, K, dtype=BF, device="cuda"), torch.empty(N, K, device="cuda")
    dh = want.normal_(generator=gen)
    det.det_tok8_glu_bwd(dh, Fh, gu, N, q, s, _laid_out(qW.T), sW.view(-1), M, Fh, K, dX, K, dW, ws(det.det_tok8_glu_bwd_ws_bytes(M, Fh, K)))
    dgu = torch.empty_like(gu)
    det.det_swiglu_bwd(dh, gu, M, Fh, dgu)
    _backward_matches(lambda r: dgu[r].to(F32), x, qW, sW, dX, dW)
