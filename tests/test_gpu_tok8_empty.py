"""The 8-bit linears and the gated block on empty tensors: nothing is written but gradients of zeros for the weights."""
import numpy as np
import pytest
import torch

import oracle
import synth
from gpu_util import dev, empty

pytestmark = pytest.mark.gpu


def test_empty_tensors():
    import paper_2609_17380_b200 as det
    Fh, K = 24, 40
    N = 2 * Fh
    qW, sW = oracle.tok8_quant(synth.normal_bf16((N, K), 0.02, seed=2))
    pad = lambda q: dev(np.pad(q, ((0, 0), (0, -q.shape[1] % 16))))
    wc, wt, sw = pad(qW), pad(np.ascontiguousarray(qW.T)), dev(sW)
    row = lambda n, dt=np.uint16: empty((0, n), dt)
    q, s, x, y, h = row(48, np.int8), row(1, np.float32), row(K), row(N), row(Fh)
    assert x.data_ptr() == 0
    det.det_tok8_quant(x, K, 0, K, q, s)
    det.det_tok8_transpose(q, 0, K, row(16, np.int8))
    det.det_tok8_linear_fwd(x, K, wc, sw, 0, N, K, y, N, q, s)
    det.det_tok8_glu_fwd(x, K, wc, sw, 0, Fh, K, h, Fh, y, N, q, s)
    for call in (lambda dw: det.det_tok8_linear_bwd(y, N, q, s, wt, sw, 0, N, K, row(K), K, dw, None),
                 lambda dw: det.det_tok8_glu_bwd(h, Fh, y, N, q, s, wt, sw, 0, Fh, K, row(K), K, dw, None)):
        dw = torch.full((N, K), 7.0, device="cuda")
        call(dw)
        torch.cuda.synchronize()
        assert not dw.any()
