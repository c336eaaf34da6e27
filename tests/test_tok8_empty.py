"""Calls of the 8-bit linears without tokens: what has a row for every token may be NULL, as the address of an empty tensor is; the weights may not."""
import pytest

import paper_2609_17380_b200 as det

ARG = -1
A = 4096                                                  # an aligned address that nothing reads or writes: without tokens only a dW is written

CALLS = {
    "det_tok8_quant": dict(X=None, ld=64, M=0, K=64, q=None, s=None, st=None),
    "det_tok8_transpose": dict(q=None, M=0, K=64, t=None, st=None),
    "det_tok8_linear_fwd": dict(X=None, ld=64, qW=A, sW=A, M=0, N=32, K=64, Y=None, ldy=32, q=None, s=None, st=None, status=None),
    "det_tok8_linear_fwd_q": dict(q=None, s=None, qW=A, sW=A, M=0, N=32, K=64, Y=None, ldy=32, st=None, status=None),
    "det_tok8_linear_bwd": dict(dY=None, ldy=32, q=None, s=None, qWt=A, sW=A, M=0, N=32, K=64, dX=None, ldx=64, dW=None, ws=None, n=0, st=None, status=None),
    "det_tok8_glu_fwd": dict(X=None, ld=64, qW=A, sW=A, M=0, F=32, K=64, h=None, ldh=32, gu=None, ldg=64, q=None, s=None, st=None, status=None),
    "det_tok8_glu_fwd_q": dict(q=None, s=None, qW=A, sW=A, M=0, F=32, K=64, h=None, ldh=32, gu=None, ldg=64, st=None, status=None),
    "det_tok8_glu_bwd": dict(dh=None, ldh=32, gu=None, ldg=64, q=None, s=None, qWt=A, sW=A, M=0, F=32, K=64, dX=None, ldx=64, dW=None, ws=None, n=0, st=None,
                             status=None),
}


@pytest.mark.parametrize("name", CALLS)
def test_no_tokens(name):
    fn, args = getattr(det.load(), name), CALLS[name]
    assert fn(*args.values()) == 0
    for x in args:
        if x in ("qW", "qWt", "sW"):
            assert fn(*{**args, x: None}.values()) == ARG, x
        if x in ("ld", "ldy", "ldh"):
            assert fn(*{**args, x: 31}.values()) == ARG, x
    assert fn(*{**args, "M": 1}.values()) == ARG and fn(*{**args, "M": -1}.values()) != 0
