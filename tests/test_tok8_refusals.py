"""What the 8-bit products with token and channel scales and AdamW with moments in 8 bits refuse: on the host, before anything is launched (addresses are
never followed, so these run without a GPU)."""
import ctypes as C

import pytest
import torch

import paper_2609_17380_b200 as det

ARG, SHAPE, ALIGN, WORKSPACE, RANGE = -1, -2, -3, -4, -5
A = 4096                                                  # an aligned address that nothing reads


def refused(code, fn, args):
    assert getattr(det.load(), fn)(*args.values()) == code, (fn, args)


def _with(base):
    return lambda **k: {**base, **k}


def test_codes_refusals():
    f = _with(dict(X=A, ld=64, M=4, K=64, q=A, s=A, st=None))
    for bad in (dict(X=None), dict(q=None), dict(s=None), dict(ld=63), dict(M=-1), dict(K=0, ld=0), dict(K=-1)):
        refused(ARG, "det_tok8_quant", f(**bad))
    refused(RANGE, "det_tok8_quant", f(K=1 << 17, ld=1 << 17))
    refused(SHAPE, "det_tok8_quant", f(M=(1 << 28) + 1))
    for bad in (dict(X=A + 1), dict(q=A + 8), dict(s=A + 2)):
        refused(ALIGN, "det_tok8_quant", f(**bad))
    refused(0, "det_tok8_quant", f(M=0))
    t = _with(dict(q=A, M=4, K=64, t=A, st=None))
    for bad, code in ((dict(q=None), ARG), (dict(t=None), ARG), (dict(M=-1), ARG), (dict(K=0), ARG), (dict(K=1 << 17), RANGE), (dict(q=A + 8), ALIGN),
                      (dict(t=A + 4), ALIGN), (dict(M=1 << 24), SHAPE), (dict(M=0), 0)):
        refused(code, "det_tok8_transpose", t(**bad))
    assert [det.det_tok8_ld(K) for K in (-5, 0, 1, 16, 17, (1 << 17) - 1)] == [0, 0, 16, 16, 32, 1 << 17]


def test_linear_refusals():
    f = _with(dict(X=A, ld=64, qW=A, sW=A, M=4, N=32, K=64, Y=A, ldy=32, q=A, s=A, st=None, status=None))
    for bad in (dict(X=None), dict(qW=None), dict(sW=None), dict(Y=None), dict(q=None), dict(s=None), dict(ld=63), dict(ldy=31), dict(M=-1), dict(N=0, ldy=0),
                dict(K=0, ld=0)):
        refused(ARG, "det_tok8_linear_fwd", f(**bad))
    refused(RANGE, "det_tok8_linear_fwd", f(K=1 << 17, ld=1 << 17))
    for bad in (dict(M=(1 << 28) + 1), dict(N=(1 << 28) + 1, ldy=(1 << 28) + 1)):
        refused(SHAPE, "det_tok8_linear_fwd", f(**bad))
    for bad in (dict(X=A + 1), dict(qW=A + 8), dict(sW=A + 2), dict(Y=A + 1), dict(q=A + 4), dict(s=A + 1)):
        refused(ALIGN, "det_tok8_linear_fwd", f(**bad))
    refused(0, "det_tok8_linear_fwd", f(M=0))
    f = _with(dict(q=A, s=A, qW=A, sW=A, M=4, N=32, K=64, Y=A, ldy=32, st=None, status=None))
    for bad, code in ((dict(q=None), ARG), (dict(s=None), ARG), (dict(ldy=31), ARG), (dict(K=1 << 17), RANGE), (dict(q=A + 8), ALIGN), (dict(M=0), 0)):
        refused(code, "det_tok8_linear_fwd_q", f(**bad))


def test_linear_backward_refusals():
    need = det.det_tok8_linear_bwd_ws_bytes(4, 32, 64)
    f = _with(dict(dY=A, ldy=32, q=A, s=A, qWt=A, sW=A, M=4, N=32, K=64, dX=A, ldx=64, dW=A, ws=A, n=need, st=None, status=None))
    for bad in (dict(dY=None), dict(q=None), dict(s=None), dict(qWt=None), dict(sW=None), dict(dX=None, dW=None), dict(ldy=31), dict(ldx=63), dict(M=-1),
                dict(N=0), dict(K=0)):
        refused(ARG, "det_tok8_linear_bwd", f(**bad))
    for bad in (dict(M=1 << 17), dict(N=1 << 17, ldy=1 << 17), dict(K=1 << 17, ldx=1 << 17)):
        refused(RANGE, "det_tok8_linear_bwd", f(**bad))
    for bad in (dict(dY=A + 1), dict(q=A + 8), dict(qWt=A + 8), dict(sW=A + 2), dict(s=A + 2), dict(dX=A + 1), dict(dW=A + 2)):
        refused(ALIGN, "det_tok8_linear_bwd", f(**bad))
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=A + 128)):
        refused(WORKSPACE, "det_tok8_linear_bwd", f(**bad))
    refused(0, "det_tok8_linear_bwd", f(M=0, ws=None, dW=None))
    assert det.det_tok8_linear_bwd_ws_bytes(0, 32, 64) == 0 and need >= 4 * 32 + 32 * 16 + 64 * 16


def test_glu_refusals():
    f = _with(dict(X=A, ld=64, qW=A, sW=A, M=4, F=32, K=64, h=A, ldh=32, gu=A, ldg=64, q=A, s=A, st=None, status=None))
    for bad in (dict(X=None), dict(qW=None), dict(sW=None), dict(h=None), dict(q=None), dict(s=None), dict(ld=63), dict(ldh=31), dict(ldg=63), dict(M=-1),
                dict(F=0), dict(K=0)):
        refused(ARG, "det_tok8_glu_fwd", f(**bad))
    refused(SHAPE, "det_tok8_glu_fwd", f(F=(1 << 27) + 1, ldh=1 << 28, ldg=1 << 29))
    refused(RANGE, "det_tok8_glu_fwd", f(K=1 << 17, ld=1 << 17))
    for bad in (dict(X=A + 1), dict(gu=A + 1), dict(h=A + 1), dict(qW=A + 8)):
        refused(ALIGN, "det_tok8_glu_fwd", f(**bad))
    refused(0, "det_tok8_glu_fwd", f(M=0, gu=None, ldg=0))
    f = _with(dict(q=A, s=A, qW=A, sW=A, M=4, F=32, K=64, h=A, ldh=32, gu=None, ldg=0, st=None, status=None))
    for bad, code in ((dict(gu=A, ldg=63), ARG), (dict(h=None), ARG), (dict(gu=A + 1, ldg=64), ALIGN), (dict(F=(1 << 27) + 1, ldh=1 << 28), SHAPE), (dict(M=0), 0)):
        refused(code, "det_tok8_glu_fwd_q", f(**bad))
    need = det.det_tok8_glu_bwd_ws_bytes(4, 32, 64)
    b = _with(dict(dh=A, ldh=32, gu=A, ldg=64, q=A, s=A, qWt=A, sW=A, M=4, F=32, K=64, dX=A, ldx=64, dW=A, ws=A, n=need, st=None, status=None))
    for bad in (dict(dh=None), dict(gu=None), dict(q=None), dict(s=None), dict(qWt=None), dict(sW=None), dict(dX=None, dW=None), dict(ldh=31), dict(ldg=63),
                dict(ldx=63), dict(M=-1), dict(F=0), dict(K=0)):
        refused(ARG, "det_tok8_glu_bwd", b(**bad))
    for bad in (dict(M=1 << 17), dict(F=1 << 16, ldh=1 << 16, ldg=1 << 17), dict(K=1 << 17, ldx=1 << 17)):
        refused(RANGE, "det_tok8_glu_bwd", b(**bad))
    for bad in (dict(dh=A + 1), dict(gu=A + 1), dict(qWt=A + 4), dict(dW=A + 1)):
        refused(ALIGN, "det_tok8_glu_bwd", b(**bad))
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=A + 16)):
        refused(WORKSPACE, "det_tok8_glu_bwd", b(**bad))


def _adamw8(**k):
    """Two tensors, the second with moments in 32 bits; k: other entries of the first."""
    tables = dict(p=[A, A], g=[A, A], m=[A, A], v=[A, A], s=[A, None], po=[A, A], mo=[A, A], vo=[A, A], so=[A, None])
    kind, n, step = [1, 0], [300, 300], 1
    for name, x in k.items():
        if name in tables:
            tables[name][0] = x
        elif name == "kind":
            kind[0] = x
        elif name == "n":
            n[0] = x
        else:
            step = x
    descs = (det.det_adamw_desc * 2)(*[det.det_adamw_desc(1e-3, 0.9, 0.95, 1e-8, 0.0, s) for s in (step, 1)])
    t = {name: (C.c_void_p * 2)(*x) for name, x in tables.items()}
    return det.load().det_adamw8_batch(descs, (C.c_int * 2)(*kind), t["p"], t["g"], t["m"], t["v"], t["s"], t["po"], t["mo"], t["vo"], t["so"],
                                       (C.c_size_t * 2)(*n), 2, None, None)


def test_adamw8_refusals():
    for bad in (dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(po=None), dict(mo=None), dict(vo=None), dict(s=None), dict(so=None), dict(kind=2),
                dict(step=0)):
        assert _adamw8(**bad) == ARG, bad
    for bad in (dict(p=A + 4), dict(p=A + 8, kind=0), dict(g=A + 8), dict(m=A + 2), dict(vo=A + 1), dict(s=A + 4), dict(so=A + 4),
                dict(s=None, so=None, m=A + 8), dict(s=None, so=None, vo=A + 4), dict(po=A + 2)):
        assert _adamw8(**bad) == ALIGN, bad
    assert _adamw8(n=1 << 40) == SHAPE
    lib = det.load()
    assert lib.det_adamw8_batch(*[None] * 12, 0, None, None) == 0 and lib.det_adamw8_batch(*[None] * 12, -1, None, None) == ARG
    assert lib.det_adamw8_batch(*[None] * 12, 1, None, None) == ARG
    one = lambda x: (C.c_void_p * 1)(x)
    for fn, order in (("det_adamw8_pack", (3, 4, 0, 1, 2)), ("det_adamw8_unpack", (0, 1, 2, 3, 4))):      # m8, v8, s, m, v
        call = lambda x, n=300: getattr(lib, fn)(*[one(x[i]) for i in order], (C.c_size_t * 1)(n), 1, None)
        for i in range(5):
            assert call([None if i == k else A for k in range(5)]) == ARG
            assert call([A + 2 if i == k else A for k in range(5)]) == ALIGN
        assert call([A] * 5, 1 << 40) == SHAPE and call([None] * 5, 0) == 0
    assert [det.det_adamw8_scale_floats(n) for n in (0, 1, 256, 257)] == [0, 2, 2, 4]


# every tensor of a table is checked as a single argument is: one on the host, of another length or of another width is refused
def test_adamw8_tables_are_checked():
    t = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)
    desc, bf, m8, v8, s = det.det_adamw_desc(1e-3, 0.9, 0.95, 1e-8, 0.0, 1), t(8, torch.int16), t(8, torch.int8), t(8, torch.uint8), t(2)
    good = dict(d=[desc], k=[det.DET_BF16], p=[bf], g=[t(8)], m=[m8], v=[v8], s=[s])
    bad = (dict(), dict(g=[t(4)]), dict(m=[t(8)]), dict(v=[t(4, torch.uint8)]), dict(s=[t(4)]), dict(s=[None]), dict(k=[det.DET_F32]), dict(k=[]),
           dict(s=[]), dict(g=[t(8, torch.int16)]))
    for change in bad:
        with pytest.raises(AssertionError):
            det.det_adamw8_batch(*{**good, **change}.values())
    for outs in (([bf], [m8], [v8], [None]), ([bf], [t(8)], [v8], [s]), ([t(4, torch.int16)], [m8], [v8], [s])):
        with pytest.raises(AssertionError):
            det.det_adamw8_batch(*good.values(), outs=outs)
    for args in (([m8], [v8], [s], [t(8)], [t(8)]), ([m8], [v8], [None], [t(8)], [t(8)]), ([m8], [v8], [s], [t(4)], [t(8)]), ([m8], [bf], [s], [t(8)], [t(8)])):
        with pytest.raises(AssertionError):
            det.det_adamw8_unpack(*args)
