"""What layer norm, the 8-bit checkpoints and the gated linear recurrence refuse: on the host, before anything is launched (addresses are
never followed, so these run without a GPU)."""
import paper_2609_17380_b200 as det

ARG, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4
A = 4096                                                  # an aligned address that nothing reads


def refused(code, fn, args):
    assert getattr(det.load(), fn)(*args.values()) == code, (fn, args)


def _with(base):
    return lambda **k: {**base, **k}


def test_layernorm_refusals():
    f = _with(dict(io=1, x=A, g=A, b=A, rows=4, D=64, eps=1e-6, y=A, mean=A, rstd=A, st=None))
    for bad in (dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(rows=-1), dict(D=0), dict(D=-8), dict(io=2), dict(io=-1)):
        refused(ARG, "det_layernorm_fwd", f(**bad))
    refused(SHAPE, "det_layernorm_fwd", f(D=8193))
    for name in ("x", "g", "b", "y"):
        refused(ALIGN, "det_layernorm_fwd", f(**{name: A + 8}))
        refused(ALIGN, "det_layernorm_fwd", f(**{name: A + 1, "D": 63}))
        refused(ALIGN, "det_layernorm_fwd", f(**{name: A + 2, "D": 63, "io": 0}))
    refused(0, "det_layernorm_fwd", f(rows=0))
    r = _with(dict(a=A, b=A, g=A, be=A, rows=4, D=64, eps=1e-6, sum=A, y=A, mean=A, rstd=A, s=A, qy=A, q8=A, e8=A, st=None))
    for bad in (dict(a=None), dict(sum=None), dict(s=None), dict(q8=None), dict(e8=None), dict(y=None)):
        refused(ARG, "det_residual_layernorm_fwd", r(**bad))
    refused(SHAPE, "det_residual_layernorm_fwd", r(D=63))
    refused(ALIGN, "det_residual_layernorm_fwd", r(q8=A + 4))
    refused(ALIGN, "det_residual_layernorm_fwd", r(qy=A + 4))
    refused(0, "det_residual_layernorm_fwd", r(rows=0))


def test_layernorm_backward_refusals():
    need = det.det_layernorm_bwd_ws_bytes(100, 64)
    f = _with(dict(io=1, dy=A, x=A, g=A, mean=A, rstd=A, rows=100, D=64, dx=A, dg=A, db=A, ws=A, n=need, st=None))
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(io=3), dict(rows=-1), dict(D=0)):
        refused(ARG, "det_layernorm_bwd", f(**bad))
    refused(SHAPE, "det_layernorm_bwd", f(D=8200))
    refused(ALIGN, "det_layernorm_bwd", f(x=A + 2))
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=A + 8), dict(ws=None, dg=None), dict(ws=None, db=None)):
        refused(WORKSPACE, "det_layernorm_bwd", f(**bad))
    r = _with(dict(dy=A, x=A, g=A, mean=A, rstd=A, rows=100, D=64, res=A, dx=A, dg=A, db=A, ws=A, n=need, st=None))
    refused(ARG, "det_layernorm_bwd_residual", r(res=None))
    refused(ALIGN, "det_layernorm_bwd_residual", r(res=A + 2))
    q = _with(dict(dy=A, q8=A, e8=A, g=A, mean=A, rstd=A, rows=100, D=64, res=A, dx=A, dg=A, db=A, ws=A, n=need, st=None))
    refused(ARG, "det_layernorm_bwd_act8", q(e8=None))
    refused(ARG, "det_layernorm_bwd_act8", q(q8=None))
    refused(ALIGN, "det_layernorm_bwd_act8", q(q8=A + 4))
    refused(0, "det_layernorm_bwd_act8", q(rows=0, dg=None, db=None))


def test_act8_refusals():
    f = _with(dict(io=1, x=A, ld=64, rows=4, D=64, q=A, e=A, st=None))
    for bad in (dict(io=5), dict(x=None), dict(ld=63), dict(rows=-1), dict(D=0, ld=0), dict(q=None), dict(e=None)):
        refused(ARG, "det_act8_pack", f(**bad))
    refused(ALIGN, "det_act8_pack", f(x=A + 1))
    refused(ALIGN, "det_act8_pack", f(x=A + 2, io=0))
    refused(SHAPE, "det_act8_pack", f(rows=2 ** 31 - 1, D=1024, ld=1024))
    u = _with(dict(io=1, q=A, e=A, rows=4, D=64, y=A, ld=64, st=None))
    for bad in (dict(io=5), dict(y=None), dict(ld=63), dict(rows=-1), dict(q=None), dict(e=None)):
        refused(ARG, "det_act8_unpack", u(**bad))
    assert det.det_act8_exp_bytes(3, 33) == 6 and det.det_act8_exp_bytes(0, 33) == 0 and det.det_act8_exp_bytes(3, -1) == 0


def test_swiglu_act8_refusals():
    f = _with(dict(gu=A, rows=4, F=64, h=A, q=A, e=A, s=None, qh=None, st=None))
    for bad in (dict(gu=None), dict(h=None), dict(q=None), dict(e=None), dict(rows=-1), dict(F=0), dict(qh=A)):
        refused(ARG, "det_swiglu_fwd_act8", f(**bad))
    for width in (8, 48):
        refused(SHAPE, "det_swiglu_fwd_act8", f(F=width))
    for bad in (dict(gu=A + 8), dict(h=A + 2), dict(q=A + 4), dict(qh=A + 4, s=A)):
        refused(ALIGN, "det_swiglu_fwd_act8", f(**bad))
    f = _with(dict(q=A, e=A, rows=4, F=64, h=A, s=None, qh=None, st=None))
    for bad, code in ((dict(h=None), ARG), (dict(qh=A), ARG), (dict(F=40), SHAPE), (dict(q=A + 4), ALIGN)):
        refused(code, "det_swiglu_act8", f(**bad))
    f = _with(dict(dh=A, q=A, e=A, rows=4, F=64, dgu=A, st=None))
    for bad, code in ((dict(e=None), ARG), (dict(dh=None), ARG), (dict(F=40), SHAPE), (dict(dgu=A + 2), ALIGN)):
        refused(code, "det_swiglu_bwd_act8", f(**bad))


def test_linrec_refusals():
    f = _with(dict(g=A, v=A, ld=128, B=2, S=9, D=64, y=A, ldy=64, fl=None, h0=None, hT=None, st=None, s=None, status=None))
    for bad in (dict(g=None), dict(v=None), dict(y=None), dict(B=-1), dict(S=-1), dict(D=0), dict(ld=62), dict(ldy=62)):
        refused(ARG, "det_linrec_fwd", f(**bad))
    for bad in (dict(D=63), dict(ld=129), dict(ldy=65), dict(S=2 ** 30 + 1), dict(B=2 ** 30)):
        refused(SHAPE, "det_linrec_fwd", f(**bad))
    for bad in (dict(g=A + 2), dict(v=A + 2), dict(y=A + 2), dict(h0=A + 4), dict(hT=A + 4), dict(st=A + 4)):
        refused(ALIGN, "det_linrec_fwd", f(**bad))
    b = _with(dict(dy=A, ldy=64, g=A, v=A, ld=128, B=2, S=9, D=64, st=A, dg=A, dv=A, ldd=128, fl=None, dhT=None, dh0=None, s=None, status=None))
    for bad in (dict(dy=None), dict(g=None), dict(dg=None), dict(dv=None), dict(st=None), dict(ldy=62), dict(ldd=62), dict(ld=62)):
        refused(ARG, "det_linrec_bwd", b(**bad))
    for bad in (dict(D=63), dict(ldd=129), dict(ldy=65)):
        refused(SHAPE, "det_linrec_bwd", b(**bad))
    for bad in (dict(dy=A + 2), dict(dg=A + 2), dict(dv=A + 2), dict(dhT=A + 4), dict(dh0=A + 4), dict(st=A + 4)):
        refused(ALIGN, "det_linrec_bwd", b(**bad))
    assert det.det_linrec_state_floats(2, 65, 10) == 180 and det.det_linrec_state_floats(2, 0, 10) == 0
