"""Layer norm, 8-bit activation checkpoints and the gated linear recurrence as cases to time, with their plain forms.

Sizes are those of the repository's configurations (the smoke step, the 1B-shaped decoder: 8192 tokens of 2048, feed-forward 8192)
and odd or ragged sizes in between."""
import math

import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
GROUP = 32                    # values of a row that share the step of a checkpoint


def listed():
    return [
        # the norm of the smoke step: what a bisection of a mismatch calls over and over
        dict(name="norm_small", kind="norm", dtype="bf16", rows=128, D=256, res=False),
        # the norm of one micro-batch of the 1B-shaped decoder, with the residual stream that runs beside it
        dict(name="norm_step", kind="norm", dtype="bf16", rows=8192, D=2048, res=True),
        # its gradient, added to the gradient that bypasses the norm
        dict(name="norm_bwd_step", kind="norm_bwd", dtype="bf16", rows=8192, D=2048, res=True),
        # an odd width and ragged rows in binary32, as an ablation of the width runs them
        dict(name="norm_bwd_odd", kind="norm_bwd", dtype="f32", rows=1531, D=1003, res=False),
        # the same gradient from the input kept in 8 bits
        dict(name="norm_ckpt_bwd", kind="norm_ckpt_bwd", dtype="bf16", rows=8192, D=2048, res=True),
        # storing and restoring the fused gate and up projection of a micro-batch, the largest activation of a layer
        dict(name="ckpt_step", kind="ckpt", dtype="bf16", rows=8192, D=16384),
        # a ragged block in binary32
        dict(name="ckpt_odd", kind="ckpt", dtype="f32", rows=1003, D=777),
        # SwiGLU of a micro-batch with its input kept in 8 bits: forward, the output again for the down projection, backward
        dict(name="swiglu_ckpt_step", kind="swiglu_ckpt", rows=8192, F=8192),
        # the recurrence of the smoke step, forward and backward
        dict(name="linrec_small", kind="linrec", B=1, S=128, D=256, reset=0, bwd=True),
        # evaluation of ragged sequences
        dict(name="linrec_fwd_odd", kind="linrec", B=3, S=1999, D=1502, reset=0, bwd=False),
        # a micro-batch of the 1B-shaped decoder, forward and backward
        dict(name="linrec_step", kind="linrec", B=4, S=2048, D=2048, reset=0, bwd=True),
        # one long packed sequence of documents, forward and backward
        dict(name="linrec_long", kind="linrec", B=1, S=65536, D=512, reset=700, bwd=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "norm_ckpt_bwd", "ckpt", "swiglu_ckpt", "linrec", "linrec"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "linrec":
        D = 2 * _log(rng, 1, 2048)
        S = min(_log(rng, 1, 65536), (1 << 24) // D)
        B = max(1, min(_log(rng, 1, 8), (1 << 24) // (S * D)))
        return dict(kind=kind, B=B, S=S, D=D, reset=rng.choice([0, 0, 3, 500]), bwd=rng.random() < 0.7)
    if kind == "swiglu_ckpt":
        F = 32 * _log(rng, 1, 256)
        return dict(kind=kind, rows=max(1, min(_log(rng, 1, 16384), (1 << 25) // F)), F=F)
    D = _log(rng, 16, 8192)
    if rng.random() < 0.5:
        D = (D + 7) // 8 * 8
    rows = max(1, min(_log(rng, 1, 65536), (1 << 25) // D))
    if kind == "ckpt":
        return dict(kind=kind, dtype=dtype, rows=rows, D=D)
    return dict(kind=kind, dtype="bf16" if kind == "norm_ckpt_bwd" else dtype, rows=rows, D=D,
                res=kind == "norm_ckpt_bwd" or (dtype == "bf16" and rng.random() < 0.5))


def _type(case):
    return F32 if case.get("dtype") == "f32" else BF


def _stream(gen, rows, D, dtype):
    """Rows as a residual stream has them: channels of different scale, a few large, a mean that is not zero."""
    x = torch.randn(rows, D, generator=gen, device="cuda")
    scale = torch.exp(0.7 * torch.randn(D, generator=gen, device="cuda"))
    shift = 0.3 * torch.randn(D, generator=gen, device="cuda")
    return x.mul_(scale).add_(shift).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    s = dict(case)
    if case["kind"] == "linrec":
        B, S, D = case["B"], case["S"], case["D"]
        # gate and value are the two halves of one projection; gates of long and short memory
        s["gv"] = torch.cat([randn(B * S, D) * 2 + 3 * randn(D).abs(), randn(B * S, D)], 1).to(BF)
        s["h0"] = randn(B, D)
        s["flags"] = (torch.rand(B, S, generator=gen, device="cuda") < 1.0 / case["reset"]).to(torch.uint8) if case["reset"] else None
        if case["bwd"]:
            s["dy"], s["dhT"] = randn(B * S, D).to(BF), randn(B, D)
        return s
    rows = case["rows"]
    if case["kind"] == "swiglu_ckpt":
        s["gu"] = _stream(gen, rows, 2 * case["F"], BF)
        s["dh"] = (randn(rows, case["F"]) * 0.01).to(BF)
        return s
    D, dt = case["D"], _type(case)
    s["x"] = _stream(gen, rows, D, dt)
    if case["kind"] == "ckpt":
        return s
    s["gamma"], s["beta"] = (1 + 0.1 * randn(D)).to(dt), (0.1 * randn(D)).to(dt)
    if case["res"]:
        s["other"] = _stream(gen, rows, D, dt)
    if case["kind"] != "norm":
        # what the forward pass left: the statistics, and the input or its checkpoint
        s["dy"] = (randn(rows, D) * 0.01).to(dt)
        var, mean = torch.var_mean(s["x"].to(F64), 1, correction=0)
        s["mean"], s["rstd"] = mean.to(F32), (var + 1e-6).rsqrt().to(F32)
        if case["kind"] == "norm_ckpt_bwd":
            s["q"], s["e"] = _pack(s.pop("x"))
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------
def _steps(e, D):
    """The step of every value from the exponent bytes [rows, groups]."""
    return (e.to(torch.int32) << 23).view(F32).repeat_interleave(GROUP, 1)[:, :D]


def _pack(x):
    rows, D = x.shape
    n = (D + GROUP - 1) // GROUP
    v = torch.zeros(rows, n * GROUP, dtype=F32, device=x.device)
    v[:, :D] = x
    v = v.view(rows, n, GROUP)
    bits = v.abs().amax(2).view(torch.int32)
    # the smallest power of two 2^E with amax <= 127 * 2^E: the exponent field of amax less 6, one more where the fraction is past 127/64
    e = ((bits >> 23) - 6 + ((bits & 0x7FFFFF) > 0x7E0000).to(torch.int32)).clamp_(min=1)
    q = torch.round(v * ((254 - e) << 23).view(F32)[:, :, None])
    return q.to(torch.int8).view(rows, n * GROUP)[:, :D].contiguous(), e.to(torch.uint8)


def _unpack(q, e):
    return q.to(F32) * _steps(e, q.shape[1])


def _sigmoid(g):
    return 1.0 / (1.0 + torch.exp(-g))


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t along dimension 1 from zero: spans of the recurrence composed with the span before, doubled each time."""
    a, u = a.clone(), u.clone()
    n, S = 1, a.shape[1]
    while n < S:
        u = torch.cat([u[:, :n], u[:, n:] + a[:, n:] * u[:, :-n]], 1)
        a = torch.cat([a[:, :n], a[:, n:] * a[:, :-n]], 1)
        n *= 2
    return u


def _plain_linrec(s):
    B, S, D = s["B"], s["S"], s["D"]
    g, v = (s["gv"][:, i * D:(i + 1) * D].to(F32).view(B, S, D) for i in (0, 1))
    f, z = _sigmoid(g), _sigmoid(-g)
    a = f if s["flags"] is None else f * (s["flags"] == 0).to(F32)[:, :, None]
    u = z * v
    u[:, 0] += a[:, 0] * s["h0"]
    h = _scan(a, u)
    out = dict(y=h.to(BF).view(B * S, D), hT=h[:, -1].clone())
    if not s["bwd"]:
        return out
    before = torch.cat([s["h0"][:, None], h[:, :-1]], 1)
    if s["flags"] is not None:
        before = before * (s["flags"] == 0).to(F32)[:, :, None]
    d = s["dy"].to(F32).view(B, S, D).clone()
    d[:, -1] += s["dhT"]
    back = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    dh = _scan(back.flip(1), d.flip(1)).flip(1)
    out.update(dg=(dh * (before - v) * f * z).to(BF).view(B * S, D), dv=(dh * z).to(BF).view(B * S, D), dh0=a[:, 0] * dh[:, 0])
    return out


def _plain(s):
    kind = s["kind"]
    if kind == "linrec":
        return _plain_linrec(s)
    if kind == "ckpt":
        return _unpack(*_pack(s["x"])).to(s["x"].dtype)
    if kind == "swiglu_ckpt":
        F = s["F"]
        gu = s["gu"].to(F32)
        w = _unpack(*_pack(s["gu"]))
        g, u, d = w[:, :F], w[:, F:], s["dh"].to(F32)
        sg = _sigmoid(g)
        dg = d * u * (sg * (1.0 + g * (1.0 - sg)))
        return dict(h=(gu[:, :F] * _sigmoid(gu[:, :F]) * gu[:, F:]).to(BF), again=(g * sg * u).to(BF),
                    dgu=torch.cat([dg, d * (g * sg)], 1).to(BF))
    if kind == "norm":
        x = s["x"]
        out = {}
        if s["res"]:
            x = out["sum"] = (x.to(F32) + s["other"].to(F32)).to(x.dtype)
        v = x.to(F32)
        mean = v.mean(1, keepdim=True)
        d = v - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + 1e-6)
        y = d * rstd * s["gamma"].to(F32) + s["beta"].to(F32)
        out.update(y=y.to(x.dtype), mean=mean.view(-1), rstd=rstd.view(-1))
        return out
    x = _unpack(s["q"], s["e"]) if kind == "norm_ckpt_bwd" else s["x"].to(F32)
    dy, rstd = s["dy"].to(F32), s["rstd"][:, None]
    xh = (x - s["mean"][:, None]) * rstd
    w = dy * s["gamma"].to(F32)
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    if s["res"]:
        dx = dx + s["other"].to(F32)
    return dict(dx=dx.to(s["dy"].dtype), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))


# ---- the framework's calls ---------------------------------------------------------------------------------
def _buf(s, name, shape, dtype):
    """A buffer that the program keeps from pass to pass."""
    key = "out_" + name
    if key not in s:
        s[key] = torch.empty(shape, dtype=dtype, device="cuda")
    return s[key]


def _own(s):
    import paper_2609_17380_b200 as det
    kind = s["kind"]
    if kind == "linrec":
        B, S, D = s["B"], s["S"], s["D"]
        T = B * S
        g = s["gv"].data_ptr()
        y, hT = _buf(s, "y", (T, D), BF), _buf(s, "hT", (B, D), F32)
        states = _buf(s, "states", det.det_linrec_state_floats(B, S, D), F32) if s["bwd"] else None
        det.det_linrec_fwd(g, g + 2 * D, 2 * D, B, S, D, y, D, flags=s["flags"], h0=s["h0"], hT=hT, states=states)
        out = dict(y=y, hT=hT)
        if s["bwd"]:
            dgv = _buf(s, "dgv", (T, 2 * D), BF)
            d, dh0 = dgv.data_ptr(), _buf(s, "dh0", (B, D), F32)
            det.det_linrec_bwd(s["dy"], D, g, g + 2 * D, 2 * D, B, S, D, states, d, d + 2 * D, 2 * D, flags=s["flags"], dhT=s["dhT"], dh0=dh0)
            out.update(dg=dgv[:, :D], dv=dgv[:, D:], dh0=dh0)
        return out
    rows = s["rows"]
    if kind == "swiglu_ckpt":
        F = s["F"]
        q, e = _buf(s, "q", (rows, 2 * F), torch.int8), _buf(s, "e", (rows, 2 * F // GROUP), torch.uint8)
        h, again, dgu = _buf(s, "h", (rows, F), BF), _buf(s, "again", (rows, F), BF), _buf(s, "dgu", (rows, 2 * F), BF)
        det.det_swiglu_fwd_act8(s["gu"], rows, F, h, q, e)
        det.det_swiglu_act8(q, e, rows, F, again)
        det.det_swiglu_bwd_act8(s["dh"], q, e, rows, F, dgu)
        return dict(h=h, again=again, dgu=dgu)
    D, dt = s["D"], _type(s)
    io = det.DET_F32 if dt == F32 else det.DET_BF16
    if kind == "ckpt":
        q, e = _buf(s, "q", (rows, D), torch.int8), _buf(s, "e", (rows, (D + GROUP - 1) // GROUP), torch.uint8)
        y = _buf(s, "y", (rows, D), dt)
        det.det_act8_pack(io, s["x"], D, rows, D, q, e)
        det.det_act8_unpack(io, q, e, rows, D, y, D)
        return y
    if kind == "norm":
        y, mean, rstd = _buf(s, "y", (rows, D), dt), _buf(s, "mean", rows, F32), _buf(s, "rstd", rows, F32)
        if s["res"]:
            total = _buf(s, "sum", (rows, D), dt)
            det.det_residual_layernorm_fwd(s["x"], s["other"], s["gamma"], s["beta"], rows, D, 1e-6, total, y, mean, rstd)
            return dict(sum=total, y=y, mean=mean, rstd=rstd)
        det.det_layernorm_fwd(io, s["x"], s["gamma"], s["beta"], rows, D, 1e-6, y, mean, rstd)
        return dict(y=y, mean=mean, rstd=rstd)
    dx, dgamma, dbeta = _buf(s, "dx", (rows, D), dt), _buf(s, "dgamma", D, F32), _buf(s, "dbeta", D, F32)
    ws = _buf(s, "ws", det.det_layernorm_bwd_ws_bytes(rows, D), torch.uint8)
    if kind == "norm_ckpt_bwd":
        det.det_layernorm_bwd_act8(s["dy"], s["q"], s["e"], s["gamma"], s["mean"], s["rstd"], rows, D, s["other"], dx, dgamma, dbeta, ws)
    elif s["res"]:
        det.det_layernorm_bwd_residual(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], rows, D, s["other"], dx, dgamma, dbeta, ws)
    else:
        det.det_layernorm_bwd(io, s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], rows, D, dx, dgamma, dbeta, ws)
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "linrec":
        n, rows = case["B"] * case["S"] * case["D"], case["B"] * case["D"]
        flags = case["B"] * case["S"] if case["reset"] else 0
        # forward: gate and value in, output out; backward: gate, value and dy in, two gradients out; the states at the ends in f32
        return dict(bytes=n * (16 if case["bwd"] else 6) + rows * (16 if case["bwd"] else 8) + flags * (2 if case["bwd"] else 1),
                    flops=n * (60 if case["bwd"] else 25))
    if kind == "swiglu_ckpt":
        n = case["rows"] * case["F"]
        kept = 2 * n + 2 * n // GROUP                                   # the checkpoint: written once, read by the two that use it
        return dict(bytes=14 * n + 3 * kept, flops=75 * n)
    n, size = case["rows"] * case["D"], 4 if case.get("dtype") == "f32" else 2
    groups = case["rows"] * ((case["D"] + GROUP - 1) // GROUP)
    if kind == "ckpt":
        return dict(bytes=2 * size * n + 2 * (n + groups), flops=5 * n)
    vec, stat = case["D"], 8 * case["rows"]
    if kind == "norm":
        return dict(bytes=n * size * (4 if case["res"] else 2) + 2 * vec * size + stat, flops=9 * n)
    x = n + groups if kind == "norm_ckpt_bwd" else n * size
    return dict(bytes=n * size * (3 if case["res"] else 2) + x + vec * size + 8 * vec + stat, flops=16 * n)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------
def _exact_kept(x):
    """The values that a checkpoint of x stands for."""
    rows, D = x.shape
    v = torch.nn.functional.pad(x.to(F64), (0, -D % GROUP)).view(rows, -1, GROUP)
    frac, exp = torch.frexp(v.abs().amax(2) / 127)                      # m / 127 = frac 2^exp with frac in [1/2, 1)
    exp = torch.where(frac == 0.5, exp - 1, exp).clamp(min=-126)        # the smallest E with m <= 127 * 2^E
    step = torch.ldexp(torch.ones_like(frac), exp)[:, :, None]
    return (torch.round(v / step) * step).view(rows, -1)[:, :D]


def _exact_linrec(s):
    B, S, D = s["B"], s["S"], s["D"]
    g, v = (s["gv"][:, i * D:(i + 1) * D].to(F64).view(B, S, D).transpose(0, 1).contiguous() for i in (0, 1))
    f, z = torch.sigmoid(g), torch.sigmoid(-g)
    keep = torch.ones(S, B, 1, dtype=F64, device=g.device) if s["flags"] is None else (s["flags"] == 0).to(F64).t()[:, :, None].contiguous()
    a, u = f * keep, z * v
    h, prev, y = s["h0"].to(F64), torch.empty_like(g), torch.empty_like(g)
    for t in range(S):
        prev[t] = h
        h = torch.addcmul(u[t], a[t], h)
        y[t] = h
    flat = lambda x: x.transpose(0, 1).reshape(B * S, D)
    out = dict(y=flat(y), hT=h)
    if not s["bwd"]:
        return out
    dy = s["dy"].to(F64).view(B, S, D).transpose(0, 1)
    carry, dh = s["dhT"].to(F64), y                                     # y is not needed any more
    out["y"] = out["y"].clone()
    for t in range(S - 1, -1, -1):
        torch.add(dy[t], carry, out=dh[t])
        carry = a[t] * dh[t]
    out.update(dg=flat(dh * (prev * keep - v) * f * z), dv=flat(dh * z), dh0=carry)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "linrec":
        return _exact_linrec(s)
    if kind == "ckpt":
        return _exact_kept(s["x"])
    if kind == "swiglu_ckpt":
        F = case["F"]

        def silu(w):
            return w[:, :F] * torch.sigmoid(w[:, :F])
        gu, w, d = s["gu"].to(F64), _exact_kept(s["gu"]), s["dh"].to(F64)
        sg = torch.sigmoid(w[:, :F])
        dg = d * w[:, F:] * sg * (1 + w[:, :F] * torch.sigmoid(-w[:, :F]))
        return dict(h=silu(gu) * gu[:, F:], again=silu(w) * w[:, F:], dgu=torch.cat([dg, d * silu(w)], 1))
    gamma, eps = s["gamma"].to(F64), 1e-6
    if kind == "norm":
        x = s["x"].to(F64)
        out = {}
        if case["res"]:
            out["sum"] = x + s["other"].to(F64)
            x = out["sum"].to(s["x"].dtype).to(F64)                     # the rounded sum is what is normalised
        var, mean = torch.var_mean(x, 1, keepdim=True, correction=0)
        rstd = 1 / torch.sqrt(var + eps)
        out.update(y=(x - mean) * rstd * gamma + s["beta"].to(F64), mean=mean.view(-1), rstd=rstd.view(-1))
        return out
    if kind == "norm_ckpt_bwd":
        step = torch.ldexp(torch.ones(s["e"].shape, dtype=F64, device="cuda"), s["e"].to(torch.int32) - 127)
        x = s["q"].to(F64) * step.repeat_interleave(GROUP, 1)[:, :case["D"]]
    else:
        x = s["x"].to(F64)
    rstd = s["rstd"].to(F64)[:, None]
    xh = (x - s["mean"].to(F64)[:, None]) * rstd
    dy = s["dy"].to(F64)
    w = dy * gamma
    D = case["D"]
    dx = rstd * (w - w.sum(1, keepdim=True) / D - xh * ((w * xh).sum(1, keepdim=True) / D))
    if case["res"]:
        dx = dx + s["other"].to(F64)
    return dict(dx=dx, dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
