"""8-bit products with scales for each token and channel, the gated feed-forward block on them and AdamW with moments in 8 bits, as cases to
time, with their plain forms.

Sizes are those of the repository's configurations (the smoke step, the 1B-shaped decoder: 8192 tokens of 2048, feed-forward 8192), single
tokens through its layers, and odd or ragged sizes in between."""
import math
import random

import torch

own = False

BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
BLOCK = 256                   # values of a tensor that share the scales of their moments
LR, BETA1, BETA2, EPS, DECAY, STEP = 3e-4, 0.9, 0.95, 1e-8, 0.1, 20


def listed():
    return [
        # one token through a square projection of the 1B-shaped decoder
        dict(name="linear_token", kind="linear", M=1, N=2048, K=2048),
        # the tokens of a few sequences through its down projection: a long contraction for few rows
        dict(name="linear_few", kind="linear", M=24, N=2048, K=8192),
        # a micro-batch through its fused query, key and value projection
        dict(name="linear_step", kind="linear", M=8192, N=6144, K=2048),
        # ragged rows and odd widths, as an ablation of the width runs them, forward
        dict(name="linear_odd", kind="linear", M=1531, N=777, K=1003),
        # both gradients of the down projection for a micro-batch
        dict(name="linear_bwd_step", kind="linear_bwd", M=8192, N=2048, K=8192),
        # one token through the gated block
        dict(name="glu_token", kind="glu", M=1, F=8192, K=2048, keep=False),
        # a micro-batch through the gated block, gate and up kept for the backward pass
        dict(name="glu_step", kind="glu", M=8192, F=8192, K=2048, keep=True),
        # its backward pass: both gradients
        dict(name="glu_bwd_step", kind="glu_bwd", M=8192, F=8192, K=2048),
        # its backward pass for ragged rows and odd widths
        dict(name="glu_bwd_odd", kind="glu_bwd", M=1003, F=1369, K=520),
        # the update of the smoke step's layer: what a bisection of a mismatch calls over and over
        dict(name="adamw_small", kind="adamw", D=256, F=512, count=0, most=0, mix=0, clip=True),
        # the update of one layer of the 1B-shaped decoder
        dict(name="adamw_layer", kind="adamw", D=2048, F=8192, count=0, most=0, mix=0, clip=True),
        # many tensors of odd lengths, some with moments in 32 bits, without a clip coefficient
        dict(name="adamw_odd", kind="adamw", D=0, F=0, count=60, most=400000, mix=5, clip=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log(rng, lo, hi)
    return max(16, n // 16 * 16) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_bwd", "glu", "glu_bwd", "adamw"])
    if kind == "adamw":
        if rng.random() < 0.4:
            D = 128 * _log(rng, 1, 16)
            return dict(kind=kind, D=D, F=128 * _log(rng, 1, 64), count=0, most=0, mix=0, clip=rng.random() < 0.5)
        count = _log(rng, 1, 200)
        return dict(kind=kind, D=0, F=0, count=count, most=_log(rng, 1000, 40000000 // count), mix=rng.randrange(1 << 20), clip=rng.random() < 0.5)
    few = rng.random() < 0.4 and not kind.endswith("bwd")
    K = _width(rng, 16, 8192)
    M = _log(rng, 1, 128) if few else _log(rng, 1, 8192)
    if kind.startswith("glu"):
        F = min(_width(rng, 16, 8192), max(16, (1 << 37) // (M * K)))
        return dict(kind=kind, M=M, F=F, K=K, **(dict(keep=rng.random() < 0.5) if kind == "glu" else {}))
    return dict(kind=kind, M=M, N=min(_width(rng, 16, 16384), max(16, (1 << 38) // (M * K))), K=K)


# ---- inputs ------------------------------------------------------------------------------------------------
def _tensors(case):
    """The tensors of an update: (values, whether the moments are in 8 bits, whether the parameters are bf16, whether they decay)."""
    if case["count"]:
        rng = random.Random(case["mix"])
        return [(_log(rng, 1, case["most"]), rng.random() < 0.8, rng.random() < 0.8, rng.random() < 0.7) for _ in range(case["count"])]
    D, F = case["D"], case["F"]
    matrices = [(n, True, True, True) for n in (3 * D * D, D * D, 2 * F * D, D * F)]
    return matrices + [(D, False, True, False), (D, False, True, False), (4, False, False, False)]


def _codes(v, dim):
    """8-bit codes, as floats, of rows or columns of v, with a scale for each; in binary32 this has the definition's bits."""
    a = v.abs().amax(dim, keepdim=True)
    s = a / torch.full_like(a, 127.0)
    inv = torch.where(s > 0, torch.ones_like(s) / s, torch.zeros_like(s))
    return torch.round((v * inv).clamp(-127.0, 127.0)), s


def _laid_out(q):
    """Codes as bytes, rows 16-byte aligned with zeros behind their end."""
    return torch.nn.functional.pad(q, (0, -q.shape[1] % 16)).to(torch.int8).contiguous()


def _stream(gen, rows, width):
    """Rows as a residual stream has them: channels of different scale, a few large; some rows are padding, all zero."""
    x = torch.randn(rows, width, generator=gen, device="cuda")
    x *= torch.exp(0.7 * torch.randn(width, generator=gen, device="cuda"))
    if rows > 8:
        x *= (torch.rand(rows, 1, generator=gen, device="cuda") > 0.02)
    return x.to(BF)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    s = dict(case)
    kind = case["kind"]
    if kind == "adamw":
        s["tensors"] = _tensors(case)
        total = sum(n + -n % BLOCK for n, *_ in s["tensors"])
        # every value has its own scale of gradients, and a value in fifty has never had one
        size = torch.exp(1.5 * randn(total) - 8) * (torch.rand(total, generator=gen, device="cuda") > 0.02)
        flat = dict(p=0.02 * randn(total), g=size * randn(total), m=0.3 * size * randn(total), r=size * (0.5 + torch.rand(total, generator=gen, device="cuda")))
        at = 0
        for name in ("p", "g", "m", "v", "scales"):
            s[name] = []
        for n, eight, bf, _ in s["tensors"]:
            p, g, m, r = (flat[k][at:at + n].clone() for k in ("p", "g", "m", "r"))
            s["p"].append(p.to(BF) if bf else p)
            s["g"].append(g)
            if eight:
                m8, sm = _kept(_blocks([m]), 127)
                r8, sr = _kept(_blocks([r]), 255)
                s["m"].append(m8.view(-1)[:n].to(torch.int8).clone())
                s["v"].append(r8.view(-1)[:n].to(torch.uint8).clone())
                s["scales"].append(torch.cat([sm, sr], 1).contiguous())
            else:
                s["m"].append(m)
                s["v"].append(r * r)
                s["scales"].append(None)
            at += n + -n % BLOCK
        s["coef"] = torch.ones(1, device="cuda") if case["clip"] else None      # a step whose gradient norm is within the limit
        return s
    M, K = case["M"], case["K"]
    N = case["N"] if "N" in case else 2 * case["F"]
    qW, s_w = _codes((0.02 * randn(N, K)).to(BF).to(F32), 1)
    s["s_w"] = s_w.view(-1)
    x = _stream(gen, M, K)
    if not kind.endswith("bwd"):
        s["x"], s["qW"] = x, _laid_out(qW)
        return s
    qX, s_x = _codes(x.to(F32), 1)
    s["qX"], s["s_x"], s["qWt"] = _laid_out(qX), s_x.view(-1), _laid_out(qW.t())
    if kind == "linear_bwd":
        s["dy"] = (0.01 * _stream(gen, M, N).to(F32)).to(BF)
        return s
    s["dh"] = (0.01 * _stream(gen, M, case["F"]).to(F32)).to(BF)
    s["gu"] = ((qX @ qW.t()) * (s_x * s["s_w"])).to(BF)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------
def _product(a, b, scale):
    return (a @ b.t()) * scale


def _plain_linear_bwd(s, dy, N):
    K, x = s["K"], s["qX"][:, :s["K"]].to(F32)
    qa, sa = _codes(dy * s["s_w"], 1)
    qg, sg = _codes(dy * s["s_x"][:, None], 0)
    return dict(dx=_product(qa, s["qWt"][:, :N].to(F32), sa).to(BF), dw=_product(qg.t(), x.t(), sg.view(-1, 1)))


def _defined_sigmoid(g):
    """1 / (1 + e^-g) by the framework's steps in binary32: the bits matter where what follows from them is put into 8-bit codes."""
    x = -g
    k = torch.round(x * float.fromhex("0x1.715476p+0"))
    r = (x - k * float.fromhex("0x1.62e400p-1")) - k * float.fromhex("0x1.7f7d1cp-20")
    p = r * float.fromhex("0x1.a01a02p-13") + float.fromhex("0x1.6c16c2p-10")
    p = p * r + float.fromhex("0x1.111112p-7")
    p = p * r + float.fromhex("0x1.555556p-5")
    p = p * r + float.fromhex("0x1.555556p-3")
    p = p * r + 0.5
    p = p * r + 1.0
    p = p * r + 1.0
    e = p * ((k.clamp(-126, 127).to(torch.int32) + 127) << 23).view(F32)
    one = torch.ones_like(e)
    return one / (one + torch.where(x < float.fromhex("-0x1.5d58a0p+6"), torch.zeros_like(e), e))


def _blocks(tensors):
    return torch.cat([torch.nn.functional.pad(t.reshape(-1).to(F32), (0, -t.numel() % BLOCK)) for t in tensors]).view(-1, BLOCK)


def _kept(x, top):
    """Codes of the values of blocks by the root of their share of the block's largest, and the largest; a root that is not zero has a code of 1 at least."""
    s = x.abs().amax(1, keepdim=True)
    inv = torch.where(s > 0, torch.ones_like(s) / s, torch.zeros_like(s))
    c = torch.round(torch.sqrt(x.abs() * inv) * float(top)).clamp(max=float(top))
    if top == 255:
        return torch.where(x > 0, c.clamp(min=1.0), c), s
    return torch.where(x < 0, -c, c), s


def _worth(c, s, top):
    t = c * float(torch.tensor(1.0) / torch.tensor(float(top)))
    return s * (t * t.abs())


def _scalars():
    f = lambda x: float(torch.tensor(x, dtype=F32))
    b1, b2 = torch.tensor(BETA1, dtype=F32), torch.tensor(BETA2, dtype=F32)
    return dict(b1=float(b1), b2=float(b2), c1=float(1 - b1), c2=float(1 - b2), eps=f(EPS), size=f(LR / (1 - BETA1 ** STEP)),
                root=f(1 / math.sqrt(1 - BETA2 ** STEP)), keep=f(1 - LR * DECAY))


def _update(p, g, m, v, decay, h):
    m = m * h["b1"] + g * h["c1"]
    v = v * h["b2"] + (g * g) * h["c2"]
    r = torch.sqrt(v)
    return p * decay - (m / (r * h["root"] + h["eps"])) * h["size"], m, v, r


def _plain_adamw(s):
    h, whole, new = _scalars(), [t[1] for t in s["tensors"]], {}
    clip = (lambda g: g * s["coef"]) if s["coef"] is not None else (lambda g: g)
    count = [(t[0] + BLOCK - 1) // BLOCK for t in s["tensors"]]
    for eight in (True, False):                                       # all tensors with moments in 8 bits at once, then the others
        which = [i for i, w in enumerate(whole) if w == eight]
        if not which:
            continue
        rows = lambda name: _blocks([s[name][i] for i in which])
        sizes = [count[i] for i in which]
        decay = torch.cat([torch.full((c, 1), h["keep"] if s["tensors"][i][3] else 1.0, device="cuda") for i, c in zip(which, sizes)])
        m, v = rows("m"), rows("v")
        if eight:
            scales = torch.cat([s["scales"][i] for i in which])
            m, r = _worth(m, scales[:, :1], 127), _worth(v, scales[:, 1:], 255)
            v = r * r
        p, m, v, r = _update(rows("p"), clip(rows("g")), m, v, decay, h)
        if eight:
            m, r = _worth(*_kept(m, 127), 127), _worth(*_kept(r, 255), 255)
            v = r * r
        new.update(zip(which, zip(torch.split(p, sizes), torch.split(m, sizes), torch.split(v, sizes))))
    every = range(len(whole))
    out = {"p_%d" % (2 if bf else 4): [new[i][0] for i in every if s["tensors"][i][2] == bf] for bf in (True, False)}
    out.update(m=[new[i][1] for i in every], v=[new[i][2] for i in every])
    return {name: torch.cat(x).view(-1).to(BF if name == "p_2" else F32) for name, x in out.items() if x}


def _plain(s):
    kind, K = s["kind"], s["K"] if "K" in s else 0
    if kind == "adamw":
        return _plain_adamw(s)
    if kind == "linear_bwd":
        return _plain_linear_bwd(s, s["dy"].to(F32), s["N"])
    if kind == "glu_bwd":
        F = s["F"]
        g, u, d = s["gu"][:, :F].to(F32), s["gu"][:, F:].to(F32), s["dh"].to(F32)
        sg = _defined_sigmoid(g)
        dgu = torch.cat([(d * u) * (sg * (g * (1.0 - sg) + 1.0)), d * (g * sg)], 1).to(BF)
        return _plain_linear_bwd(s, dgu.to(F32), 2 * F)
    qx, sx = _codes(s["x"].to(F32), 1)
    y = _product(qx, s["qW"][:, :K].to(F32), sx * s["s_w"]).to(BF)
    if kind == "linear":
        return y
    g, u = y[:, :s["F"]].to(F32), y[:, s["F"]:].to(F32)
    h = (g / (1.0 + torch.exp(-g)) * u).to(BF)
    return dict(h=h, gu=y) if s["keep"] else h


# ---- the framework's calls ---------------------------------------------------------------------------------
def _buf(s, name, shape, dtype):
    """A buffer that the program keeps from pass to pass."""
    key = "out_" + name
    if key not in s:
        s[key] = torch.empty(shape, dtype=dtype, device="cuda")
    return s[key]


def _own_adamw(s):
    import paper_2609_17380_b200 as det
    if "outs" not in s:
        # a flat buffer for the parameters of each type and for each moment as numbers, every tensor at a multiple of a block
        tensors = s["tensors"]
        s["flat"], parts = {}, {}
        for name, which, dtype in (("p_2", [t[2] for t in tensors], BF), ("p_4", [not t[2] for t in tensors], F32), ("m", [True] * len(tensors), F32),
                                   ("v", [True] * len(tensors), F32)):
            sizes = [t[0] + -t[0] % BLOCK for t, w in zip(tensors, which) if w]
            if sizes:
                s["flat"][name] = torch.zeros(sum(sizes), dtype=dtype, device="cuda")
                split = iter(torch.split(s["flat"][name], sizes))
                parts[name] = [next(split)[:t[0]] if w else None for t, w in zip(tensors, which)]
        p = [parts["p_2" if t[2] else "p_4"][i] for i, t in enumerate(tensors)]
        new = lambda name, k: [torch.empty_like(x) if t[1] else parts[name][i] for i, (x, t) in enumerate(zip(s[k], tensors))]
        s["outs"] = (p, new("m", "m"), new("v", "v"), [None if x is None else torch.empty_like(x) for x in s["scales"]])
        s["numbers"] = [[x[i] for i, t in enumerate(tensors) if t[1]] for x in (*s["outs"][1:], parts["m"], parts["v"])]
        s["descs"] = [det.det_adamw_desc(LR, BETA1, BETA2, EPS, DECAY if t[3] else 0.0, STEP) for t in tensors]
        s["kinds"] = [det.DET_BF16 if t[2] else det.DET_F32 for t in tensors]
    det.det_adamw8_batch(s["descs"], s["kinds"], s["p"], s["g"], s["m"], s["v"], s["scales"], s["coef"], outs=s["outs"])
    det.det_adamw8_unpack(*s["numbers"])
    return s["flat"]


def _own(s):
    import paper_2609_17380_b200 as det
    kind = s["kind"]
    if kind == "adamw":
        return _own_adamw(s)
    M, K = s["M"], s["K"]
    if kind.endswith("bwd"):
        N = s["N"] if kind == "linear_bwd" else 2 * s["F"]
        dx, dw = _buf(s, "dx", (M, K), BF), _buf(s, "dw", (N, K), F32)
        if kind == "linear_bwd":
            ws = _buf(s, "ws", det.det_tok8_linear_bwd_ws_bytes(M, N, K), torch.uint8)
            det.det_tok8_linear_bwd(s["dy"], N, s["qX"], s["s_x"], s["qWt"], s["s_w"], M, N, K, dx, K, dw, ws)
        else:
            ws = _buf(s, "ws", det.det_tok8_glu_bwd_ws_bytes(M, s["F"], K), torch.uint8)
            det.det_tok8_glu_bwd(s["dh"], s["F"], s["gu"], N, s["qX"], s["s_x"], s["qWt"], s["s_w"], M, s["F"], K, dx, K, dw, ws)
        return dict(dx=dx, dw=dw)
    # the codes of the tokens and their scales stay for the backward pass
    qx, sx = _buf(s, "qx", (M, det.det_tok8_ld(K)), torch.int8), _buf(s, "sx", M, F32)
    if kind == "linear":
        y = _buf(s, "y", (M, s["N"]), BF)
        det.det_tok8_linear_fwd(s["x"], K, s["qW"], s["s_w"], M, s["N"], K, y, s["N"], qx, sx)
        return y
    F = s["F"]
    h, gu = _buf(s, "h", (M, F), BF), _buf(s, "gu", (M, 2 * F), BF) if s["keep"] else None
    det.det_tok8_glu_fwd(s["x"], K, s["qW"], s["s_w"], M, F, K, h, F, gu, 2 * F, qx, sx)
    return dict(h=h, gu=gu) if s["keep"] else h


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "adamw":
        total = {True: 0, False: 0}
        bytes_ = 0
        for n, eight, bf, _ in _tensors(case):
            total[eight] += n
            # parameters in and out, gradient in (and out, clipped), moments in and out; 8-bit moments as numbers besides
            bytes_ += n * ((4 if bf else 8) + (8 if case["clip"] else 4) + (4 + 2 + 8 if eight else 16))
        return dict(bytes=bytes_ + total[True] // BLOCK * 16, flops=40 * total[True] + 15 * total[False])
    M, K = case["M"], case["K"]
    N = case["N"] if "N" in case else 2 * case["F"]
    if kind == "linear":
        return dict(bytes=2 * M * K + N * K + 4 * N + 2 * M * N, flops=2 * M * N * K)
    if kind == "linear_bwd":
        return dict(bytes=2 * M * N + M * K + N * K + 4 * (M + N) + 2 * M * K + 4 * N * K, flops=4 * M * N * K)
    F = case["F"]
    if kind == "glu":
        return dict(bytes=2 * M * K + N * K + 4 * N + 2 * M * F + (4 * M * F if case["keep"] else 0), flops=2 * M * N * K)
    return dict(bytes=6 * M * F + M * K + N * K + 4 * (M + N) + 2 * M * K + 4 * N * K, flops=4 * M * N * K)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------
def _exact_codes(v, dim):
    """The codes are defined through binary32 numbers: the scale, its reciprocal and the product with it, each the nearest one."""
    near = lambda x: x.to(F32).to(F64)
    s = near(v.abs().amax(dim, keepdim=True) / 127)
    inv = near(1 / s).masked_fill(s == 0, 0.0)
    return torch.round(near(v * inv).clamp(-127, 127)), s


def _exact_linear_bwd(s, dy, N):
    near = lambda x: x.to(F32).to(F64)
    qa, sa = _exact_codes(near(dy * s["s_w"].to(F64)), 1)
    qg, sg = _exact_codes(near(dy * s["s_x"].to(F64)[:, None]), 0)
    return dict(dx=torch.einsum("mn,kn->mk", qa, s["qWt"][:, :N].to(F64)) * sa,
                dw=torch.einsum("mn,mk->nk", qg, s["qX"][:, :s["K"]].to(F64)) * sg.view(-1, 1))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "adamw":
        # the moments are codes that follow from binary32 numbers: they have no value in 64 bits, the parameters do
        ps = {"p_2": [], "p_4": []}
        for i, (n, eight, bf, decays) in enumerate(s["tensors"]):
            g, p = s["g"][i].to(F64), s["p"][i].to(F64)
            m, v = s["m"][i].to(F64), s["v"][i].to(F64)
            if eight:
                sm, sr = (s["scales"][i][:, k].to(F64).repeat_interleave(BLOCK)[:n] for k in (0, 1))
                m, v = sm * torch.sign(m) * (m / 127).square(), (sr * (v / 255).square()).square()
            m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
            step = (m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
            p = p * (1 - LR * (DECAY if decays else 0.0)) - LR * step
            ps["p_2" if bf else "p_4"].append(torch.nn.functional.pad(p, (0, -n % BLOCK)))
        return dict({name: torch.cat(x) for name, x in ps.items() if x}, m=None, v=None)
    if kind == "linear_bwd":
        return _exact_linear_bwd(s, s["dy"].to(F64), case["N"])
    if kind == "glu_bwd":
        F = case["F"]
        g, u, d = s["gu"][:, :F].to(F64), s["gu"][:, F:].to(F64), s["dh"].to(F64)
        f = torch.sigmoid(g)
        dgu = torch.cat([d * u * f * (1 + g * torch.sigmoid(-g)), d * g * f], 1).to(BF).to(F64)
        # the weights' gradient in binary32 is finer than what the codes of a rounded gradient leave undecided: no value in 64 bits
        return dict(_exact_linear_bwd(s, dgu, 2 * F), dw=None)
    qx, sx = _exact_codes(s["x"].to(F64), 1)
    y = torch.einsum("mk,nk->mn", qx, s["qW"][:, :case["K"]].to(F64)) * (sx * s["s_w"].to(F64))
    if kind == "linear":
        return y
    kept = y.to(BF).to(F64)                                           # gate and up are rounded before the activation
    g, u = kept[:, :case["F"]], kept[:, case["F"]:]
    h = g * torch.sigmoid(g) * u
    return dict(h=h, gu=y) if case["keep"] else h
