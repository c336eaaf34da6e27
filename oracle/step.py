"""Oracle-side replay of one full training step (TEST INFRASTRUCTURE ONLY).

Plain numpy orchestration of the oracle's C functions in the order the paper states a step: forward,
gradient, reduction of the micro-batch gradients in the cluster's order (Algorithm 1 + 2), clip, AdamW,
hash.  Written independently of the CUDA-side driver; they share only the seeded inputs.
"""
import numpy as np

import oracle as O
from oracle import v2 as O2

LINEARS = ("w_qkv", "w_o", "w_gu", "w_down")


def _kv(cfg):
    return cfg.get("n_kv_heads") or cfg["n_heads"]


def _window(cfg, l):
    """Sliding-window layers (Sec. 3.1): every `full_every`-th layer and the last one attend to everything."""
    W = cfg.get("window", 0)
    if not W or l == cfg["n_layers"] - 1 or (l + 1) % cfg.get("full_every", 5) == 0:
        return 0
    return W


def _specs(cfg):
    D, Fh, V, L = cfg["d_model"], cfg["ffn"], cfg["vocab"], cfg["n_layers"]
    nq = D + 2 * 128 * _kv(cfg)
    shift = ("", "_shift") if _layer(cfg) else ("",)
    norm = lambda name: [(name + part, (D,)) for part in shift]
    s = [("embed", (V, D))]
    if cfg.get("embed_norm"):
        s += norm("embed_norm")
    for l in range(L):
        s += norm("l%d.attn_norm" % l) + [("l%d.w_qkv" % l, (2 * D if _recurrent(cfg, l) else nq, D)), ("l%d.w_o" % l, (D, D))]
        s += norm("l%d.ffn_norm" % l) + [("l%d.w_gu" % l, (2 * Fh, D)), ("l%d.w_down" % l, (D, Fh))]
        s += [] if _by_token(cfg) else [("l%d.s_x" % l, (4,))]
    return s + norm("final_norm") + [("lm_head", (V, D))]


def _layer(cfg):
    return cfg.get("norm", "rms") == "layer"


def _by_token(cfg):
    """Linears whose scales follow the values, by token and output channel, in place of the learned steps."""
    return cfg.get("linear", "lsq") == "token"


def _linear(cfg, P, sw, l, w, i, x):
    name = "l%d.%s" % (l, w)
    if _by_token(cfg):
        return O.tok8_linear_fwd(x, P[name])[0]
    return O.linear_fwd(x, P[name], P["l%d.s_x" % l][i:i + 1], sw[name])[0]


def _linear_bwd(cfg, P, G, ds, sw, l, w, i, dy, x):
    """The gradient of the linear's input; the weights' goes to G, the step's to ds."""
    name = "l%d.%s" % (l, w)
    if _by_token(cfg):
        dx, G[name] = O.tok8_linear_bwd(dy, x, P[name])
        return dx
    dx, G[name], d = O.linear_bwd(dy, x, P[name], P["l%d.s_x" % l][i:i + 1], sw[name], cfg.get("hadamard_block", 128))
    ds[i] = d[0]
    return dx


def _recurrent(cfg, l):
    return l in cfg.get("recurrent", ())


def _norm(cfg, P, name, x):
    """The norm's output and its statistics (mean, rstd; no mean for RMSNorm)."""
    if _layer(cfg):
        y, mean, rstd = O.layernorm_fwd(x, P[name], P[name + "_shift"], 1e-6, bf=True)
        return y, (mean, rstd)
    y, rstd = O.rmsnorm_fwd(x, P[name], 1e-6, bf=True)
    return y, (None, rstd)


def _norm_bwd(cfg, P, G, name, dy, x, stat, past=None):
    """Gradient of the norm's input, with that of what bypasses it (past) added; gain's and shift's go to G."""
    if _layer(cfg):
        dx, G[name], G[name + "_shift"] = O.layernorm_bwd(dy, x, P[name], stat[0], stat[1], past, bf=True)
        return dx
    dx, G[name] = O.rmsnorm_bwd(dy, x, P[name], stat[1], bf=True)
    return dx if past is None else O.residual_add(past, dx)


def _kept(cfg, x):
    """What the backward pass has of an activation: itself, or what its 8-bit checkpoint stands for."""
    return O.act8_unpack(*O.act8_pack(x)) if cfg.get("act8") else x


def _attention(cfg, l, a, rope):
    H, S, B, D, Hkv = cfg["n_heads"], cfg["seq"], cfg["micro_batch"], cfg["d_model"], _kv(cfg)
    # the paper's block: gain-free RMS norm of every query and key head, then the rotary embedding
    qk = np.ascontiguousarray(a["qkv"][:, :D + 128 * Hkv]).reshape(-1, 128)
    if cfg.get("qk_norm"):
        a["qk_pre"] = qk
        qk, a["rstd_qk"] = O.rmsnorm_fwd(qk, None, 1e-6, bf=True)
    if rope is not None:
        qk = O.rope(qk.reshape(B * S, H + Hkv, 128), S, rope[0], rope[1]).reshape(-1, 128)
    a["qkr"] = np.ascontiguousarray(np.concatenate([qk.reshape(B * S, -1), a["qkv"][:, D + 128 * Hkv:]], 1))
    a["att"], a["lse"] = O.attn_fwd(a["qkr"], B, H, S, Hkv=Hkv, window=_window(cfg, l), int8_pv=bool(cfg.get("pv_int8")))


def forward(cfg, P, sw, tok, calibrate=False):
    """Returns (saved activations, loss pieces).  With calibrate, every activation step is set from its input."""
    L, S, B = cfg["n_layers"], cfg["seq"], cfg["micro_batch"]
    inp = tok[:, :-1].reshape(-1)
    x = O.embed_fwd(inp, P["embed"])
    saved = {"inp": inp, "layers": []}
    if cfg.get("embed_norm"):
        saved["x_emb"] = x
        x, saved["stat_emb"] = _norm(cfg, P, "embed_norm", x)
    rope = cfg.get("rope_tables")
    for l in range(L):
        sx = P.get("l%d.s_x" % l)
        a = {"x": x}
        a["n1"], a["stat1"] = _norm(cfg, P, "l%d.attn_norm" % l, x)
        if calibrate:
            sx[0] = O.lsq_act_scale_init(a["n1"])[0]
        a["qkv"] = _linear(cfg, P, sw, l, "w_qkv", 0, a["n1"])
        if _recurrent(cfg, l):
            a["att"], _, a["states"] = O.linrec_fwd(a["qkv"], B, S)
        else:
            _attention(cfg, l, a, rope)
        if calibrate:
            sx[1] = O.lsq_act_scale_init(a["att"])[0]
        o = _linear(cfg, P, sw, l, "w_o", 1, a["att"])
        a["h"] = O.residual_add(x, o)
        a["n2"], a["stat2"] = _norm(cfg, P, "l%d.ffn_norm" % l, a["h"])
        if calibrate:
            sx[2] = O.lsq_act_scale_init(a["n2"])[0]
        a["gu"] = _linear(cfg, P, sw, l, "w_gu", 2, a["n2"])
        a["act"] = O.swiglu_fwd(a["gu"])
        if calibrate:
            sx[3] = O.lsq_act_scale_init(a["act"])[0]
        dn = _linear(cfg, P, sw, l, "w_down", 3, a["act"])
        x = O.residual_add(a["h"], dn)
        saved["layers"].append(a)
    saved["xf"] = x
    saved["nf"], saved["statf"] = _norm(cfg, P, "final_norm", x)
    # arithmetic version 2 (cfg["arith"] == 2) replaces the LM-head contractions by the order-free ones of oracle/v2
    saved["logits"] = (O2 if cfg.get("arith", 1) == 2 else O).lmhead_fwd(saved["nf"], P["lm_head"])
    return saved


def _attention_bwd(cfg, l, a, d_att, rope):
    H, S, B, D, Hkv = cfg["n_heads"], cfg["seq"], cfg["micro_batch"], cfg["d_model"], _kv(cfg)
    d_qkv = O.attn_bwd(d_att, a["qkr"], a["att"], a["lse"], B, H, S, Hkv=Hkv, window=_window(cfg, l),
                       fixq=bool(cfg.get("dq_fixed")))
    dqk = np.ascontiguousarray(d_qkv[:, :D + 128 * Hkv]).reshape(-1, 128)
    if rope is not None:
        dqk = O.rope(dqk.reshape(B * S, H + Hkv, 128), S, rope[0], rope[1], inverse=True).reshape(-1, 128)
    if cfg.get("qk_norm"):
        dqk, _ = O.rmsnorm_bwd(dqk, a["qk_pre"], None, a["rstd_qk"], bf=True)
    return np.ascontiguousarray(np.concatenate([dqk.reshape(B * S, -1), d_qkv[:, D + 128 * Hkv:]], 1))


def microbatch_grad(cfg, P, sw, tok):
    """Forward + backward of one micro-batch; returns (flat f32 gradient in canonical order, mean loss)."""
    L, S, B = cfg["n_layers"], cfg["seq"], cfg["micro_batch"]
    rope = cfg.get("rope_tables")
    sv = forward(cfg, P, sw, tok)
    labels = tok[:, 1:].reshape(-1).astype(np.int32)
    T = labels.size
    _, lse, loss_mean, _, _ = O.xent_fwd(sv["logits"], labels, cfg.get("z_weight", 0.0))
    dlog = O.xent_bwd(sv["logits"], labels, lse, cfg.get("z_weight", 0.0), np.float32(1.0 / T))
    G = {}
    d_nf, G["lm_head"] = (O2 if cfg.get("arith", 1) == 2 else O).lmhead_bwd(dlog, sv["nf"], P["lm_head"])
    dx = _norm_bwd(cfg, P, G, "final_norm", d_nf, sv["xf"], sv["statf"])
    for l in reversed(range(L)):
        a = sv["layers"][l]
        ds = np.zeros(4, np.float32)
        gu = _kept(cfg, a["gu"])
        act = O.swiglu_fwd(gu) if cfg.get("act8") else a["act"]         # made again from what was kept
        d_act = _linear_bwd(cfg, P, G, ds, sw, l, "w_down", 3, dx, act)
        d_gu = O.swiglu_bwd(d_act, gu)
        d_n2 = _linear_bwd(cfg, P, G, ds, sw, l, "w_gu", 2, d_gu, a["n2"])
        d_h = _norm_bwd(cfg, P, G, "l%d.ffn_norm" % l, d_n2, _kept(cfg, a["h"]), a["stat2"], dx)
        d_att = _linear_bwd(cfg, P, G, ds, sw, l, "w_o", 1, d_h, a["att"])
        if _recurrent(cfg, l):
            d_qkv, _ = O.linrec_bwd(d_att, _kept(cfg, a["qkv"]), a["states"], B, S)
        else:
            d_qkv = _attention_bwd(cfg, l, a, d_att, rope)
        d_n1 = _linear_bwd(cfg, P, G, ds, sw, l, "w_qkv", 0, d_qkv, a["n1"])
        dx = _norm_bwd(cfg, P, G, "l%d.attn_norm" % l, d_n1, _kept(cfg, a["x"]), a["stat1"], d_h)
        if not _by_token(cfg):
            G["l%d.s_x" % l] = ds
    if cfg.get("embed_norm"):
        dx = _norm_bwd(cfg, P, G, "embed_norm", dx, sv["x_emb"], sv["stat_emb"])
    G["embed"] = O.embed_bwd(sv["inp"], dx, cfg["vocab"])
    flat = np.concatenate([np.asarray(G[name], np.float32).reshape(-1) for name, _ in _specs(cfg)])
    return flat, float(loss_mean[0])


def run_step(cfg, params, tokens, opt=None, calibrate=True):
    """One optimizer step.  cfg: dict (n_layers, d_model, n_heads, ffn, vocab, seq, micro_batch, mesh=(accum,
    dp_shard, dp_replicate), optional hadamard_block, z_weight, lr, betas, eps, wd, clip, step; the paper's block:
    n_kv_heads, qk_norm, rope_tables=(cos, sin) f32 [seq, 64], embed_norm, window, full_every; other blocks: norm = "layer", recurrent = layers
    with the gated linear recurrence, act8 = activations in 8 bits for the backward pass, linear = "token" = linears with token and channel scales, state8 =
    moments of the matrices in 8 bits).
    params: dict name -> numpy (uint16 bf16 bits / float32 steps).  tokens: [n_mb, micro_batch, seq+1]."""
    P = {k: np.array(v, copy=True) for k, v in params.items()}
    specs = _specs(cfg)
    accum, shard, rep = cfg["mesh"]
    assert tokens.shape[0] == accum * shard * rep
    sw = {}
    for l in range(cfg["n_layers"] if not _by_token(cfg) else 0):
        for w in LINEARS:
            sw["l%d.%s" % (l, w)] = O.lsq_weight_scale(P["l%d.%s" % (l, w)])
    if calibrate and not _by_token(cfg):
        forward(cfg, P, sw, tokens[0], calibrate=True)
    n = sum(int(np.prod(s)) for _, s in specs)
    acc = O.Accum(accum, shard, rep, n)
    losses = []
    for mb in range(tokens.shape[0]):
        g, loss = microbatch_grad(cfg, P, sw, tokens[mb])
        acc.push(g)
        losses.append(loss)
    g = acc.result()
    offs = np.cumsum([0] + [int(np.prod(s)) for _, s in specs])
    views = [g[offs[i]:offs[i + 1]] for i in range(len(specs))]
    norm, coef = O.grad_norm(views, cfg.get("clip", 1.0))
    g = O.scale(g, coef)
    # with state8 the moments of the matrices are codes and scales, one tensor's behind the other's; the others' are in 32 bits, likewise
    eight = [bool(cfg.get("state8")) and len(shape) > 1 for _, shape in specs]
    size = [int(np.prod(shape)) for _, shape in specs]
    if opt is None:
        n32, n8 = sum(k for k, e in zip(size, eight) if not e), [k for k, e in zip(size, eight) if e]
        opt = {"m": np.zeros(n32, np.float32), "v": np.zeros(n32, np.float32), "m8": np.zeros(sum(n8), np.int8), "v8": np.zeros(sum(n8), np.uint8),
               "s": np.zeros((sum(-(-k // O.ADAMW8_BLOCK) for k in n8), 2), np.float32)}
    st = {k: x.copy() for k, x in opt.items()}
    lr, (b1, b2), eps, wd, t = cfg.get("lr", 3e-4), cfg.get("betas", (0.9, 0.95)), cfg.get("eps", 1e-8), cfg.get("wd", 0.1), cfg.get("step", 1)
    hashes, at32, at8, ats = {}, 0, 0, 0
    for i, (name, shape) in enumerate(specs):
        sl, k = slice(offs[i], offs[i + 1]), size[i]
        decay = wd if (name == "lm_head" or name.split(".")[-1] in LINEARS) else 0.0
        if eight[i]:
            c, b = slice(at8, at8 + k), slice(ats, ats + -(-k // O.ADAMW8_BLOCK))
            p, st["m8"][c], st["v8"][c], st["s"][b] = O.adamw8(P[name].reshape(-1), g[sl], st["m8"][c], st["v8"][c], st["s"][b], lr, b1, b2, eps, decay, t)
            at8, ats = c.stop, b.stop
        else:
            c = slice(at32, at32 + k)
            p, st["m"][c], st["v"][c] = O.adamw(P[name].reshape(-1), g[sl], st["m"][c], st["v"][c], lr, b1, b2, eps, decay, t)
            at32 = c.stop
        P[name] = p.reshape(shape)
        hashes[name] = O.tensor_hash(P[name])
    hashes["grad"] = O.tensor_hash(g)
    hashes["adam_m"], hashes["adam_v"] = O.tensor_hash(st["m"]), O.tensor_hash(st["v"])
    if cfg.get("state8"):
        hashes.update(adam_m8=O.tensor_hash(st["m8"]), adam_v8=O.tensor_hash(st["v8"]), adam_scales=O.tensor_hash(st["s"]))
    return {"params": P, "m": st["m"], "v": st["v"], "opt": st, "grad": g, "loss": float(np.mean(losses)), "losses": losses,
            "grad_norm": float(norm), "coef": float(coef), "hashes": hashes}
