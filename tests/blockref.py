"""Layer norm, 8-bit checkpoints and the gated linear recurrence in 64 bits, with bounds on how far the binary32 definition may be
off (u = 2^-24, half a step of binary32 relative to the value; a bf16 output adds 2^-8 of it)."""
import numpy as np

import synth

U, UBF = 2.0 ** -24, 2.0 ** -8


def wide(x):
    """float64 of bf16 bit patterns (uint16) or of float32."""
    return (synth.from_bf16(x) if x.dtype == np.uint16 else x).astype(np.float64)


def layernorm(x, gamma, beta, eps):
    """y, mean, rstd and the bound on y's error before its last rounding.  The mean is a tree of depth n = log2 D and one product: off by
    (n + 2) u mean|x|.  d = x - mean adds its own rounding.  The variance is a tree of n + 2 roundings over squares of d, whose errors count twice, and
    1/sqrt halves that and adds three roundings: rstd is off by (n + 6) u + max err(d) / sigma relative to itself."""
    x, D = wide(x), x.shape[1]
    n = np.ceil(np.log2(D)) + 2
    mean = x.mean(1, keepdims=True)
    d = x - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    err_mean = (n + 1) * U * np.abs(x).mean(1, keepdims=True)
    err_d = err_mean + U * np.abs(d)
    rel = (n + 6) * U + err_d.max(1, keepdims=True) * rstd
    g = 1.0 if gamma is None else wide(gamma)
    b = 0.0 if beta is None else wide(beta)
    y = d * rstd * g + b
    err = np.abs(g) * rstd * (err_d + np.abs(d) * (rel + 3 * U)) + 2 * U * (np.abs(y) + np.abs(b))
    return dict(y=y, mean=mean[:, 0], rstd=rstd[:, 0], err_y=err, err_mean=err_mean[:, 0], err_rstd=(rel * rstd)[:, 0])


def layernorm_bwd(dy, x, gamma, mean, rstd, res=None):
    """dx, dgamma, dbeta for the given statistics and bounds: xhat is off by 2 u, w by u, c1 and c2 by a tree of depth n and what goes in."""
    dy, x, mean, rstd = wide(dy), wide(x), mean.astype(np.float64)[:, None], rstd.astype(np.float64)[:, None]
    rows, D = x.shape
    n, nr = np.ceil(np.log2(D)) + 2, np.ceil(np.log2(max(rows, 2)))
    xh = (x - mean) * rstd
    w = dy * (1.0 if gamma is None else wide(gamma))
    c1, c2 = w.mean(1, keepdims=True), (w * xh).mean(1, keepdims=True)
    e1 = (n + 2) * U * np.abs(w).mean(1, keepdims=True)
    e2 = (n + 5) * U * np.abs(w * xh).mean(1, keepdims=True)
    dx = rstd * (w - c1 - xh * c2)
    err = rstd * (e1 + np.abs(xh) * e2 + U * (4 * np.abs(w) + 3 * np.abs(c1) + 6 * np.abs(xh * c2)))
    if res is not None:
        dx = dx + wide(res)
        err = err + U * np.abs(dx)
    prod = dy * xh
    return dict(dx=dx, err_dx=err, dgamma=prod.sum(0), err_dgamma=(nr + 4) * U * np.abs(prod).sum(0), dbeta=dy.sum(0),
                err_dbeta=(nr + 1) * U * np.abs(dy).sum(0))


def act8(x):
    """The values that a checkpoint of x stands for, and the steps."""
    x = wide(x)
    out, steps = np.empty_like(x), np.empty_like(x)
    for lo in range(0, x.shape[1], 32):
        v = x[:, lo:lo + 32]
        m = np.abs(v).max(1, keepdims=True)
        E = np.ceil(np.log2(np.maximum(m, 2.0 ** -200) / 127))
        E += m > 127 * 2.0 ** E                  # log2 rounds
        E -= m <= 127 * 2.0 ** (E - 1)
        step = 2.0 ** np.maximum(E, -126)
        out[:, lo:lo + 32], steps[:, lo:lo + 32] = np.rint(v / step) * step, step
    return out, steps


def _gate(g):
    e = np.exp(-np.abs(g))
    m = e / (1 + e)
    return np.where(g >= 0, 1 - m, m), np.where(g >= 0, m, 1 - m)


def linrec(gv, B, S, flags=None, h0=None):
    """h, hT and bounds.  A gate is off by at most 12 u of itself (its exponential by 8 u, a division, a difference to 1 that is at least a half), a
    product and a sum per row, the composition of spans less than two roundings a row more: every row adds 16 u of what it handles."""
    D = gv.shape[1] // 2
    gv = wide(gv).reshape(B, S, 2 * D)
    f, z = _gate(gv[..., :D])
    u = z * gv[..., D:]
    keep = np.ones((B, S, 1)) if flags is None else (np.asarray(flags).reshape(B, S, 1) == 0)
    s = np.zeros((B, D)) if h0 is None else h0.astype(np.float64)
    mag, err = np.abs(s), np.zeros((B, D))
    h, prev, errs = np.empty_like(u), np.empty_like(u), np.empty_like(u)
    for t in range(S):
        prev[:, t] = np.where(keep[:, t], s, 0)
        a = np.where(keep[:, t], f[:, t], 0.0)
        err = a * err + 16 * U * (a * mag + np.abs(u[:, t]))
        mag = a * mag + np.abs(u[:, t])
        s = np.where(keep[:, t], f[:, t] * s, 0) + u[:, t]
        h[:, t], errs[:, t] = s, err
    return dict(h=h.reshape(B * S, D), err_h=errs.reshape(B * S, D), hT=s, err_hT=err, prev=prev, f=f, z=z, keep=keep)


def linrec_bwd(dy, gv, B, S, flags=None, h0=None, dhT=None):
    """dg, dv, dh0 and bounds: the gradient of the state grows errors as the state does; a product or two for each output."""
    D = gv.shape[1] // 2
    r = linrec(gv, B, S, flags, h0)
    f, z, keep, prev = r["f"], r["z"], r["keep"], r["prev"]
    v = wide(gv).reshape(B, S, 2 * D)[..., D:]
    dy = wide(dy).reshape(B, S, D)
    c = np.zeros((B, D)) if dhT is None else dhT.astype(np.float64)
    mag, err = np.abs(c), np.zeros((B, D))
    dh, errs = np.empty_like(dy), np.empty_like(dy)
    for t in range(S - 1, -1, -1):
        dh[:, t] = dy[:, t] + c
        err = err + 2 * U * (np.abs(dy[:, t]) + mag)
        mag = mag + np.abs(dy[:, t])
        errs[:, t] = err
        a = np.where(keep[:, t], f[:, t], 0.0)
        c, err, mag = a * dh[:, t], a * err + 16 * U * a * mag, a * mag
    err_prev = np.concatenate([np.zeros((B, 1, D)), r["err_h"].reshape(B, S, D)[:, :-1]], 1)
    fz, diff = f * z, prev - v
    dg, dv = dh * diff * fz, dh * z
    err_dg = fz * (errs * np.abs(diff) + np.abs(dh) * (err_prev + U * np.abs(diff))) + 30 * U * np.abs(dg)
    out = lambda x: x.reshape(B * S, D)
    return dict(dg=out(dg), err_dg=out(err_dg), dv=out(dv), err_dv=out(errs * z + 16 * U * np.abs(dv)), dh0=c, err_dh0=err)


def close(got, want, err, bf=False, what=""):
    """|got - want| within the bound, with the last rounding of a bf16 output; results below 2^-126 flush to zero."""
    got = wide(got) if got.dtype == np.uint16 else np.asarray(got, np.float64)
    tol = err + (UBF if bf else U) * (np.abs(want) + err) + 2.0 ** -125
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(got - want)[bad].max()))
