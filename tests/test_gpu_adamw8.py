"""AdamW with moments in 8 bits on the GPU against the oracle, bit for bit (the oracle's own pins against 64 bits are in test_oracle_tok8.py)."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import assert_same_bits, dev, empty, host

pytestmark = pytest.mark.gpu
F = np.float32
H = (3e-4, 0.9, 0.95, 1e-8)


@pytest.fixture(scope="module")
def det():
    import paper_2609_17380_b200 as d
    d.load()
    return d


def same(got, want, what):
    want = np.ascontiguousarray(want)
    wide = lambda x: synth.from_bf16(x) if x.dtype == np.uint16 else x
    nan = np.isnan(wide(want)) if want.dtype in (np.uint16, np.float32) else np.zeros(want.shape, bool)
    if nan.any():
        assert np.array_equal(np.isnan(wide(got)), nan), what
        got, want = got[~nan], want[~nan]
    assert_same_bits(got, want, what)


def gradient(n, seed):
    """Values of very different scale, some zero, a block of zeros."""
    g = synth.normal_f32((n,), 1.0, seed=seed, tid=3) * np.exp(3 * synth.normal_f32((n,), 1.0, seed=seed, tid=4) - 8)
    g[synth.randint((n,), 20, seed=seed, tid=5) == 0] = 0
    if n > 600:
        g[256:512] = 0
    return g.astype(F)


def _tensors(sizes, seed):
    """Parameters of either type and moments of either width, in turn."""
    out = []
    for i, n in enumerate(sizes):
        p = synth.normal_f32((n,), 0.02, seed=seed, tid=100 + i)
        out.append(dict(n=n, p=synth.to_bf16(p) if i % 2 == 0 else p, eight=i % 4 < 3, wd=0.1 if i % 3 else 0.0, m=np.zeros(n, F), v=np.zeros(n, F),
                        m8=np.zeros(n, np.int8), v8=np.zeros(n, np.uint8), s=np.zeros((-(-n // 256), 2), F)))
    return out


SIZES = [1, 3, 4, 255, 256, 257, 1000, 2048, 4099, 0, 511, 30000, 7, 512]


@pytest.mark.parametrize("clip", [None, 1.0, 0.37])
def test_three_updates(det, clip):
    ts = _tensors(SIZES, 1)
    st = [dict(p=dev(t["p"]), m=dev(t["m8"] if t["eight"] else t["m"]), v=dev(t["v8"] if t["eight"] else t["v"]), s=dev(t["s"]) if t["eight"] else None)
          for t in ts]
    kinds = [det.DET_BF16 if t["p"].dtype == np.uint16 else det.DET_F32 for t in ts]
    coef = dev(np.array([clip], F)) if clip is not None else None
    for step in (1, 2, 3):
        gs = [gradient(t["n"], 10 * step + i) for i, t in enumerate(ts)]
        dg = [dev(g) for g in gs]
        descs = [det.det_adamw_desc(*H, t["wd"], step) for t in ts]
        det.det_adamw8_batch(descs, kinds, *([x[k] for x in st] if k != "g" else dg for k in ("p", "g", "m", "v", "s")), coef)
        for t, g, x, d in zip(ts, gs, st, dg):
            if clip is not None:
                g = oracle.scale(g, F(clip)) if t["n"] else g
            same(host(d), g, "gradient")
            if t["eight"]:
                t["p"], t["m8"], t["v8"], t["s"] = oracle.adamw8(t["p"], g, t["m8"], t["v8"], t["s"], *H, t["wd"], step)
                same(host(x["m"]), t["m8"], "m %d" % t["n"])
                same(host(x["v"]), t["v8"], "v %d" % t["n"])
                same(host(x["s"]), t["s"], "scales %d" % t["n"])
            else:
                t["p"], t["m"], t["v"] = oracle.adamw(t["p"], g, t["m"], t["v"], *H, t["wd"], step)
                same(host(x["m"]), t["m"], "m %d" % t["n"])
                same(host(x["v"]), t["v"], "v %d" % t["n"])
            same(host(x["p"], t["p"].dtype), t["p"], "p %d" % t["n"])


def test_elsewhere_leaves_the_inputs(det):
    """The new state in buffers of its own is that in place, and the old one stays; nothing is written behind a tensor's end."""
    import torch
    ts = [t for t in _tensors(SIZES, 2) if t["n"]]
    for i, t in enumerate(ts):
        t["m8"], t["v8"], t["s"] = oracle.adamw8_pack(gradient(t["n"], 50 + i), gradient(t["n"], 80 + i) ** 2)
    lists = lambda: [[dev(t[k]) for t in ts] for k in ("p", "m8", "v8", "s")]
    kinds, descs = [det.DET_BF16 if t["p"].dtype == np.uint16 else det.DET_F32 for t in ts], [det.det_adamw_desc(*H, t["wd"], 9) for t in ts]
    gs = [dev(gradient(t["n"], 30 + i)) for i, t in enumerate(ts)]
    here, old = lists(), lists()
    room = [[torch.full((x.numel() + 16,), 77, dtype=x.dtype, device="cuda") for x in part] for part in old]
    outs = [[r[:x.numel()].view(x.shape) for r, x in zip(a, b)] for a, b in zip(room, old)]
    run = lambda a, outs=None: det.det_adamw8_batch(descs, kinds, a[0], gs, a[1], a[2], a[3], None, outs=outs)
    run(here)
    run(old, tuple(outs))
    for part, want, got, kept in zip(("p", "m8", "v8", "s"), here, room, old):
        for t, w, g, k in zip(ts, want, got, kept):
            assert torch.equal(g[:w.numel()].view(torch.uint8), w.reshape(-1).view(torch.uint8)), part
            assert (g[w.numel():] == 77).all(), part
            same(host(k, t[part].dtype), t[part], part)


def test_many_tensors(det):
    """More tensors than one launch takes."""
    ts = _tensors([1 + 7 * i % 700 for i in range(300)], 3)
    gs = [gradient(t["n"], i) for i, t in enumerate(ts)]
    args = [[dev(t["p"]) for t in ts], [dev(g) for g in gs], [dev(t["m8"] if t["eight"] else t["m"]) for t in ts],
            [dev(t["v8"] if t["eight"] else t["v"]) for t in ts], [dev(t["s"]) if t["eight"] else None for t in ts]]
    det.det_adamw8_batch([det.det_adamw_desc(*H, t["wd"], 4) for t in ts], [det.DET_BF16 if t["p"].dtype == np.uint16 else det.DET_F32 for t in ts], *args)
    for i, (t, g) in enumerate(zip(ts, gs)):
        want = oracle.adamw8(t["p"], g, t["m8"], t["v8"], t["s"], *H, t["wd"], 4) if t["eight"] else oracle.adamw(t["p"], g, t["m"], t["v"], *H, t["wd"], 4)
        same(host(args[0][i], t["p"].dtype), want[0], "p")
        same(host(args[2][i]), want[1], "m")
        same(host(args[3][i]), want[2], "v")


@pytest.mark.parametrize("n", [1, 5, 256, 700, 4096, 10001])
def test_codes_and_numbers(det, n):
    m, v = gradient(n, 6), gradient(n, 7) ** 2
    if n > 4000:                       # blocks that are not finite, hold subnormals, and the ends of the range
        m[5], v[300], m[600], v[601] = np.nan, np.inf, F(1e-40), F(1e-44)
        m[1024:1280], v[1024:1280] = F(3e38), F(3e38)
        m[1300], v[1301] = F(1.2e-38), F(1.2e-38)
        m[2048:2304], v[2048:2304] = m[2048:2304] * F(1e-30), v[2048:2304] * F(1e-25)
    m8, v8, s = empty((n,), np.int8), empty((n,), np.uint8), empty((-(-n // 256), 2), F)
    det.det_adamw8_pack([dev(m), dev(m)], [dev(v), dev(v)], [m8, empty((n,), np.int8)], [v8, empty((n,), np.uint8)],
                        [s, empty((-(-n // 256), 2), F)])
    om, ov, os_ = oracle.adamw8_pack(m, v)
    same(host(s), os_, "scales")
    same(host(m8), om, "m")
    same(host(v8), ov, "v")
    bm, bv = empty((n,), F), empty((n,), F)
    det.det_adamw8_unpack([m8], [v8], [s], [bm], [bv])
    wm, wv = oracle.adamw8_unpack(om, ov, os_)
    same(host(bm), wm, "m back")
    same(host(bv), wv, "v back")


def test_not_finite(det):
    """A gradient that is not finite makes its block's moments NaN, and no other's."""
    n = 1024
    p, g = synth.normal_bf16((n,), 0.02, seed=1), gradient(n, 2)
    g[300], g[700] = np.nan, np.inf
    m8, v8, s = oracle.adamw8_pack(gradient(n, 3), gradient(n, 4) ** 2)
    args = [[dev(x)] for x in (p, g, m8, v8, s)]
    for step in (3, 4):
        det.det_adamw8_batch([det.det_adamw_desc(*H, 0.1, step)], [det.DET_BF16], *args)
        p, m8, v8, s = oracle.adamw8(p, g, m8, v8, s, *H, 0.1, step)
        for x, w in zip([args[0]] + args[2:], (p, m8, v8, s)):
            same(host(x[0], w.dtype).reshape(w.shape), w, "state")
        assert np.array_equal(np.isnan(s).any(1), [False, True, True, False])


def test_graph(det):
    import torch
    n = 5000
    p, g, m8, v8, s = (dev(x) for x in (synth.normal_bf16((n,), 0.02, seed=1), gradient(n, 2), *oracle.adamw8_pack(gradient(n, 3), gradient(n, 4) ** 2)))
    step = lambda: det.det_adamw8_batch([det.det_adamw_desc(*H, 0.1, 5)], [det.DET_BF16], [p], [g], [m8], [v8], [s])
    hp, hm, hv, hs = host(p, np.uint16).copy(), host(m8).copy(), host(v8).copy(), host(s).copy()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step()
    for k in range(2):
        g.copy_(dev(gradient(n, 40 + k)))
        graph.replay()
    torch.cuda.synchronize()
    for grad in (gradient(n, 2), gradient(n, 40), gradient(n, 41)):
        hp, hm, hv, hs = oracle.adamw8(hp, grad, hm, hv, hs, *H, 0.1, 5)
    for x, w in ((p, hp), (m8, hm), (v8, hv), (s, hs)):
        same(host(x, w.dtype).reshape(w.shape), w, "state")
