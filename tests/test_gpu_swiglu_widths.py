"""SwiGLU over rows of any width and address, and the step that makes it again from activations kept in 8 bits: against the oracle, bit for bit."""
import numpy as np
import pytest

import oracle
import synth
from gpu_util import assert_same_bits, dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,F", [(1, 1), (3, 7), (37, 100), (129, 509), (1000, 1001), (5, 8), (0, 9)])
def test_any_width(rows, F):
    """One element off an aligned address where the width allows it; what lies in front and behind stays."""
    import torch

    import paper_2609_17380_b200 as det
    gu = synth.normal_bf16((rows, 2 * F), 2.0, seed=6, tid=1)
    if F > 6 and rows:
        gu[0, :6] = synth.to_bf16(np.array([-200.0, 200.0, 90.0, -90.0, np.inf, 0.0], np.float32))
    off = 1 if F % 8 else 8
    src, dst = torch.full((gu.size + 32,), 77, dtype=torch.int16, device="cuda"), torch.full((rows * F + 32,), 77, dtype=torch.int16, device="cuda")
    src[off:off + gu.size] = dev(gu).reshape(-1)
    det.det_swiglu_fwd(src.data_ptr() + 2 * off, rows, F, dst.data_ptr() + 2 * off)
    torch.cuda.synchronize()
    assert (dst[:off] == 77).all() and (dst[off + rows * F:] == 77).all()
    assert_same_bits(host(dst, np.uint16)[off:off + rows * F].reshape(rows, F), oracle.swiglu_fwd(gu), "h")


@pytest.mark.parametrize("kw", [dict(ffn=100), dict(ffn=509, state8=True), dict(ffn=200, norm="layer", recurrent=(1,)), dict(ffn=672)])
def test_steps_with_activations_in_8_bits(kw):
    """Feed-forward widths of which no group of 32 values ends with the gates, and one of which one does."""
    import torch
    from oracle import step as ostep
    from paper_2609_17380_b200 import step as dstep
    cfg = dstep.ModelConfig(n_layers=2, d_model=256, n_heads=2, vocab=512, seq=128, micro_batch=1, mesh=(1, 2, 1), linear="token", act8=True, **kw)
    params = synth.model_params(cfg.as_dict(), seed=1)
    r = dstep.Replay(cfg)
    r.load_params(params)
    opt = None
    for step in (1, 2):
        cfg.step = step
        tokens = synth.model_tokens(cfg.as_dict(), cfg.n_microbatches, seed=step)
        got = r.step(torch.from_numpy(np.ascontiguousarray(tokens, dtype=np.int32)).cuda())
        want = ostep.run_step(cfg.as_dict(), params, tokens, opt=opt)
        params, opt = want["params"], want["opt"]
        assert got["status"] == 0 and got["losses"] == [np.float32(x) for x in want["losses"]]
        bad = [k for k, h in want["hashes"].items() if got["hashes"][k] != h]
        assert not bad and set(got["hashes"]) == set(want["hashes"]), (step, bad)
