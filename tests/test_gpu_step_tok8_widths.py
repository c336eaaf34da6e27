"""Replayed steps with 8-bit linears by token and channel at feed-forward widths that are no multiple of the 16 bytes that a row of codes is padded to,
against the oracle's step: every hash."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu

BLOCK = dict(n_layers=2, d_model=256, n_heads=2, vocab=512, seq=128, micro_batch=1, mesh=(1, 2, 1), linear="token")


@pytest.mark.parametrize("kw", [dict(ffn=100), dict(ffn=392, state8=True), dict(ffn=509), dict(ffn=1001, recurrent=(0,))])
def test_two_steps_match_the_oracle(kw):
    """The second step starts from weights that the first one moved."""
    import torch
    from oracle import step as ostep
    from paper_2609_17380_b200 import step as dstep
    cfg = dstep.ModelConfig(**BLOCK, **kw)
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
