"""Replayed steps with 8-bit linears by token and channel and with moments in 8 bits, against the oracle's step: every hash."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu

SMALL = dict(n_layers=2, d_model=256, n_heads=2, ffn=512, vocab=512, seq=128, micro_batch=1, mesh=(1, 2, 1))


@pytest.mark.parametrize("kw", [
    dict(SMALL, linear="token"),
    dict(SMALL, state8=True),
    dict(SMALL, linear="token", state8=True, mesh=(2, 1, 2)),
    # a feed-forward width that is no multiple of a tile, activations in 8 bits, a recurrent layer, layer norm
    dict(SMALL, linear="token", state8=True, ffn=672, act8=True, norm="layer", recurrent=(1,)),
    # grouped queries with QK-norm and RoPE, an embedding norm
    dict(n_layers=2, d_model=512, n_heads=4, n_kv_heads=1, ffn=384, vocab=512, seq=192, micro_batch=2, mesh=(1, 1, 1), qk_norm=True, rope=True,
         embed_norm=True, linear="token", state8=True),
])
def test_two_steps_match_the_oracle(kw):
    """The second step starts from moments that are not zero."""
    import torch
    from oracle import step as ostep
    from paper_2609_17380_b200 import step as dstep
    kw = dict(kw)
    if kw.pop("rope", False):
        kw["rope_tables"] = synth.rope_tables(kw["seq"])
    cfg = dstep.ModelConfig(**kw)
    params = synth.model_params(cfg.as_dict(), seed=1)
    r = dstep.Replay(cfg)
    r.load_params(params)
    opt = None
    for step in (1, 2):
        cfg.step = step
        tokens = synth.model_tokens(cfg.as_dict(), cfg.n_microbatches, seed=step)
        tok = torch.from_numpy(np.ascontiguousarray(tokens, dtype=np.int32)).cuda()
        if step == 1:
            r.calibrate(tok[0])
        got = r.step(tok)
        want = ostep.run_step(cfg.as_dict(), params, tokens, opt=opt, calibrate=step == 1)
        params, opt = want["params"], want["opt"]
        assert got["status"] == 0 and got["losses"] == [np.float32(x) for x in want["losses"]]
        bad = [k for k, h in want["hashes"].items() if got["hashes"][k] != h]
        assert not bad and set(got["hashes"]) == set(want["hashes"]), (step, bad)


def test_state_file_takes_the_codes_along(tmp_path):
    """A step after a saved state gives the hashes that it gives without the file; another kind of state is refused."""
    import torch
    from paper_2609_17380_b200 import step as dstep
    tok = [torch.from_numpy(np.ascontiguousarray(synth.model_tokens(dict(SMALL), 2, seed=s), dtype=np.int32)).cuda() for s in (1, 2)]
    r = dstep.Replay(dstep.ModelConfig(**SMALL, linear="token", state8=True))
    r.init_params_on_device(3)
    r.step(tok[0])
    r.cfg.step = 2
    path = str(tmp_path / "state.npz")
    r.save_state(path)
    want = r.step(tok[1])["hashes"]
    other = dstep.Replay(dstep.ModelConfig(**SMALL, linear="token", state8=True))
    other.load_state(path)
    assert other.cfg.step == 2 and other.step(tok[1])["hashes"] == want
    for kw in (dict(linear="token"), dict(state8=True), dict()):
        with pytest.raises(ValueError):
            dstep.Replay(dstep.ModelConfig(**SMALL, **kw)).load_state(path)


def test_moments_in_8_bits_save_memory():
    from paper_2609_17380_b200 import step as dstep
    size = lambda r: sum(t.numel() * t.element_size() for t in (r.m, r.v, r.m8, r.v8, r.ms))
    whole, small = (size(dstep.Replay(dstep.ModelConfig(**SMALL, state8=e))) for e in (False, True))
    assert small < whole / 3.5
