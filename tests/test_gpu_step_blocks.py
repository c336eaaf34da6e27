"""Replayed steps of blocks with layer norm, recurrent layers and activations in 8 bits, against the oracle's step: every hash."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu

SMALL = dict(n_layers=2, d_model=256, n_heads=2, ffn=512, vocab=512, seq=128, micro_batch=1, mesh=(1, 2, 1))


def _run(kw, seed=0):
    from oracle import step as ostep
    from paper_2609_17380_b200 import step as dstep
    kw = dict(kw)
    if kw.pop("rope", False):
        kw["rope_tables"] = synth.rope_tables(kw["seq"])
    cfg = dstep.ModelConfig(**kw)
    params = synth.model_params(cfg.as_dict(), seed=seed)
    for name in params:                                    # gains and shifts that are not their start values
        if name.endswith("norm") or name.endswith("norm_shift"):
            params[name] = synth.normal_bf16(params[name].shape, 0.1, mean=0.0 if name.endswith("shift") else 1.0, seed=seed + 7, tid=len(name))
    tokens = synth.model_tokens(cfg.as_dict(), cfg.n_microbatches, seed=seed)
    return cfg, dstep.run_step(cfg, params, tokens), ostep.run_step(cfg.as_dict(), params, tokens)


@pytest.mark.parametrize("kw", [
    dict(SMALL, norm="layer"),
    dict(SMALL, act8=True),
    dict(SMALL, recurrent=(0,)),
    dict(SMALL, norm="layer", recurrent=(0, 1), act8=True, mesh=(2, 1, 2)),
    # every second layer recurrent, grouped queries with QK-norm and RoPE in the others, an embedding norm
    dict(n_layers=3, d_model=512, n_heads=4, n_kv_heads=1, ffn=384, vocab=512, seq=256, micro_batch=2, mesh=(1, 1, 1), qk_norm=True, rope=True,
         embed_norm=True, norm="layer", recurrent=(1,), act8=True),
    dict(n_layers=2, d_model=256, n_heads=2, ffn=256, vocab=256, seq=192, micro_batch=2, mesh=(1, 1, 1), pv_int8=True, act8=True, recurrent=(1,)),
])
def test_step_hashes_match_oracle(kw):
    cfg, got, want = _run(kw)
    assert got["status"] == 0
    assert got["losses"] == [np.float32(x) for x in want["losses"]]
    assert np.float32(got["grad_norm"]) == np.float32(want["grad_norm"])
    bad = [k for k, h in want["hashes"].items() if got["hashes"][k] != h]
    assert not bad and set(got["hashes"]) == set(want["hashes"]), bad
    assert abs(got["loss"] - np.log(cfg.vocab)) < 0.5      # random init: loss ~ log V


def test_separate_quantiser_passes_give_the_same_hashes():
    import torch
    from paper_2609_17380_b200 import step as dstep
    cfg = dstep.ModelConfig(**dict(SMALL, norm="layer", recurrent=(1,), act8=True))
    params = synth.model_params(cfg.as_dict(), seed=3)
    tok = torch.from_numpy(np.ascontiguousarray(synth.model_tokens(cfg.as_dict(), 2, seed=3), dtype=np.int32)).cuda()
    out = []
    for fuse in (True, False):
        r = dstep.Replay(cfg)
        r.fuse_quant = fuse
        r.load_params(params)
        r.calibrate(tok[0])
        out.append(r.step(tok)["hashes"])
    assert out[0] == out[1]


def test_checkpoints_in_8_bits_save_memory():
    """The activations of a layer take less than two thirds of what they take whole."""
    from paper_2609_17380_b200 import step as dstep
    size = lambda r: sum(t.numel() * t.element_size() for a in r.act for t in a.values())
    whole, small = (size(dstep.Replay(dstep.ModelConfig(**dict(SMALL, ffn=1024, act8=a)))) for a in (False, True))
    assert small < 2 * whole / 3
