"""Host side of the blocks with layer norm and recurrent layers: the driver, the oracle and the synthetic inputs agree on the parameters."""
import numpy as np
import pytest

import synth
from oracle import step as ostep
from paper_2609_17380_b200 import step as dstep


@pytest.mark.parametrize("kw", [dict(), dict(norm="layer"), dict(recurrent=(0, 2)), dict(norm="layer", recurrent=(1,), embed_norm=True, n_kv_heads=1)])
def test_parameter_lists_agree(kw):
    cfg = dstep.ModelConfig(n_layers=3, d_model=256, n_heads=2, ffn=384, vocab=512, seq=128, micro_batch=1, mesh=(1, 1, 1), **kw)
    ours = [(n, s) for n, s, _ in dstep.param_specs(cfg)]
    assert ours == list(ostep._specs(cfg.as_dict())) == [(n, s) for n, s, _ in synth.model_param_specs(cfg.as_dict())]
    params = synth.model_params(cfg.as_dict())
    shifts = [n for n in params if n.endswith("_shift")]
    assert len(shifts) == (0 if cfg.norm == "rms" else 7 + bool(cfg.embed_norm)) and not any(params[n].any() for n in shifts)
    for l in range(3):
        assert params["l%d.w_qkv" % l].shape[0] == (512 if l in cfg.recurrent else cfg.qkv_width)


def test_oracle_step_learns_from_every_parameter():
    """No gradient of the block is lost: every parameter of a step moves."""
    cfg = dict(n_layers=2, d_model=128, n_heads=1, ffn=128, vocab=128, seq=128, micro_batch=1, mesh=(1, 1, 1), norm="layer", recurrent=(1,), act8=True,
               lr=1e-2)
    params = synth.model_params(cfg, seed=5)
    tok = synth.model_tokens(cfg, 1, seed=5)
    first = ostep.run_step(cfg, params, tok)
    for name, p in first["params"].items():
        assert not np.array_equal(p, params[name]), name
    assert np.isfinite(first["loss"]) and abs(first["loss"] - np.log(128)) < 0.5
