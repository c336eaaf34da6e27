"""A state file says what its numbers are: a configuration with parameters of other places or meanings refuses it (on the CPU, nothing is launched)."""
import numpy as np
import pytest
import torch

from paper_2609_17380_b200 import step as dstep


def _replay(**kw):
    cfg = dict(n_layers=2, d_model=512, n_heads=4, ffn=256, vocab=512, seq=64, micro_batch=1, mesh=(1, 1, 1))
    cfg.update(kw)
    r = dstep.Replay(dstep.ModelConfig(**cfg), device="cpu")
    for n, t in enumerate((r.pbf, r.sx, r.m, r.v)):
        t.copy_(torch.arange(t.numel()) % 1000 + n)
    return r


def _state(r):
    return [t.clone() for t in (r.pbf, r.sx, r.m, r.v)]


def _loads(saved, kw, path):
    r = _replay(**kw)
    for t in (r.pbf, r.sx, r.m, r.v):
        t.zero_()
    r.load_state(path)
    return all(torch.equal(a, b) for a, b in zip(_state(r), _state(saved)))


@pytest.mark.parametrize("kw", [dict(), dict(recurrent=(0,)), dict(recurrent=(0, 1), norm="layer"), dict(recurrent=(1,), n_kv_heads=2), dict(norm="layer", act8=True)])
def test_the_same_configuration_takes_it(kw, tmp_path):
    path = str(tmp_path / "state.npz")
    r = _replay(**kw)
    r.cfg.step = 5
    r.save_state(path)
    assert _loads(r, kw, path)
    # how activations are kept, or the order in which the layers were named, is no matter of the state
    assert _loads(r, dict(kw, act8=not kw.get("act8", False), recurrent=list(reversed(kw.get("recurrent", ())))), path)


@pytest.mark.parametrize("one,other", [
    (dict(recurrent=(0,)), dict(recurrent=(1,))),                                     # as many numbers, in another order
    (dict(n_kv_heads=2), dict(n_kv_heads=2, recurrent=(0,))),                         # w_qkv of the same shape: queries, keys and values, or gate and value
    (dict(n_kv_heads=2, recurrent=(0, 1)), dict(n_kv_heads=2)),
    (dict(n_layers=1, vocab=512, ffn=256), dict(n_layers=1, vocab=512, ffn=512)),
    (dict(norm="layer"), dict()),
    # 2 * 512 + 3 * 256 rows of 512 values in another division
    (dict(n_layers=1, ffn=256, vocab=896), dict(n_layers=1, ffn=512, vocab=512)),
])
def test_another_configuration_refuses_it(one, other, tmp_path):
    path = str(tmp_path / "state.npz")
    _replay(**one).save_state(path)
    r = _replay(**other)
    before = _state(r)
    with pytest.raises(ValueError, match="does not match this configuration"):
        r.load_state(path)
    assert all(torch.equal(a, b) for a, b in zip(before, _state(r)))


def test_a_file_without_a_layout(tmp_path):
    """By the lengths alone, where no layer is recurrent."""
    for kw, ok in ((dict(), True), (dict(norm="layer"), True), (dict(recurrent=(0,)), False)):
        path, r = str(tmp_path / "state.npz"), _replay(**kw)
        np.savez(path, pbf=r.pbf.numpy(), sx=r.sx.numpy(), m=r.m.numpy(), v=r.v.numpy(), step=np.array([3], np.int64))
        if ok:
            assert _loads(r, kw, path)
        else:
            with pytest.raises(ValueError, match="recurrent"):
                r.load_state(path)
    r = _replay()
    np.savez(path, pbf=r.pbf.numpy()[:-8], sx=r.sx.numpy(), m=r.m.numpy(), v=r.v.numpy(), step=np.array([3], np.int64))
    with pytest.raises(ValueError, match="does not match this configuration"):
        r.load_state(path)
