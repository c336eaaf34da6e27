"""Host side of the step with 8-bit linears by token and channel: every buffer of codes has room for rows of codes as the library lays them out."""
import pytest
import torch

import paper_2609_17380_b200 as det
from paper_2609_17380_b200 import step as dstep

BLOCK = dict(n_layers=2, d_model=256, n_heads=2, vocab=512, seq=128, micro_batch=1, mesh=(1, 1, 1))


# widths that are no multiple of 16 bytes, of which a row of codes is one
@pytest.mark.parametrize("act8", [False, True])
@pytest.mark.parametrize("ffn", [100, 392, 509, 1001, 512])
def test_rows_of_codes_have_room(ffn, act8):
    cfg = dstep.ModelConfig(**BLOCK, ffn=ffn, linear="token", act8=act8, recurrent=(1,))
    r = dstep.Replay(cfg, device="cpu")
    T, D = cfg.tokens_per_microbatch, cfg.d_model
    for l in range(cfg.n_layers):
        a = r.act[l]
        for name, K in (("qx_qkv", D), ("qx_o", D), ("qx_gu", D), ("qx_down", ffn)):
            q = r.shared[name] if act8 and name == "qx_down" else a[name]
            assert q.dtype == torch.int8 and q.numel() == T * det.det_tok8_ld(K), (l, name)
            assert a["sx" + name[2:]].numel() == T
        for w, (N, K) in dict(w_qkv=(cfg.mixer_width(l), D), w_o=(D, D), w_gu=(2 * ffn, D), w_down=(D, ffn)).items():
            d = r.lin[(l, w)]
            assert d["qW"].numel() == N * det.det_tok8_ld(K) and d["qWt"].numel() == K * det.det_tok8_ld(N) and d["s_w"].numel() == N, (l, w)


def test_rows_of_codes_with_a_learned_step_are_not_padded():
    r = dstep.Replay(dstep.ModelConfig(**BLOCK, ffn=384), device="cpu")
    assert [r.act[0][n].numel() for n in ("qx_qkv", "qx_o", "qx_gu", "qx_down")] == [128 * 256] * 3 + [128 * 384]


def test_parts_of_the_state_by_name():
    """Codes, scales and moments of a parameter lie where the update takes them from, whatever buffer they are asked of; together they are the whole buffers."""
    r = dstep.Replay(dstep.ModelConfig(**BLOCK, ffn=100, linear="token", state8=True), device="cpu")
    for buf, matrices in ((r.m8, True), (r.v8, True), (r.ms, True), (r.m, False), (r.v, False)):
        at = 0
        for name, shape, _ in r.specs:
            n = shape[0] * (shape[1] if len(shape) > 1 else 1)
            if (len(shape) > 1) != matrices:
                with pytest.raises(KeyError):
                    r.g(buf, name)
                continue
            n = det.det_adamw8_scale_floats(n) if buf is r.ms else n
            part = r.g(buf, name)
            assert part.numel() == n and part.data_ptr() == buf.data_ptr() + at * buf.element_size(), name
            at += n
        assert at == buf.numel()
