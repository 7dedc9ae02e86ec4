"""What the int8 blocks refuse: every tensor whose shape, type or device is not what the library would read, before anything is launched."""
import pytest
import torch

import paper_2405_18832_amd as moe
from paper_2405_18832_amd import int8_layer as il

T, D, F, E, K = 6, 64, 96, 8, 2
BF = torch.bfloat16
META = torch.device("meta")


@pytest.fixture
def on_cpu(monkeypatch):
    """Blocks of CPU tensors: their weights are not laid out, and the first call of a forward pass refuses them."""
    monkeypatch.setattr(il, "moe_quantize_weights_int", lambda *a, **k: None)


def moe_args(**kw):
    a = dict(T=T, d_model=D, d_ff=F, E=E, k=K, w1=torch.zeros(E, 2 * F, D, dtype=BF), w2=torch.zeros(E, D, F, dtype=BF), w_gate=torch.zeros(E, D, dtype=BF),
             norm_weight=torch.ones(D), gate_bias=torch.zeros(E), choice_bias=torch.zeros(E), b1=torch.zeros(E, 2 * F), b2=torch.zeros(E, D))
    a.update(kw)
    return a


def dense_args(**kw):
    a = dict(T=T, d_model=D, d_ff=F, w1=torch.zeros(2 * F, D), w2=torch.zeros(D, F), norm_weight=torch.ones(D), b1=torch.zeros(2 * F), b2=torch.zeros(D))
    a.update(kw)
    return a


@pytest.mark.parametrize("match,kw", [
    ("w_gate", dict(w_gate=torch.zeros(E, D))), ("w_gate", dict(w_gate=torch.zeros(D, E, dtype=BF))), ("w_gate", dict(w_gate=torch.zeros(E, D, dtype=BF, device=META))),
    ("norm_weight", dict(norm_weight=torch.ones(D - 1))), ("norm_weight", dict(norm_weight=torch.ones(D, dtype=torch.int32))),
    ("norm_weight", dict(norm_weight=torch.ones(D, device=META))), ("gate_bias", dict(gate_bias=torch.zeros(E + 1))),
    ("choice_bias", dict(choice_bias=torch.zeros(1, E))), ("choice_bias", dict(choice_bias=torch.zeros(E, device=META))),
    ("b1", dict(b1=torch.zeros(E, F))), ("b2", dict(b2=torch.zeros(E, F))), ("b2", dict(b2=torch.zeros(E, D, dtype=torch.float64))),
    ("w1 is", dict(w1=torch.zeros(E, F, D, dtype=BF))), ("w1 is", dict(gated=False)), ("w1 is", dict(w2=torch.zeros(E + 1, D, F, dtype=BF))),
    ("w1 is", dict(w2=torch.zeros(E, D, F, dtype=BF, device=META))), ("fp32, bf16 or int8", dict(w1=torch.zeros(E, 2 * F, D, dtype=torch.float16))),
    ("scales belong", dict(w1=torch.zeros(E, 2 * F, D, dtype=torch.int8))), ("scales belong", dict(w1_scales=torch.ones(E, 2 * F))),
    ("one scale", dict(w2=torch.zeros(E, D, F, dtype=torch.int8), w2_scales=torch.ones(E, F))),
    ("weights' device", dict(w2=torch.zeros(E, D, F, dtype=torch.int8), w2_scales=torch.ones(E, D, device=META))),
    ("weights' device", dict(w2=torch.zeros(E, D, F, dtype=torch.int8), w2_scales=torch.ones(E, D, dtype=torch.int32))),
    ("T = -1", dict(T=-1)), ("eps", dict(eps=-1.0)), ("eps", dict(eps=float("nan"))), ("activation", dict(activation="swish")), ("score", dict(score="linear")),
    ("routing", dict(groups=3)), ("routing", dict(groups=0)), ("routing", dict(groups=4, groups_kept=5)), ("routing", dict(groups=8, groups_kept=1)),
    ("routing", dict(group_top=3)), ("routing", dict(groups=8, groups_kept=8, group_top=2)), ("routing", dict(scale=float("inf"))),
    ("routing", dict(k=E + 1)), ("refuses", dict(k=0)), ("refuses", dict(T=1 << 30)),
    ("refuses", dict(d_model=80, w1=torch.zeros(E, 2 * F, 80, dtype=BF), w2=torch.zeros(E, 80, F, dtype=BF), w_gate=torch.zeros(E, 80, dtype=BF),
                     norm_weight=None, b2=None)),
])
def test_moe_block_refuses(on_cpu, match, kw):
    with pytest.raises(ValueError, match=match):
        il.Int8MoEBlock(**moe_args(**kw))


@pytest.mark.parametrize("match,kw", [
    ("norm_weight", dict(norm_weight=torch.ones(D + 1))), ("b1", dict(b1=torch.zeros(F))), ("b2", dict(b2=torch.zeros(1, D))), ("w1 is", dict(w1=torch.zeros(F, D))),
    ("w1 is", dict(w2=torch.zeros(F, D))), ("w1 is", dict(w2=torch.zeros(D, F, device=META))), ("scales belong", dict(w2=torch.zeros(D, F, dtype=torch.int8))),
    ("one scale", dict(w1=torch.zeros(2 * F, D, dtype=torch.int8), w1_scales=torch.ones(F))), ("T = -2", dict(T=-2)), ("d_model = 0", dict(d_model=0)),
    ("activation", dict(activation=2)),
])
def test_dense_block_refuses(on_cpu, match, kw):
    with pytest.raises(ValueError, match=match):
        il.Int8DenseBlock(**dense_args(**kw))


@pytest.mark.parametrize("make", [lambda: il.Int8MoEBlock(**moe_args()), lambda: il.Int8DenseBlock(**dense_args())])
def test_forward_refuses(on_cpu, make):
    block = make()
    x = torch.zeros(T, D, dtype=BF)
    for bad in (x.float(), x[:, :-1], x[:-1], torch.zeros(T, D, dtype=BF, device=META)):
        with pytest.raises(ValueError, match="x: expected"):
            block.forward(bad)
        with pytest.raises(ValueError, match="residual: expected"):
            block.forward(x, bad)
    with pytest.raises(ValueError, match="T = -3"):
        block.resized(-3)
    with pytest.raises(ValueError, match="CUDA"):       # CPU tensors get as far as the first call
        block.forward(x, x)


def test_longest_contraction(on_cpu):
    with pytest.raises(ValueError, match="131071"):
        il.Int8Weights(torch.zeros(1, 1, moe.MOE_INT_MAX_K + 1, dtype=torch.int8, device=META), torch.ones(1, 1, device=META))
