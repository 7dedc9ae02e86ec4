"""What the 8-bit blocks refuse: every tensor whose shape, type or device is not what the library would read, before anything is launched."""
import pytest
import torch

import paper_2405_18832_amd as moe
from paper_2405_18832_amd import quant_layer as ql

T, D, F, E, K = 6, 64, 96, 4, 2
BF = torch.bfloat16


@pytest.fixture
def on_cpu(monkeypatch):
    """Blocks of CPU tensors: their weights are not laid out, and the first call of a forward pass refuses them."""
    monkeypatch.setattr(ql, "moe_quantize_weights", lambda *a, **k: None)


def moe_args(**kw):
    a = dict(T=T, d_model=D, d_ff=F, E=E, k=K, w1=torch.zeros(E, F, D, dtype=BF), w2=torch.zeros(E, D, F, dtype=BF),
             w_gate=torch.zeros(E, D, dtype=BF), norm_weight=torch.ones(D), gate_bias=torch.zeros(E), b1=torch.zeros(E, F), b2=torch.zeros(E, D))
    a.update(kw)
    return a


def dense_args(**kw):
    a = dict(T=T, d_model=D, d_ff=F, w1=torch.zeros(F, D), w2=torch.zeros(D, F), norm_weight=torch.ones(D), b1=torch.zeros(F), b2=torch.zeros(D))
    a.update(kw)
    return a


META = torch.device("meta")


@pytest.mark.parametrize("match,kw", [
    ("w_gate", dict(w_gate=torch.zeros(E, D))), ("w_gate", dict(w_gate=torch.zeros(E, D + 1, dtype=BF))),
    ("w_gate", dict(w_gate=torch.zeros(D, E, dtype=BF))), ("w_gate", dict(w_gate=torch.zeros(E, D, dtype=BF, device=META))),
    ("norm_weight", dict(norm_weight=torch.ones(D - 1))), ("norm_weight", dict(norm_weight=torch.ones(1, D))),
    ("norm_weight", dict(norm_weight=torch.ones(D, dtype=torch.int32))), ("norm_weight", dict(norm_weight=torch.ones(D, device=META))),
    ("gate_bias", dict(gate_bias=torch.zeros(E + 1))), ("b1", dict(b1=torch.zeros(E, D))), ("b1", dict(b1=torch.zeros(F))),
    ("b2", dict(b2=torch.zeros(E, F))), ("b2", dict(b2=torch.zeros(E, D, dtype=torch.float64))),
    ("w1 is", dict(w1=torch.zeros(E, D, F, dtype=BF))), ("w1 is", dict(w2=torch.zeros(E + 1, D, F, dtype=BF))),
    ("w1 is", dict(w2=torch.zeros(E, D, F, dtype=BF, device=META))), ("fp32, bf16 or e4m3", dict(w1=torch.zeros(E, F, D, dtype=torch.float16))),
    ("scales belong", dict(w1=torch.zeros(E, F, D).to(torch.float8_e4m3fn))), ("scales belong", dict(w1_scales=torch.ones(E, 1, 1))),
    ("one scale", dict(w2=torch.zeros(E, D, F).to(torch.float8_e4m3fn), w2_scales=torch.ones(E, 1, 2))),
    ("weights' device", dict(w2=torch.zeros(E, D, F).to(torch.float8_e4m3fn), w2_scales=torch.ones(E, 1, 1, device=META))),
    ("T = -1", dict(T=-1)), ("eps", dict(eps=-1.0)), ("eps", dict(eps=float("nan"))), ("eps", dict(eps=float("inf"))),
    ("refuses", dict(k=E + 1)), ("refuses", dict(k=0)), ("refuses", dict(T=1 << 30)),
    ("refuses", dict(d_model=80, w1=torch.zeros(E, F, 80, dtype=BF), w2=torch.zeros(E, 80, F, dtype=BF), w_gate=torch.zeros(E, 80, dtype=BF),
                     norm_weight=None, b2=None)),
])
def test_moe_block_refuses(on_cpu, match, kw):
    with pytest.raises(ValueError, match=match):
        ql.QuantMoEBlock(**moe_args(**kw))


@pytest.mark.parametrize("match,kw", [
    ("norm_weight", dict(norm_weight=torch.ones(D + 1))), ("norm_weight", dict(norm_weight=torch.ones(D, device=META))),
    ("b1", dict(b1=torch.zeros(D))), ("b2", dict(b2=torch.zeros(F))), ("b2", dict(b2=torch.zeros(1, D))),
    ("w1 is", dict(w1=torch.zeros(D, F))), ("w1 is", dict(w2=torch.zeros(F, D))), ("w1 is", dict(w2=torch.zeros(D, F, device=META))),
    ("fp32, bf16 or e4m3", dict(w2=torch.zeros(D, F, dtype=torch.int8))), ("T = -2", dict(T=-2)), ("d_model = 0", dict(d_model=0)),
    ("eps", dict(eps=-1e-6)), ("refuses", dict(T=1 << 30)),
])
def test_dense_block_refuses(on_cpu, match, kw):
    with pytest.raises(ValueError, match=match):
        ql.QuantDenseBlock(**dense_args(**kw))


@pytest.mark.parametrize("make,args", [(ql.QuantMoEBlock, moe_args), (ql.QuantDenseBlock, dense_args)])
def test_forward_refuses(on_cpu, make, args):
    block = make(**args())
    good = torch.zeros(T, D, dtype=BF)
    for bad in (torch.zeros(T, D), torch.zeros(T - 1, D, dtype=BF), torch.zeros(T + 1, D, dtype=BF), torch.zeros(T, D + 32, dtype=BF),
                torch.zeros(T * D, dtype=BF), torch.zeros(T, D, dtype=torch.float16), torch.zeros(T, D, dtype=BF, device=META)):
        with pytest.raises(ValueError, match="^x: expected"):
            block.forward(bad)
        with pytest.raises(ValueError, match="^residual: expected"):
            block.forward(good, bad)
    with pytest.raises(ValueError, match="expected a CUDA tensor"):
        block.forward(good, good)
    with pytest.raises(ValueError, match="^x: expected"):
        block.resized(T - 1).forward(good)
    with pytest.raises(ValueError, match="T = -1"):
        block.resized(-1)


@pytest.mark.parametrize("dtype", [torch.float32, BF, torch.float16])
def test_weights_and_biases_of_other_types(on_cpu, dtype):
    """A bf16 checkpoint's norm weight and biases: the library reads fp32, so that is what the blocks keep."""
    v = lambda *s: torch.nn.Parameter(torch.linspace(-1, 1, s[0] * (s[1] if len(s) > 1 else 1)).view(s).to(dtype))
    block = ql.QuantMoEBlock(**moe_args(norm_weight=v(D), gate_bias=v(E), b1=v(E, F), b2=v(D, E).t()))
    for name, want in (("norm_weight", v(D)), ("gate_bias", v(E)), ("b1", v(E, F)), ("b2", v(D, E).t())):
        t = getattr(block, name)
        assert t.dtype == torch.float32 and t.is_contiguous() and not t.requires_grad and torch.equal(t, want.float()), name
    block = ql.QuantDenseBlock(**dense_args(norm_weight=v(D), b1=v(F), b2=v(D)))
    for name, want in (("norm_weight", v(D)), ("b1", v(F)), ("b2", v(D))):
        assert getattr(block, name).dtype == torch.float32 and torch.equal(getattr(block, name), want.float()), name


def test_refused_choices(on_cpu):
    for make, args in ((ql.QuantMoEBlock, moe_args), (ql.QuantDenseBlock, dense_args)):
        with pytest.raises((KeyError, ValueError)):
            make(**args(sums="bf16"))
        with pytest.raises((KeyError, ValueError)):
            make(**args(activation="tanh"))
        assert make(**args(sums="units")).first.out_dtype == moe.MOE_E4M3 | moe.MOE_QUANT_UNIT_SUMS
