"""The 8-bit blocks as a program uses them: no tokens, sizes, tensors that do not fit."""
import pytest
import torch

from test_quant_gpu import block_inputs, say

pytestmark = pytest.mark.gpu


def moe_block(T, d=128, f=256, E=8, k=2, seed=5, **kw):
    from paper_2405_18832_amd.quant_layer import QuantMoEBlock
    gen, new, x, r = block_inputs(T, d, seed)
    w1, w2 = (new(E, f, d) / d ** 0.5).bfloat16(), (new(E, d, f) / f ** 0.5).bfloat16()
    return QuantMoEBlock(T, d, f, E, k, w1, w2, new(E, d).bfloat16(), torch.exp(0.2 * new(d)), **kw), x, r


def dense_block(T, d=128, f=256, seed=5, **kw):
    from paper_2405_18832_amd.quant_layer import QuantDenseBlock
    gen, new, x, r = block_inputs(T, d, seed)
    return QuantDenseBlock(T, d, f, new(f, d) / d ** 0.5, new(d, f) / f ** 0.5, torch.exp(0.2 * new(d)), **kw), x, r


def test_blocks_without_tokens(gpu_lib):
    """An empty batch gives empty rows, from a block made for it and from one resized to it, and the block goes on with others."""
    say("[case] blocks, T = 0")
    for make in (moe_block, dense_block):
        block, x, r = make(33)
        want = [t.clone() for t in block.forward(x, r)]
        for empty in (block.resized(0), make(0)[0]):
            y, stream = empty.forward(x[:0], r[:0])
            assert y.shape == stream.shape == (0, 128)
            y, stream = empty.forward(x[:0])
            assert y.shape == stream.shape == (0, 128)
            again = empty.resized(33)
            if empty.w1 is block.w1:
                assert all(torch.equal(a, b) for a, b in zip(again.forward(x, r), want))
    block, x, r = moe_block(0)
    block.forward(x, r, H=3)
    torch.cuda.synchronize()
    assert block.counts.cpu().tolist() == [0] * 8 and block.offsets.cpu().tolist() == [0] * 9 and block.hot_mask.cpu().tolist() == [1] * 3 + [0] * 5


@pytest.mark.parametrize("make", [moe_block, dense_block])
def test_forward_refuses_what_it_would_misread(gpu_lib, make):
    """Too few rows, another type, another layout: an error, and nothing is launched."""
    say("[case] blocks refuse rows")
    block, x, r = make(33)
    want = [t.clone() for t in block.forward(x, r)]
    for bad in (x[:32], x.float(), x.half(), x[:, :96], x.flatten(), x.cpu(), x.t().contiguous().t()):
        for args in ((bad, r), (x, bad)):
            with pytest.raises(ValueError):
                block.forward(*args)
    torch.cuda.synchronize()
    assert torch.equal(block.out, want[0]) and torch.equal(block.stream, want[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_constants_of_other_types(gpu_lib, dtype):
    """A norm weight and biases in 16 bits act as the same numbers in fp32."""
    from paper_2405_18832_amd.quant_layer import QuantDenseBlock, QuantMoEBlock
    say(f"[case] blocks with constants in {dtype}")
    T, d, f, E = 50, 64, 96, 4
    gen, new, x, r = block_inputs(T, d, 3)
    w1, w2, gate = new(E, f, d).bfloat16(), new(E, d, f).bfloat16(), new(E, d).bfloat16()
    c = dict(norm_weight=torch.exp(0.2 * new(d)).to(dtype), gate_bias=new(E).to(dtype), b1=new(E, f).to(dtype), b2=new(E, d).to(dtype))
    a, b = (QuantMoEBlock(T, d, f, E, 2, w1, w2, gate, **{k: g(v) for k, v in c.items()}) for g in (lambda t: t, lambda t: t.float()))
    assert all(torch.equal(u, v) for u, v in zip(a.forward(x, r), b.forward(x, r)))
    c = dict(norm_weight=c["norm_weight"], b1=c["b1"][0], b2=c["b2"][0])
    a, b = (QuantDenseBlock(T, d, f, w1[0], w2[0], **{k: g(v) for k, v in c.items()}) for g in (lambda t: t, lambda t: t.float()))
    assert all(torch.equal(u, v) for u, v in zip(a.forward(x, r), b.forward(x, r)))


def test_units_of_the_blocks_sums(gpu_lib):
    """sums="units" changes how the products are added, by less than an output's rounding: both forms of a block agree to a few of its steps."""
    say("[case] blocks with sums by the 8-bit units")
    for make in (moe_block, dense_block):
        a, x, r = make(300)
        b, _, _ = make(300, sums="units")
        ya, yb = a.forward(x, r)[0].float(), b.forward(x, r)[0].float()
        assert torch.equal(a.stream, b.stream) and torch.equal(a.x8.codes.view(torch.uint8), b.x8.codes.view(torch.uint8))
        # an e4m3 code in the middle may go the other way: 2^-3 of one of 256 hidden values, a bf16 step of the output
        assert (ya - yb).norm() <= 2.0 ** -6 * ya.norm()
