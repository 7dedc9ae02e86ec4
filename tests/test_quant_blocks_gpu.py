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
