"""Sizes of the 8-bit calls at which a launch's own limits lie."""
import pytest
import torch

from oracle import quant_oracle as qo
from test_quant_gpu import codes_of, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [((1 << 24) + 5, 1025), ((1 << 25) + 3, 520), ((1 << 26) + 7, 3)])
def test_norm_of_many_rows(gpu_lib, rows, d):
    """More rows than one direction of a launch has blocks of threads for: one, two and four rows per block."""
    moe = gpu_lib
    say(f"[case] moe_norm_quantize {rows} x {d}")
    pick = sorted({0, 1, 4095, (1 << 22) - 1, 1 << 22, (1 << 24) - 1, (1 << 24), (1 << 24) + 1, rows - 5, rows - 1})
    x = torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda")
    few = torch.randn((len(pick), d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(d)).bfloat16()
    x[pick] = few
    pitch, nb = moe.moe_quant_pitch(d), qo.blocks(d)
    q = torch.full((rows, pitch), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, nb), -1.0, device="cuda")
    moe.moe_norm_quantize(rows, d, "bf16", x, None, None, 1e-6, None, None, q, s)
    want_q, want_s = torch.empty((len(pick), pitch), dtype=torch.uint8, device="cuda"), torch.empty((len(pick), nb), device="cuda")
    moe.moe_norm_quantize(len(pick), d, "bf16", few, None, None, 1e-6, None, None, want_q, want_s)
    torch.cuda.synchronize()
    assert torch.equal(q[pick], want_q) and torch.equal(s[pick], want_s)
    q[pick], s[pick] = 0, qo.TINY
    assert not q.view(torch.int32).any() and bool((s == qo.TINY).all())      # every other row is zeros
