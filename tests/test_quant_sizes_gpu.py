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


@pytest.mark.parametrize("E,N", [(1, 1 << 24), (2, 32768 * 128), (3, 32768 * 128 + 1), (1, 65536 * 128 + 300)])
def test_weights_of_many_rows(gpu_lib, E, N):
    """Matrices with more blocks of 128 rows than one direction of a launch has blocks, up to the largest that the calls accept."""
    moe = gpu_lib
    say(f"[case] moe_quantize_weights {E} x {N} x 1")
    w = torch.zeros((E, N, 1), device="cuda")
    codes = torch.arange(N, device="cuda") % 128 % 5            # 448 m, 0, -224 m, 112 m, 7 m / 2: codes of a block whose scale is m
    value = torch.tensor([448.0, 0.0, -224.0, 112.0, 3.5], device="cuda")[codes]
    m = 1.0 + torch.arange(qo.blocks(N), device="cuda") % 1000
    for e in range(E):
        w[e, :, 0] = value * m.repeat_interleave(128)[:N] * (e + 1)
    dst = torch.full((moe.moe_quant_weight_bytes(E, N, 1),), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((E, qo.blocks(N), 1), -1.0, device="cuda")
    moe.moe_quantize_weights(E, N, 1, "f32", w, dst, scales)
    torch.cuda.synchronize()
    want = torch.zeros(qo.blocks(N) * 128, device="cuda")
    want[:N] = value
    for e in range(E):
        assert torch.equal(scales[e, :, 0], m * (e + 1))
        got = dst.view(E, -1)[e].view(-1, 2, 4, 16, 16)         # row r of a fragment begins at byte 16 r, its one column there
        assert torch.equal(got[:, 0, 0, :, 0].flatten().view(torch.float8_e4m3fn).float(), want)
        assert not got[:, 1].any() and not got[:, 0, 1:].any() and not got[:, 0, 0, :, 1:].any()
