"""Sizes of the 8-bit calls at which a launch's own limits lie."""
import numpy as np
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


def guarded(shape, dtype, fill):
    """A buffer with rows before and behind it that nobody may write."""
    buf = torch.full((shape[0] + 64, *shape[1:]), fill, dtype=dtype, device="cuda")
    return buf, buf[32:-32]


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("A,N", [(300, 256), (4000, 512), (9001, 2048)])
def test_offsets_that_are_none(gpu_lib, A, N, out):
    """Offsets that give every other expert all rows, go back, or lie outside: every access stays inside, and as all experts have the same weights,
    a row that is anybody's is right."""
    moe = gpu_lib
    say(f"[case] offsets that are none {A} x {N} {out}")
    E, K = 130, 256
    gen = torch.Generator(device="cuda").manual_seed(A)
    rows = torch.randint(-4, 5, (A, K), device="cuda", generator=gen).float()
    w = torch.randint(-4, 5, (1, N, K), device="cuda", generator=gen).float()
    packed = torch.empty(moe.moe_quant_weight_bytes(E, N, K), dtype=torch.uint8, device="cuda")
    moe.moe_quantize_weights(E, N, K, "e4m3", w.to(torch.float8_e4m3fn).expand(E, N, K).contiguous(), packed, None)
    one, ones = torch.ones((A, 2), device="cuda"), torch.ones((E, qo.blocks(N), 2), device="cuda")
    shape = moe.make_quant_shape(A, N, K, E, 1, "none", out)
    ws = torch.empty(moe.moe_quant_workspace_bytes(shape), dtype=torch.uint8, device="cuda")

    def call(offsets):
        buf, y = guarded((A, N), {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}[out], 77)
        sbuf, s = guarded((A, qo.blocks(N)), torch.float32, -1.0) if out == "e4m3" else (None, None)
        moe.moe_quant_expert_linear(shape, rows.to(torch.float8_e4m3fn), one, None, torch.tensor(offsets, dtype=torch.int32, device="cuda"), None, packed,
                                    ones, None, y, s, ws)
        torch.cuda.synchronize()
        for b in (buf, sbuf):
            assert b is None or ((b[:32] == b[0, 0]).all() and (b[-32:] == b[0, 0]).all() and b[0, 0] in (77, -1.0))
        return y, s

    want = call([0] + [A] * E)
    for offsets in ([A * (e % 2) for e in range(E + 1)], [0, A, -5, 2 ** 31 - 1] * 32 + [0, A, 0], [2 ** 31 - 1 if e % 2 else -2 ** 31 for e in range(E + 1)]):
        for got, ref in zip(call(offsets), want):
            assert got is None or torch.equal(got, ref)


def test_offsets_that_are_none_in_a_large_call(gpu_lib):
    """2^25 rows that 512 experts claim, in 16 column groups: 2^31 units, were they not held to the rows' own."""
    moe = gpu_lib
    say("[case] offsets that are none, 2^25 rows")
    A, N, K, E = 1 << 25, 2048, 128, 1024
    packed = torch.empty(moe.moe_quant_weight_bytes(E, N, K), dtype=torch.uint8, device="cuda")
    w = torch.zeros((E, N, K), dtype=torch.uint8, device="cuda")
    w[:, :, 0] = 0x38                                              # one
    moe.moe_quantize_weights(E, N, K, "e4m3", w, packed, None)
    rows = torch.zeros((A, K), dtype=torch.uint8, device="cuda")
    rows[:, 0] = 0x38
    scales = 1.0 + (torch.arange(A, device="cuda") % 7).float()
    offsets = torch.tensor([A * (e % 2) for e in range(E + 1)], dtype=torch.int32, device="cuda")
    shape = moe.make_quant_shape(A, N, K, E, 1, "none", "e4m3")
    y = torch.full((A, N), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((A, N // 128), -1.0, device="cuda")
    ws = torch.empty(moe.moe_quant_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    moe.moe_quant_expert_linear(shape, rows, scales, None, offsets, None, packed, torch.ones((E, N // 128, 1), device="cuda"), None, y, s, ws)
    torch.cuda.synchronize()
    want = torch.from_numpy(np.arange(1, 8, dtype=np.float32) / np.float32(448)).cuda()     # torch divides by a number with its reciprocal
    assert torch.equal(s, want[torch.arange(A, device="cuda") % 7][:, None].expand(-1, N // 128))
    assert bool((y.view(torch.int64) == 0x7e7e7e7e7e7e7e7e).all())
