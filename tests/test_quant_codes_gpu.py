"""One rule for codes, whichever kernel writes them: v / scale in fp32, to the nearest e4m3 value, ties to even.

Every value here is known to the last bit: m * t in a block whose largest is 448 * m, so that the scale is m and the quotient t, which is
the middle between two codes (and now and then a code).  A reciprocal's rounding would move such a quotient to one side.
"""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo
from test_quant_gpu import VALUES, codes_of, say, workspace

pytestmark = pytest.mark.gpu

# 448, then middles between two codes of every size, both signs, as sums of two codes
HIGH, LOW = np.zeros(128), np.zeros(128)
HIGH[0] = 448.0
for i in range(1, 128):
    e, step = i % 11 - 5, (i // 11) % 8
    HIGH[i], LOW[i] = (8 + step) * 2.0 ** e, 2.0 ** (e - 1)
    if i % 2:
        HIGH[i], LOW[i] = -HIGH[i], -LOW[i]
HIGH, LOW = np.where(np.abs(HIGH) > 224, HIGH / 2, HIGH), np.where(np.abs(HIGH) > 224, LOW / 2, LOW)
HIGH[0] = 448.0
WANT = qo.nearest(HIGH + LOW)


def multipliers(n):
    return 1.0 + np.arange(n) % 1000


def test_the_quotients_are_middles():
    q = (HIGH + LOW)[1:]
    assert np.array_equal(qo.nearest(HIGH), HIGH) and np.array_equal(qo.nearest(LOW), LOW)
    assert (np.abs(q) < 448).all() and (np.abs(np.abs(WANT[1:] - q) - np.abs(LOW[1:])) == 0).all()


@pytest.mark.parametrize("sums", ["f32", "units"])
@pytest.mark.parametrize("T,blocks,K", [(1, 1, 128), (64, 1, 512), (64, 20, 512), (60, 3, 256), (64, 100, 128), (100, 3, 130), (2000, 8, 128), (5000, 16, 256)])
def test_codes_of_products(gpu_lib, T, blocks, K, sums):
    moe = gpu_lib
    say(f"[case] codes of products {T} x {128 * blocks} x {K} {sums}")
    N = 128 * blocks
    last = min(K, 300) - 1                                     # the two codes lie in the first and the last block
    w = np.zeros((1, N, K), dtype=np.float32)
    w[0, :, 0], w[0, :, last] = np.tile(HIGH, blocks), np.tile(LOW, blocks)
    packed = torch.empty(moe.moe_quant_weight_bytes(1, N, K), dtype=torch.uint8, device="cuda")
    moe.moe_quantize_weights(1, N, K, "e4m3", torch.from_numpy(w).cuda().to(torch.float8_e4m3fn), packed, None)
    rows = torch.zeros((T, moe.moe_quant_pitch(K)), device="cuda")
    rows[:, 0] = rows[:, last] = 1
    m = multipliers(T)
    scales = torch.from_numpy(np.repeat(m[:, None], qo.blocks(K), 1).astype(np.float32)).cuda()
    shape = moe.make_quant_shape(T, N, K, 1, 1, "none", "e4m3", sums=sums)
    y = torch.full((T, N), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((T, blocks), -1.0, device="cuda")
    moe.moe_quant_linear(shape, rows.to(torch.float8_e4m3fn), scales, packed, torch.ones((1, blocks, qo.blocks(K)), device="cuda"), None, y, s,
                         workspace(moe, shape))
    torch.cuda.synchronize()
    assert np.array_equal(s.cpu().numpy(), np.repeat(m[:, None], blocks, 1))
    got = VALUES[codes_of(y)].reshape(T, blocks, 128)
    assert (got == WANT).all(), np.argwhere(got != WANT)[:5]


@pytest.mark.parametrize("up", [1.0, 2.0 ** -120, 2.0 ** 100])
def test_codes_of_weights(gpu_lib, up):
    moe = gpu_lib
    say(f"[case] codes of weights x {up}")
    E = 1000
    m = multipliers(E)
    w = np.broadcast_to((HIGH + LOW)[None, None], (E, 3, 128)) * m[:, None, None] * up
    packed = torch.empty(moe.moe_quant_weight_bytes(E, 3, 128), dtype=torch.uint8, device="cuda")
    s = torch.empty((E, 1, 1), device="cuda")
    moe.moe_quantize_weights(E, 3, 128, "f32", torch.from_numpy(w.astype(np.float32)).cuda(), packed, s)
    torch.cuda.synchronize()
    assert np.array_equal(s.cpu().numpy().ravel(), (m * up).astype(np.float32))
    codes = codes_of(packed).reshape(E, 8, 2, 4, 16, 16).transpose(0, 1, 4, 2, 3, 5).reshape(E, 128, 128)[:, :3]
    assert (VALUES[codes] == WANT).all(), np.argwhere(VALUES[codes] != WANT)[:5]


def test_codes_of_random_weights(gpu_lib):
    """Against fp32 division itself, scales of every size (the tiniest among them)."""
    moe = gpu_lib
    say("[case] codes of random weights")
    rng = np.random.default_rng(8)
    E = 500
    w = (rng.standard_normal((E, 128, 128)) * np.exp2(rng.integers(-134, 100, (E, 1, 1)))).astype(np.float32)
    packed = torch.empty(moe.moe_quant_weight_bytes(E, 128, 128), dtype=torch.uint8, device="cuda")
    s = torch.empty((E, 1, 1), device="cuda")
    moe.moe_quantize_weights(E, 128, 128, "f32", torch.from_numpy(w).cuda(), packed, s)
    torch.cuda.synchronize()
    scales = np.maximum(np.abs(w).max((1, 2)) / np.float32(448), np.float32(qo.TINY))
    assert np.array_equal(s.cpu().numpy().ravel(), scales)
    codes = codes_of(packed).reshape(E, 8, 2, 4, 16, 16).transpose(0, 1, 4, 2, 3, 5).reshape(E, 128, 128)
    want = qo.nearest((w / scales[:, None, None]).astype(np.float64))
    assert (VALUES[codes] == want).all(), np.argwhere(VALUES[codes] != want)[:5]
