"""How exact the sums of the 8-bit products are, for outputs that would hide it: bf16 and e4m3.

By default sums are fp32, so that the bound of test_quant_gpu.py for fp32 outputs, SUM(K) = (132 + ceil(K / 128)) 2^-23 of sum |a| |w| + |bias|,
holds for every type's result before it is rounded.

With MOE_QUANT_UNIT_SUMS eight neighbouring columns are added as one group, whose products are cut at step = 2^-13 2^floor(log2 largest).
Products of codes have 8 bits, so that only those below 2^-6 of the largest one's power of two lose something: less than step and at most
themselves, c = min(|p|, step).  The losses go towards zero and the signs are random: independent, of mean 0, so that their sum is beyond 8
sqrt(sum c^2) with a probability of 2 exp(-32) (Hoeffding's bound) and never beyond sum c; its rms is at most sqrt(sum c^2).
"""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo
from test_quant_gpu import HALF, LINEAR, VALUES, Product, check_rows, codes_of, say, sum_error, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", LINEAR)
def test_sums_are_fp32(gpu_lib, T, N, K, out):
    moe = gpu_lib
    say(f"[case] fp32 sums {T} x {N} x {K} {out}")
    p = Product(moe, T, N, K, seed=1)
    for act, bias in (("none", False), ("gelu", True)):
        shape = moe.make_quant_shape(T, N, K, 1, 1, act, out)
        y, sc = p.buffers(T, out)
        moe.moe_quant_linear(shape, p.d_a, p.d_as, p.d_w, p.d_ws, torch.from_numpy(p.bias).cuda() if bias else None, y, sc, workspace(moe, shape))
        torch.cuda.synchronize()
        check_rows(y, sc, *p.reference(slice(None), 0, act, bias, "f32"), out)


def cut(a, w):
    """(sum c, sqrt(sum c^2)) of the products of a row a [K] with every row of w [N, K]; the values' scales are theirs."""
    N, K = w.shape
    pad = -K % 8
    p = np.abs(np.pad(a[None] * w, ((0, 0), (0, pad)))).reshape(N, -1, 8)
    top = p.max(2, keepdims=True)
    step = 2.0 ** -13 * 2.0 ** np.floor(np.log2(np.where(top > 0, top, 1)))
    c = np.where(p < 128 * step, np.minimum(p, step), 0)
    return c.sum((1, 2)), np.sqrt((c * c).sum((1, 2)))


@pytest.mark.parametrize("sums", ["f32", "units"])
@pytest.mark.parametrize("T,N,K", [(1, 300, 384), (40, 130, 384), (64, 520, 2048), (100, 256, 1000), (2000, 1024, 640), (5000, 2048, 384)])
def test_what_a_bias_leaves_of_large_sums(gpu_lib, T, N, K, sums):
    """Equal rows, and biases that take away what every sum should be: what is left are the errors, which no rounding hides."""
    moe = gpu_lib
    say(f"[case] sums less themselves {T} x {N} x {K} {sums}")
    p = Product(moe, 1, N, K, seed=2)
    # the scales as powers of two: the products' bits are the codes'
    p.a_scales, p.w_scales = np.exp2(np.floor(np.log2(p.a_scales))), np.exp2(np.floor(np.log2(p.w_scales)))
    a, w = VALUES[codes_of(p.d_a)][0, :K] * qo.spread(p.a_scales.astype(np.float64), 1, K)[0], p.weights(0)
    want, size = qo.linear(a[None], w)
    bias = -want[0].astype(np.float32)
    left = want[0] + bias.astype(np.float64)
    err = sum_error(K) * (size[0] + np.abs(bias))
    most, rms = cut(a, w)
    d_a, d_as = p.d_a.expand(T, -1).contiguous(), torch.from_numpy(p.a_scales).cuda().expand(T, -1).contiguous()
    d_ws, d_bias = torch.from_numpy(p.w_scales).cuda(), torch.from_numpy(bias).cuda()
    for out in ("bf16", "e4m3"):
        shape = moe.make_quant_shape(T, N, K, 1, 1, "none", out, sums=sums)
        y, sc = p.buffers(T, out)
        moe.moe_quant_linear(shape, d_a, d_as, p.d_w, d_ws, d_bias, y, sc, workspace(moe, shape))
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.uint8), y[:1].view(torch.uint8).expand(T, -1))      # equal rows stay equal, wherever they are
        bound = err if sums == "f32" else err + np.minimum(most, 8 * rms)
        check_rows(y[:1], None if sc is None else sc[:1], left[None], bound[None], out)
        if out == "bf16":
            off = y[0].float().cpu().numpy().astype(np.float64) - left
            far = np.sqrt((err ** 2).mean()) + (0 if sums == "f32" else np.sqrt((rms ** 2).mean()))
            assert np.sqrt((off * off).mean()) <= far * (1 + HALF["bf16"]), (np.sqrt((off * off).mean()), far)


@pytest.mark.parametrize("T,N,K", [(1, 16, 256), (64, 130, 256), (64, 130, 4096), (100, 256, 256), (300, 512, 512), (5000, 2048, 256)])
def test_large_products_that_cancel(gpu_lib, T, N, K):
    """448 * 448 - 448 * 448 + six ones in every eight columns: six, in sums of at least 24 bits."""
    moe = gpu_lib
    say(f"[case] products that cancel {T} x {N} x {K}")
    row = torch.ones((T, K), device="cuda")
    row[:, 0::8] = row[:, 1::8] = 448
    w = torch.ones((1, N, K), device="cuda")
    w[:, :, 0::8], w[:, :, 1::8] = 448, -448
    packed = torch.empty(moe.moe_quant_weight_bytes(1, N, K), dtype=torch.uint8, device="cuda")
    moe.moe_quantize_weights(1, N, K, "e4m3", w.to(torch.float8_e4m3fn), packed, None)
    one = torch.ones((T, qo.blocks(K)), device="cuda")
    ones = torch.ones((1, qo.blocks(N), qo.blocks(K)), device="cuda")
    for out in ("f32", "bf16"):
        shape = moe.make_quant_shape(T, N, K, 1, 1, "none", out)
        y = torch.zeros((T, N), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
        moe.moe_quant_linear(shape, row.to(torch.float8_e4m3fn), one, packed, ones, None, y, None, workspace(moe, shape))
        assert (y == 6 * K // 8).all(), y[0, 0]
