"""Streamed experts of the 8-bit products on the paths that an encoder pass takes: units of 256 columns (more units of 128 than the GPU has
CUs, in a call of 65 rows and more), and weights of more than 32 MB, which are read as what is read once."""
import numpy as np
import pytest
import torch

from oracle import quant_oracle as qo
from test_quant_gpu import Product, check_rows, say, workspace

pytestmark = pytest.mark.gpu

CACHED = 32 << 20


def check_grouped(moe, sizes, k, N, K, out, sums, masked, act, seed=0):
    E, A, rng = len(sizes), sum(sizes), np.random.default_rng(seed)
    p = Product(moe, A // k, N, K, E, seed)
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    perm = rng.permutation(A).astype(np.int32)
    mask = (rng.random(E) < 0.8).astype(np.uint8) if masked else None
    shape = moe.make_quant_shape(A, N, K, E, k, act, out, sums=sums)
    y, sc = p.buffers(A, out)
    before = (y.clone(), None if sc is None else sc.clone())
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, dev(perm), dev(offsets), dev(mask), p.d_w, p.d_ws, dev(p.bias), y, sc, workspace(moe, shape))
    torch.cuda.synchronize()
    for e in range(E):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        if s.start == s.stop:
            continue
        if masked and not mask[e]:
            assert torch.equal(y[s], before[0][s]) and (sc is None or torch.equal(sc[s], before[1][s]))
            continue
        y_ref, err = p.reference(perm[s] // k, e, act, True, "f32" if sums == "f32" else out)
        check_rows(y[s], None if sc is None else sc[s], y_ref, err, out)


# 70 experts of 0 to 64 rows, every number of row fragments and its ends among them, and an even sum
SIZES = [1, 17, 33, 49, 64, 16, 32, 48, 0, 2, 15, 31, 47, 63, 34, 50] * 4 + [64, 64, 1, 8, 7, 0]


@pytest.mark.parametrize("out,sums", [("f32", "f32"), ("bf16", "f32"), ("bf16", "units"), ("e4m3", "f32"), ("e4m3", "units")])
@pytest.mark.parametrize("N,K", [(520, 300), (512, 64), (1000, 128), (520, 1100), (700, 500)])
def test_units_of_256_columns(gpu_lib, N, K, out, sums):
    """Two blocks of columns per unit and the odd one left over, contractions of one block to nine, past the ring of three."""
    moe = gpu_lib
    say(f"[case] streamed units of 256 columns {N} x {K} {out} {sums}")
    streamed = sum(n > 0 for n in SIZES)
    assert streamed * qo.blocks(N) > torch.cuda.get_device_properties(0).multi_processor_count and sum(SIZES) % 2 == 0 and max(SIZES) <= 64
    check_grouped(moe, SIZES, 2, N, K, out, sums, masked=False, act="gelu")
    check_grouped(moe, SIZES + [300, 70], 1, N, K, out, sums, masked=True, act="relu", seed=1)        # tiles in the same launch


@pytest.mark.parametrize("out,sums", [("f32", "f32"), ("bf16", "f32"), ("bf16", "units"), ("e4m3", "f32"), ("e4m3", "units")])
@pytest.mark.parametrize("sizes,N,K", [
    ([0] * 7 + [64] + [0] * 20 + [3, 1] + [0] * 10, 1024, 1024),                     # 68 rows: units of 128 columns beside tiles
    ([1] * 30 + [0] * 5 + [29], 1024, 1024),                                        # 59 rows, a unit for each expert's columns
    ([0] * 39 + [9], 1024, 1024),                                                   # 9 rows: the contraction is cut
    ([1, 0, 40], 4000, 4096),
])
def test_weights_that_no_cache_holds(gpu_lib, sizes, N, K, out, sums):
    moe = gpu_lib
    say(f"[case] weights read once {sum(sizes)} rows x {N} x {K} {out} {sums}")
    assert moe.moe_quant_weight_bytes(len(sizes), N, K) > CACHED
    check_grouped(moe, sizes, 1, N, K, out, sums, masked=False, act="none")


@pytest.mark.parametrize("out,sums", [("f32", "f32"), ("bf16", "units"), ("e4m3", "f32")])
@pytest.mark.parametrize("T", [1, 33, 64])
def test_a_matrix_that_no_cache_holds(gpu_lib, T, out, sums):
    moe = gpu_lib
    N, K = 4100, 8192
    say(f"[case] a matrix read once {T} x {N} x {K} {out} {sums}")
    assert moe.moe_quant_weight_bytes(1, N, K) > CACHED
    p = Product(moe, T, N, K)
    shape = moe.make_quant_shape(T, N, K, 1, 1, "none", out, sums=sums)
    y, sc = p.buffers(T, out)
    moe.moe_quant_linear(shape, p.d_a, p.d_as, p.d_w, p.d_ws, torch.from_numpy(p.bias).cuda(), y, sc, workspace(moe, shape))
    torch.cuda.synchronize()
    check_rows(y, sc, *p.reference(slice(None), 0, "none", True, "f32" if sums == "f32" else out), out)
