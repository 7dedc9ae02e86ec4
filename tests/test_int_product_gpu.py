"""int8 products against exact sums of whole numbers (oracle/int_oracle.py).

Tolerance, u = 2^-24 (half a step of fp32): the sum is exact; its conversion, the product of the two scales and the multiply-add round once each, so
that the value before the activation is within 2 u of |sa sw sum| plus u of itself: BEFORE = 3 u (|sa sw sum| + |z|).  GeLU and SiLU have slopes of at
most 1.13 and are themselves within 1e-6 max(1, |z|) of 64 bits.  The output is rounded once: half a step, 2^-24 (fp32) or 2^-8 (bf16).
"""
import sys

import numpy as np
import pytest
import torch

from oracle import int_oracle as io
from oracle import quant_oracle as qo

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def workspace(moe, shape):
    n = moe.moe_int_workspace_bytes(shape)
    assert n > 0
    return torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda")


def within(y, z, size, act, out):
    want = io.activate(z, act)
    err = 3 * 2.0 ** -24 * (size + np.abs(z))
    if act in ("gelu", "silu"):
        err = 1.13 * err + 1e-6 * np.maximum(1.0, np.abs(z))
    err = err * (1 + HALF[out]) + HALF[out] * np.abs(want) + 2.0 ** -126
    got = y.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= err)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


class Problem:
    def __init__(self, moe, rows, N, K, E=1, seed=0, extreme=False):
        rng = self.rng = np.random.default_rng(seed)
        self.moe, self.N, self.K, self.E = moe, N, K, E
        draw = (lambda s: rng.choice(np.array([-128, -127, 127], dtype=np.int8), s)) if extreme else (lambda s: rng.integers(-128, 128, s).astype(np.int8))
        self.a, self.w = draw((rows, K)), draw((E, N, K))
        self.sa = np.exp(rng.normal(size=rows)).astype(np.float32)
        self.sw = (np.exp(0.3 * rng.normal(size=(E, N))) / (5000 * np.sqrt(K))).astype(np.float32)
        self.bias = rng.normal(size=(E, N)).astype(np.float32)
        full = np.full((rows, moe.moe_quant_pitch(K)), 0, dtype=np.int8)
        full[:, :K] = self.a
        self.d_a, self.d_sa, self.d_sw, self.d_bias = dev(full), dev(self.sa), dev(self.sw), dev(self.bias)
        self.d_w = torch.empty(moe.moe_quant_weight_bytes(E, N, K), dtype=torch.int8, device="cuda")
        moe.moe_quantize_weights_int(E, N, K, "i8", dev(self.w), self.d_w, None)

    def linear(self, T, act, bias, out, offset=0):
        moe, N = self.moe, self.N
        shape = moe.make_quant_shape(T, N, self.K, 1, 1, act, out)
        y = torch.full(((T + 1) * N + offset,), 77.0, dtype=DT[out], device="cuda")[offset:].view(T + 1, N)
        moe.moe_int_linear(shape, self.d_a, self.d_sa, self.d_w, self.d_sw, self.d_bias if bias else None, y, workspace(moe, shape))
        torch.cuda.synchronize()
        assert (y[T:] == 77).all()
        z, size = io.product(self.a[:T], self.sa[:T], self.w[0], self.sw[0], self.bias[0] if bias else None)
        within(y[:T], z, size, act, out)
        return y

    def experts(self, sizes, k, act, bias, out, gather=True, mask=None, behind=0):
        """Rows of all experts and `behind` more, which belong to none."""
        moe, N, E = self.moe, self.N, self.E
        A = sum(sizes) + behind
        assert A % k == 0 and len(sizes) == E
        offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        perm = self.rng.permutation(A).astype(np.int32) if gather else None
        shape = moe.make_quant_shape(A, N, self.K, E, k if gather else 1, act, out)
        y = torch.full((A, N), 77.0, dtype=DT[out], device="cuda")
        moe.moe_int_expert_linear(shape, self.d_a, self.d_sa, dev(perm), dev(offsets), dev(mask), self.d_w, self.d_sw, self.d_bias if bias else None, y,
                                  workspace(moe, shape))
        torch.cuda.synchronize()
        for e in range(E):
            s = slice(int(offsets[e]), int(offsets[e + 1]))
            if s.start == s.stop:
                continue
            if mask is not None and not mask[e]:
                assert (y[s] == 77).all()
                continue
            rows = perm[s] // k if gather else np.arange(s.start, s.stop)
            z, size = io.product(self.a[rows], self.sa[rows], self.w[e], self.sw[e], self.bias[e] if bias else None)
            within(y[s], z, size, act, out)
        assert (y[offsets[-1]:] == 77).all()
        return y


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N,K", [(1, 1), (7, 40), (128, 128), (130, 129), (300, 1000), (1000, 513), (2048, 256), (264, 2048)])
def test_linear_sizes(gpu_lib, N, K, out):
    p = Problem(gpu_lib, 700, N, K)
    for i, T in enumerate([1, 2, 15, 16, 17, 33, 48, 64, 65, 100, 128, 129, 200, 255, 256, 257, 384, 700]):
        say(f"[case] int linear {T} x {N} x {K} {out}")
        p.linear(T, ["none", "relu", "gelu", "silu"][i % 4], i % 3 != 0, out, offset=i % 2)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", [(1, 2048, 8192), (32, 4096, 2048), (64, 640, 4100), (300, 4096, 512), (2500, 1024, 384), (5000, 2048, 128), (4200, 2050, 300),
                                   (9000, 1100, 640)])
def test_linear_large(gpu_lib, T, N, K, out):
    """Several units per block, each kind of tile, a contraction of one block and of many; weights of 16 MB."""
    say(f"[case] int linear {T} x {N} x {K} {out}")
    Problem(gpu_lib, T, N, K, seed=T).linear(T, "none", True, out)


def test_sums_are_exact_at_the_longest_contraction(gpu_lib):
    """Codes of -128 throughout: the sum is within 2^14 of 2^31.  What is left of it after taking the largest part away is exact too."""
    moe, K = gpu_lib, gpu_lib.MOE_INT_MAX_K
    say("[case] int longest contraction")
    for T in (3, 70):
        p = Problem(moe, T, 20, K, extreme=True)
        p.a[:], p.w[:, :10] = -128, -128
        p.a[1, :] = 127
        p.sa[:], p.sw[:] = 1, 1
        full = np.zeros((T, moe.moe_quant_pitch(K)), dtype=np.int8)
        full[:, :K] = p.a
        p.d_a, p.d_sa, p.d_sw = dev(full), dev(p.sa), dev(p.sw)
        moe.moe_quantize_weights_int(1, 20, K, "i8", dev(p.w), p.d_w, None)
        y = p.linear(T, "none", False, "f32")
        exact = p.a.astype(np.int64) @ p.w[0].astype(np.int64).T
        assert exact.max() == 128 * 128 * K and np.array_equal(y[:T].cpu().numpy(), exact.astype(np.float32))


SIZES = [1, 17, 33, 49, 64, 16, 32, 48, 0, 2, 15, 31, 47, 63, 34, 50]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", [(1, 100, 1700), (3, 130, 14000), (16, 2000, 9000), (40, 300, 20011), (64, 2048, 4096), (64, 8192, 2048), (64, 4100, 16400), (5, 1, 131071),
                                   (64, 16, 131071)])
def test_linear_of_few_rows(gpu_lib, T, N, K, out):
    """Contractions that are cut into many parts, into a few and not at all, of unequal lengths."""
    test_linear_large(gpu_lib, T, N, K, out)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("sizes,k,N,K", [
    ([3, 0, 1, 0], 2, 200, 300), ([0, 0, 0, 64], 1, 1024, 2048), ([0, 65], 1, 130, 256), ([64, 65, 0, 129, 1, 257, 130, 0], 2, 384, 200),
    (SIZES * 4, 2, 520, 300), (SIZES * 4 + [300, 70], 1, 520, 128), ([400, 0, 3, 5, 0, 0, 90, 700], 2, 1000, 640), ([2] * 200 + [0] * 300, 1, 256, 384),
    ([1000, 1, 64, 65, 66, 128, 129, 255, 256, 257], 1, 260, 130), ([0] * 9, 1, 64, 64), ([1] * 30 + [0] * 5 + [28], 1, 1024, 1024),
])
def test_experts(gpu_lib, sizes, k, N, K, masked, out):
    say(f"[case] int experts {sum(sizes)} rows of {len(sizes)} k {k} x {N} x {K} masked {masked} {out}")
    rng = np.random.default_rng(len(sizes))
    behind = (-sum(sizes)) % k + 2 * k
    p = Problem(gpu_lib, sum(sizes) + behind, N, K, len(sizes))
    mask = rng.integers(0, 2, len(sizes)).astype(np.uint8) if masked else None
    p.experts(sizes, k, "silu", True, out, mask=mask, behind=behind)
    p.experts(sizes, 1, "relu", False, out, gather=False, mask=mask)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("sizes,N,K", [
    ([4000, 5000, 100, 3, 64, 120, 0, 65, 1, 30], 1024, 300), ([9000, 0, 0, 0], 1100, 128), ([8500] + [7, 0, 90] * 60, 1024, 384), ([5000, 5000, 128, 127], 1024, 1100),
    ([3000, 1] * 2 + [66] * 9, 3000, 200), ([2, 9100, 60], 1024, 130), ([1500] * 5 + [5] * 5, 1300, 520),
])
def test_experts_side_by_side(gpu_lib, sizes, N, K, masked, out):
    """A round of long tiles and more, which some of the CUs leave to the others while they do what memory bounds; sums of one to nine blocks."""
    say(f"[case] int experts side by side {sum(sizes)} rows of {len(sizes)} x {N} x {K} masked {masked} {out}")
    behind = (-sum(sizes)) % 2
    p = Problem(gpu_lib, sum(sizes) + behind, N, K, len(sizes))
    mask = (np.random.default_rng(3).random(len(sizes)) < 0.8).astype(np.uint8) if masked else None
    p.experts(sizes, 2, "gelu" if masked else "relu", True, out, mask=mask, behind=behind)


@pytest.mark.parametrize("sizes,N,K", [([0] * 7 + [64] + [0] * 20 + [3, 1] + [0] * 10, 1024, 1024), ([0] * 39 + [9], 1024, 1024), ([1, 0, 40], 4000, 4096)])
def test_weights_that_no_cache_holds(gpu_lib, sizes, N, K):
    say(f"[case] int weights read once {sum(sizes)} rows of {len(sizes)} x {N} x {K}")
    assert gpu_lib.moe_quant_weight_bytes(len(sizes), N, K) > 32 << 20
    Problem(gpu_lib, sum(sizes), N, K, len(sizes)).experts(sizes, 1, "none", True, "f32")


def test_offsets_and_perm_that_are_none(gpu_lib):
    """Wrong offsets and places give wrong rows, inside the buffers."""
    moe = gpu_lib
    N, K, E = 200, 260, 6
    for A in (40, 300):
        p = Problem(moe, A, N, K, E)
        shape = moe.make_quant_shape(A, N, K, E, 2, "none", "f32")
        guard = torch.full((A + 64, N), 77.0, device="cuda")
        for offsets in ([0, 1 << 30, -5, 3, 1 << 30, 7, 2], [0, A, 0, A, 0, A, 0], [-(1 << 31)] * 7, [(1 << 31) - 1] * 7, [5, 4, 3, 2, 1, 0, A]):
            say(f"[case] int wrong offsets {A} {offsets}")
            perm = np.random.default_rng(1).integers(-(1 << 31), (1 << 31) - 1, A).astype(np.int32)
            moe.moe_int_expert_linear(shape, p.d_a, p.d_sa, dev(perm), dev(np.array(offsets, dtype=np.int32)), None, p.d_w, p.d_sw, p.d_bias, guard,
                                      workspace(moe, shape))
            torch.cuda.synchronize()
            assert (guard[A:] == 77).all()


def test_scales_that_are_none(gpu_lib):
    """A row of NaN scale is NaN, its neighbours are not; so is a channel."""
    moe = gpu_lib
    for T in (5, 300):
        say(f"[case] int NaN scales {T}")
        p = Problem(moe, T, 150, 200)
        p.d_sa[3], p.d_sw[0, 7] = float("nan"), float("nan")
        shape = moe.make_quant_shape(T, 150, 200, 1, 1, "relu", "f32")
        y = torch.empty((T, 150), device="cuda")
        moe.moe_int_linear(shape, p.d_a, p.d_sa, p.d_w, p.d_sw, None, y, workspace(moe, shape))
        torch.cuda.synchronize()
        nan = torch.isnan(y)
        want = torch.zeros_like(nan)
        want[3], want[:, 7] = True, True
        assert torch.equal(nan, want)


def test_results_do_not_depend_on_the_cut(gpu_lib):
    """The same rows alone, in a streamed call, a cut one and a tiled one, bit for bit; and every call again."""
    moe = gpu_lib
    N, K = 384, 4096
    say("[case] int cuts")
    p = Problem(moe, 600, N, K)
    ys = {T: p.linear(T, "silu", True, "f32")[:T].clone() for T in (1, 40, 64, 65, 300, 600)}
    for T, y in ys.items():
        assert torch.equal(y, ys[600][:T]), T
        assert torch.equal(p.linear(T, "silu", True, "f32")[:T], y)
