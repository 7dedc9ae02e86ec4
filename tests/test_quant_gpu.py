"""GPU parity of the 8-bit layers with the 64-bit reference (oracle/quant_oracle.py).

Tolerances, from the arithmetic and the formats (u = 2^-24, half a step of fp32):
  norm: a sum of d squares in chains of at most 8 and a tree (d <= 16384: 8 + 8 + 6 + 4 additions, relative error of each u, halved by the
    square root), mean, eps, root, quotient and two products: n is within 30 u = 1.8e-6 of the 64-bit value; rows that are read twice
    (d > 16384) add d / 2048 additions.  NORM = 3e-6 covers both at the lengths used.
  product: every product of two codes is exact in fp32.  A sum of the 128 of a block is at most 128 steps of 2^-23 (a matrix unit
    may truncate) of the sum of magnitudes off, scaling and adding up ceil(K / 128) blocks that many more, bias and the two scales'
    product 4: SUM(K) = (132 + ceil(K / 128)) 2^-23 of sum |a| |w| + |bias|.  GeLU has a slope of at most 1.13 and is itself
    within 1e-6 max(1, |z|) of 64 bits.
    bf16 and e4m3 outputs may come from the matrix units for 8-bit operands, which add products in groups of eight and cut seven of them at
    2^-13 of the largest one's power of two: at most 7 2^-13 of the sum of the groups' largest, so of sum |a| |w|.  The cuts go towards zero,
    so with random signs they are independent, of mean 0 and a variance of at most 2^-26 / 3 of the largest one's square each; the groups'
    largest squares add up to at most sum a^2 w^2: CUT = 8 standard deviations = 8 2^-13 sqrt(7 / 3 sum a^2 w^2), where that is less.
  rounding to the output: half a step, 2^-24 (fp32), 2^-8 (bf16), 2^-4 (e4m3; below 2^-6 times the scale 2^-10 times the scale), of a value that
    is itself off by the error above.
"""
import ctypes
import sys

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import quant_oracle as qo

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NORM = 3e-6
VALUES = qo.code_values()


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def sum_error(K):
    return (132 + qo.blocks(K)) * 2.0 ** -23


def cut_error(a, w):
    """CUT of every row of `a` with every row of `w`."""
    return np.minimum(7 * 2.0 ** -13 * (np.abs(a) @ np.abs(w).T), 8 * 2.0 ** -13 * np.sqrt(7 / 3 * ((a * a) @ (w * w).T)))


def torch_dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def rounded(v, dtype):
    return wl.round_to_storage(v.astype(np.float32), dtype)


def codes_of(t):
    return t.cpu().view(torch.uint8).numpy()


def assert_codes(q, scales, ref, error, pad_from):
    """Quantised rows against 64-bit values `ref` that the device knows to `error` (absolute, per element): the scale follows the block's
    maximum, every code is a nearest one of a value within the error, and codes past the end are zero."""
    R, C = ref.shape
    assert not q[:, pad_from:].any()
    nb = qo.blocks(C)
    got = VALUES[q[:, :C]]
    for b in range(nb):
        s = slice(b * qo.BLOCK, min(C, (b + 1) * qo.BLOCK))
        most, slack = np.abs(ref[:, s]).max(1), error[:, s].max(1)
        want = np.maximum(most / qo.TOP, qo.TINY)
        assert (np.abs(scales[:, b] - want) <= slack / qo.TOP + 2.0 ** -22 * want).all()
        v, e = ref[:, s] / scales[:, b:b + 1], error[:, s] / scales[:, b:b + 1] + 2.0 ** -22 * np.abs(ref[:, s] / scales[:, b:b + 1])
        lo, hi = qo.nearest(np.clip(v - e, -460, 460)), qo.nearest(np.clip(v + e, -460, 460))
        bad = ~((got[:, s] >= lo) & (got[:, s] <= hi))
        assert not bad.any(), (b, np.argwhere(bad)[:5], v[bad][:5], got[:, s][bad][:5])


# ---- norm -----------------------------------------------------------------------------------------------------------
def run_norm(moe, x, res, w, eps, dtype, want_sum=True, want_norm=True, offset=0):
    rows, d = x.shape
    td = torch_dtype(dtype)

    def dev(a, t):
        if a is None:
            return None
        buf = torch.empty(a.size + offset, dtype=t, device="cuda")      # `offset` elements in: not 16-byte aligned
        buf[offset:].copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).reshape(-1).to(t))
        return buf[offset:].view(a.shape)

    new = lambda: torch.full((rows * d + offset,), 7.0, dtype=td, device="cuda")[offset:].view(rows, d)
    s, n = (new() if want_sum else None), (new() if want_norm else None)
    q = torch.full((rows, moe.moe_quant_pitch(d)), 0x55, dtype=torch.uint8, device="cuda")
    sc = torch.full((rows, qo.blocks(d)), -1.0, device="cuda")
    moe.moe_norm_quantize(rows, d, dtype, dev(x, td), dev(res, td), dev(w, torch.float32), eps, s, n, q, sc)
    torch.cuda.synchronize()
    out = [None if t is None else t.float().cpu().numpy().astype(np.float64) for t in (s, n)]
    return out[0], out[1], codes_of(q), sc.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 5), (1, 127), (2, 128), (5, 130), (7, 768), (4, 1000), (33, 2048), (1, 2049), (6, 4104),
                                    (2, 16384), (2, 16390), (3, 20480), (1, 40000)])
def test_norm(gpu_lib, dtype, rows, d):
    say(f"[case] moe_norm_quantize {dtype} {rows} x {d}")
    rng = np.random.default_rng(rows * 100003 + d)
    for res in (False, True):
        for weight in (False, True):
            x = rounded(rng.standard_normal((rows, d)) * np.exp(rng.standard_normal((rows, 1))), dtype)
            r = rounded(3 * rng.standard_normal((rows, d)), dtype) if res else None
            w = np.exp(0.3 * rng.standard_normal(d)).astype(np.float32) if weight else None
            s, n, q, sc = run_norm(gpu_lib, x, r, w, 1e-5, dtype, want_sum=weight, want_norm=res, offset=int(weight and not res))
            total = x if r is None else rounded(x + r, dtype)                # one fp32 addition, one rounding
            if weight:
                assert np.array_equal(s, total.astype(np.float64))
            ref = qo.norm(total.astype(np.float64), None if w is None else w.astype(np.float64), 1e-5)
            if res:
                assert (np.abs(n - ref) <= (HALF[dtype] + NORM) * np.abs(ref) * 1.001).all()
            assert_codes(q, sc, ref, NORM * np.abs(ref), d)


def test_norm_special_rows(gpu_lib):
    """Rows of zeros, a NaN, an infinity, tiny and large values: a bad value stays in its row, and codes past the end stay zero."""
    say("[case] moe_norm_quantize special rows")
    d = 300
    x = np.random.default_rng(3).standard_normal((6, d)).astype(np.float32)
    x[0] = 0
    x[1, 200] = np.nan
    x[2, 7] = -np.inf
    x[3] *= 1e-18
    x[4] *= 1e15
    s, n, q, sc = run_norm(gpu_lib, x, None, None, 0.0, "f32")
    v = VALUES[q[:, :d]]
    for row in (0, 1):                 # 0 / sqrt(0), and a NaN in the sum of squares
        assert np.isnan(v[row]).all() and np.isnan(sc[row]).all() and np.isnan(n[row]).all()
    assert np.isnan(n[2, 7]) and np.isnan(v[2, :128]).all() and not v[2, 128:].any() and (sc[2, 1:] == qo.TINY).all()
    assert not q[:, d:].any()
    ref = qo.norm(x[3:].astype(np.float64), None, 0.0)
    assert_codes(q[3:], sc[3:], ref, NORM * np.abs(ref), d)
    s, n, q, sc = run_norm(gpu_lib, x[:1], None, None, 1e-6, "f32")
    assert not q.any() and (sc == qo.TINY).all() and not n.any()


def test_norm_in_place(gpu_lib):
    """The sum may replace x or the residual, also in rows that are read twice."""
    moe = gpu_lib
    for d in (512, 20000):
        say(f"[case] moe_norm_quantize in place, {d}")
        gen = torch.Generator(device="cuda").manual_seed(d)
        x, r = (torch.randn((5, d), device="cuda", generator=gen).bfloat16() for _ in range(2))
        q = [torch.empty((5, moe.moe_quant_pitch(d)), dtype=torch.uint8, device="cuda") for _ in range(3)]
        sc = [torch.empty((5, qo.blocks(d)), device="cuda") for _ in range(3)]
        s = torch.empty_like(x)
        x1, r1 = x.clone(), r.clone()
        moe.moe_norm_quantize(5, d, "bf16", x, r, None, 1e-6, s, None, q[0], sc[0])
        moe.moe_norm_quantize(5, d, "bf16", x1, r, None, 1e-6, x1, None, q[1], sc[1])
        moe.moe_norm_quantize(5, d, "bf16", x, r1, None, 1e-6, r1, None, q[2], sc[2])
        assert torch.equal(x1, s) and torch.equal(r1, s)
        for i in (1, 2):
            assert torch.equal(q[0], q[i]) and torch.equal(sc[0], sc[i])


# ---- weights --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (1, 16, 128), (2, 130, 200), (3, 128, 256), (1, 300, 96)])
def test_weights(gpu_lib, E, N, K):
    moe = gpu_lib
    say(f"[case] moe_quantize_weights {E} x {N} x {K}")
    rng = np.random.default_rng(E * 7 + N + K)
    codes = rng.integers(0, 256, (E, N, K), dtype=np.uint8)
    dst = torch.full((moe.moe_quant_weight_bytes(E, N, K),), 0x55, dtype=torch.uint8, device="cuda")
    moe.moe_quantize_weights(E, N, K, "e4m3", torch.from_numpy(codes).cuda(), dst, None)
    assert np.array_equal(codes_of(dst), np.concatenate([qo.pack(c) for c in codes]))
    for dtype in ("f32", "bf16"):
        w = rounded(rng.standard_normal((E, N, K)) * np.exp(rng.standard_normal((E, N, 1))), dtype)
        w[0, :128, :128] *= 0 if N > 128 else 1
        sc = torch.full((E, qo.blocks(N), qo.blocks(K)), -1.0, device="cuda")
        moe.moe_quantize_weights(E, N, K, dtype, torch.from_numpy(w).to(torch_dtype(dtype)).cuda(), dst, sc)
        got, sc = codes_of(dst).reshape(E, -1), sc.cpu().numpy().astype(np.float64)
        for e in range(E):
            want = qo.weight_scales(w[e].astype(np.float64))
            assert (np.abs(sc[e] - want) <= 2.0 ** -23 * want).all()
            # unpack by packing the positions
            order = np.full(got.shape[1], -1, dtype=np.int64)
            for byte in range(4):
                part = qo.pack(((np.arange(N * K) + 1) >> (8 * byte) & 255).astype(np.uint8).reshape(N, K)).astype(np.int64)
                order = np.where(byte == 0, part, order + (part << (8 * byte)))
            assert not got[e][order == 0].any()
            flat = np.empty(N * K, dtype=np.uint8)
            flat[order[order > 0] - 1] = got[e][order > 0]
            v = w[e].astype(np.float64) / qo.spread(sc[e], N, K)
            lo, hi = qo.nearest(v - 2.0 ** -22 * np.abs(v)), qo.nearest(v + 2.0 ** -22 * np.abs(v))
            c = VALUES[flat].reshape(N, K)
            assert ((c >= lo) & (c <= hi)).all()


@pytest.mark.parametrize("dtype", ["e4m3", "bf16", "f32"])
@pytest.mark.parametrize("N,K", [(130, 200), (128, 256), (17, 131)])
def test_weights_from_any_address(gpu_lib, N, K, dtype):
    """Weights that begin on a multiple of their element's size only."""
    moe = gpu_lib
    say(f"[case] moe_quantize_weights from odd addresses {N} x {K} {dtype}")
    w = torch.randn((2, N, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(N + K))
    w = w.to(torch.float8_e4m3fn).view(torch.uint8) if dtype == "e4m3" else w.to(torch_dtype(dtype))
    got = []
    for offset in (0, 1, 3):
        src = torch.empty(w.numel() + offset, dtype=w.dtype, device="cuda")[offset:].view(w.shape)
        src.copy_(w)
        dst = torch.full((moe.moe_quant_weight_bytes(2, N, K),), 0x55, dtype=torch.uint8, device="cuda")
        sc = None if dtype == "e4m3" else torch.full((2, qo.blocks(N), qo.blocks(K)), -1.0, device="cuda")
        moe.moe_quantize_weights(2, N, K, dtype, src, dst, sc)
        got.append((dst, sc))
    for dst, sc in got[1:]:
        assert torch.equal(dst, got[0][0]) and (sc is None or torch.equal(sc, got[0][1]))


# ---- products -------------------------------------------------------------------------------------------------------
class Product:
    """Seeded operands of a product, their values for the reference and their device copies."""

    def __init__(self, moe, T, N, K, E=1, seed=0, spread=1.0):
        rng = np.random.default_rng(seed * 1000003 + T * 1009 + N * 31 + K * 7 + E)
        self.moe, self.T, self.N, self.K, self.E, self.rng = moe, T, N, K, E, rng
        a = rng.standard_normal((T, K)) * np.exp(spread * rng.standard_normal((T, 1)))
        q, s = qo.quantize_rows(a)
        self.a_scales = s.astype(np.float32)
        self.a = qo.dequantize_rows(q, self.a_scales.astype(np.float64))
        pitch = moe.moe_quant_pitch(K)
        aq = np.zeros((T, pitch), dtype=np.float32)
        aq[:, :K] = q
        w = qo.nearest(np.clip(rng.standard_normal((E, N, K)) * 112, -448, 448))
        self.w_scales = (np.exp(0.3 * rng.standard_normal((E, qo.blocks(N), qo.blocks(K)))) / 112 / K ** 0.5).astype(np.float32)
        self.w_codes = w
        self.d_a = torch.from_numpy(aq).cuda().to(torch.float8_e4m3fn)
        self.d_as, self.d_ws = torch.from_numpy(self.a_scales).cuda(), torch.from_numpy(self.w_scales).cuda()
        self.d_w = torch.empty(moe.moe_quant_weight_bytes(E, N, K), dtype=torch.uint8, device="cuda")
        moe.moe_quantize_weights(E, N, K, "e4m3", torch.from_numpy(w.astype(np.float32)).cuda().to(torch.float8_e4m3fn), self.d_w, None)
        self.bias = (0.5 * rng.standard_normal((E, N))).astype(np.float32)

    def weights(self, e):
        return self.w_codes[e] * qo.spread(self.w_scales[e].astype(np.float64), self.N, self.K)

    def reference(self, rows, e, act, bias, out):
        """(values, error bound of the result before it is rounded to `out`) of rows of `a` with matrix e."""
        y, size = qo.linear(self.a[rows], self.weights(e), self.bias[e].astype(np.float64) if bias else None, act)
        err = sum_error(self.K) * size
        if out != "f32":
            err = err + cut_error(self.a[rows], self.weights(e))
        if act == "gelu":
            err = 1.13 * err + 1e-6 * np.maximum(1, size)
        return y, err

    def buffers(self, rows, out, offset=0):
        moe, N = self.moe, self.N
        if out == "e4m3":
            return (torch.full((rows, moe.moe_quant_pitch(N)), 0x55, dtype=torch.uint8, device="cuda"),
                    torch.full((rows, qo.blocks(N)), -1.0, device="cuda"))
        return torch.full((rows * N + offset,), 7.0, dtype=torch_dtype(out), device="cuda")[offset:].view(rows, N), None


def workspace(moe, shape):
    return torch.empty(moe.moe_quant_workspace_bytes(shape), dtype=torch.uint8, device="cuda").fill_(0xff)


def check_rows(got, scales, ref, err, out):
    if out == "e4m3":
        assert_codes(codes_of(got), scales.cpu().numpy().astype(np.float64), ref, err, ref.shape[1])
    else:
        v = got.float().cpu().numpy().astype(np.float64)
        bad = ~(np.abs(v - ref) <= err + HALF[out] * (np.abs(ref) + err))
        assert not bad.any(), (np.argwhere(bad)[:5], v[bad][:5], ref[bad][:5], err[bad][:5])


LINEAR = [(1, 1, 1), (1, 16, 128), (2, 100, 130), (16, 128, 256), (17, 48, 7), (33, 384, 500), (48, 130, 384), (64, 200, 640), (65, 256, 128),
          (100, 129, 1000), (128, 256, 256), (200, 512, 2048), (257, 384, 512), (300, 260, 1152), (520, 768, 256), (700, 130, 96), (1000, 520, 768),
          # enough units for tiles of 128 and of 256 rows; contractions shorter than the rings
          (3000, 1024, 128), (2950, 1000, 200), (5000, 2048, 100), (5001, 2050, 384), (4900, 2048, 640)]


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", LINEAR)
def test_linear(gpu_lib, T, N, K, out):
    moe = gpu_lib
    say(f"[case] moe_quant_linear {T} x {N} x {K} {out}")
    p = Product(moe, T, N, K)
    for act, bias, offset in (("none", False, 0), ("relu", True, 1), ("gelu", True, 0)):
        shape = moe.make_quant_shape(T, N, K, 1, 1, act, out)
        y, sc = p.buffers(T, out, offset)
        moe.moe_quant_linear(shape, p.d_a, p.d_as, p.d_w, p.d_ws, torch.from_numpy(p.bias).cuda() if bias else None, y, sc, workspace(moe, shape))
        torch.cuda.synchronize()
        check_rows(y, sc, *p.reference(slice(None), 0, act, bias, out), out)


def grouped_case(p, sizes, k, rng):
    """Rows in expert order with `sizes` rows each; with k > 1 a permutation of T k assignments."""
    A = sum(sizes)
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    perm = rng.permutation(A).astype(np.int32)
    return A, offsets, perm


GROUPS = {
    "empty_and_small": ([0, 1, 0, 5, 17, 0, 40], 2, 200, 260),
    "one": ([9], 1, 130, 128),
    "all_empty_but_last": ([0] * 40 + [30], 2, 64, 300),
    "tile_edges": ([16, 32, 64, 63, 65, 128, 129, 1], 2, 256, 384),
    "large_and_small": ([300, 3, 0, 260, 70, 1, 130, 512], 2, 384, 512),
    "many": ([1, 0, 2] * 340, 2, 32, 64),
    "long": ([700, 2], 1, 520, 2176),
    # every kind of tile and streamed experts in one launch, with tiles of 256 and of 128 rows
    "all_kinds": ([1300, 70, 3, 0, 256, 190, 2000, 64, 1000, 257, 17, 65], 2, 2048, 300),
    "all_kinds_128": ([1300, 70, 3, 0, 256, 190, 64, 900, 257, 17, 65], 2, 1000, 200),
}


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("name", list(GROUPS))
def test_expert_linear(gpu_lib, name, out):
    moe = gpu_lib
    sizes, k, N, K = GROUPS[name]
    say(f"[case] moe_quant_expert_linear {name} {out}")
    E = len(sizes)
    rng = np.random.default_rng(E + N)
    A = sum(sizes)
    for gather in (True, False):
        kk = k if gather and A % k == 0 else 1
        p = Product(moe, A // kk, N, K, E)
        A, offsets, perm = grouped_case(p, sizes, kk, rng)
        source = perm // kk if gather else np.arange(A)
        for mask in (None, (rng.random(E) < 0.6).astype(np.uint8)):
            act, bias = ("relu", True) if gather else ("none", False)
            shape = moe.make_quant_shape(A, N, K, E, kk, act, out)
            y, sc = p.buffers(A, out)
            before = (y.clone(), None if sc is None else sc.clone())
            moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, torch.from_numpy(perm).cuda() if gather else None, torch.from_numpy(offsets).cuda(),
                                        None if mask is None else torch.from_numpy(mask).cuda(), p.d_w, p.d_ws,
                                        torch.from_numpy(p.bias).cuda() if bias else None, y, sc, workspace(moe, shape))
            torch.cuda.synchronize()
            for e in range(E):
                s = slice(int(offsets[e]), int(offsets[e + 1]))
                if s.start == s.stop:
                    continue
                if mask is not None and not mask[e]:
                    assert torch.equal(y[s], before[0][s]) and (sc is None or torch.equal(sc[s], before[1][s]))
                    continue
                check_rows(y[s], None if sc is None else sc[s], *p.reference(source[s], e, act, bias, out), out)


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("T,N,K", [(3, 256, 1024), (60, 200, 300), (300, 384, 640), (5000, 2048, 300)])
def test_outlier_columns(gpu_lib, T, N, K, out):
    """One column of every block a hundred times the others, as activations have them: what a matrix unit may cut is largest there."""
    moe = gpu_lib
    say(f"[case] outlier columns {T} x {N} x {K} {out}")
    p = Product(moe, T, N, K)
    a = p.rng.standard_normal((T, K))
    a[:, 5::128] *= 100
    q, s = qo.quantize_rows(a)
    p.a_scales = s.astype(np.float32)
    p.a = qo.dequantize_rows(q, p.a_scales.astype(np.float64))
    padded = np.zeros((T, moe.moe_quant_pitch(K)), dtype=np.float32)
    padded[:, :K] = q
    p.d_a, p.d_as = torch.from_numpy(padded).cuda().to(torch.float8_e4m3fn), torch.from_numpy(p.a_scales).cuda()
    shape = moe.make_quant_shape(T, N, K, 1, 1, "none", out)
    y, sc = p.buffers(T, out)
    moe.moe_quant_linear(shape, p.d_a, p.d_as, p.d_w, p.d_ws, None, y, sc, workspace(moe, shape))
    torch.cuda.synchronize()
    check_rows(y, sc, *p.reference(slice(None), 0, "none", False, out), out)


@pytest.mark.parametrize("out", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("rows", [5, 64, 900])
def test_nothing_to_do(gpu_lib, rows, out):
    """Every expert masked out, and rows that are no expert's: nothing is written."""
    moe = gpu_lib
    say(f"[case] no expert runs, {rows} rows {out}")
    E, N, K = 3, 256, 200
    p = Product(moe, rows, N, K, E)
    shape = moe.make_quant_shape(rows, N, K, E, 1, "relu", out)
    cut = torch.tensor([0, rows // 2, rows // 2, rows], dtype=torch.int32, device="cuda")
    for offsets, mask in ((cut, torch.zeros(E, dtype=torch.uint8, device="cuda")), (torch.zeros_like(cut), None)):
        y, sc = p.buffers(rows, out)
        before = (y.clone(), None if sc is None else sc.clone())
        moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, None, offsets, mask, p.d_w, p.d_ws, None, y, sc, workspace(moe, shape))
        torch.cuda.synchronize()
        assert torch.equal(y, before[0]) and (sc is None or torch.equal(sc, before[1]))


def test_bad_values_stay_where_they_are(gpu_lib):
    """A NaN scale spoils its row, a masked expert's NaN weights nobody, and the products of the other rows keep their bits."""
    moe = gpu_lib
    say("[case] NaN rows and weights")
    sizes = [20, 0, 150, 300]
    E, N, K, A = 4, 256, 300, 470
    p = Product(moe, A, N, K, E)
    off = torch.tensor([0, 20, 20, 170, 470], dtype=torch.int32, device="cuda")
    mask = torch.tensor([1, 1, 0, 1], dtype=torch.uint8, device="cuda")
    for out in ("f32", "e4m3"):
        shape = moe.make_quant_shape(A, N, K, E, 1, "relu", out)
        y0, s0 = p.buffers(A, out)
        moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, None, off, mask, p.d_w, p.d_ws, None, y0, s0, workspace(moe, shape))
        bad_s, bad_w = p.d_as.clone(), p.d_ws.clone()
        bad_s[3, 1] = float("nan")
        bad_s[400, 0] = float("inf")
        bad_s[20:170] = float("nan")            # rows of the masked expert
        bad_w[2] = float("nan")
        y, s = p.buffers(A, out)
        moe.moe_quant_expert_linear(shape, p.d_a, bad_s, None, off, mask, p.d_w, bad_w, None, y, s, workspace(moe, shape))
        torch.cuda.synchronize()
        for row in (3, 400):
            v = VALUES[codes_of(y)[row]] if out == "e4m3" else y[row].float().cpu().numpy()
            assert not np.isfinite(v).any() if row == 3 else not np.isfinite(v).all()
        keep = torch.ones(A, dtype=torch.bool)
        keep[[3, 400]] = False
        assert torch.equal(y[keep.cuda()].view(torch.uint8), y0[keep.cuda()].view(torch.uint8))
        if s is not None:
            assert torch.equal(s[keep.cuda()], s0[keep.cuda()])


def test_wrong_indices_stay_inside(gpu_lib):
    """perm and offsets out of range are clamped: rows in range are right, the others are products of some row."""
    moe = gpu_lib
    say("[case] perm and offsets out of range")
    p = Product(moe, 40, 64, 200, 3)
    A = 40
    perm = np.arange(A, dtype=np.int32)
    perm[5], perm[6] = -7, 2 ** 31 - 1
    off = np.array([0, 10, 2 ** 30, 12], dtype=np.int32)          # expert 1: rows 10 ..., expert 2: none
    shape = moe.make_quant_shape(A, 64, 200, 3, 1, "none", "f32")
    y, _ = p.buffers(A, "f32")
    moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, torch.from_numpy(perm).cuda(), torch.from_numpy(off).cuda(), None, p.d_w, p.d_ws, None, y,
                                None, workspace(moe, shape))
    torch.cuda.synchronize()
    source = np.clip(perm, 0, A - 1)
    check_rows(y[:10], None, *p.reference(source[:10], 0, "none", False, "f32"), "f32")
    check_rows(y[10:], None, *p.reference(source[10:], 1, "none", False, "f32"), "f32")


def test_rows_past_32_bits(gpu_lib):
    """Rows whose bytes lie further than 2^32 from the first."""
    moe = gpu_lib
    say("[case] rows past 32 bits")
    T, N, K = 70000, 16, 65536
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = torch.zeros((T, K), dtype=torch.uint8, device="cuda")
    sc = torch.ones((T, K // 128), device="cuda")
    pick = [0, 1, 32767, 32768, 65535, 65536, 69999]
    for r in pick:
        q[r] = torch.randn(K, device="cuda", generator=gen).to(torch.float8_e4m3fn).view(torch.uint8)
    w = torch.randn((1, N, K), device="cuda", generator=gen).to(torch.float8_e4m3fn)
    packed = torch.empty(moe.moe_quant_weight_bytes(1, N, K), dtype=torch.uint8, device="cuda")
    moe.moe_quantize_weights(1, N, K, "e4m3", w, packed, None)
    ws = torch.ones((1, 1, K // 128), device="cuda")
    shape = moe.make_quant_shape(T, N, K)
    y = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
    moe.moe_quant_linear(shape, q, sc, packed, ws, None, y, None, workspace(moe, shape))
    a, b = VALUES[codes_of(q[pick])], VALUES[codes_of(w[0])]
    ref, size = qo.linear(a, b)
    check_rows(y[pick], None, ref, sum_error(K) * size + cut_error(a, b), "bf16")
    y[pick] = 0
    assert not y.any()


def test_same_bits_again_and_on_another_stream(gpu_lib):
    moe = gpu_lib
    say("[case] repeats and streams")
    p = Product(moe, 700, 384, 1000, 3)
    off = torch.tensor([0, 30, 330, 700], dtype=torch.int32, device="cuda")
    shape = moe.make_quant_shape(700, 384, 1000, 3, 1, "gelu", "e4m3")
    want, want_s = p.buffers(700, "e4m3")
    moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, None, off, None, p.d_w, p.d_ws, None, want, want_s, workspace(moe, shape))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in range(4):
        y, s = p.buffers(700, "e4m3")
        ws = workspace(moe, shape)
        torch.cuda.synchronize()
        if i % 2:
            with torch.cuda.stream(side):
                moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, None, off, None, p.d_w, p.d_ws, None, y, s, ws)
        else:
            moe.moe_quant_expert_linear(shape, p.d_a, p.d_as, None, off, None, p.d_w, p.d_ws, None, y, s, ws, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(y, want) and torch.equal(s, want_s)


def test_in_a_graph(gpu_lib):
    """Norm and both products captured once, replayed with changing inputs and eager work between."""
    moe = gpu_lib
    say("[case] graph capture")
    moe.moe_init()
    T, d, f, E = 300, 256, 512, 4
    p, p2 = Product(moe, T, f, d, E), Product(moe, T, d, f, E)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    x, r = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    s1, s2 = moe.make_quant_shape(T, f, d, E, 1, "relu", "e4m3"), moe.make_quant_shape(T, d, f, E, 1, "none", "f32")
    w1, w2 = workspace(moe, s1), workspace(moe, s2)
    q, sc = torch.empty((T, d), dtype=torch.uint8, device="cuda"), torch.empty((T, d // 128), device="cuda")
    h, hs = p.buffers(T, "e4m3")

    def steps(total, y):
        moe.moe_norm_quantize(T, d, "bf16", x, r, None, 1e-6, total, None, q, sc)
        moe.moe_quant_expert_linear(s1, q, sc, None, off, None, p.d_w, p.d_ws, None, h, hs, w1)
        moe.moe_quant_expert_linear(s2, h, hs, None, off, None, p2.d_w, p2.d_ws, None, y, None, w2)

    total, y = torch.zeros_like(x), torch.zeros((T, d), device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        steps(total, y)
    for i, cut in enumerate(([0, 10, 20, 300, 300], [0, 0, 150, 150, 300], [0, 300, 300, 300, 300], [0, 1, 2, 3, 300])):
        gen = torch.Generator(device="cuda").manual_seed(i)
        x.copy_(torch.randn((T, d), device="cuda", generator=gen))
        r.copy_(torch.randn((T, d), device="cuda", generator=gen))
        off.copy_(torch.tensor(cut, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        got = (total.clone(), y.clone())
        want = (torch.empty_like(x), torch.empty_like(y))
        steps(*want)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i


# ---- the blocks that run them together -----------------------------------------------------------------------------
def block_inputs(T, d, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(s, device="cuda", generator=gen)
    return gen, new, new(T, d).bfloat16(), (3 * new(T, d)).bfloat16()


def check_norm(block, x, residual, d):
    total = wl.round_to_storage(x.float().cpu().numpy() + residual.float().cpu().numpy(), "bf16").astype(np.float64)
    assert np.array_equal(block.stream.float().cpu().numpy(), total)
    ref = qo.norm(total, block.norm_weight.cpu().numpy().astype(np.float64), block.eps)
    assert_codes(codes_of(block.x8.codes), block.x8.scales.cpu().numpy().astype(np.float64), ref, NORM * np.abs(ref), d)
    return ref


def unpacked(weights, e):
    """Values of matrix e of QuantWeights, from the codes in the products' layout."""
    N, K = weights.N, weights.K
    nb, kb = qo.blocks(N) * 8, qo.blocks(K)
    codes = weights.codes.view(weights.E, -1)[e].cpu().numpy().reshape(nb, kb, 2, 4, 16, 16).transpose(0, 4, 1, 2, 3, 5).reshape(nb * 16, kb * 128)
    return VALUES[codes[:N, :K]] * qo.spread(weights.scales[e].cpu().numpy().astype(np.float64), N, K)


def row_values(rows, C):
    return qo.dequantize_rows(VALUES[codes_of(rows.codes)[:, :C]], rows.scales.cpu().numpy().astype(np.float64))


@pytest.mark.parametrize("T,d,f,E,k,H,act", [(1, 256, 512, 16, 2, -1, "relu"), (33, 96, 160, 5, 1, -1, "gelu"), (700, 256, 384, 6, 2, -1, "relu"),
                                             (300, 128, 256, 40, 2, 3, "relu")])
def test_moe_block(gpu_lib, T, d, f, E, k, H, act):
    """Every step of the block against the reference on what the step before left on the device."""
    from oracle import moe_oracle as orc
    from paper_2405_18832_amd.quant_layer import QuantMoEBlock
    say(f"[case] QuantMoEBlock T={T} d={d} f={f} E={E} k={k} H={H} {act}")
    gen, new, x, r = block_inputs(T, d, T + d)
    w1, w2 = (new(E, f, d) / d ** 0.5).bfloat16(), (new(E, d, f) / f ** 0.5).bfloat16()
    bias = 0.3 * new(E) if H >= 0 else None
    block = QuantMoEBlock(T, d, f, E, k, w1, w2, (0.3 * new(E, d)).bfloat16(), torch.exp(0.2 * new(d)), gate_bias=bias, b1=0.3 * new(E, f),
                          b2=0.3 * new(E, d), activation=act)
    block.y_perm.fill_(float("nan"))
    out, stream = block.forward(x, r, H)
    torch.cuda.synchronize()
    assert out is block.out and stream is block.stream
    ref = check_norm(block, x, r, d)
    normed = block.normed.float().cpu().numpy()
    assert (np.abs(normed - ref) <= (HALF["bf16"] + NORM) * np.abs(ref) * 1.001).all()
    route = orc.route(normed, block.w_gate.float().cpu().numpy(), None if bias is None else bias.cpu().numpy(), k, True)
    idx = block.topk_idx.cpu().numpy()
    sure = route["margin"] >= 1e-4
    assert np.array_equal(idx[sure], route["idx"][sure])
    perm, inv = (t.cpu().numpy() for t in (block.perm, block.inv_perm))
    off, mask = block.offsets.cpu().numpy(), np.ones(E, dtype=bool) if H < 0 else block.hot_mask.cpu().numpy().astype(bool)
    assert mask.sum() == (E if H < 0 else H)
    a, h = row_values(block.x8, d), row_values(block.h8, f)
    y = block.y_perm.cpu().numpy().astype(np.float64)
    for e in range(E):
        s = slice(off[e], off[e + 1])
        if s.start == s.stop:
            continue
        if not mask[e]:
            assert np.isnan(y[s]).all()                     # not written
            continue
        v, size = qo.linear(a[perm[s] // k], unpacked(block.w1, e), block.b1[e].cpu().numpy().astype(np.float64), act)
        err = sum_error(d) * size + cut_error(a[perm[s] // k], unpacked(block.w1, e))
        if act == "gelu":
            err = 1.13 * err + 1e-6 * np.maximum(1, size)
        assert_codes(codes_of(block.h8.codes[s]), block.h8.scales[s].cpu().numpy().astype(np.float64), v, err, f)
        v, size = qo.linear(h[s], unpacked(block.w2, e), block.b2[e].cpu().numpy().astype(np.float64))
        assert (np.abs(y[s] - v) <= sum_error(f) * size + HALF["f32"] * np.abs(v)).all()
    gate = block.topk_w.cpu().numpy().astype(np.float64)
    want, size = np.zeros((T, d)), np.zeros((T, d))
    for j in range(k):
        on = mask[idx[:, j]]
        rows = y[inv.reshape(T, k)[:, j]]
        want[on] += gate[on, j:j + 1] * rows[on]
        size[on] += np.abs(gate[on, j:j + 1] * rows[on])
    got = out.float().cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= HALF["bf16"] * np.abs(want) * 1.001 + 8 * HALF["f32"] * size).all()


def test_block_of_another_size_and_refusals(gpu_lib):
    from paper_2405_18832_amd.quant_layer import QuantMoEBlock, QuantWeights
    say("[case] QuantMoEBlock resized")
    gen, new, x, r = block_inputs(200, 128, 5)
    w1, w2 = (new(8, 256, 128) / 11).bfloat16(), (new(8, 128, 256) / 16).bfloat16()
    block = QuantMoEBlock(200, 128, 256, 8, 2, w1, w2, new(8, 128).bfloat16())
    whole = block.forward(x, r)[0].clone()
    one = block.resized(1)
    assert one.w1 is block.w1 and one.out.shape == (1, 128)
    out, _ = one.forward(x[7:8].contiguous(), r[7:8].contiguous())
    # the gate's sums are taken another way for few tokens: the same experts, weights to fp32
    assert torch.equal(one.topk_idx[0], block.topk_idx[7])
    assert (out.float() - whole[7].float()).abs().max() <= 2.0 ** -6 * whole[7].float().abs().max()
    with pytest.raises(ValueError):
        QuantWeights(w1, torch.ones((8, 2, 1), device="cuda"))
    with pytest.raises(ValueError):
        QuantWeights(w1.to(torch.float8_e4m3fn), torch.ones((8, 1, 1), device="cuda"))
    with pytest.raises(ValueError):
        QuantMoEBlock(200, 128, 256, 8, 2, w2, w1, new(8, 128).bfloat16())


@pytest.mark.parametrize("T,d,f", [(1, 256, 1024), (40, 130, 300), (600, 256, 512)])
def test_dense_block(gpu_lib, T, d, f):
    from paper_2405_18832_amd.quant_layer import QuantDenseBlock
    say(f"[case] QuantDenseBlock T={T} d={d} f={f}")
    gen, new, x, r = block_inputs(T, d, T + d)
    block = QuantDenseBlock(T, d, f, new(f, d) / d ** 0.5, new(d, f) / f ** 0.5, torch.exp(0.2 * new(d)), b1=0.3 * new(f), b2=0.3 * new(d))
    out, _ = block.forward(x, r)
    torch.cuda.synchronize()
    check_norm(block, x, r, d)
    a, w = row_values(block.x8, d), unpacked(block.w1, 0)
    v, size = qo.linear(a, w, block.b1.cpu().numpy().astype(np.float64), "relu")
    assert_codes(codes_of(block.h8.codes), block.h8.scales.cpu().numpy().astype(np.float64), v, sum_error(d) * size + cut_error(a, w), f)
    a, w = row_values(block.h8, f), unpacked(block.w2, 0)
    v, size = qo.linear(a, w, block.b2.cpu().numpy().astype(np.float64))
    check_rows(out, None, v, sum_error(f) * size + cut_error(a, w), "bf16")
