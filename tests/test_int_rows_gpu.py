"""int8 rows and weights against the 64-bit reference (oracle/int_oracle.py).

Codes are the definition's whole numbers, so they are equal.  Scales, u = 2^-24 (half a step of fp32): the largest magnitude rounded to fp32 and divided,
2 u (with none or ReLU, gated: 3 u); behind GeLU and SiLU it may be the fp32 activation's, which is taken where its error is below 2^-17 of itself; the norm's factor on top, a sum of d squares in chains of 8, of the chunks that a lane keeps and of the lanes (d <= 20000: 8 + 8 + 6 + 8
additions, halved by the square root), mean, eps, root and quotient: 24 u together.  NORM = 3e-6 covers 50 u; the norm's two products are in it.
"""
import sys

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import int_oracle as io
from oracle import quant_oracle as qo

pytestmark = pytest.mark.gpu

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NORM = 3e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def dev(a, dtype="f32", offset=0):
    """On the device as `dtype`, `offset` elements behind an aligned address."""
    if a is None:
        return None
    flat = torch.zeros(a.size + offset, dtype=DT[dtype], device="cuda")
    flat[offset:] = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(-1)).to(DT[dtype]).cuda()
    return flat[offset:].view(a.shape)


def host(t):
    return t.double().cpu().numpy()


def rounded(v, dtype):
    return wl.round_to_storage(np.ascontiguousarray(v, dtype=np.float32), dtype)


def check_rows(q, scales, v, factor, tol, C):
    q, scales = q.cpu().numpy(), scales.double().cpu().numpy()
    want, want_s = io.quantize_rows(v, factor)
    assert not q[:, C:].any()                                   # codes past the end
    assert np.array_equal(np.isnan(scales), np.isnan(want_s))
    fine = ~np.isnan(want_s)
    assert (np.abs(scales - want_s)[fine] <= tol * want_s[fine]).all()
    wrong = np.argwhere(q[:, :C] != want)
    assert not len(wrong), (len(wrong), [(r, c, q[r, c], want[r, c], v[r, c]) for r, c in wrong[:5]])


def norm_case(moe, x, res, w, eps, dtype, sum_to=None, norm_out=True, offset=0):
    rows, d = x.shape
    dx, dres, dw = dev(x, dtype, offset), dev(res, dtype, offset), dev(w, "f32", offset)
    total = {None: torch.empty_like(dx) if res is not None else None, "x": dx, "residual": dres}[sum_to]
    n = torch.empty_like(dx) if norm_out else None
    q = torch.full((rows + 1, moe.moe_quant_pitch(d)), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 1,), 77.0, device="cuda")
    moe.moe_norm_quantize_int(rows, d, dtype, dx, dres, dw, eps, total, n, q, s)
    torch.cuda.synchronize()
    assert (q[rows:] == 77).all() and s[rows] == 77            # nothing behind the last row
    exact = x.astype(np.float64) if res is None else rounded(x.astype(np.float32) + res.astype(np.float32), dtype).astype(np.float64)
    if total is not None:
        assert np.array_equal(host(total), exact, equal_nan=True)
    u, rho = io.norm_parts(exact, w, eps)
    check_rows(q[:rows], s[:rows], u, rho, NORM, d)
    if n is not None:
        want = u * rho
        fine = np.isfinite(want)
        assert (np.abs(host(n) - want)[fine] <= (HALF[dtype] * (1 + NORM) + NORM) * np.abs(want)[fine] + 2.0 ** -126).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (5, 128), (1, 2048), (33, 512), (34, 513), (9, 1000), (7, 1024), (6, 2047), (5, 2049), (4, 4096), (3, 5000),
                                    (3, 9001), (2, 16384), (3, 16392), (2, 20000)])
def test_norm_sizes(gpu_lib, rows, d, dtype):
    say(f"[case] norm {rows} x {d} {dtype}")
    rng = np.random.default_rng(rows * 100003 + d)
    x, res = rounded(rng.normal(size=(rows, d)), dtype), rounded(3 * rng.normal(size=(rows, d)), dtype)
    w = np.exp(0.2 * rng.normal(size=d)).astype(np.float32)
    norm_case(gpu_lib, x, res, w, 1e-6, dtype)
    norm_case(gpu_lib, x, None, None, 0.0, dtype, norm_out=False)
    norm_case(gpu_lib, x, res, w, 1e-5, dtype, sum_to="x", offset=1)
    norm_case(gpu_lib, x, res, None, 1e-5, dtype, sum_to="residual", offset=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [96, 1001, 2048, 17000])
def test_norm_values(gpu_lib, d, dtype):
    """Many rows at once: ties between two codes, outlier columns, ranges that fp32's quotients do not cover, rows that are none."""
    say(f"[case] norm values {d} {dtype}")
    rng = np.random.default_rng(d)
    x = rng.normal(size=(400, d))
    x[0] = 0
    x[1] = rng.integers(-127, 128, d) / 2                       # halves: with 127 in the row every odd one is a tie
    x[1, d // 2] = 127
    x[2] = rng.integers(-127, 128, d) / 2
    x[2, 0] = 63.5
    x[3, ::17] *= 1000
    x[4] *= 1e-30
    x[5] *= 1e18                                                # squares of 1e36
    x[6] *= 1e-36
    x[7, d - 1] = np.nan
    x[8, 0] = np.inf
    x[9, 5] = -np.inf
    x[10] = 2.0 ** -60
    x[11] = -1.0
    x[12, :] = 0
    x[12, 3] = 1e-20
    for i in range(13, 60):                                     # ties of a row's own scale
        m = 127 * 2.0 ** rng.integers(-9, 9)
        x[i] = rng.integers(-127, 128, d) * (m / 254)
        x[i, rng.integers(d)] = m
    norm_case(gpu_lib, rounded(x, dtype), None, None, 1e-6, dtype)
    w = np.exp(rng.normal(size=d)).astype(np.float32)
    w[::29] = 100
    norm_case(gpu_lib, rounded(x, dtype), rounded(np.where(np.abs(x) < 100, rng.normal(size=x.shape), 0), dtype), w, 1e-6, dtype)


def test_norm_products_beyond_fp32(gpu_lib):
    """s w leaves fp32's range and the norm does not."""
    say("[case] norm, large products")
    rng = np.random.default_rng(3)
    x = rng.normal(size=(6, 640)) * 1e16
    w = (np.exp(rng.normal(size=640)) * 1e25).astype(np.float32)
    norm_case(gpu_lib, rounded(x, "f32"), None, w, 1e-6, "f32")
    norm_case(gpu_lib, rounded(x, "f32"), None, (w * np.float32(1e12)).astype(np.float32), 1e-6, "f32")     # and here it does: NaN rows


def act_case(moe, h, act, gated, dtype, offsets=None, mask=None, offset=0):
    rows, f = h.shape[0], h.shape[1] // (2 if gated else 1)
    q = torch.full((rows + 1, moe.moe_quant_pitch(f)), 77, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 1,), 77.0, device="cuda")
    i32 = lambda a: None if a is None else torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()
    m = None if mask is None else torch.from_numpy(np.asarray(mask, dtype=np.uint8)).cuda()
    moe.moe_act_quantize_int(rows, f, dtype, dev(h, dtype, offset), gated, act, 0 if offsets is None else len(offsets) - 1, i32(offsets), m, q, s)
    torch.cuda.synchronize()
    h = h.astype(np.float64)
    with np.errstate(invalid="ignore"):
        v = io.activate(h[:, :f], act) * (h[:, f:] if gated else 1.0)
    run = np.ones(rows, dtype=bool)
    if offsets is not None:
        run[:] = False
        for e in range(len(offsets) - 1):
            run[offsets[e]:offsets[e + 1]] = mask is None or mask[e] != 0
    idle = torch.from_numpy(np.concatenate([~run, [True]])).cuda()
    assert (q[idle] == 77).all() and (s[idle] == 77).all()      # other rows are left as they were
    at = torch.from_numpy(np.flatnonzero(run)).cuda()
    check_rows(q[at], s[at], v[run], None, 2.0 ** -17 if act in ("gelu", "silu") else 2.0 ** -22, f)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_act_sizes(gpu_lib, act, gated, dtype):
    say(f"[case] act {act} gated {gated} {dtype}")
    rng = np.random.default_rng(7)
    for rows, f in [(1, 1), (5, 9), (3, 128), (9, 512), (10, 520), (3, 1001), (7, 2048), (2, 2050), (3, 4096), (64, 8192), (2, 8200), (2, 16384), (2, 19999)]:
        h = rng.normal(size=(rows, f * (1 + gated))) * np.exp(0.5 * rng.normal(size=(rows, 1)))
        act_case(gpu_lib, rounded(h, dtype), act, gated, dtype, offset=rows % 3)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("f", [200, 3000, 9000])
def test_act_values(gpu_lib, act, gated, dtype, f):
    say(f"[case] act values {act} gated {gated} {dtype} {f}")
    rng = np.random.default_rng(f + gated)
    h = rng.normal(size=(300, f * (1 + gated)))
    h[0] = 0
    h[1, f - 1] = np.nan
    h[2, 0] = np.inf
    h[3] = -np.abs(h[3]) - 5                                     # only the tails of GeLU and SiLU
    h[4] = -np.abs(h[4]) - 11
    h[5] = -np.abs(h[5]) - 30
    h[6] *= 1e-20
    h[7] *= 1e-37
    h[8] *= 100
    h[9, :f] = rng.integers(-127, 128, f) / 2
    h[9, 0] = 127
    h[9, f:] = 1
    h[10] = -1
    h[11, ::19] *= 300
    for i in range(12, 40):
        m = 127 * 2.0 ** rng.integers(-9, 9)
        h[i, :f] = rng.integers(-127, 128, f) * (m / 254)
        h[i, rng.integers(f)] = m
        h[i, f:] = 2.0 ** rng.integers(-3, 3)
    if gated:                                                   # a second factor that brings a tail back
        h[40, :f] = -12.5 - np.abs(h[40, :f])
        h[40, f:] *= 1e32
        h[41, 5], h[41, f + 5] = -13.3, 1e38
        h[42, 5], h[42, f + 5] = -90.0, 1e37
    act_case(gpu_lib, rounded(h, dtype), act, gated, dtype)


@pytest.mark.parametrize("f", [300, 2048])
@pytest.mark.parametrize("masked", [False, True])
def test_act_of_experts(gpu_lib, f, masked):
    """Rows of experts that do not run and rows behind the last one are left as they were."""
    say(f"[case] act of experts {f} masked {masked}")
    rng = np.random.default_rng(5)
    for E in (1, 5, 64, 65, 1024):
        sizes = rng.integers(0, 4, E)
        offsets = np.concatenate([[0], np.cumsum(sizes)])
        act_case(gpu_lib, rounded(rng.normal(size=(offsets[-1] + 3, 2 * f)), "bf16"), "silu", 1, "bf16", offsets,
                 rng.integers(0, 2, E) if masked else None)


def test_act_many_rows(gpu_lib):
    """More rows than 2^16 blocks; every value of bf16 as a row's content."""
    say("[case] act many rows")
    v = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    x = wl.bf16_bits_to_f32(v)
    x = x[np.isfinite(x) & (np.abs(x) < 1e4)]
    rng = np.random.default_rng(0)
    h = x[rng.integers(0, len(x), (70000, 40))]
    act_case(gpu_lib, h, "silu", 1, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32", "i8"])
@pytest.mark.parametrize("E,N,K", [(1, 1, 1), (2, 16, 128), (3, 33, 129), (1, 200, 1000), (2, 130, 65)])
def test_weights(gpu_lib, E, N, K, dtype):
    moe = gpu_lib
    say(f"[case] weights {E} x {N} x {K} {dtype}")
    rng = np.random.default_rng(N * K)
    if dtype == "i8":
        codes = rng.integers(-128, 128, (E, N, K)).astype(np.int8)
        src, scales = torch.from_numpy(codes).cuda(), None
    else:
        w = rounded(rng.normal(size=(E, N, K)) * np.exp(rng.normal(size=(E, N, 1))), dtype)
        if N > 20:
            w[0, 3], w[0, 7, K // 2], w[0, 9, 0], w[0, 11] = 0, np.nan, np.inf, w[0, 11] * 1e-37
            w = rounded(w, dtype)
        src, scales = dev(w, dtype, 1), torch.empty((E, N), device="cuda")
        codes, want = zip(*[io.quantize_weights(w[e]) for e in range(E)])
    dst = torch.full((moe.moe_quant_weight_bytes(E, N, K),), 77, dtype=torch.int8, device="cuda")
    moe.moe_quantize_weights_int(E, N, K, dtype, src, dst, scales)
    torch.cuda.synchronize()
    if scales is not None:
        assert np.array_equal(scales.cpu().numpy(), np.stack(want), equal_nan=True)
    got = dst.cpu().numpy().view(np.uint8).reshape(E, -1)
    for e in range(E):
        assert np.array_equal(got[e], qo.pack(codes[e].view(np.uint8)))
