"""Numbers of elements that 32 bits do not count, and strides of the grid's second direction: rows picked out of large calls against the same rows alone or
the 64-bit reference."""
import sys

import numpy as np
import pytest
import torch

from oracle import int_oracle as io
from test_int_product_gpu import within, workspace
from test_int_rows_gpu import NORM, check_rows, host

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def picked(rows):
    return torch.tensor([0, 1, 255, rows // 2, rows - 257, rows - 2, rows - 1], device="cuda")


@pytest.mark.parametrize("T,N,K", [(270000, 8192, 128), (70000, 128, 65536)])
def test_products(gpu_lib, T, N, K):
    """2.2e9 outputs; rows of 4.6 GB, which tiles of 256 rows do not address."""
    moe = gpu_lib
    say(f"[case] int linear {T} x {N} x {K}")
    g = torch.Generator(device="cuda").manual_seed(T)
    a = torch.randint(-128, 128, (T, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-128, 128, (1, N, K), dtype=torch.int8, device="cuda", generator=g)
    sa, sw = torch.rand(T, device="cuda", generator=g), torch.rand((1, N), device="cuda", generator=g) / (5000 * K ** 0.5)
    packed = torch.empty(moe.moe_quant_weight_bytes(1, N, K), dtype=torch.int8, device="cuda")
    moe.moe_quantize_weights_int(1, N, K, "i8", w, packed, None)
    shape = moe.make_quant_shape(T, N, K)
    y = torch.empty((T, N), dtype=BF, device="cuda")
    moe.moe_int_linear(shape, a, sa, packed, sw, None, y, workspace(moe, shape))
    at = picked(T)
    z, size = io.product(a[at].cpu().numpy(), host(sa[at]), w[0].cpu().numpy(), host(sw[0]))
    within(y[at], z, size, "none", "bf16")


def test_experts(gpu_lib):
    """The same behind a permutation, grouped: 2.2e9 outputs of rows that 8 assignments share."""
    moe = gpu_lib
    A, N, K, E, k = 280000, 8192, 64, 5, 8
    say(f"[case] int experts {A} x {N} x {K}")
    rng = np.random.default_rng(1)
    g = torch.Generator(device="cuda").manual_seed(1)
    a = torch.randint(-128, 128, (A // k, 128), dtype=torch.int8, device="cuda", generator=g)
    a[:, K:] = 0
    w = torch.randint(-128, 128, (E, N, K), dtype=torch.int8, device="cuda", generator=g)
    sa, sw = torch.rand(A // k, device="cuda", generator=g), torch.rand((E, N), device="cuda", generator=g) / (5000 * K ** 0.5)
    packed = torch.empty(moe.moe_quant_weight_bytes(E, N, K), dtype=torch.int8, device="cuda")
    moe.moe_quantize_weights_int(E, N, K, "i8", w, packed, None)
    perm, offsets = rng.permutation(A).astype(np.int32), np.array([0, 100000, 100003, 100003, 279990, A], dtype=np.int32)
    shape = moe.make_quant_shape(A, N, K, E, k)
    y = torch.empty((A, N), dtype=BF, device="cuda")
    moe.moe_int_expert_linear(shape, a, sa, torch.from_numpy(perm).cuda(), torch.from_numpy(offsets).cuda(), None, packed, sw, None, y, workspace(moe, shape))
    for p in (0, 99999, 100001, 100003, 150000, 279989, 279990, A - 1):
        e = int(np.searchsorted(offsets, p, side="right")) - 1
        row = torch.tensor([perm[p] // k], device="cuda")
        z, size = io.product(a[row, :K].cpu().numpy(), host(sa[row]), w[e].cpu().numpy(), host(sw[e]))
        within(y[p:p + 1], z, size, "none", "bf16")


@pytest.mark.parametrize("rows,d", [(140000, 16384), (9000000, 128)])
def test_rows(gpu_lib, rows, d):
    """2.3e9 values; more rows than the grid's first direction takes blocks."""
    moe = gpu_lib
    say(f"[case] int rows {rows} x {d}")
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, d), dtype=BF, device="cuda", generator=g)
    q, s = torch.empty((rows, d), dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    n = torch.empty_like(x)
    at = picked(rows)
    moe.moe_norm_quantize_int(rows, d, "bf16", x, None, None, 1e-6, None, n, q, s)
    u, rho = io.norm_parts(host(x[at]), None, 1e-6)
    check_rows(q[at], s[at], u, rho, NORM, d)
    assert (np.abs(host(n[at]) - u * rho) <= (2.0 ** -8 * (1 + NORM) + NORM) * np.abs(u * rho)).all()
    del n
    for gated in (0, 1):
        half = d // (1 + gated)
        moe.moe_act_quantize_int(rows, half, "bf16", x, gated, "silu", 0, None, None, q, s)
        h = host(x[at])
        codes = q.view(-1)[:rows * moe.moe_quant_pitch(half)].view(rows, -1)
        check_rows(codes[at], s[at], io.activate(h[:, :half], "silu") * (h[:, half:] if gated else 1.0), None, 2.0 ** -17, half)


def test_router(gpu_lib):
    """2.2e9 logits."""
    moe = gpu_lib
    T, E, d, k = 2150000, 1024, 32, 8
    say(f"[case] router of {T} tokens, {E} experts")
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = torch.randn((T, d), dtype=BF, device="cuda", generator=g), torch.randn((E, d), dtype=BF, device="cuda", generator=g)
    logits = torch.empty((T, E), device="cuda")
    shape = moe.make_shape(T, d, 32, E, k, "bf16", True)
    moe.moe_gate_logits(shape, x, w, None, logits)
    at = picked(T)
    want = host(x[at]) @ host(w).T
    assert (np.abs(host(logits[at]) - want) <= (d + 2) * 2.0 ** -23 * (np.abs(host(x[at])) @ np.abs(host(w)).T)).all()
    i32 = dict(dtype=torch.int32, device="cuda")
    idx, weight, counts, offsets = torch.empty((T, k), **i32), torch.empty((T, k), device="cuda"), torch.empty(E, **i32), torch.empty(E + 1, **i32)
    ws = torch.empty(moe.moe_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    balance = 0.05 * torch.randn(E, device="cuda", generator=g)
    moe.moe_route_logits(shape, moe.make_routing("sigmoid", 8, 4, 2, 2.5), "f32", logits, balance, idx, weight, counts, offsets, -1, None, ws)
    want, want_w = io.route(host(logits[at]), k, "sigmoid", host(balance), 8, 4, 2, True, 2.5)
    assert np.array_equal(idx[at].cpu().numpy(), want) and np.allclose(host(weight[at]), want_w, rtol=2.0 ** -19)
    assert torch.equal(counts.long(), torch.bincount(idx.view(-1), minlength=E)) and torch.equal(offsets[1:].long(), counts.long().cumsum(0))
