"""Router logits and routing by scores against the 64-bit reference (oracle/int_oracle.py, oracle/moe_oracle.py).

Logits, u = 2^-23 (a matrix unit may truncate): a sum of d products of which each is exact in fp32 (bf16) or rounded once (fp32), in any order: at most
(d + 2) u of sum |x| |w| + |b|.  Experts, counts and offsets are whole numbers and equal.  Weights: scores in 64 bits or fp32, a quotient and a product:
within 2^-19 of themselves (fp32 scores are exponentials of a difference that is |l| 2^-24 off, |l| < 16).
"""
import sys

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import int_oracle as io
from oracle import moe_oracle as orc

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def rounded(v, dtype):
    return wl.round_to_storage(np.ascontiguousarray(v, dtype=np.float32), dtype)


def dev(a, dtype="f32", offset=0):
    if a is None:
        return None
    flat = torch.zeros(a.size + offset, dtype=DT[dtype], device="cuda")
    flat[offset:] = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(-1)).to(DT[dtype]).cuda()
    return flat[offset:].view(a.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,E,offset", [(1, 32, 1, 0), (1, 2048, 128, 0), (7, 96, 5, 0), (16, 64, 16, 1), (33, 1024, 130, 0), (64, 768, 64, 0), (200, 2048, 256, 0),
                                          (777, 800, 60, 0), (1000, 64, 1024, 0), (3000, 512, 256, 0), (5003, 1056, 128, 0), (4500, 768, 8, 3), (9000, 256, 100, 0)])
def test_logits(gpu_lib, T, d, E, dtype, offset):
    moe = gpu_lib
    say(f"[case] logits {T} x {d} x {E} {dtype} offset {offset}")
    rng = np.random.default_rng(T + d)
    x, w = rounded(rng.normal(size=(T, d)), dtype), rounded(rng.normal(size=(E, d)) / np.sqrt(d), dtype)
    for b in (None, rng.normal(size=E).astype(np.float32)):
        out = torch.full((T + 1, E), 77.0, device="cuda")
        moe.moe_gate_logits(moe.make_shape(T, d, 32, E, 1, dtype, False), dev(x, dtype, offset), dev(w, dtype, offset), dev(b), out)
        torch.cuda.synchronize()
        assert (out[T:] == 77).all()
        x64, w64 = x.astype(np.float64), w.astype(np.float64)
        want, size = orc.gate_logits(x64, w64, b), np.abs(x64) @ np.abs(w64).T + (0 if b is None else np.abs(b))
        assert (np.abs(out[:T].double().cpu().numpy() - want) <= (d + 2) * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,E", [(1300, 96, 64), (2101, 64, 50), (4500, 160, 40), (9000, 64, 33), (13001, 96, 64), (700, 416, 256), (3001, 224, 200), (9001, 96, 65), (13007, 64, 72),
                                   (70000, 32, 7), (66000, 32, 16)])
def test_logits_of_blocks_of_every_size(gpu_lib, T, d, E, dtype):
    test_logits(gpu_lib, T, d, E, dtype, 0)


@pytest.mark.parametrize("d", [1, 3, 30, 33, 130, 1001])
def test_logits_of_odd_widths(gpu_lib, d):
    test_logits(gpu_lib, 50, d, 20, "f32", 1)
    test_logits(gpu_lib, 2100, d, 20, "f32", 0)


def test_logits_of_rows_that_are_none(gpu_lib):
    """An infinity or a NaN stays in its token's and its expert's logits, also where widths end inside a step."""
    moe = gpu_lib
    for T, d, dtype in [(20, 96, "bf16"), (3000, 96, "bf16"), (20, 36, "f32"), (3000, 36, "f32"), (3000, 32, "f32"), (3000, 64, "bf16")]:
        say(f"[case] logits with infinities {T} x {d} {dtype}")
        rng = np.random.default_rng(d)
        x, w = rounded(np.abs(rng.normal(size=(T, d))) + 0.1, dtype), rounded(np.abs(rng.normal(size=(24, d))) + 0.1, dtype)
        x[4, d - 1], x[5, 0], w[3, d - 1] = np.inf, np.nan, -np.inf
        out = torch.empty((T, 24), device="cuda")
        moe.moe_gate_logits(moe.make_shape(T, d, 32, 24, 1, dtype, False), dev(x, dtype), dev(w, dtype), None, out)
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        with np.errstate(invalid="ignore"):
            want = x.astype(np.float64) @ w.astype(np.float64).T
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
        fine = np.isfinite(want)
        assert np.allclose(got[fine], want[fine], rtol=1e-4)


def run_route(moe, logits, k, dtype="f32", H=-1, offset=0, balance=None, score="softmax", groups=1, kept=1, top=1, renormalize=False, scale=1.0):
    T, E = logits.shape
    shape = moe.make_shape(T, 32, 32, E, k, "bf16", renormalize)
    i32 = dict(dtype=torch.int32, device="cuda")
    idx, w = torch.full((T + 1, k), 77, **i32), torch.full((T + 1, k), 77.0, device="cuda")
    counts, offsets, hot = torch.full((E + 1,), 77, **i32), torch.full((E + 2,), 77, **i32), torch.full((E + 1,), 77, dtype=torch.uint8, device="cuda")
    ws = torch.full((moe.moe_workspace_bytes(shape),), 0x5a, dtype=torch.uint8, device="cuda")
    moe.moe_route_logits(shape, moe.make_routing(score, groups, kept, top, scale), dtype, dev(logits, dtype, offset), dev(balance, "f32", offset), idx, w,
                         counts, offsets, H, hot if H >= 0 else None, ws)
    torch.cuda.synchronize()
    assert (idx[T:] == 77).all() and (w[T:] == 77).all() and counts[E] == 77 and offsets[E + 1] == 77 and hot[E] == 77
    return idx[:T].cpu().numpy(), w[:T].double().cpu().numpy(), counts[:E].cpu().numpy(), offsets[:E + 1].cpu().numpy(), hot[:E].cpu().numpy()


def check_route(moe, logits, k, dtype="f32", H=-1, offset=0, **rule):
    T, E = logits.shape
    idx, w, counts, offsets, hot = run_route(moe, logits, k, dtype, H, offset, **rule)
    want, want_w = io.route(logits, k, **rule)
    wrong = np.argwhere((idx != want).any(axis=1))[:, 0]
    assert not len(wrong), (len(wrong), wrong[:3], idx[wrong[:3]], want[wrong[:3]])
    assert np.array_equal(np.isnan(w), np.isnan(want_w))
    fine = ~np.isnan(want_w)
    assert (np.abs(w - want_w)[fine] <= 2.0 ** -19 * np.abs(want_w)[fine] + 2.0 ** -126).all()
    n = np.bincount(want.reshape(-1), minlength=E)
    assert np.array_equal(counts, n) and np.array_equal(offsets, np.concatenate([[0], np.cumsum(n)]))
    if H >= 0:
        assert np.array_equal(hot, orc.hot_mask_top_h(n, H))



@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("balanced", [False, True])
@pytest.mark.parametrize("T,E,k,groups,kept,top", [
    (1, 1, 1, 1, 1, 1), (1, 8, 8, 1, 1, 1), (3, 128, 8, 8, 4, 2), (64, 64, 6, 1, 1, 1), (65, 256, 8, 8, 4, 2), (100, 60, 4, 3, 2, 1), (257, 16, 2, 16, 5, 1),
    (300, 17, 3, 1, 1, 1), (700, 160, 6, 8, 3, 1), (130, 1024, 8, 64, 20, 2), (90, 1000, 8, 4, 2, 2), (2000, 256, 8, 8, 4, 2), (40, 300, 8, 60, 7, 2),
    (2300, 32, 4, 4, 2, 2), (2200, 400, 5, 1, 1, 1),
])
def test_route(gpu_lib, T, E, k, groups, kept, top, balanced, score):
    say(f"[case] route {T} tokens {E} experts k {k} groups {groups}/{kept} top {top} balance {balanced} {score}")
    rng = np.random.default_rng(T * E)
    logits = rng.normal(size=(T, E)).astype(np.float32) * 1.5
    balance = (0.1 * rng.normal(size=E)).astype(np.float32) if balanced else None
    rule = dict(score=score, balance=balance, groups=groups, kept=kept, top=top)
    check_route(gpu_lib, logits, k, **rule, renormalize=True, scale=2.5)
    check_route(gpu_lib, logits, k, H=E // 3, offset=1, **rule)
    check_route(gpu_lib, rounded(logits, "bf16"), k, dtype="bf16", offset=E % 2, **rule)           # ties


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,kept,top", [(64, 1, 1, 1), (256, 8, 4, 2), (96, 8, 4, 1), (600, 4, 3, 2)])
def test_scores_next_to_each_other(gpu_lib, E, groups, kept, top, score):
    """Logits a step of fp32 or less than a step of their scores apart, equal ones, saturated ones; a bias that nearly makes up for the difference."""
    rng = np.random.default_rng(E)
    T, k = 300, 8
    base = rng.normal(size=(T, E)).astype(np.float32)
    near = rng.choice(rng.normal(size=6).astype(np.float32), (T, E))
    near = np.nextafter(near, np.where(rng.random((T, E)) < 0.5, np.inf, -np.inf).astype(np.float32)).astype(np.float32)
    large = (rng.choice([-120, -30, 18, 30, 60], (T, E)) + rng.integers(0, 3, (T, E)) * 0.25).astype(np.float32)
    p = 1 / (1 + np.exp(-base[0].astype(np.float64))) if score == "sigmoid" else np.exp(base[0].astype(np.float64)) / np.exp(base[0].astype(np.float64)).sum()
    level = (0.75 - p).astype(np.float32)                         # p + bias = 0.75 +- 2^-25
    for name, logits, balance in [("near", near, None), ("near, balanced", near, (0.01 * rng.integers(-2, 3, E)).astype(np.float32)), ("large", large, None),
                                  ("large, balanced", large, (0.25 * rng.integers(0, 2, E)).astype(np.float32)), ("level", np.tile(base[:1], (T, 1)), level)]:
        say(f"[case] route next to each other: {name} {E} experts {groups} groups {score}")
        if name.startswith("large") and score == "softmax" and balance is not None:
            continue          # choices of 0.25 + 1e-20 and 0.25 + 2e-20 are one number in 64 bits, and their order there no property of the formula
        check_route(gpu_lib, logits, k, score=score, balance=balance, groups=groups, kept=kept, top=top, renormalize=score == "softmax")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("balanced", [False, True])
@pytest.mark.parametrize("T,E,groups,kept,top", [(40, 16, 1, 1, 1), (40, 128, 4, 2, 2), (300, 256, 8, 4, 2), (40, 512, 8, 8, 1)])
def test_experts_that_are_not_there(gpu_lib, T, E, groups, kept, top, balanced, score):
    say(f"[case] route masked {T} tokens {E} experts {groups} groups {score} {balanced}")
    rng = np.random.default_rng(E)
    logits = rng.normal(size=(T, E)).astype(np.float32)
    logits[:, ::3] = -np.inf
    logits[1] = -np.inf                                            # no expert at all
    logits[2, 1:] = -np.inf                                        # one
    logits[3, E // 2:] = -np.inf
    logits[4, 5], logits[5] = np.nan, np.nan
    logits[6, 1] = np.inf
    logits[7, 1], logits[7, 2] = np.inf, np.nan
    balance = (0.1 * rng.normal(size=E)).astype(np.float32) if balanced else None
    for renormalize in (False, True):
        check_route(gpu_lib, logits, 8, score=score, balance=balance, groups=groups, kept=kept, top=top, renormalize=renormalize, H=4)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,groups,kept,top", [(20, 16, 1, 1, 1), (33, 64, 8, 3, 2), (40, 128, 4, 2, 2), (300, 256, 8, 4, 2), (40, 512, 8, 5, 1)])
def test_biases_that_are_no_numbers(gpu_lib, T, E, groups, kept, top, score):
    """A bias of -infinity or NaN takes its expert out, one of infinity takes it first, a large one leaves nothing of the scores' order.  A group of infinity
    and nothing else has no sum of two and comes last."""
    rng = np.random.default_rng(E + T)
    logits = rng.normal(size=(T, E)).astype(np.float32)
    logits[0, E - 1], logits[1, 3] = -np.inf, np.nan
    plain = (0.1 * rng.normal(size=E)).astype(np.float32)
    out, first, large, alone = (plain.copy() for _ in range(4))
    out[::5], out[1::7] = -np.inf, np.nan
    first[E // 2 + 1], first[3] = np.inf, np.inf
    large[:E // 2] = 1e30
    alone[:E // groups] = -np.inf
    alone[1] = np.inf
    for name, balance in [("out", out), ("first", first), ("large", large), ("alone", alone), ("all out", np.full(E, -np.inf, dtype=np.float32))]:
        say(f"[case] route with a bias {name}: {T} tokens {E} experts {groups} groups {score}")
        check_route(gpu_lib, logits, 6, score=score, balance=balance, groups=groups, kept=kept, top=top, renormalize=True, H=3)


def test_no_tokens(gpu_lib):
    say("[case] route of no tokens")
    moe, E = gpu_lib, 20
    s = moe.make_shape(0, 32, 32, E, 2, "bf16", True)
    ws = torch.empty(moe.moe_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    counts, offsets, hot = (torch.full((n,), 77, dtype=t, device="cuda") for n, t in ((E, torch.int32), (E + 1, torch.int32), (E, torch.uint8)))
    moe.moe_route_logits(s, moe.make_routing("sigmoid"), "f32", None, None, None, None, counts, offsets, 3, hot, ws)
    torch.cuda.synchronize()
    assert not counts.any() and not offsets.any() and hot.tolist() == [1] * 3 + [0] * 17


def test_agrees_with_the_layers_own_routing(gpu_lib):
    """Softmax without bias and groups on the logits of moe_gate_logits is moe_route, but for tokens whose logits are a rounding apart."""
    moe = gpu_lib
    say("[case] route against moe_route")
    rng = np.random.default_rng(11)
    T, d, E, k = 600, 512, 64, 2
    x, w = dev(rounded(rng.normal(size=(T, d)), "bf16"), "bf16"), dev(rounded(0.1 * rng.normal(size=(E, d)), "bf16"), "bf16")
    s = moe.make_shape(T, d, 32, E, k, "bf16", True)
    i32 = dict(dtype=torch.int32, device="cuda")
    ws = torch.empty(moe.moe_workspace_bytes(s), dtype=torch.uint8, device="cuda")
    a = (torch.empty((T, k), **i32), torch.empty((T, k), device="cuda"), torch.empty(E, **i32), torch.empty(E + 1, **i32))
    b = tuple(torch.empty_like(t) for t in a)
    margin, logits = torch.empty(T, device="cuda"), torch.empty((T, E), device="cuda")
    moe.moe_route(s, x, w, None, a[0], a[1], margin, a[2], a[3], -1, None, ws)
    moe.moe_gate_logits(s, x, w, None, logits)
    moe.moe_route_logits(s, moe.make_routing(), "f32", logits, None, *b, -1, None, ws)
    torch.cuda.synchronize()
    ok = margin > 1e-4
    assert ok.float().mean() > 0.95 and torch.equal(a[0][ok], b[0][ok]) and torch.allclose(a[1][ok], b[1][ok], rtol=2e-4)
