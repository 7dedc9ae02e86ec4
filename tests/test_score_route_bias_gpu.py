"""Routing by scores where a finite choice bias takes experts out: whatever its size, the k best of the kept groups are chosen, each once.

The kernel orders choices in fp32 within a range of +-8 and leaves the rest to 64 bits, so biases lie on both sides of its end, and the kept groups hold k experts, one or
two more, or many.
"""
import sys

import numpy as np
import pytest

from test_score_route_gpu import check_route, rounded, run_route

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def biases(rng, E, value):
    plain = (0.1 * rng.normal(size=E)).astype(np.float32)
    one, some, most = plain.copy(), plain.copy(), plain.copy()
    one[E // 2] = value
    some[::3] = value
    most[1:] = value
    return {"one": one, "some": some, "all but one": most, "all": np.full(E, value, dtype=np.float32), "all, apart": plain + np.float32(value)}


# kept experts: k, k + 1, k + 2, many; numbers that do and do not fill the lanes' places
SIZES = [(4, 4, 1, 1, 1), (8, 8, 1, 1, 1), (8, 7, 1, 1, 1), (10, 8, 1, 1, 1), (5, 3, 1, 1, 1), (8, 2, 4, 1, 1), (16, 8, 4, 2, 2), (20, 8, 5, 2, 1), (32, 8, 8, 2, 2), (36, 8, 4, 1, 2),
         (30, 8, 3, 1, 2), (64, 8, 8, 1, 2), (70, 7, 10, 1, 2), (128, 8, 16, 1, 1), (130, 6, 13, 1, 2), (256, 8, 8, 4, 2), (640, 8, 1, 1, 1), (1024, 8, 16, 1, 2), (80, 8, 20, 2, 2)]


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,k,groups,kept,top", SIZES)
def test_finite_biases_that_take_experts_out(gpu_lib, E, k, groups, kept, top, score):
    rng = np.random.default_rng(E * k)
    logits = (1.5 * rng.normal(size=(200, E))).astype(np.float32)
    for value in (-6.5, -7.5, -7.9, -8.0, -10.0, -1e4, -1e9):
        for name, balance in biases(rng, E, value).items():
            say(f"[case] bias {value} on {name} of {E} experts, k {k}, {kept} of {groups} groups by {top}, {score}")
            rule = dict(score=score, balance=balance, groups=groups, kept=kept, top=top)
            check_route(gpu_lib, logits, k, renormalize=True, H=2, **rule)
            check_route(gpu_lib, rounded(logits[:20], "bf16"), k, dtype="bf16", **rule)         # one block
            idx = run_route(gpu_lib, logits, k, **rule)[0]
            assert all(len(set(row)) == k and len(set(row // (E // groups))) <= kept for row in idx)


def test_softmax_of_one_large_score_and_many_small_ones(gpu_lib):
    """1024 experts: a score of nearly one, 63 of half a step of fp32 or so beside it (which a running sum of 32 bits would lose, one by one), and a bias between what is
    left of it with and without them."""
    u = 2.0 ** -24
    for first, place in [(0, 20), (0, 700), (64 * 15 + 3, 20), (1, 1000)]:
        logits = np.full((40, 1024), -50.0, dtype=np.float32)
        lane = [64 * j + 4 * (first % 64 // 4) + i for j in range(16) for i in range(4)]       # the experts of a lane
        logits[:, lane] = -16.75
        logits[:, first] = 0
        for t in range(40):                                     # fewer and fewer of them
            logits[t, lane[64 - t:]] = np.where(np.asarray(lane[64 - t:]) == first, 0, -50).astype(np.float32)
        for steps in (8, 24, 40, 52):
            say(f"[case] softmax of 1024 experts, one large, bias {steps} steps below one at {place}")
            balance = np.zeros(1024, dtype=np.float32)
            balance[place] = 1 - steps * u
            for k in (1, 3):
                check_route(gpu_lib, logits, k, balance=balance)
            check_route(gpu_lib, logits, 2, balance=balance, groups=16, kept=8, top=1)


def test_groups_whose_choices_cancel(gpu_lib):
    """Two groups of two experts with biases of 7.25 and -8.75: the sums are near zero, the choices' roundings are not.  The scores are such that with fp32 scores to nearest
    the roundings add up, 12 steps of 2^-24 for each group, the other way round for one than for the other, and the better group's sum is less than a step above."""
    u, up, down = 2.0 ** -24, 7.25, -8.75
    l = np.arange(1 << 21, dtype=np.float64) * 2.0 ** -25 + 0.3
    l = l.astype(np.float32)
    p = 1 / (1 + np.exp(-l.astype(np.float64))) / u
    part, n = p % 16, np.floor(p / 16)                          # choices near 8: multiples of 16 steps, near 7: of 8
    part8, n8 = p % 8, np.floor(p / 8)
    even, even8 = n % 2 == 0, n8 % 2 == 0
    a1, a2 = np.flatnonzero(even8 & (part8 > 4.2) & (part8 < 4.45)), np.flatnonzero(even & (part > 8.2) & (part < 8.45))
    b1, b2 = np.flatnonzero(even8 & (part8 > 4.5) & (part8 < 4.7)), np.flatnonzero(~even & (part > 7.55) & (part < 7.8))
    at = {int(n8[i]): i for i in b1}
    rng = np.random.default_rng(1)
    rows = []
    while len(rows) < 4096:
        i, j, h = rng.choice(a1), rng.choice(a2), rng.choice(b2)
        g = at.get(int(n8[i] + 2 * n[j] - 2 * n[h]))
        if g is not None and p[i] + p[j] > p[g] + p[h] + 0.1:
            rows.append([l[i], l[j], l[g], l[h]])
    logits = np.asarray(rows, dtype=np.float32)
    logits[1::2] = logits[1::2][:, [2, 3, 0, 1]]
    balance = np.array([up, down, up, down], dtype=np.float32)
    for k in (1, 2):
        say(f"[case] groups whose choices cancel, k {k}")
        check_route(gpu_lib, logits, k, score="sigmoid", balance=balance, groups=2, kept=1, top=2)
    wide = np.full((4096, 32), -20.0, dtype=np.float32)         # more groups, others far below
    wide[:, [8, 9, 24, 25]] = logits
    balance = np.full(32, -9.0, dtype=np.float32)
    balance[[8, 9, 24, 25]] = up, down, up, down
    check_route(gpu_lib, wide, 4, score="sigmoid", balance=balance, groups=4, kept=1, top=2)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("balanced", [False, True])
@pytest.mark.parametrize("E,k,groups,kept,top", [(8, 3, 2, 1, 1), (32, 6, 4, 2, 1), (64, 8, 8, 2, 2), (256, 8, 8, 1, 1), (80, 8, 20, 3, 1), (600, 8, 4, 2, 2)])
def test_masked_experts_of_the_kept_groups_come_before_other_groups(gpu_lib, E, k, groups, kept, top, balanced, score):
    """Where fewer than k experts are left in the kept groups, the others are those groups' masked ones, lowest index first: never an expert of a group that was dropped."""
    say(f"[case] masked experts of kept groups {E} k {k} groups {groups}/{kept} top {top} {score} {balanced}")
    rng = np.random.default_rng(E + k)
    size, T = E // groups, 60
    logits = rng.normal(size=(T, E)).astype(np.float32)
    best = np.stack([rng.permutation(groups)[:kept] for _ in range(T)])
    for t in range(T):
        for g in best[t]:                                       # two large ones each, the rest masked
            logits[t, g * size:(g + 1) * size] = -np.inf
            logits[t, g * size + rng.permutation(size)[:2]] = [6, 5]
    balance = (0.01 * rng.normal(size=E)).astype(np.float32) if balanced else None
    idx, w, counts, offsets, _ = run_route(gpu_lib, logits, k, score=score, balance=balance, groups=groups, kept=kept, top=top)
    l = logits.astype(np.float64)
    p = 1 / (1 + np.exp(-l)) if score == "sigmoid" else np.exp(l) / np.exp(l).sum(axis=1, keepdims=True)
    short = 0
    for t in range(T):
        c = np.where(np.isneginf(l[t]), -np.inf, p[t] + balance if balanced else l[t])
        of = np.where(np.isneginf(l[t]), -np.inf, p[t]) if top == 2 and not balanced else c
        value = np.sort(of.reshape(groups, size), axis=1)[:, size - top:].sum(axis=1)
        stay = set(sorted(range(groups), key=lambda g: (-value[g], g))[:kept])
        want = sorted((e for e in range(E) if e // size in stay), key=lambda e: (-c[e], e))[:k]
        assert list(idx[t]) == want and ((w[t] > 0) == (c[want] > -np.inf)).all(), (t, idx[t], want)
        short += np.isneginf(c[want[-1]])
    assert short >= T // 2
    assert np.array_equal(counts, np.bincount(idx.reshape(-1), minlength=E))
