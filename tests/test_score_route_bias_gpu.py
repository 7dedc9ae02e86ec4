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
