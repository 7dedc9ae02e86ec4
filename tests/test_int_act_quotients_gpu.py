"""Rows to int8 behind a gated activation where a second factor makes the row's largest value of a gate whose activation fp32 holds less exactly than the others', or not at
all: every code of the row is a quotient by it.
"""
import sys

import numpy as np
import pytest

from test_int_rows_gpu import act_case, rounded

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("f", [40, 700, 2048, 9000, 33000])
def test_largest_value_of_a_negative_gate(gpu_lib, act, dtype, f):
    """From -2 to where the activation is next to nothing, and past that (-12 for GeLU, -80 for SiLU)."""
    say(f"[case] act, largest value of a negative gate: {act} {dtype} {f}")
    rng = np.random.default_rng(f)
    rows = 120 if f < 20000 else 24
    h = np.zeros((rows, 2 * f))
    h[:, :f], h[:, f:] = 0.5 * rng.normal(size=(rows, f)), rng.normal(size=(rows, f))
    ends = (-2, -4, -8, -11.9, -12.1, -12.8, -13.1) if act == "gelu" else (-2, -8, -25, -60, -79, -80.5, -86)
    for r in range(rows):
        z = ends[r % 7] + 0.05 * rng.normal()
        size = abs(z) * np.exp(-z * z / 2) / (abs(z) * 2.5066) if act == "gelu" else abs(z) * np.exp(z)        # of the activation
        at = rng.integers(f)
        h[r, at], h[r, f + at] = z, min(3.0 / size, 3e38) * rng.choice([-1, 1]) * rng.uniform(0.7, 1)
        if r % 3 == 0:                                          # another one next to it
            to = rng.integers(f)
            h[r, to], h[r, f + to] = z, h[r, f + at] * (1 + 2.0 ** -7 * rng.integers(-1, 2))
    act_case(gpu_lib, rounded(h, dtype), act, 1, dtype)


def test_rows_of_which_only_the_tail_is_left(gpu_lib):
    """A tail's value that is the row's largest beside small ones, an infinity or a NaN beside or on it."""
    say("[case] act, tails beside small values")
    rng = np.random.default_rng(2)
    for act, z in (("gelu", -12.6), ("silu", -85.0)):
        h = np.zeros((12, 1200))
        h[:, :600], h[:, 600:] = rng.normal(size=(12, 600)), rng.normal(size=(12, 600)) * 10.0 ** -np.arange(0, 48, 4)[:, None]
        h[:, 77], h[:, 677] = z, 2e38
        h[9, 677], h[10, 677], h[11, 77] = np.inf, np.nan, -np.inf
        act_case(gpu_lib, rounded(h, "f32"), act, 1, "f32")


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("f", [40, 700, 9000])
def test_gates_below_the_normal_numbers(gpu_lib, act, dtype, f):
    """The other factor brings back what the gate's rounding there would have lost."""
    say(f"[case] act gates below the normal numbers {act} {dtype} {f}")
    rng = np.random.default_rng(f)
    step = 2.0 ** (-149 if dtype == "f32" else -133)
    h = np.zeros((40, 2 * f))
    g, u = h[:, :f], h[:, f:]
    for r in range(40):
        places = [0, f - 1] if r % 4 == 0 else rng.permutation(f)[:1 + r] if r % 4 == 1 else np.arange(f)
        g[r], u[r] = 1e-7 * rng.normal(size=f), rng.normal(size=f)
        g[r, places] = rng.integers(1, 9 if r < 20 else 100, len(places)) * step * rng.choice([-1, 1], len(places))
        u[r, places] = 2.0 ** (125 if dtype == "f32" else 109) * rng.uniform(0.5, 2, len(places))
        if r % 4 == 3:
            u[r, ::2] *= 2.0 ** -30                             # what is left there is below the others' half steps
    act_case(gpu_lib, rounded(h, dtype), act, 1, dtype)
