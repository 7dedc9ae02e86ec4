"""Router logits of as many tokens as the call takes: rows picked out of them against the 64-bit reference."""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_most_tokens(gpu_lib):
    """2^30 - 1 tokens: more threads than one launch counts (2^32 - 1), 69 GB of x."""
    moe = gpu_lib
    T, E, d = 0x3fffffff, 2, 32
    print(f"[case] logits of {T} tokens", file=sys.stderr, flush=True)
    at = torch.tensor([0, 1, 63, 64, 12345, T // 2, T - 129, T - 128, T - 127, T - 65, T - 64, T - 63, T - 2, T - 1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.zeros((T, d), dtype=BF, device="cuda")
    rows, w = torch.randn((len(at), d), device="cuda", generator=g).to(BF), torch.randn((E, d), device="cuda", generator=g).to(BF)
    x[at] = rows
    logits = torch.full((T, E), 7.0, device="cuda")
    shape = moe.make_shape(T, d, 32, E, 1, "bf16", False)
    bias = torch.tensor([0.5, 0.25], device="cuda")
    moe.moe_gate_logits(shape, x, w, bias, logits)
    a, b = rows.double().cpu().numpy(), w.double().cpu().numpy()
    want = a @ b.T + bias.double().cpu().numpy()
    assert (np.abs(logits[at].double().cpu().numpy() - want) <= (d + 2) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T + 0.5)).all()
    others = torch.ones(T, dtype=torch.bool, device="cuda")
    others[at] = False
    assert int(((logits[:, 0] != 0.5) & others).sum()) == 0 and int(((logits[:, 1] != 0.25) & others).sum()) == 0      # every row is written, once or alike
