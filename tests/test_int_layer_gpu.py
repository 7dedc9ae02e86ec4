"""The int8 blocks, step by step against the 64-bit reference from what the step before left, and as they are run: in graphs, on two streams, for tokens
that are not there.

Tolerances are those of the steps' own tests (test_int_rows_gpu, test_int_product_gpu, test_score_route_gpu); the combine adds k products in fp32, (k + 1) 2^-24
of the sum of magnitudes, and rounds to bf16 once, 2^-8.
"""
import sys

import numpy as np
import pytest
import torch

from oracle import int_oracle as io
from oracle import moe_oracle as orc
from paper_2405_18832_amd import int8_layer as il
from test_int_product_gpu import within
from test_int_rows_gpu import HALF, NORM, check_rows, host

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def tensors(seed, *shapes, dtype=BF, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(s, device="cuda", generator=g) * std).to(dtype) for s in shapes]


def moe_block(T, d, f, E, k, gated=True, activation="silu", biases=True, dtype=BF, **rule):
    w1, = tensors(1, (E, f * (1 + gated), d), std=d ** -0.5)
    w2, = tensors(2, (E, d, f), std=f ** -0.5)
    gate, = tensors(3, (E, d), std=2 * d ** -0.5)
    vec = lambda seed, *s: tensors(seed, s, dtype=torch.float32, std=0.1)[0]
    kw = dict(gate_bias=vec(4, E), b1=vec(5, E, f * (1 + gated)), b2=vec(6, E, d)) if biases else {}
    if rule.pop("balanced", False):
        kw["choice_bias"] = vec(7, E)
    norm = 1 + vec(8, d)
    block = il.Int8MoEBlock(T, d, f, E, k, w1.to(dtype), w2.to(dtype), gate, norm, gated=gated, activation=activation, **kw, **rule)
    return block, w1.to(dtype), w2.to(dtype)


def check_first_rows(b, x, residual):
    s = host(b.stream)
    want = host(x) if residual is None else host((x.float() + residual.float()).to(BF))
    assert np.array_equal(s, want)
    u, rho = io.norm_parts(s, host(b.norm_weight), b.eps)
    check_rows(b.x8.codes, b.x8.scales, u, rho, NORM, b.d_model)
    return u * rho


def check_product(out, rows, scales, w, bias):
    """Against the weights' own int8 form, from the rows that the block made."""
    codes, ws = io.quantize_weights(w.float().cpu().numpy())
    q = rows.cpu().numpy()[:, :w.shape[1]]
    z, size = io.product(q, host(scales), codes, ws, None if bias is None else host(bias))
    within(out, z, size, "none", "f32" if out.dtype == torch.float32 else "bf16")


RULES = [dict(), dict(score="sigmoid", balanced=True, groups=4, groups_kept=2, group_top=2, scale=2.5), dict(renormalize=False, groups=2)]


@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("T,d,f,E,k,gated,activation,H", [(1, 64, 96, 8, 2, True, "silu", -1), (33, 128, 200, 16, 4, True, "gelu", -1), (300, 96, 64, 8, 2, False, "relu", 3),
                                                          (700, 256, 300, 32, 8, True, "silu", 9), (150, 64, 128, 8, 1, False, "none", 0)])
def test_moe_block(gpu_lib, T, d, f, E, k, gated, activation, H, rule):
    say(f"[case] int8 block {T} x {d} x {f}, {E} experts, k {k}, gated {gated} {activation} H {H} {rule}")
    rule = dict(rule)
    if rule.get("groups") == 2:
        rule["groups_kept"] = 2
    b, w1, w2 = moe_block(T, d, f, E, k, gated, activation, biases=H != 3, **rule)
    x, residual = tensors(10, (T, d), (T, d))
    b.out.fill_(77)
    y, stream = b.forward(x, residual, H)
    torch.cuda.synchronize()
    n = check_first_rows(b, x, residual)
    normed = host(b.normed)
    assert (np.abs(normed - n) <= (HALF["bf16"] * (1 + NORM) + NORM) * np.abs(n)).all()
    gate = host(b.w_gate)
    bias = None if b.gate_bias is None else host(b.gate_bias)
    want, size = orc.gate_logits(normed, gate, bias), np.abs(normed) @ np.abs(gate).T + (0 if bias is None else np.abs(bias))
    assert (np.abs(host(b.logits) - want) <= (d + 2) * 2.0 ** -23 * size).all()
    r = b.routing
    idx, weight = io.route(host(b.logits), k, "sigmoid" if r.score else "softmax", None if b.choice_bias is None else host(b.choice_bias), r.groups, r.groups_kept,
                           r.group_top, b.renormalize, r.scale)
    assert np.array_equal(b.topk_idx.cpu().numpy(), idx) and np.allclose(host(b.topk_w), weight, rtol=2.0 ** -19, atol=0)
    counts = np.bincount(idx.reshape(-1), minlength=E)
    assert np.array_equal(b.counts.cpu().numpy(), counts)
    on = np.ones(E, dtype=bool) if H < 0 else orc.hot_mask_top_h(counts, H).astype(bool)
    perm, inv = orc.stable_permutation(idx, E)[:2]
    assert np.array_equal(b.perm.cpu().numpy(), perm)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    for e in np.flatnonzero(on & (counts > 0)):
        s = slice(offsets[e], offsets[e + 1])
        rows = torch.from_numpy(perm[s].astype(np.int64) // k).cuda()
        check_product(b.h[s], b.x8.codes[rows], b.x8.scales[rows], w1[e], None if b.b1 is None else b.b1[e])
        h = host(b.h[s])
        v = io.activate(h[:, :f], activation) * (h[:, f:] if gated else 1.0)
        check_rows(b.h8.codes[s], b.h8.scales[s], v, None, 2.0 ** -17, f)
        check_product(b.y_perm[s], b.h8.codes[s], b.h8.scales[s], w2[e], None if b.b2 is None else b.b2[e])
    y_perm = host(b.y_perm)
    total, size = np.zeros((T, d)), np.zeros((T, d))
    inv = b.inv_perm.cpu().numpy().reshape(T, k)
    for j in range(k):
        term = np.where(on[idx[:, j]][:, None], host(b.topk_w)[:, j:j + 1] * y_perm[inv[:, j]], 0.0)
        total, size = total + term, size + np.abs(term)
    err = (k + 1) * 2.0 ** -24 * size
    assert (np.abs(host(y) - total) <= err * (1 + HALF["bf16"]) + HALF["bf16"] * np.abs(total)).all()


@pytest.mark.parametrize("T,d,f,gated,activation", [(1, 100, 70, True, "silu"), (17, 128, 129, False, "gelu"), (90, 200, 300, True, "relu"), (1100, 256, 512, True, "silu")])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_dense_block(gpu_lib, T, d, f, gated, activation, dtype):
    say(f"[case] int8 dense block {T} x {d} x {f} gated {gated} {activation} {dtype}")
    w1, w2 = (t.to(dtype) for t in tensors(1, (f * (1 + gated), d), (d, f), std=0.1))
    b1, b2 = tensors(2, (f * (1 + gated),), (d,), dtype=torch.float32)
    norm, = tensors(3, (d,), dtype=torch.float16)
    b = il.Int8DenseBlock(T, d, f, w1, w2, norm, b1=b1, b2=b2, activation=activation, gated=gated, eps=1e-5)
    x, residual = tensors(4, (T, d), (T, d))
    for res in (residual, None):
        y, stream = b.forward(x, res)
        torch.cuda.synchronize()
        check_first_rows(b, x, res)
        check_product(b.h, b.x8.codes, b.x8.scales, w1, b.b1)
        h = host(b.h)
        check_rows(b.h8.codes, b.h8.scales, io.activate(h[:, :f], activation) * (h[:, f:] if gated else 1.0), None, 2.0 ** -17, f)
        check_product(y, b.h8.codes, b.h8.scales, w2, b.b2)


def test_near_the_layer_in_full_precision(gpu_lib):
    """Rounding to int8 leaves an error of max / (127 sqrt 12) of a value, so of (max / rms) / 440 of the rms: 0.0095 for normal rows (max / rms 4.2), 0.0085 for the
    channels of w1 and w2 (3.7), 0.018 for gated rows (8).  Both halves of the first product are sqrt(0.0095^2 + 0.0085^2) = 0.013 off, their gated
    product 1.1 sqrt 2 times that, 0.02; the output sqrt(0.02^2 + 0.018^2 + 0.0085^2) = 0.028, and the worst of 200 rows up to half as much again."""
    say("[case] int8 block against full precision")
    T, d, f, E, k = 200, 512, 768, 8, 2
    b, w1, w2 = moe_block(T, d, f, E, k, biases=False)
    x, residual = tensors(10, (T, d), (T, d))
    y, _ = b.forward(x, residual)
    torch.cuda.synchronize()
    n, idx, w = host(b.normed), b.topk_idx.cpu().numpy(), host(b.topk_w)
    want = np.zeros((T, d))
    for e in range(E):
        t, j = np.nonzero(idx == e)
        h = n[t] @ host(w1[e]).T
        want[t] += w[t, j][:, None] * ((io.activate(h[:, :f], "silu") * h[:, f:]) @ host(w2[e]).T)
    off = np.linalg.norm(host(y) - want, axis=1) / np.linalg.norm(want, axis=1)
    say(f"worst row {off.max():.4f}")
    assert off.max() <= 0.04


def test_a_checkpoints_codes(gpu_lib):
    """int8 codes with their scales are used as they are: the block of quantised weights again."""
    say("[case] int8 block of a checkpoint's codes")
    T, d, f, E, k = 40, 64, 96, 8, 2
    b, w1, w2 = moe_block(T, d, f, E, k, biases=False)
    codes = [[io.quantize_weights(w[e].float().cpu().numpy()) for e in range(E)] for w in (w1, w2)]
    q1, q2 = (torch.from_numpy(np.stack([c for c, _ in cs])).cuda() for cs in codes)
    s1, s2 = (torch.from_numpy(np.stack([s for _, s in cs])).cuda() for cs in codes)
    c = il.Int8MoEBlock(T, d, f, E, k, q1, q2, b.w_gate, b.norm_weight, w1_scales=s1, w2_scales=s2)
    x, = tensors(10, (T, d))
    assert torch.equal(b.forward(x)[0], c.forward(x)[0])


def test_other_numbers_of_tokens(gpu_lib):
    """Blocks of other T share weights, and a token's output does not depend on the others'."""
    say("[case] int8 block resized")
    b, _, _ = moe_block(700, 256, 300, 32, 8, score="sigmoid", balanced=True, groups=4, groups_kept=2, group_top=2)
    x, residual = tensors(10, (700, 256), (700, 256))
    y = b.forward(x, residual)[0].clone()
    logits = b.logits.clone()
    for T in (0, 1, 5, 65, 200):
        s = b.resized(T)
        got, stream = s.forward(x[:T].contiguous(), residual[:T].contiguous())
        torch.cuda.synchronize()
        assert got.shape == (T, 256) and s.w1 is b.w1
        same = (s.logits == logits[:T]).all(1)                   # logits of few tokens are summed in another order
        ok = same & (s.topk_w == b.topk_w[:T]).all(1) & (s.topk_idx == b.topk_idx[:T]).all(1)
        assert torch.equal(got[ok], y[:T][ok])
        assert torch.allclose(got.float(), y[:T].float(), rtol=2.0 ** -6, atol=2.0 ** -6 * y.float().abs().max().item())


def test_block_in_a_graph(gpu_lib):
    """Captured and replayed with other inputs, with eager work between the replays; two graphs of one block share its buffers and run in turn."""
    say("[case] int8 block in graphs")
    b, _, _ = moe_block(130, 128, 200, 16, 4, score="sigmoid", balanced=True)
    x, residual = tensors(10, (130, 128), (130, 128))
    xs = [t.contiguous() for t in tensors(11, *[(130, 128)] * 4)]
    want = []
    for t in xs:
        want.append([v.clone() for v in b.forward(t, residual)] + [b.forward(t, residual, 5)[0].clone()])
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.forward(x, residual)
    torch.cuda.current_stream().wait_stream(side)
    for H in (-1, 5):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(b.forward(x, residual, H))
        graphs.append(g)
    for i, t in enumerate(xs):
        x.copy_(t)
        for n, g in enumerate(graphs):
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(b.out, want[i][0 if n == 0 else 2]) and torch.equal(b.stream, want[i][1])
            b.resized(3).forward(x[:3].contiguous())             # eager work in between
    assert all(o[0] is b.out for o in outs)


def test_blocks_on_two_streams(gpu_lib):
    """Two blocks at once, each on a stream of its own, bit for bit what each gives alone."""
    say("[case] int8 blocks on two streams")
    blocks = [moe_block(T, 256, 300, 32, 8, score="sigmoid", balanced=True, groups=4, groups_kept=2, group_top=2)[0] for T in (900, 60)]
    xs = [tensors(20 + i, (b.T, 256))[0] for i, b in enumerate(blocks)]
    alone = [b.forward(x)[0].clone() for b, x in zip(blocks, xs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b in blocks:
            b.out.zero_()
        torch.cuda.synchronize()
        for s, b, x in zip(streams, blocks, xs):
            with torch.cuda.stream(s):
                for _ in range(3):
                    b.forward(x)
        torch.cuda.synchronize()
        for b, want in zip(blocks, alone):
            assert torch.equal(b.out, want)
