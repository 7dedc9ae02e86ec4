"""A token's output does not depend on the others': blocks of other numbers of tokens, given the same logits (whose sums' order goes by that number), bit for bit."""
import pytest
import torch

from paper_2405_18832_amd import int8_layer as il
from test_int_layer_gpu import moe_block, say, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("H", [-1, 32])
def test_tokens_by_themselves(gpu_lib, monkeypatch, score, H):
    say(f"[case] int8 block resized, logits given, {score} H {H}")
    b, _, _ = moe_block(700, 256, 300, 32, 8, score=score, balanced=True, groups=4, groups_kept=2, group_top=2)
    x, residual = tensors(10, (700, 256), (700, 256))
    y, stream = (t.clone() for t in b.forward(x, residual, H))
    logits, idx, w = b.logits.clone(), b.topk_idx.clone(), b.topk_w.clone()
    for T in (1, 5, 32, 33, 65, 200, 699):
        monkeypatch.setattr(il, "moe_gate_logits", lambda layer, n, w_gate, bias, out: out.copy_(logits[:out.shape[0]]))
        s = b.resized(T)
        got, of = s.forward(x[:T].contiguous(), residual[:T].contiguous(), H)
        torch.cuda.synchronize()
        assert torch.equal(s.topk_idx, idx[:T]) and torch.equal(s.topk_w, w[:T])
        assert torch.equal(of, stream[:T]) and torch.equal(got, y[:T])
