"""Feed-forward blocks in int8 with a scale per token and output channel, as a pre-norm model runs them: their tensors on the device and the calls into
the C ABI.

`Int8MoEBlock`: residual addition and RMS norm with an int8 output, routing by scores on the norm in bf16, both expert products on int8 rows and
weights with the activation (gated or not) between them, combine.  `Int8DenseBlock`: the same for dense layers and shared experts.  No arithmetic
happens here.

    block = Int8MoEBlock(T, d_model, d_ff, E, k, w1, w2, w_gate, norm_weight, score="sigmoid", choice_bias=bias, groups=8, groups_kept=4, group_top=2)
    y, stream = block.forward(x, residual)     # stream = x + residual continues; y is the next block's x

gated (the default): w1 [E, 2 d_ff, d_model], act(first d_ff rows' outputs) * the others'; else w1 [E, d_ff, d_model].  w2 [E, d_model, d_ff].  Weights are fp32
or bf16, which are quantised, or a checkpoint's int8 codes with their scales per output channel, w1_scales [E, rows of w1], w2_scales [E, d_model].

Workspaces are made once for a step of T tokens; a block of another T shares the weights through `resized`.  The library reads addresses, so that
shapes, types and devices are checked here, with ValueError: x, residual and w_gate are bf16, the norm's weight and the biases of any floating type
(kept as fp32).
"""
from __future__ import annotations

import copy
import math
from typing import Optional

import torch

from . import (make_quant_shape, make_routing, make_shape, moe_act_quantize_int, moe_combine, moe_gate_logits, moe_int_expert_linear, moe_int_linear,
               moe_int_workspace_bytes, moe_norm_quantize_int, moe_permute, moe_quant_pitch, moe_quant_weight_bytes, moe_quantize_weights_int,
               moe_route_logits, moe_workspace_bytes, MOE_INT_MAX_K, MOE_MAX_GROUPS)
from .quant_layer import _check, _fp32

_DTYPES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.int8: "i8"}
_ACTIVATIONS = ("none", "relu", "gelu", "silu")


class Int8Weights:
    """E matrices [E, N, K] in the products' layout and their scales [E, N].  `w`: fp32 or bf16 weights, which are quantised, or int8 codes with
    their `scales`."""

    def __init__(self, w: torch.Tensor, scales: Optional[torch.Tensor] = None):
        if w.dim() != 3 or w.dtype not in _DTYPES:
            raise ValueError(f"weights are [E, N, K] in fp32, bf16 or int8, got {list(w.shape)} of {w.dtype}")
        self.E, self.N, self.K = w.shape
        if moe_quant_weight_bytes(self.E, self.N, self.K) == 0 or self.K > MOE_INT_MAX_K:
            raise ValueError(f"weights of {list(w.shape)}: 1 <= E <= 1024, 1 <= N <= 2^24, 1 <= K <= {MOE_INT_MAX_K}")
        if (w.dtype == torch.int8) != (scales is not None):
            raise ValueError("scales belong to int8 codes")
        if scales is not None and tuple(scales.shape) != (self.E, self.N):
            raise ValueError("one scale per matrix and output channel")
        if scales is not None and (scales.device != w.device or not scales.is_floating_point()):
            raise ValueError("scales are floating-point numbers on the weights' device")
        self.codes = torch.empty(moe_quant_weight_bytes(self.E, self.N, self.K), dtype=torch.int8, device=w.device)
        self.scales = scales.float().contiguous() if scales is not None else torch.empty((self.E, self.N), device=w.device)
        moe_quantize_weights_int(self.E, self.N, self.K, _DTYPES[w.dtype], w, self.codes, None if scales is not None else self.scales)


class _Rows:
    """int8 rows [R, C]."""

    def __init__(self, R: int, C: int, device):
        self.codes = torch.empty((R, moe_quant_pitch(C)), dtype=torch.int8, device=device)
        self.scales = torch.empty(R, device=device)


class _Block:
    def _check_sizes(self):
        if self.T < 0 or self.d_model < 1 or self.d_ff < 1:
            raise ValueError(f"T = {self.T}, d_model = {self.d_model}, d_ff = {self.d_ff}")
        if not (math.isfinite(self.eps) and self.eps >= 0):
            raise ValueError(f"eps = {self.eps}")
        if self.activation not in _ACTIVATIONS:
            raise ValueError(f"activation is one of {', '.join(_ACTIVATIONS)}, got {self.activation!r}")
        self.width = self.d_ff * (2 if self.gated else 1)       # of the first product

    def _row_buffers(self, rows: int, norm_out: bool):
        d, dev, bf16 = self.d_model, self.device, torch.bfloat16
        self.stream = torch.empty((self.T, d), dtype=bf16, device=dev)
        self.normed = torch.empty((self.T, d), dtype=bf16, device=dev) if norm_out else None
        self.x8 = _Rows(self.T, d, dev)
        self.h = torch.empty((rows, self.width), dtype=bf16, device=dev)
        self.h8 = _Rows(rows, self.d_ff, dev)
        self.out = torch.empty((self.T, d), dtype=bf16, device=dev)

    def _norm(self, x, residual):
        _check("x", x, (self.T, self.d_model), self.device, (torch.bfloat16,))
        if residual is not None:
            _check("residual", residual, (self.T, self.d_model), self.device, (torch.bfloat16,))
        moe_norm_quantize_int(self.T, self.d_model, "bf16", x, residual, self.norm_weight, self.eps, self.stream, self.normed, self.x8.codes,
                              self.x8.scales)

    def _workspace(self, shape):
        size = moe_int_workspace_bytes(shape)
        if size == 0:
            raise ValueError(f"products that the library refuses: T = {self.T}, d_model = {self.d_model}, d_ff = {self.d_ff}")
        return torch.empty(size, dtype=torch.uint8, device=self.device)

    def resized(self, T: int):
        """The same block for T tokens: weights shared, buffers of its own."""
        other = copy.copy(self)
        other.T = T
        other._check_sizes()
        other._buffers()
        return other


class Int8MoEBlock(_Block):
    def __init__(self, T, d_model, d_ff, E, k, w1, w2, w_gate, norm_weight=None, *, w1_scales=None, w2_scales=None, gate_bias=None, choice_bias=None,
                 b1=None, b2=None, activation="silu", gated=True, score="softmax", groups=1, groups_kept=1, group_top=1, scale=1.0, renormalize=True,
                 eps=1e-6):
        self.T, self.d_model, self.d_ff, self.E, self.k = T, d_model, d_ff, E, k
        self.device, self.eps, self.activation, self.gated, self.renormalize = w1.device, eps, activation, bool(gated), renormalize
        dev = self.device
        self._check_sizes()
        if score not in ("softmax", "sigmoid"):
            raise ValueError(f"score is softmax or sigmoid, got {score!r}")
        if not (1 <= groups <= MOE_MAX_GROUPS and E % groups == 0 and 1 <= groups_kept <= groups and groups_kept * (E // groups) >= k and group_top in (1, 2)
                and (groups == 1 or E // groups >= group_top) and math.isfinite(scale)):
            raise ValueError(f"routing that the library refuses: {E} experts in {groups} groups, {groups_kept} of them kept by their {group_top} largest, "
                             f"k = {k}, scale = {scale}")
        self.routing = make_routing(score, groups, groups_kept, group_top, scale)
        if tuple(w1.shape) != (E, self.width, d_model) or tuple(w2.shape) != (E, d_model, d_ff) or w2.device != dev:
            raise ValueError("w1 is [E, 2 d_ff (gated) or d_ff, d_model], w2 [E, d_model, d_ff], on one device")
        _check("w_gate", w_gate, (E, d_model), dev, (torch.bfloat16,))
        self.w_gate = w_gate.contiguous()
        self.norm_weight = _fp32("norm_weight", norm_weight, (d_model,), dev)
        self.gate_bias, self.choice_bias = _fp32("gate_bias", gate_bias, (E,), dev), _fp32("choice_bias", choice_bias, (E,), dev)
        self.b1, self.b2 = _fp32("b1", b1, (E, self.width), dev), _fp32("b2", b2, (E, d_model), dev)
        self.layer = self._layer()
        self.w1, self.w2 = Int8Weights(w1, w1_scales), Int8Weights(w2, w2_scales)
        self._buffers()

    def _layer(self):
        # routing, permutation and combine know the layer by its tokens, experts and d_model; d_ff plays no part in them
        layer = make_shape(self.T, self.d_model, 32, self.E, self.k, "bf16", self.renormalize)
        if moe_workspace_bytes(layer) == 0:
            raise ValueError(f"a layer that the library refuses (d_model is a multiple of 32, k <= E <= 1024, k <= 8): T = {self.T}, "
                             f"d_model = {self.d_model}, E = {self.E}, k = {self.k}")
        return layer

    def _buffers(self):
        T, k, E, dev = self.T, self.k, self.E, self.device
        A = T * k
        self.layer = self._layer()
        self.first = make_quant_shape(A, self.width, self.d_model, E, k, "none", "bf16")
        self.second = make_quant_shape(A, self.d_model, self.d_ff, E, 1, "none", "f32")
        self.ws1, self.ws2 = self._workspace(self.first), self._workspace(self.second)
        self._row_buffers(A, norm_out=True)
        i32 = torch.int32
        self.logits = torch.empty((T, E), device=dev)
        self.topk_idx = torch.empty((T, k), dtype=i32, device=dev)
        self.topk_w = torch.empty((T, k), device=dev)
        self.counts = torch.empty(E, dtype=i32, device=dev)
        self.offsets = torch.empty(E + 1, dtype=i32, device=dev)
        self.perm, self.inv_perm = (torch.empty(A, dtype=i32, device=dev) for _ in range(2))
        self.hot_mask = torch.empty(E, dtype=torch.uint8, device=dev)
        self.y_perm = torch.empty((A, self.d_model), device=dev)
        self.ws = torch.empty(moe_workspace_bytes(self.layer), dtype=torch.uint8, device=dev)

    def forward(self, x, residual=None, H: int = -1):
        """(the block's output, the residual stream x + residual), both [T, d_model] bf16 and overwritten by the next call.  H >= 0: the
        share of the H experts with the most tokens."""
        self._norm(x, residual)
        mask = self.hot_mask if H >= 0 else None
        moe_gate_logits(self.layer, self.normed, self.w_gate, self.gate_bias, self.logits)
        moe_route_logits(self.layer, self.routing, "f32", self.logits, self.choice_bias, self.topk_idx, self.topk_w, self.counts, self.offsets, H, mask,
                         self.ws)
        moe_permute(self.layer, None, self.topk_idx, self.offsets, self.perm, self.inv_perm, None, self.ws)
        moe_int_expert_linear(self.first, self.x8.codes, self.x8.scales, self.perm, self.offsets, mask, self.w1.codes, self.w1.scales, self.b1, self.h,
                              self.ws1)
        moe_act_quantize_int(self.T * self.k, self.d_ff, "bf16", self.h, self.gated, self.activation, self.E, self.offsets if H >= 0 else None, mask,
                             self.h8.codes, self.h8.scales)
        moe_int_expert_linear(self.second, self.h8.codes, self.h8.scales, None, self.offsets, mask, self.w2.codes, self.w2.scales, self.b2, self.y_perm,
                              self.ws2)
        moe_combine(self.layer, self.y_perm, self.inv_perm, self.topk_idx, self.topk_w, mask, self.out)
        return self.out, self.stream


class Int8DenseBlock(_Block):
    def __init__(self, T, d_model, d_ff, w1, w2, norm_weight=None, *, w1_scales=None, w2_scales=None, b1=None, b2=None, activation="silu", gated=True,
                 eps=1e-6):
        self.T, self.d_model, self.d_ff = T, d_model, d_ff
        self.device, self.eps, self.activation, self.gated = w1.device, eps, activation, bool(gated)
        dev = self.device
        self._check_sizes()
        if tuple(w1.shape) != (self.width, d_model) or tuple(w2.shape) != (d_model, d_ff) or w2.device != dev:
            raise ValueError("w1 is [2 d_ff (gated) or d_ff, d_model], w2 [d_model, d_ff], on one device")
        self.norm_weight = _fp32("norm_weight", norm_weight, (d_model,), dev)
        self.b1, self.b2 = _fp32("b1", b1, (self.width,), dev), _fp32("b2", b2, (d_model,), dev)
        one = lambda t: None if t is None else t[None]
        self.w1, self.w2 = Int8Weights(w1[None], one(w1_scales)), Int8Weights(w2[None], one(w2_scales))
        self._buffers()

    def _buffers(self):
        self.first = make_quant_shape(self.T, self.width, self.d_model, 1, 1, "none", "bf16")
        self.second = make_quant_shape(self.T, self.d_model, self.d_ff, 1, 1, "none", "bf16")
        self.ws1, self.ws2 = self._workspace(self.first), self._workspace(self.second)
        self._row_buffers(self.T, norm_out=False)

    def forward(self, x, residual=None):
        """(the block's output, the residual stream x + residual), both [T, d_model] bf16 and overwritten by the next call."""
        self._norm(x, residual)
        moe_int_linear(self.first, self.x8.codes, self.x8.scales, self.w1.codes, self.w1.scales, self.b1, self.h, self.ws1)
        moe_act_quantize_int(self.T, self.d_ff, "bf16", self.h, self.gated, self.activation, 0, None, None, self.h8.codes, self.h8.scales)
        moe_int_linear(self.second, self.h8.codes, self.h8.scales, self.w2.codes, self.w2.scales, self.b2, self.out, self.ws2)
        return self.out, self.stream
