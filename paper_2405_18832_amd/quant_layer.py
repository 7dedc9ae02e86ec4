"""Feed-forward blocks in 8 bits, as a pre-norm model runs them: their tensors on the device and the calls into the C ABI.

`QuantMoEBlock`: residual addition and RMS norm with a quantised output, routing on the norm in bf16, both expert products on e4m3 rows
and weights, combine.  `QuantDenseBlock`: the same for the dense layers between the expert layers.  No arithmetic happens here.

    block = QuantMoEBlock(T, d_model, d_ff, E, k, w1, w2, w_gate, norm_weight)      # w1 [E, d_ff, d_model], w2 [E, d_model, d_ff]
    y, stream = block.forward(x, residual)     # stream = x + residual continues; y is the next block's x

Sums are fp32; with sums="units" those of bf16 and e4m3 outputs come from the matrix units for 8-bit operands, which are faster for many
tokens and less exact (moe.h, MOE_QUANT_UNIT_SUMS).

Both products of a step of T tokens use workspaces that are made once; a block of another T shares the weights through `resized`.

The library reads addresses, so that shapes, types and devices are checked here, with ValueError: x, residual and w_gate are bf16, the norm's
weight and the biases of any floating type (kept as fp32).
"""
from __future__ import annotations

import copy
import math
from typing import Optional

import torch

from . import (make_quant_shape, make_shape, moe_combine, moe_norm_quantize, moe_permute, moe_quant_expert_linear, moe_quant_linear,
               moe_quant_pitch, moe_quant_weight_bytes, moe_quant_workspace_bytes, moe_quantize_weights, moe_route, moe_workspace_bytes)

_DTYPES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float8_e4m3fn: "e4m3"}


def _blocks(n: int) -> int:
    return moe_quant_pitch(n) // 128


def _check(name: str, t: torch.Tensor, shape: tuple, device, dtypes: tuple) -> None:
    if t.shape != shape or t.dtype not in dtypes or t.device != device:
        raise ValueError(f"{name}: expected {list(shape)} of {' or '.join(str(d) for d in dtypes)} on {device}, "
                         f"got {list(t.shape)} of {t.dtype} on {t.device}")


def _fp32(name: str, t: Optional[torch.Tensor], shape: tuple, device) -> Optional[torch.Tensor]:
    """A norm weight or bias as the library reads it."""
    if t is None:
        return None
    _check(name, t, shape, device, (torch.float32, torch.bfloat16, torch.float16))
    return t.detach().float().contiguous()


class QuantWeights:
    """E matrices [E, N, K] in the products' layout and their scales.  `w`: fp32 or bf16 weights, which are quantised, or a checkpoint's
    e4m3 codes with their `scales` [E, ceil(N / 128), ceil(K / 128)]."""

    def __init__(self, w: torch.Tensor, scales: Optional[torch.Tensor] = None):
        if w.dim() != 3 or w.dtype not in _DTYPES:
            raise ValueError(f"weights are [E, N, K] in fp32, bf16 or e4m3, got {list(w.shape)} of {w.dtype}")
        self.E, self.N, self.K = w.shape
        if moe_quant_weight_bytes(self.E, self.N, self.K) == 0:
            raise ValueError(f"weights of {list(w.shape)}: 1 <= E <= 1024, 1 <= N, K <= 2^24")
        if (w.dtype == torch.float8_e4m3fn) != (scales is not None):
            raise ValueError("scales belong to e4m3 codes")
        if scales is not None and tuple(scales.shape) != (self.E, _blocks(self.N), _blocks(self.K)):
            raise ValueError("one scale per matrix and 128 x 128 block")
        if scales is not None and scales.device != w.device:
            raise ValueError("scales are on the weights' device")
        self.codes = torch.empty(moe_quant_weight_bytes(self.E, self.N, self.K), dtype=torch.uint8, device=w.device)
        self.scales = scales.float().contiguous() if scales is not None else torch.empty(
            (self.E, _blocks(self.N), _blocks(self.K)), device=w.device)
        moe_quantize_weights(self.E, self.N, self.K, _DTYPES[w.dtype], w, self.codes, None if scales is not None else self.scales)


class _Rows:
    """Quantised rows [R, C]."""

    def __init__(self, R: int, C: int, device):
        self.codes = torch.empty((R, moe_quant_pitch(C)), dtype=torch.float8_e4m3fn, device=device)
        self.scales = torch.empty((R, _blocks(C)), device=device)


class _Block:
    def _check_sizes(self):
        if self.T < 0 or self.d_model < 1 or self.d_ff < 1:
            raise ValueError(f"T = {self.T}, d_model = {self.d_model}, d_ff = {self.d_ff}")
        if not (math.isfinite(self.eps) and self.eps >= 0):
            raise ValueError(f"eps = {self.eps}")

    def _norm_buffers(self, norm_out: bool):
        d, dev = self.d_model, self.device
        self.stream = torch.empty((self.T, d), dtype=torch.bfloat16, device=dev)
        self.normed = torch.empty((self.T, d), dtype=torch.bfloat16, device=dev) if norm_out else None
        self.x8 = _Rows(self.T, d, dev)
        self.out = torch.empty((self.T, d), dtype=torch.bfloat16, device=dev)

    def _norm(self, x, residual):
        _check("x", x, (self.T, self.d_model), self.device, (torch.bfloat16,))
        if residual is not None:
            _check("residual", residual, (self.T, self.d_model), self.device, (torch.bfloat16,))
        moe_norm_quantize(self.T, self.d_model, "bf16", x, residual, self.norm_weight, self.eps, self.stream, self.normed, self.x8.codes,
                          self.x8.scales)

    def _workspace(self, shape):
        size = moe_quant_workspace_bytes(shape)
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


class QuantMoEBlock(_Block):
    def __init__(self, T, d_model, d_ff, E, k, w1, w2, w_gate, norm_weight=None, *, w1_scales=None, w2_scales=None, gate_bias=None, b1=None,
                 b2=None, activation="relu", renormalize=True, eps=1e-6, sums="f32"):
        self.T, self.d_model, self.d_ff, self.E, self.k, self.sums = T, d_model, d_ff, E, k, sums
        self.device, self.eps, self.activation, self.renormalize = w1.device, eps, activation, renormalize
        dev = self.device
        self._check_sizes()
        if tuple(w1.shape) != (E, d_ff, d_model) or tuple(w2.shape) != (E, d_model, d_ff) or w2.device != dev:
            raise ValueError("w1 is [E, d_ff, d_model], w2 [E, d_model, d_ff], on one device")
        _check("w_gate", w_gate, (E, d_model), dev, (torch.bfloat16,))
        self.w_gate = w_gate
        self.norm_weight, self.gate_bias = _fp32("norm_weight", norm_weight, (d_model,), dev), _fp32("gate_bias", gate_bias, (E,), dev)
        self.b1, self.b2 = _fp32("b1", b1, (E, d_ff), dev), _fp32("b2", b2, (E, d_model), dev)
        self.layer = self._layer()
        self.w1, self.w2 = QuantWeights(w1, w1_scales), QuantWeights(w2, w2_scales)
        self._buffers()

    def _layer(self):
        layer = make_shape(self.T, self.d_model, self.d_ff, self.E, self.k, "bf16", self.renormalize)
        if moe_workspace_bytes(layer) == 0:
            raise ValueError(f"a layer that the library refuses (d_model and d_ff are multiples of 32, k <= E <= 1024, k <= 8): T = {self.T}, "
                             f"d_model = {self.d_model}, d_ff = {self.d_ff}, E = {self.E}, k = {self.k}")
        return layer

    def _buffers(self):
        T, k, E, dev = self.T, self.k, self.E, self.device
        A = T * k
        self.layer = self._layer()
        self.first = make_quant_shape(A, self.d_ff, self.d_model, E, k, self.activation, "e4m3", self.sums)
        self.second = make_quant_shape(A, self.d_model, self.d_ff, E, 1, "none", "f32")
        self.ws1, self.ws2 = self._workspace(self.first), self._workspace(self.second)
        self._norm_buffers(norm_out=True)
        i32 = torch.int32
        self.topk_idx = torch.empty((T, k), dtype=i32, device=dev)
        self.topk_w = torch.empty((T, k), device=dev)
        self.counts = torch.empty(E, dtype=i32, device=dev)
        self.offsets = torch.empty(E + 1, dtype=i32, device=dev)
        self.perm, self.inv_perm = (torch.empty(A, dtype=i32, device=dev) for _ in range(2))
        self.hot_mask = torch.empty(E, dtype=torch.uint8, device=dev)
        self.h8 = _Rows(A, self.d_ff, dev)
        self.y_perm = torch.empty((A, self.d_model), device=dev)
        self.ws = torch.empty(moe_workspace_bytes(self.layer), dtype=torch.uint8, device=dev)

    def forward(self, x, residual=None, H: int = -1):
        """(the block's output, the residual stream x + residual), both [T, d_model] bf16 and overwritten by the next call.  H >= 0: the
        share of the H experts with the most tokens."""
        self._norm(x, residual)
        mask = self.hot_mask if H >= 0 else None
        moe_route(self.layer, self.normed, self.w_gate, self.gate_bias, self.topk_idx, self.topk_w, None, self.counts, self.offsets, H, mask,
                  self.ws)
        moe_permute(self.layer, None, self.topk_idx, self.offsets, self.perm, self.inv_perm, None, self.ws)
        moe_quant_expert_linear(self.first, self.x8.codes, self.x8.scales, self.perm, self.offsets, mask, self.w1.codes, self.w1.scales, self.b1,
                                self.h8.codes, self.h8.scales, self.ws1)
        moe_quant_expert_linear(self.second, self.h8.codes, self.h8.scales, None, self.offsets, mask, self.w2.codes, self.w2.scales, self.b2,
                                self.y_perm, None, self.ws2)
        moe_combine(self.layer, self.y_perm, self.inv_perm, self.topk_idx, self.topk_w, mask, self.out)
        return self.out, self.stream


class QuantDenseBlock(_Block):
    def __init__(self, T, d_model, d_ff, w1, w2, norm_weight=None, *, w1_scales=None, w2_scales=None, b1=None, b2=None, activation="relu",
                 eps=1e-6, sums="f32"):
        self.T, self.d_model, self.d_ff, self.sums = T, d_model, d_ff, sums
        self.device, self.eps, self.activation = w1.device, eps, activation
        dev = self.device
        self._check_sizes()
        if tuple(w1.shape) != (d_ff, d_model) or tuple(w2.shape) != (d_model, d_ff) or w2.device != dev:
            raise ValueError("w1 is [d_ff, d_model], w2 [d_model, d_ff], on one device")
        self.norm_weight = _fp32("norm_weight", norm_weight, (d_model,), dev)
        self.b1, self.b2 = _fp32("b1", b1, (d_ff,), dev), _fp32("b2", b2, (d_model,), dev)
        one = lambda t: None if t is None else t[None]
        self.w1, self.w2 = QuantWeights(w1[None], one(w1_scales)), QuantWeights(w2[None], one(w2_scales))
        self._buffers()

    def _buffers(self):
        self.first = make_quant_shape(self.T, self.d_ff, self.d_model, 1, 1, self.activation, "e4m3", self.sums)
        self.second = make_quant_shape(self.T, self.d_model, self.d_ff, 1, 1, "none", "bf16", self.sums)
        self.ws1, self.ws2 = self._workspace(self.first), self._workspace(self.second)
        self._norm_buffers(norm_out=False)
        self.h8 = _Rows(self.T, self.d_ff, self.device)

    def forward(self, x, residual=None):
        """(the block's output, the residual stream x + residual), both [T, d_model] bf16 and overwritten by the next call."""
        self._norm(x, residual)
        moe_quant_linear(self.first, self.x8.codes, self.x8.scales, self.w1.codes, self.w1.scales, self.b1, self.h8.codes, self.h8.scales, self.ws1)
        moe_quant_linear(self.second, self.h8.codes, self.h8.scales, self.w2.codes, self.w2.scales, self.b2, self.out, None, self.ws2)
        return self.out, self.stream
