// C ABI of the routing by scores and of the int8 layers: argument validation on the host, then asynchronous launches on the caller's stream.
#include <cmath>

#include "int8.hpp"

using namespace moe;

namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool is_activation(int act) { return act == MOE_ACT_NONE || act == MOE_ACT_RELU || act == MOE_ACT_GELU || act == MOE_ACT_SILU; }
moe_status from_hip(hipError_t e) { return e == hipSuccess ? MOE_OK : MOE_ERR_HIP; }

// A shape that the layer's calls take, its d_ff and k aside.
moe_status check_router(const moe_shape* s) {
    if (s == nullptr || s->T < 0 || s->d_model <= 0 || s->E <= 0) return MOE_ERR_INVALID_ARG;
    if (s->dtype != MOE_F32 && s->dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (s->E > MOE_MAX_E || s->T > 0x3fffffff) return MOE_ERR_UNSUPPORTED;
    if (s->dtype == MOE_BF16 && s->d_model % 32 != 0) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

moe_status check_routing(const moe_shape& s, const moe_routing* r) {
    if (r == nullptr || (r->score != MOE_SCORE_SOFTMAX && r->score != MOE_SCORE_SIGMOID)) return MOE_ERR_INVALID_ARG;
    if (r->groups < 1 || s.E % r->groups != 0 || r->groups_kept < 1 || r->groups_kept > r->groups) return MOE_ERR_INVALID_ARG;
    if (r->groups > MOE_MAX_GROUPS) return MOE_ERR_UNSUPPORTED;
    const int size = s.E / r->groups;
    if (r->groups_kept * size < s.k) return MOE_ERR_INVALID_ARG;
    if (r->group_top != 1 && r->group_top != 2) return MOE_ERR_INVALID_ARG;
    if (r->groups > 1 && size < r->group_top) return MOE_ERR_INVALID_ARG;
    if (!std::isfinite(r->scale)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

moe_status check_matrices(int32_t E, int32_t N, int32_t K) {
    if (E < 1 || N < 1 || K < 1) return MOE_ERR_INVALID_ARG;
    if (E > MOE_MAX_E || N > kMaxQuantDim || K > MOE_INT_MAX_K) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

moe_status check_product(const moe_quant_shape* s) {
    if (s == nullptr || s->rows < 0 || s->k < 1) return MOE_ERR_INVALID_ARG;
    const moe_status st = check_matrices(s->E, s->N, s->K);
    if (st != MOE_OK) return st;
    if (s->out_dtype != MOE_F32 && s->out_dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (!is_activation(s->activation)) return MOE_ERR_UNSUPPORTED;
    if (s->rows % s->k != 0) return MOE_ERR_INVALID_ARG;
    if (s->k > MOE_MAX_K) return MOE_ERR_UNSUPPORTED;
    // int32 numbers of rows and of the kernels' units (row tiles of 16 rows at least x 16 columns)
    if (s->rows > 0x3fffffff) return MOE_ERR_UNSUPPORTED;
    const long long tiles = s->rows / 16 + s->E, columns = (static_cast<long long>(s->N) + 15) / 16;
    if (tiles * columns > 0x3fffffffLL) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

moe_status product(const moe_quant_shape* s, const void* a, const float* a_scales, const int32_t* perm, const int32_t* offsets,
                   const uint8_t* mask, const void* w, const float* w_scales, const float* bias, void* out, void* ws, size_t ws_bytes, void* stream,
                   bool grouped) {
    const moe_status st = check_product(s);
    if (st != MOE_OK) return st;
    if (!grouped && (s->E != 1 || s->k != 1)) return MOE_ERR_INVALID_ARG;
    if (s->rows == 0) return MOE_OK;
    if (a == nullptr || a_scales == nullptr || w == nullptr || w_scales == nullptr || out == nullptr) return MOE_ERR_INVALID_ARG;
    if (grouped && offsets == nullptr) return MOE_ERR_INVALID_ARG;
    if (!aligned(a, 16) || !aligned(w, 16) || !aligned(out, elem_size(s->out_dtype)) || !aligned(a_scales, 4) || !aligned(w_scales, 4) ||
        !aligned(bias, 4) || !aligned(perm, 4) || !aligned(offsets, 4))
        return MOE_ERR_INVALID_ARG;
    if (ws == nullptr || !aligned(ws, 256) || ws_bytes < int_product_workspace(*s)) return MOE_ERR_WORKSPACE;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    const QuantArgs args{static_cast<const uint8_t*>(a), a_scales, perm, offsets, mask, static_cast<const uint8_t*>(w), w_scales, bias,
                         out, nullptr, s->rows, s->N, s->K, s->E, perm != nullptr ? s->k : 1, s->activation, s->out_dtype, false};
    return from_hip(launch_int_product(args, ws, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

moe_status moe_gate_logits(const moe_shape* shape, const void* x, const void* w_gate, const float* gate_bias, float* logits, void* stream) {
    const moe_status st = check_router(shape);
    if (st != MOE_OK) return st;
    if (shape->T == 0) return MOE_OK;
    const size_t es = elem_size(shape->dtype);
    if (x == nullptr || w_gate == nullptr || logits == nullptr) return MOE_ERR_INVALID_ARG;
    if (!aligned(x, es) || !aligned(w_gate, es) || !aligned(gate_bias, 4) || !aligned(logits, 4)) return MOE_ERR_INVALID_ARG;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    return from_hip(launch_gate_logits(*shape, x, w_gate, gate_bias, logits, static_cast<hipStream_t>(stream)));
}

moe_status moe_route_logits(const moe_shape* shape, const moe_routing* routing, int32_t logits_dtype, const void* logits,
                            const float* choice_bias, int32_t* topk_idx, float* topk_w, int32_t* counts, int32_t* offsets, int32_t H,
                            uint8_t* hot_mask, void* ws, size_t ws_bytes, void* stream) {
    moe_status st = layer_shape_status(shape);
    if (st == MOE_OK) st = check_routing(*shape, routing);
    if (st != MOE_OK) return st;
    if (logits_dtype != MOE_F32 && logits_dtype != MOE_BF16) return MOE_ERR_INVALID_ARG;
    if (counts == nullptr || offsets == nullptr || (H >= 0 && hot_mask == nullptr)) return MOE_ERR_INVALID_ARG;
    if (shape->T > 0 && (logits == nullptr || topk_idx == nullptr || topk_w == nullptr)) return MOE_ERR_INVALID_ARG;
    if (!aligned(logits, elem_size(logits_dtype)) || !aligned(choice_bias, 4) || !aligned(topk_idx, 4) || !aligned(topk_w, 4) || !aligned(counts, 4) ||
        !aligned(offsets, 4))
        return MOE_ERR_INVALID_ARG;
    if (ws == nullptr || !aligned(ws, 256) || ws_bytes < ws_layout(*shape).total) return MOE_ERR_WORKSPACE;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    const ScoreArgs args{logits, logits_dtype == MOE_BF16, choice_bias, topk_idx, topk_w, counts, offsets, hot_mask,
                         reinterpret_cast<int32_t*>(static_cast<char*>(ws) + ws_layout(*shape).hist),
                         shape->T, shape->E, shape->k, H, routing->score == MOE_SCORE_SIGMOID, shape->renormalize != 0,
                         routing->groups, routing->groups_kept, routing->group_top, routing->scale};
    return from_hip(launch_route_logits(args, static_cast<hipStream_t>(stream)));
}

moe_status moe_quantize_weights_int(int32_t E, int32_t N, int32_t K, int32_t src_dtype, const void* src, void* dst, float* scales, void* stream) {
    const moe_status st = check_matrices(E, N, K);
    if (st != MOE_OK) return st;
    if (src_dtype != MOE_F32 && src_dtype != MOE_BF16 && src_dtype != MOE_I8) return MOE_ERR_INVALID_ARG;
    if (src == nullptr || dst == nullptr || src == dst || (src_dtype != MOE_I8 && scales == nullptr)) return MOE_ERR_INVALID_ARG;
    if (!aligned(dst, 16) || !aligned(src, src_dtype == MOE_I8 ? 1 : elem_size(src_dtype)) || !aligned(scales, 4)) return MOE_ERR_INVALID_ARG;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    return from_hip(launch_quantize_weights_int(E, N, K, src_dtype, src, static_cast<uint8_t*>(dst), scales, static_cast<hipStream_t>(stream)));
}

moe_status moe_norm_quantize_int(int32_t rows, int32_t d, int32_t dtype, const void* x, const void* residual, const float* weight, float eps,
                                 void* sum_out, void* norm_out, void* q, float* q_scales, void* stream) {
    if (rows < 0 || d < 1 || (dtype != MOE_F32 && dtype != MOE_BF16) || !(eps >= 0.f) || std::isinf(eps)) return MOE_ERR_INVALID_ARG;
    if (d > kMaxQuantDim || rows > 0x3fffffff) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    if (x == nullptr || q == nullptr || q_scales == nullptr) return MOE_ERR_INVALID_ARG;
    const size_t es = elem_size(dtype);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(sum_out, es) || !aligned(norm_out, es) || !aligned(weight, 4) || !aligned(q, 16) ||
        !aligned(q_scales, 4))
        return MOE_ERR_INVALID_ARG;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    const IntRowArgs args{x, residual, weight, eps, sum_out, norm_out, nullptr, nullptr, static_cast<uint8_t*>(q), q_scales, rows, d, 0, MOE_ACT_NONE,
                          false};
    return from_hip(launch_norm_quantize_int(args, dtype, static_cast<hipStream_t>(stream)));
}

moe_status moe_act_quantize_int(int32_t rows, int32_t f, int32_t dtype, const void* h, int32_t gated, int32_t activation, int32_t E,
                                const int32_t* offsets, const uint8_t* mask, void* q, float* q_scales, void* stream) {
    if (rows < 0 || f < 1 || (dtype != MOE_F32 && dtype != MOE_BF16) || (gated != 0 && gated != 1)) return MOE_ERR_INVALID_ARG;
    if (offsets != nullptr ? E < 1 : mask != nullptr) return MOE_ERR_INVALID_ARG;
    if (!is_activation(activation)) return MOE_ERR_UNSUPPORTED;
    if (f > kMaxQuantDim || rows > 0x3fffffff || (offsets != nullptr && E > MOE_MAX_E)) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    if (h == nullptr || q == nullptr || q_scales == nullptr || h == q) return MOE_ERR_INVALID_ARG;
    if (!aligned(h, elem_size(dtype)) || !aligned(q, 16) || !aligned(q_scales, 4) || !aligned(offsets, 4)) return MOE_ERR_INVALID_ARG;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    const IntRowArgs args{h, nullptr, nullptr, 0.f, nullptr, nullptr, offsets, mask, static_cast<uint8_t*>(q), q_scales, rows, f, E, activation, gated != 0};
    return from_hip(launch_act_quantize_int(args, dtype, static_cast<hipStream_t>(stream)));
}

size_t moe_int_workspace_bytes(const moe_quant_shape* shape) { return check_product(shape) == MOE_OK ? int_product_workspace(*shape) : 0; }

moe_status moe_int_linear(const moe_quant_shape* shape, const void* a, const float* a_scales, const void* w, const float* w_scales,
                          const float* bias, void* out, void* ws, size_t ws_bytes, void* stream) {
    return product(shape, a, a_scales, nullptr, nullptr, nullptr, w, w_scales, bias, out, ws, ws_bytes, stream, false);
}

moe_status moe_int_expert_linear(const moe_quant_shape* shape, const void* a, const float* a_scales, const int32_t* perm,
                                 const int32_t* offsets, const uint8_t* mask, const void* w, const float* w_scales, const float* bias,
                                 void* out, void* ws, size_t ws_bytes, void* stream) {
    return product(shape, a, a_scales, perm, offsets, mask, w, w_scales, bias, out, ws, ws_bytes, stream, true);
}

}  // extern "C"
