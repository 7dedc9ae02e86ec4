// C ABI of the 8-bit layers: argument validation on the host, then asynchronous launches on the caller's stream.
#include <cmath>

#include "quant.hpp"

using namespace moe;

namespace {

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
size_t element_bytes(int dtype) { return dtype == MOE_F32 ? 4 : dtype == MOE_BF16 ? 2 : 1; }

moe_status check_matrices(int32_t E, int32_t N, int32_t K) {
    if (E < 1 || N < 1 || K < 1) return MOE_ERR_INVALID_ARG;
    if (E > MOE_MAX_E || N > kMaxQuantDim || K > kMaxQuantDim) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

int out_type(const moe_quant_shape& s) { return s.out_dtype & ~MOE_QUANT_UNIT_SUMS; }

moe_status check_product(const moe_quant_shape* s) {
    if (s == nullptr || s->rows < 0 || s->k < 1) return MOE_ERR_INVALID_ARG;
    const moe_status st = check_matrices(s->E, s->N, s->K);
    if (st != MOE_OK) return st;
    const int out = out_type(*s);
    if (out != MOE_BF16 && out != MOE_E4M3 && s->out_dtype != MOE_F32) return MOE_ERR_INVALID_ARG;      // fp32 outputs have fp32 sums
    if (s->activation != MOE_ACT_NONE && s->activation != MOE_ACT_RELU && s->activation != MOE_ACT_GELU) return MOE_ERR_UNSUPPORTED;
    if (s->rows % s->k != 0) return MOE_ERR_INVALID_ARG;
    if (s->k > MOE_MAX_K) return MOE_ERR_UNSUPPORTED;
    // int32 numbers of rows and of the kernels' units (row tiles of 16 rows at least x 16 columns)
    if (s->rows > 0x3fffffff) return MOE_ERR_UNSUPPORTED;
    const long long tiles = s->rows / 16 + s->E, columns = (static_cast<long long>(s->N) + 15) / 16;
    if (tiles * columns > 0x3fffffffLL) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

moe_status product(const moe_quant_shape* s, const void* a, const float* a_scales, const int32_t* perm, const int32_t* offsets,
                   const uint8_t* mask, const void* w, const float* w_scales, const float* bias, void* out, float* out_scales, void* ws,
                   size_t ws_bytes, void* stream, bool grouped) {
    const moe_status st = check_product(s);
    if (st != MOE_OK) return st;
    if (!grouped && (s->E != 1 || s->k != 1)) return MOE_ERR_INVALID_ARG;
    if (s->rows == 0) return MOE_OK;
    if (a == nullptr || a_scales == nullptr || w == nullptr || w_scales == nullptr || out == nullptr) return MOE_ERR_INVALID_ARG;
    if (grouped && offsets == nullptr) return MOE_ERR_INVALID_ARG;
    const int type = out_type(*s);
    if ((type == MOE_E4M3) != (out_scales != nullptr)) return MOE_ERR_INVALID_ARG;
    if (!aligned(a, 16) || !aligned(w, 16) || !aligned(out, type == MOE_E4M3 ? 16 : element_bytes(type)))
        return MOE_ERR_INVALID_ARG;
    if (!aligned(a_scales, 4) || !aligned(w_scales, 4) || !aligned(bias, 4) || !aligned(out_scales, 4) || !aligned(perm, 4) ||
        !aligned(offsets, 4))
        return MOE_ERR_INVALID_ARG;
    if (ws == nullptr || !aligned(ws, 256) || ws_bytes < quant_product_workspace(*s)) return MOE_ERR_WORKSPACE;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    const QuantArgs args{static_cast<const uint8_t*>(a), a_scales, perm, offsets, mask, static_cast<const uint8_t*>(w), w_scales, bias,
                         out, out_scales, s->rows, s->N, s->K, s->E, perm != nullptr ? s->k : 1, s->activation, type,
                         s->out_dtype != type};
    return launch_quant_product(args, ws, static_cast<hipStream_t>(stream)) == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // namespace

extern "C" {

size_t moe_quant_pitch(int32_t n) { return n < 1 ? 0 : quant_pitch(n); }

size_t moe_quant_weight_bytes(int32_t E, int32_t N, int32_t K) {
    return check_matrices(E, N, K) == MOE_OK ? E * quant_matrix_bytes(N, K) : 0;
}

moe_status moe_quantize_weights(int32_t E, int32_t N, int32_t K, int32_t src_dtype, const void* src, void* dst, float* scales,
                                void* stream) {
    const moe_status st = check_matrices(E, N, K);
    if (st != MOE_OK) return st;
    if (src_dtype != MOE_F32 && src_dtype != MOE_BF16 && src_dtype != MOE_E4M3) return MOE_ERR_INVALID_ARG;
    if (src == nullptr || dst == nullptr || src == dst || (src_dtype != MOE_E4M3 && scales == nullptr)) return MOE_ERR_INVALID_ARG;
    if (!aligned(dst, 16) || !aligned(src, element_bytes(src_dtype)) || !aligned(scales, 4)) return MOE_ERR_INVALID_ARG;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    return launch_quantize_weights(E, N, K, src_dtype, src, static_cast<uint8_t*>(dst), scales, static_cast<hipStream_t>(stream)) ==
                   hipSuccess
               ? MOE_OK
               : MOE_ERR_HIP;
}

moe_status moe_norm_quantize(int32_t rows, int32_t d, int32_t dtype, const void* x, const void* residual, const float* weight, float eps,
                             void* sum_out, void* norm_out, void* q, float* q_scales, void* stream) {
    if (rows < 0 || d < 1 || (dtype != MOE_F32 && dtype != MOE_BF16) || !(eps >= 0.f) || std::isinf(eps)) return MOE_ERR_INVALID_ARG;
    if (d > kMaxQuantDim || rows > 0x3fffffff) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    if (x == nullptr || q == nullptr || q_scales == nullptr) return MOE_ERR_INVALID_ARG;
    const size_t es = element_bytes(dtype);
    if (!aligned(x, es) || !aligned(residual, es) || !aligned(sum_out, es) || !aligned(norm_out, es) || !aligned(weight, 4) ||
        !aligned(q, 16) || !aligned(q_scales, 4))
        return MOE_ERR_INVALID_ARG;
    if (ensure_ready() != hipSuccess) return MOE_ERR_HIP;
    return launch_norm_quantize(rows, d, dtype, x, residual, weight, eps, sum_out, norm_out, static_cast<uint8_t*>(q), q_scales,
                                static_cast<hipStream_t>(stream)) == hipSuccess
               ? MOE_OK
               : MOE_ERR_HIP;
}

size_t moe_quant_workspace_bytes(const moe_quant_shape* shape) {
    return check_product(shape) == MOE_OK ? quant_product_workspace(*shape) : 0;
}

moe_status moe_quant_linear(const moe_quant_shape* shape, const void* a, const float* a_scales, const void* w, const float* w_scales,
                            const float* bias, void* out, float* out_scales, void* ws, size_t ws_bytes, void* stream) {
    return product(shape, a, a_scales, nullptr, nullptr, nullptr, w, w_scales, bias, out, out_scales, ws, ws_bytes, stream, false);
}

moe_status moe_quant_expert_linear(const moe_quant_shape* shape, const void* a, const float* a_scales, const int32_t* perm,
                                   const int32_t* offsets, const uint8_t* mask, const void* w, const float* w_scales, const float* bias,
                                   void* out, float* out_scales, void* ws, size_t ws_bytes, void* stream) {
    return product(shape, a, a_scales, perm, offsets, mask, w, w_scales, bias, out, out_scales, ws, ws_bytes, stream, true);
}

}  // extern "C"
