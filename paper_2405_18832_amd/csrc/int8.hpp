// Shared parts of the int8 layers: rounding to codes, launches.  Rows of codes have the pitch of quant.hpp's rows and one scale each, packed
// weights its layout and one scale per output channel.
#pragma once

#include "quant.hpp"

namespace moe {

static_assert(128ll * 128 * MOE_INT_MAX_K <= 0x7fffffffll, "sums of products of codes down to -128 stay within int32");

#ifdef __HIPCC__
constexpr float kIntMax = 127.f;

// z / (1 + exp(-z)), by the hardware's exponential and reciprocal (a unit of the last place each, so 2 u, u = 2^-24): the constant is 0.22 u off, the argument's product u,
// so the result (1.25 |z| + 6) u of itself.
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f)); }

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = row16_max(v);
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return max(max(a, b), max(c, d));
}
#endif

struct IntRowArgs {
    const void *x, *residual;           // norm: rows and residual; activation: rows [f] or [2 f]
    const float* weight;
    float eps;
    void *sum_out, *norm_out;
    const int32_t* offsets;             // activation: rows of experts with mask[e] == 0 are left out
    const uint8_t* mask;
    uint8_t* q;
    float* q_scales;
    int rows, d, E, act;
    bool gated;
};

// csrc/int_rows.hip
hipError_t launch_norm_quantize_int(const IntRowArgs& a, int dtype, hipStream_t stream);
hipError_t launch_quantize_weights_int(int E, int N, int K, int src_dtype, const void* src, uint8_t* dst, float* scales, hipStream_t stream);
// csrc/int_act.hip
hipError_t launch_act_quantize_int(const IntRowArgs& a, int dtype, hipStream_t stream);
// csrc/int_linear.hip
size_t int_product_workspace(const moe_quant_shape& s);
hipError_t launch_int_product(const QuantArgs& a, void* ws, hipStream_t stream);
// csrc/score_route.hip
hipError_t launch_gate_logits(const moe_shape& s, const void* x, const void* w_gate, const float* bias, float* logits, hipStream_t stream);
struct ScoreArgs {
    const void* logits;
    bool bf16;                          // logits' type: bf16, else fp32
    const float* balance;
    int32_t* idx;
    float* weight;
    int32_t *counts, *offsets;
    uint8_t* hot_mask;
    int32_t* hist;                      // workspace [ceil(T / 16) + 1][E]
    int T, E, k, H;
    bool sigmoid, renormalize;
    int groups, kept, top;
    float scale;
};
hipError_t launch_route_logits(const ScoreArgs& a, hipStream_t stream);

}  // namespace moe
