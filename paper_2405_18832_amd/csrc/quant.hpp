// Shared parts of the 8-bit layers: the e4m3 conversions, the layout of quantised rows and packed weights, launches.
#pragma once

#include "common.hpp"

namespace moe {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(8))) int32_t i32x8;

constexpr int kQuantBlock = MOE_QUANT_BLOCK;        // values per scale, in both directions for weights
constexpr int kFragBytes = 16 * kQuantBlock;        // a packed fragment: 16 rows of one block of columns
constexpr int kMaxQuantDim = 1 << 24;               // N, K, d

inline __host__ __device__ int quant_blocks(int n) { return (n + kQuantBlock - 1) / kQuantBlock; }
inline __host__ __device__ size_t quant_pitch(int n) { return static_cast<size_t>(quant_blocks(n)) * kQuantBlock; }
inline __host__ __device__ size_t quant_matrix_bytes(int N, int K) { return quant_pitch(N) * quant_pitch(K); }

#ifdef __HIPCC__
constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 1.17549435e-38f;        // 2^-126: blocks of zeros have a scale that can be divided by

// Four values as e4m3 codes, to nearest, ties to even; NaN becomes the NaN code.  (gfx950 converts to the OCP format.)
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true));
}

// Magnitudes are compared as integers: a NaN is larger than infinity, infinity larger than any number, so that neither is lost in a
// block's maximum (fmaxf would drop a NaN).
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale of a block from its largest magnitude; NaN if that is NaN or infinity.
__device__ __forceinline__ float block_scale(uint32_t most) {
    if (most >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    return fmaxf(__uint_as_float(most) / kE4m3Max, kMinScale);
}

// v / scale of a block's values as fp32 division rounds it, which a product with the reciprocal does not (of the middles between two codes it
// puts one in eight on a side): the product, corrected by its remainder, which is exact.  Tiny scales are taken up first, so that no remainder
// falls below fp32's range.  Three operations more per value than the product: 16384 x 8192 x 2048 with GeLU 554 -> 579 us.
struct BlockQuotient {
    float up, by, inv;
    __device__ __forceinline__ explicit BlockQuotient(float scale)
        : up(scale < 0x1p-64f ? 0x1p64f : 1.f), by(scale * up), inv(1.f / by) {}
    __device__ __forceinline__ float operator()(float v) const {
        v *= up;
        const float q = v * inv;
        return fmaf(fmaf(-q, by, v), inv, q);
    }
};

// Maximum over the 16 lanes of a row of lanes, in every one of them (DPP rotations within the row).
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x128, 0xF, 0xF, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x124, 0xF, 0xF, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x122, 0xF, 0xF, false)));
    v = max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x121, 0xF, 0xF, false)));
    return v;
}
#endif

// What a product is launched with: the shape and the caller's pointers.
struct QuantArgs {
    const uint8_t* a;
    const float* a_scales;
    const int32_t* perm;        // NULL: row p of the product is row p of `a`
    const int32_t* offsets;     // NULL: one matrix, all rows
    const uint8_t* mask;
    const uint8_t* w;
    const float* w_scales;
    const float* bias;
    void* out;
    float* out_scales;
    int rows, N, K, E, k, act, out_dtype;
    bool unit_sums;             // blocks' sums by the matrix units for 8-bit operands
    bool once = false;          // streamed weights are not kept in the caches
};

// csrc/quant_rows.hip
hipError_t launch_quantize_weights(int E, int N, int K, int src_dtype, const void* src, uint8_t* dst, float* scales, hipStream_t stream);
hipError_t launch_norm_quantize(int rows, int d, int dtype, const void* x, const void* residual, const float* weight, float eps,
                                void* sum_out, void* norm_out, uint8_t* q, float* q_scales, hipStream_t stream);
// csrc/quant_linear.hip
size_t quant_product_workspace(const moe_quant_shape& s);
hipError_t launch_quant_product(const QuantArgs& a, void* ws, hipStream_t stream);

}  // namespace moe
