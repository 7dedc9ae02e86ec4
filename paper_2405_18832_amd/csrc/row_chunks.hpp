// Chunks of 8 values of a row, the rows' kernels' unit of access.
#pragma once

#include "quant.hpp"

namespace moe {

// 16 bytes at an address that is a multiple of the element's size only: one access all the same, as the machine takes them
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t any_u32x4;
typedef __attribute__((ext_vector_type(4), aligned(4))) float any_f32x4;

template <typename ST> struct Eight;
template <> struct Eight<uint16_t> {
    static __device__ __forceinline__ void load(const uint16_t* p, float (&v)[8]) {
        const any_u32x4 w = *reinterpret_cast<const any_u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float (&v)[8]) {
        *reinterpret_cast<any_u32x4*>(p) =
            any_u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
    static __device__ __forceinline__ float round(float v) { return bf16_to_f32(f32_to_bf16(v)); }
};
template <> struct Eight<float> {
    static __device__ __forceinline__ void load(const float* p, float (&v)[8]) {
        const any_f32x4 a = *reinterpret_cast<const any_f32x4*>(p), b = *reinterpret_cast<const any_f32x4*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
        *reinterpret_cast<any_f32x4*>(p) = any_f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<any_f32x4*>(p + 4) = any_f32x4{v[4], v[5], v[6], v[7]};
    }
    static __device__ __forceinline__ float round(float v) { return v; }
};

// 8 values from column `c` of a row of d; those past the end are zero.  WHOLE: d is a multiple of 8, no row ends inside a chunk.
template <typename ST, bool WHOLE>
__device__ __forceinline__ void load8(const ST* row, int c, int d, float (&v)[8]) {
    if constexpr (WHOLE) {
        if (c < d) {
            Eight<ST>::load(row + c, v);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    } else {
        if (c + 8 <= d) {
            Eight<ST>::load(row + c, v);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < d ? Storage<ST>::load(row + c + i) : 0.f;
    }
}
template <typename ST, bool WHOLE>
__device__ __forceinline__ void store8(ST* row, int c, int d, const float (&v)[8]) {
    if constexpr (WHOLE) {
        if (c < d) Eight<ST>::store(row + c, v);
    } else {
        if (c + 8 <= d) {
            Eight<ST>::store(row + c, v);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < d) Storage<ST>::store(row + c + i, v[i]);
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

}  // namespace moe
