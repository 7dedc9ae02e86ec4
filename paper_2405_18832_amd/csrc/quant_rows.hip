// Quantised rows and weights: the RMS norm in front of a layer with the residual's addition, and the weights' layout.
#include <algorithm>
#include <type_traits>

#include "quant.hpp"

namespace moe {

// ---- moe_norm_quantize ----------------------------------------------------------------------------------------------
// One pass over the data: the row is read once (x, residual), kept in registers as fp32, its squares are summed, and sum, norm and
// codes are written from the registers.  Bound by memory: per value 2 or 4 + 4 bytes in, 1 to 9 out; 16384 x 2048 (bf16, all outputs)
// 57 us = 5.3 TB/s (a copy of 2 GiB: 4.9); 5000 x 1024 11.6 us, of which 3 are a launch.
//
// A lane holds chunks of 8 consecutive values, so that 16 lanes are a block of 128 (its maximum takes four DPP rotations) and a
// wavefront covers 512 values per chunk; chunk c of a row is done by wavefront c % WPR of the row's WPR wavefronts: as many as it has chunks, up
// to four (5000 x 300 with four for the one chunk 13.8 us, with one 11.6; 5000 x 1024 12.3, 11.6).  Rows need no alignment: a chunk
// is one access of 16 bytes wherever it begins (5000 x 300 with an access per value 11.6 us, now 7.0).

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

// Whether v, with the rounding errors that it has from its way through fp32 (a few steps), may lie on the other side of the middle
// between two codes than the number it stands for.  From 2^-6 on codes have 3 bits behind the leading one; below (one value in 10^4 of
// a normal block, more where a few values are much larger than the others) nothing is said.
__device__ __forceinline__ bool next_to_a_border(float v) {
    const uint32_t m = magnitude(v);
    const int32_t past = static_cast<int32_t>(m & 0xfffffu) - 0x80000;
    return m >= 0x3c800000u ? past >= -16 && past <= 16 : m != 0;
}

// The same quotients from 64 bits, for chunks in which one is next to a border: s w is exact there, and divided by the
// block's largest the row's rho goes out.  Each is left as the fp32 number with an odd last bit next to it, which rounds to the code that
// it rounds to itself.  By whole wavefronts.  How many chunks that are depends on the values: 5 % of normal ones, 24 % where one column is
// 1000 times the others, 65 % where one in every block is 100 times the others; in a captured graph 16384 x 2048 then take 62.5, 62.1 and 67.7 us,
// 2048 x 768 6.6, 7.0 and 7.3, one row 3.1, 3.4 and 3.5.
__device__ __forceinline__ void exact_codes(const float (&s)[8], const float* w, int c, int d, float rho, uint32_t most, float (&n)[8]) {
    double u[8], top = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] = static_cast<double>(s[i]);
        if (w != nullptr) u[i] *= static_cast<double>(w[i]);
        if (c + i < d) top = fmax(top, fabs(u[i]));
    }
    auto with = [&](auto control) {
        const uint64_t v = __double_as_longlong(top);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(control)::value, 0xF, 0xF, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), decltype(control)::value, 0xF, 0xF, false);
        top = fmax(top, __longlong_as_double(static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo)));
    };
    with(std::integral_constant<int, 0x128>{});
    with(std::integral_constant<int, 0x124>{});
    with(std::integral_constant<int, 0x122>{});
    with(std::integral_constant<int, 0x121>{});
    const double ratio = fmin(static_cast<double>(kE4m3Max) / top, static_cast<double>(rho) / static_cast<double>(kMinScale));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double v = u[i] * ratio;
        const float f = static_cast<float>(v);
        const double back = static_cast<double>(f);
        uint32_t bits = __float_as_uint(f);
        if (back != v && (bits & 1u) == 0) bits += fabs(v) > fabs(back) ? 1u : ~0u;
        if (c + i < d && most < 0x7f800000u) n[i] = __uint_as_float(bits);
    }
}

constexpr int kNormWaves = 4;               // wavefronts of a block
constexpr int kNormValues = 512;            // values of a wavefront's chunk

struct NormArgs {
    const void *x, *residual;
    const float* weight;
    float eps;
    void *sum_out, *norm_out;
    uint8_t* q;
    float* q_scales;
    int rows, d;
};

// NV: chunks that a wavefront keeps in registers; 0: rows longer than any variant keeps, which are read a second time.
template <typename ST, int WPR, int NV, bool WHOLE>
__global__ __launch_bounds__(kNormWaves * 64) void norm_quantize_kernel(const NormArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % WPR;
    const int row = (blockIdx.y * gridDim.x + blockIdx.x) * (kNormWaves / WPR) + wave / WPR;
    const bool live = row < a.rows;                         // the block meets at a barrier below
    const int d = a.d;
    const size_t at = static_cast<size_t>(live ? row : 0) * d;
    const ST* x = static_cast<const ST*>(a.x) + at;
    const ST* res = a.residual ? static_cast<const ST*>(a.residual) + at : nullptr;
    ST* sum_out = a.sum_out ? static_cast<ST*>(a.sum_out) + at : nullptr;
    ST* norm_out = a.norm_out ? static_cast<ST*>(a.norm_out) + at : nullptr;
    const size_t pitch = quant_pitch(d);
    uint8_t* q = a.q + static_cast<size_t>(live ? row : 0) * pitch;
    float* q_scales = a.q_scales + static_cast<size_t>(live ? row : 0) * (pitch / kQuantBlock);
    const int chunks = (static_cast<int>(pitch) + kNormValues - 1) / kNormValues;
    auto column = [&](int chunk) { return chunk * kNormValues + lane * 8; };
    auto read_sum = [&](int chunk, float (&s)[8]) {
        load8<ST, WHOLE>(x, column(chunk), d, s);
        if (res != nullptr) {
            float r[8];
            load8<ST, WHOLE>(res, column(chunk), d, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = Eight<ST>::round(s[i] + r[i]);
        }
    };

    float kept[NV > 0 ? NV : 1][8];
    float squares = 0.f;
    if (live) {
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (j * WPR + part < chunks) {
                    read_sum(j * WPR + part, kept[j]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) kept[j][i] = 0.f;
                }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float p = 0.f;                              // short chains: the rounding error of a sum grows with its length
#pragma unroll
                for (int i = 0; i < 8; ++i) p = fmaf(kept[j][i], kept[j][i], p);
                squares += p;
            }
        } else {
            for (int c = part; c < chunks; c += WPR) {
                read_sum(c, kept[0]);
                float p = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) p = fmaf(kept[0][i], kept[0][i], p);
                squares += p;
            }
        }
    }
    squares = wave_sum(squares);
    if constexpr (WPR > 1) {
        __shared__ float parts[kNormWaves];
        if (lane == 0) parts[wave] = squares;
        __syncthreads();
        squares = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) squares += parts[wave / WPR * WPR + w];
    }
    if (!live) return;
    const float rho = 1.f / sqrtf(squares / static_cast<float>(d) + a.eps);

    auto finish = [&](int chunk, float (&s)[8]) {
        const int c = column(chunk);
        if (sum_out != nullptr) store8<ST, WHOLE>(sum_out, c, d, s);
        uint32_t most = 0;
        float w[8], n[8];
        if (a.weight != nullptr) load8<float, WHOLE>(a.weight, c, d, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] = s[i] * rho;
            if (a.weight != nullptr) n[i] *= w[i];
            most = max(most, c + i < d ? magnitude(n[i]) : 0u);
        }
        if (norm_out != nullptr) store8<ST, WHOLE>(norm_out, c, d, n);
        most = row16_max(most);
        const float scale = block_scale(most), inv = 1.f / scale;
        bool unsure = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            n[i] = c + i < d ? n[i] * inv : 0.f;            // zeros past the end, also where the scale is NaN
            unsure |= next_to_a_border(n[i]);
        }
        if (__ballot(unsure && most < 0x7f800000u) != 0) exact_codes(s, a.weight != nullptr ? w : nullptr, c, d, rho, most, n);
        if (c < static_cast<int>(pitch)) {
            *reinterpret_cast<uint2*>(q + c) = uint2{pack_e4m3x4(n[0], n[1], n[2], n[3]), pack_e4m3x4(n[4], n[5], n[6], n[7])};
            if ((lane & 15) == 0) q_scales[c / kQuantBlock] = scale;
        }
    };
    if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j * WPR + part < chunks) finish(j * WPR + part, kept[j]);
    } else {
        for (int c = part; c < chunks; c += WPR) {
            read_sum(c, kept[0]);
            finish(c, kept[0]);
        }
    }
}

template <typename ST, bool WHOLE>
static hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
    const int chunks = static_cast<int>((quant_pitch(a.d) + kNormValues - 1) / kNormValues);
    const dim3 block(kNormWaves * 64);
    // a launch counts at most 2^32 - 1 threads in one direction: 2^24 blocks are one too many
    constexpr int kAcross = 1 << 22;
    auto go = [&](auto kernel, int wpr) {
        const int per_block = kNormWaves / wpr, blocks = (a.rows + per_block - 1) / per_block;
        kernel<<<dim3(blocks < kAcross ? blocks : kAcross, (blocks + kAcross - 1) / kAcross), block, 0, stream>>>(a);
    };
    // as many wavefronts per row as it has chunks
    if (chunks == 1) go(norm_quantize_kernel<ST, 1, 1, WHOLE>, 1);
    else if (chunks == 2) go(norm_quantize_kernel<ST, 2, 1, WHOLE>, 2);
    else if (chunks <= kNormWaves) go(norm_quantize_kernel<ST, 4, 1, WHOLE>, 4);
    else if (chunks <= 2 * kNormWaves) go(norm_quantize_kernel<ST, 4, 2, WHOLE>, 4);
    else if (chunks <= 8 * kNormWaves) go(norm_quantize_kernel<ST, 4, 8, WHOLE>, 4);
    else go(norm_quantize_kernel<ST, 4, 0, WHOLE>, 4);
    return hipGetLastError();
}

hipError_t launch_norm_quantize(int rows, int d, int dtype, const void* x, const void* residual, const float* weight, float eps,
                                void* sum_out, void* norm_out, uint8_t* q, float* q_scales, hipStream_t stream) {
    const NormArgs a{x, residual, weight, eps, sum_out, norm_out, q, q_scales, rows, d};
    const bool whole = d % 8 == 0;
    if (dtype == MOE_BF16) return whole ? launch_norm<uint16_t, true>(a, stream) : launch_norm<uint16_t, false>(a, stream);
    return whole ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream);
}

// ---- moe_quantize_weights -------------------------------------------------------------------------------------------
// A block of threads per 128 x 128 block of a matrix.  Thread t holds columns 16 (t % 8) ... of rows t / 8 + 32 i, so that eight lanes read
// whole lines of a row (of one-byte codes; of wider types two and four) and store 16 bytes at the place that the products' loads want
// them (moe.h), eight neighbours 128 bytes.  In between the block's maximum and the codes.  Bound by memory: 32 matrices of 8192 x 2048 read and
// written at 4.8 TB/s (e4m3, 223 us), 4.9 (bf16, 330 us), 5.8 (fp32, 461 us); 64 of 1000 x 1501 at 3.7 to 4.9.
typedef __attribute__((ext_vector_type(4), aligned(1))) uint32_t any_codes16;

template <typename ST>      // float, uint16_t (bf16) or uint8_t (codes)
__global__ __launch_bounds__(256) void quantize_weights_kernel(const ST* __restrict__ src, uint8_t* __restrict__ dst,
                                                               float* __restrict__ scales, int N, int K, int parts) {
    // the row blocks of a matrix may need several of the grid's second direction
    const int kb = blockIdx.x, e = blockIdx.z / parts, nb = (blockIdx.z - e * parts) * gridDim.y + blockIdx.y;
    const int kblocks = gridDim.x, nblocks = quant_blocks(N);
    if (nb >= nblocks) return;
    const int piece = threadIdx.x & 7, r0 = threadIdx.x >> 3;
    const int c0 = kb * kQuantBlock + piece * 16;
    auto row_of = [&](int i) { return nb * kQuantBlock + r0 + 32 * i; };
    auto from = [&](int i) { return src + (static_cast<size_t>(e) * N + min(row_of(i), N - 1)) * K + c0; };
    uint32_t codes[4][4];
    if constexpr (std::is_same_v<ST, uint8_t>) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row_of(i) < N && c0 + 16 <= K) {
                const any_codes16 v = *reinterpret_cast<const any_codes16*>(from(i));
#pragma unroll
                for (int q = 0; q < 4; ++q) codes[i][q] = v[q];
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    codes[i][q] = 0;
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if (row_of(i) < N && c0 + 4 * q + b < K) codes[i][q] |= static_cast<uint32_t>(from(i)[4 * q + b]) << (8 * b);
                }
            }
        }
    } else {
        float v[4][2][8];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (row_of(i) < N && c0 + 8 * h + 8 <= K) {
                    Eight<ST>::load(from(i) + 8 * h, v[i][h]);
                } else {
#pragma unroll
                    for (int b = 0; b < 8; ++b) v[i][h][b] = row_of(i) < N && c0 + 8 * h + b < K ? Storage<ST>::load(from(i) + 8 * h + b) : 0.f;
                }
#pragma unroll
                for (int b = 0; b < 8; ++b) most = max(most, magnitude(v[i][h][b]));
            }
        __shared__ uint32_t all[4];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), o, 64)));
        if ((threadIdx.x & 63) == 0) all[threadIdx.x >> 6] = most;
        __syncthreads();
        most = max(max(all[0], all[1]), max(all[2], all[3]));
        const float scale = block_scale(most);
        const BlockQuotient of(scale);
        if (threadIdx.x == 0) scales[(static_cast<size_t>(e) * nblocks + nb) * kblocks + kb] = scale;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float* u = v[i][q >> 1] + 4 * (q & 1);
                codes[i][q] = pack_e4m3x4(of(u[0]), of(u[1]), of(u[2]), of(u[3]));
                // columns and rows past the end stay zero in a block whose scale is NaN
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (row_of(i) >= N || c0 + 4 * q + b >= K) codes[i][q] &= ~(0xffu << (8 * b));
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 32 * i;
        uint8_t* frag = dst + ((static_cast<size_t>(e) * nblocks * 8 + nb * 8 + (r >> 4)) * kblocks + kb) * kFragBytes;
        *reinterpret_cast<uint4*>(frag + (piece >> 2) * 1024 + ((piece & 3) * 16 + (r & 15)) * 16) =
            uint4{codes[i][0], codes[i][1], codes[i][2], codes[i][3]};
    }
}

hipError_t launch_quantize_weights(int E, int N, int K, int src_dtype, const void* src, uint8_t* dst, float* scales, hipStream_t stream) {
    constexpr int kAcross = 32768;              // blocks of the grid's second and third direction: at most 65535
    static_assert(MOE_MAX_E * (kMaxQuantDim / kQuantBlock / kAcross) <= 65535, "of the third");
    const int nblocks = quant_blocks(N), parts = (nblocks + kAcross - 1) / kAcross;
    const dim3 grid(quant_blocks(K), std::min(nblocks, kAcross), E * parts), block(256);
    auto go = [&](auto* from) { quantize_weights_kernel<<<grid, block, 0, stream>>>(from, dst, scales, N, K, parts); };
    if (src_dtype == MOE_F32) go(static_cast<const float*>(src));
    else if (src_dtype == MOE_BF16) go(static_cast<const uint16_t*>(src));
    else go(static_cast<const uint8_t*>(src));
    return hipGetLastError();
}

}  // namespace moe
