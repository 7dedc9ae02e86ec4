// Rows as int8.  A row's codes are the whole numbers next to 127 v / max |v|, of its values v as real numbers (ties to even): v is computed in fp32, and where
// the quotient lies so close to the middle between two codes that fp32's errors could have moved it across, again in 64 bits.  The row's factor
// cancels in the quotient, so that of the norm only s w enters.  The quotient's divisor is then the largest magnitude in 64 bits: of the few values
// whose fp32 magnitude is next to the largest one.
#pragma once

#include <algorithm>
#include <cfloat>
#include <type_traits>
#include <utility>

#include "int8.hpp"
#include "row_chunks.hpp"

namespace moe {

namespace {

constexpr int kChunk = 512;             // values of a wavefront's chunk, 8 per lane

// f(0), ..., f(N - 1) with the numbers known when compiled: a loop that the compiler leaves one would put what it indexes into memory.
template <typename F, int... I>
__device__ __forceinline__ void unrolled(F f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
    unrolled(f, std::make_integer_sequence<int, N>{});
}

// Relative errors that fp32 quotients are allowed: products of two or three roundings, twice over.
constexpr float kProductSlack = 0x1p-21f;

struct Codes8 {
    uint32_t lo, hi, unsure;            // codes 0 ... 3, 4 ... 7; a bit for each that 64 bits have to decide
};
// Whole numbers next to v * ratio, ties to even: the sum with 1.5 2^23 has them in its low bits.  slack(i): relative error of the product i.
template <typename Slack>
__device__ __forceinline__ Codes8 codes8(const float (&v)[8], float ratio, Slack slack) {
    constexpr float kShift = 12582912.f;
    uint32_t r[8];
    float off[8], most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = v[i] * ratio, s = t + kShift;
        r[i] = __float_as_uint(s);
        off[i] = fmaf(fabsf(t), slack(i), fabsf(t - (s - kShift)));
        most = fmaxf(most, off[i]);
    }
    Codes8 c;
    c.lo = __builtin_amdgcn_perm(__builtin_amdgcn_perm(r[3], r[2], 0x0c0c0400), __builtin_amdgcn_perm(r[1], r[0], 0x0c0c0400), 0x05040100);
    c.hi = __builtin_amdgcn_perm(__builtin_amdgcn_perm(r[7], r[6], 0x0c0c0400), __builtin_amdgcn_perm(r[5], r[4], 0x0c0c0400), 0x05040100);
    c.unsure = 0;
    if (most > 0.5f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c.unsure |= off[i] > 0.5f ? 1u << i : 0u;
    }
    return c;
}
// What the wavefronts of a block tell each other; a row's are neighbours.
template <int WAVES>
struct RowShared {
    float squares[WAVES], slack[WAVES];
    uint32_t most[WAVES];
    double top[WAVES];
};

__device__ __forceinline__ float wave_total(float v) {
    auto add = [&](auto control) {
        v += __uint_as_float(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), decltype(control)::value, 0xF, 0xF, false));
    };
    add(std::integral_constant<int, 0x128>{});
    add(std::integral_constant<int, 0x124>{});
    add(std::integral_constant<int, 0x122>{});
    add(std::integral_constant<int, 0x121>{});
    auto lane = [&](int l) { return __uint_as_float(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(v)), l)); };
    return (lane(0) + lane(16)) + (lane(32) + lane(48));
}
// Largest of the lanes' numbers, which are not negative: most often one lane has one that is not zero.
__device__ __forceinline__ double wave_top(double v) {
    uint64_t have = __ballot(v > 0.0);
    double top = 0.0;
    while (have != 0) {
        const int l = __builtin_ctzll(have);
        have &= have - 1;
        const uint64_t bits = __double_as_longlong(v);
        const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(bits), l));
        const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(bits >> 32), l));
        top = fmax(top, __longlong_as_double(static_cast<int64_t>(hi << 32 | lo)));
    }
    return top;
}

// A row's quotients: 127 v / top, or, where the scale is the smallest one (the largest value is below 127 * 2^-126), v * factor * 2^126.
struct Quotient {
    double top, factor;
    bool tiny;
    __device__ __forceinline__ double operator()(double v) const { return tiny ? v * factor * 0x1p+126 : v * 127.0 / top; }
};

// From a row's fp32 values to its codes and scale; called by all wavefronts of a block, the row's WPR among them.
//   each(f): f(chunk, values [8], slack) for the wavefront's chunks; slack: twice the relative error of the values, negative where some of the lane's are left out,
//   which are zero then (all of these are computed in 64 bits).
//   exact(chunk, i): the value in 64 bits.   most: bits of the row's largest magnitude.   slack: the row's largest, below 2^-17 where quotients by that magnitude, and
//   the scale, may be taken from it; 2^-17 at least where values are left out.   factor: what the values are multiplied by for the scale.   bad: the row is none.
// Codes are written from fp32, a quotient's error being that of its value and that of the largest, half of either slack; those in doubt, most often none or a few of a
// row, are written again, for which the row's largest value in 64 bits is needed first.  Where fp32's is not exact enough all are, as quotients by that.
template <int WPR, int WAVES, typename Each, typename Exact>
__device__ __forceinline__ void write_row(RowShared<WAVES>& shared, bool live, bool bad, uint32_t most, float slack, double factor, int d, uint8_t* q,
                                          float* q_scale, Each each, Exact exact) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w0 = wave - wave % WPR;
    const int pitch = static_cast<int>(quant_pitch(d));
    const float largest = __uint_as_float(most);
    const double largest_out = static_cast<double>(largest) * factor;
    // values too large or too small for fp32's quotients, or a scale that might be the smallest one: all of them from 64 bits
    const bool extreme = !(largest >= 0x1p-100f && largest <= 0x1p+100f) || !(largest_out >= 0x1p-110 && largest_out <= 0x1p+110);
    const float ratio = extreme ? 0.f : kIntMax / largest;
    const bool loose = !(slack < 0x1p-17f);
    bool doubt = false;
    if (live) {
        each([&](int chunk, const float (&v)[8], float own) __attribute__((always_inline)) {
            const int c = chunk * kChunk + lane * 8;
            const Codes8 codes = codes8(v, ratio, [&](int) { return fmaf(0.5f, own, 0.5f * slack); });
            doubt |= codes.unsure != 0 || own < 0.f;
            if (c < pitch) *reinterpret_cast<uint2*>(q + c) = bad || extreme ? uint2{0, 0} : uint2{codes.lo, codes.hi};
        });
    }
    doubt = live && !bad && (doubt || extreme || loose);
    bool any = __ballot(doubt) != 0;
    if constexpr (WPR > 1) any = __syncthreads_or(any) != 0;
    double top = largest;
    if (any) {                                              // the same for the block, or the wavefront where rows are one wavefront's
        top = 0.0;
        if (live && !bad) {
            each([&](int chunk, const float (&v)[8], float own) __attribute__((always_inline)) {
                const int c = chunk * kChunk + lane * 8;
                const float least = extreme || own < 0.f ? 0.f : largest * (1.f - (own + slack + 0x1p-16f));
                uint32_t next = 0;                          // values that may be the largest
#pragma unroll
                for (int i = 0; i < 8; ++i) next |= fabsf(v[i]) >= least ? 1u << i : 0u;
                next &= c + 8 <= d ? 0xffu : c < d ? 0xffu >> (c + 8 - d) : 0u;
                while (next != 0) {
                    const int i = __builtin_ctz(next);
                    next &= next - 1;
                    top = fmax(top, fabs(exact(chunk, i)));
                }
            });
        }
        top = wave_top(top);
        if constexpr (WPR > 1) {
            if (lane == 0) shared.top[wave] = top;
            __syncthreads();
            top = 0.0;
#pragma unroll
            for (int w = 0; w < WPR; ++w) top = fmax(top, shared.top[w0 + w]);
        }
        if (live) {
            bad = bad || !(top * factor <= static_cast<double>(FLT_MAX));
            const Quotient quotient{top, factor, top * factor < 127.0 * 0x1p-126};
            const bool again = loose && !extreme;
            const float by = again ? kIntMax / static_cast<float>(top) : ratio, divisor = again ? 0x1p-22f : 0.5f * slack;
            each([&](int chunk, const float (&v)[8], float own) __attribute__((always_inline)) {
                const int c = chunk * kChunk + lane * 8;
                const Codes8 codes = codes8(v, by, [&](int) { return fmaf(0.5f, own, divisor); });
                if (again && c < pitch) *reinterpret_cast<uint2*>(q + c) = bad ? uint2{0, 0} : uint2{codes.lo, codes.hi};
                uint32_t unsure = extreme || own < 0.f || bad ? 0xffu : codes.unsure;
                while (unsure != 0) {
                    const int i = __builtin_ctz(unsure);
                    unsure &= unsure - 1;
                    if (c + i < d) q[c + i] = bad ? 0 : static_cast<uint8_t>(static_cast<int>(rint(quotient(exact(chunk, i)))));
                }
            });
        }
    }
    if (live && wave == w0 && lane == 0) {
        const double out = top * factor;
        *q_scale = bad ? __uint_as_float(0x7fc00000u) : out < 127.0 * 0x1p-126 ? kMinScale : static_cast<float>(out) / kIntMax;
    }
}

// Blocks of WAVES wavefronts, WPR for each row.
template <int WPR, int WAVES, typename Kernel>
void launch_rows(Kernel kernel, const IntRowArgs& a, hipStream_t stream) {
    // a launch counts at most 2^32 - 1 threads in one direction
    constexpr int kAcross = 1 << 21, per_block = WAVES / WPR;
    const int blocks = (a.rows + per_block - 1) / per_block;
    kernel<<<dim3(std::min(blocks, kAcross), (blocks + kAcross - 1) / kAcross), dim3(WAVES * 64), 0, stream>>>(a);
}

// go(WPR, WAVES, NV): as many wavefronts per row as keep busy; where there are rows enough for all CUs, longer rows are left to fewer (GB/s, gated SiLU in
// bf16, one wavefront per row, four with a chunk each, four chunks each, sixteen: 20000 x 700 2500, 1660, -, -; 20011 x 2048 4100, 4700, -, -; 8000 x 4096 -, -,
// 4900, 3100; 8000 x 8192 -, -, 4500, 3900).
constexpr int kFewRows = 1024;
template <int WPR, int WAVES, int NV, typename Go>
void row_variant(Go go) {
    go(std::integral_constant<int, WPR>{}, std::integral_constant<int, WAVES>{}, std::integral_constant<int, NV>{});
}
template <typename Go>
void with_row_variant(const IntRowArgs& a, Go go) {
    const int chunks = (a.d + kChunk - 1) / kChunk;
    const bool many = a.rows >= kFewRows;
    if (chunks <= 2 && many) row_variant<1, 4, 2>(go);
    else if (chunks <= 4) row_variant<4, 4, 1>(go);
    else if (chunks <= 8 && many) row_variant<4, 4, 2>(go);
    else if (chunks <= 16 && many) row_variant<4, 4, 4>(go);
    else if (chunks <= 16) row_variant<16, 16, 1>(go);
    else if (chunks <= 32 && many) row_variant<8, 8, 4>(go);
    else if (chunks <= 64) row_variant<16, 16, 4>(go);
    else row_variant<16, 16, 0>(go);
}

}  // namespace

}  // namespace moe
