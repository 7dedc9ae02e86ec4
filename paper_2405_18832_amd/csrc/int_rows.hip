// Rows and weights as int8: the norm in front of a layer, the activation between its products, the weights' layout.
//
// A row's codes are the whole numbers next to 127 v / max |v|, of its values v as real numbers (ties to even): v is computed in fp32, and where the
// quotient lies so close to the middle between two codes that fp32's errors could have moved it across, again in 64 bits.  The row's factor
// cancels in the quotient, so that of the norm only s w enters.  The quotient's divisor is the largest magnitude in 64 bits: of the few values
// whose fp32 magnitude is next to the largest one.
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
__device__ __forceinline__ void put_code(Codes8& c, int i, double t) {
    const uint32_t code = static_cast<uint32_t>(static_cast<int>(rint(t))) & 0xffu, shift = 8 * (i & 3), keep = ~(0xffu << shift);
    if (i < 4) c.lo = (c.lo & keep) | code << shift;
    else c.hi = (c.hi & keep) | code << shift;
}
__device__ __forceinline__ float pick(const float (&v)[8], int i) {
    float r = v[0];
#pragma unroll
    for (int n = 1; n < 8; ++n) r = i == n ? v[n] : r;
    return r;
}

// What the wavefronts of a block tell each other; a row's are neighbours.
template <int WAVES>
struct RowShared {
    float squares[WAVES];
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

// ---- moe_norm_quantize_int -------------------------------------------------------------------------------------------
// NV: chunks that a wavefront keeps in registers; 0: rows longer than any variant keeps, which are read again.
template <typename ST, int WPR, int WAVES, int NV, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64) void norm_int_kernel(const IntRowArgs a) {
    __shared__ RowShared<WAVES> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % WPR, w0 = wave - part;
    const int row = (blockIdx.y * gridDim.x + blockIdx.x) * (WAVES / WPR) + wave / WPR;
    const bool live = row < a.rows;                         // the block meets at barriers below
    const int d = a.d;
    const size_t at = static_cast<size_t>(live ? row : 0) * d;
    const ST* x = static_cast<const ST*>(a.x) + at;
    const ST* res = a.residual ? static_cast<const ST*>(a.residual) + at : nullptr;
    const size_t pitch = quant_pitch(d);
    const int chunks = (d + kChunk - 1) / kChunk;
    auto column = [&](int chunk) { return chunk * kChunk + lane * 8; };
    auto read_sum = [&](int chunk, float (&s)[8]) {
        load8<ST, WHOLE>(x, column(chunk), d, s);
        if (res != nullptr) {
            float r[8];
            load8<ST, WHOLE>(res, column(chunk), d, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = Eight<ST>::round(s[i] + r[i]);
        }
    };
    auto times_weight = [&](int chunk, const float (&s)[8], float (&w)[8], float (&u)[8]) {
        if (a.weight != nullptr) load8<float, WHOLE>(a.weight, column(chunk), d, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = a.weight != nullptr ? s[i] * w[i] : s[i];
    };

    float kept[NV > 0 ? NV : 1][8];
    auto each = [&](auto f) __attribute__((always_inline)) {       // f(chunk, its sums)
        if constexpr (NV > 0) {
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) f(j * WPR + part, kept[j]);
            });
        } else {
            for (int c = part; c < chunks; c += WPR) {
                read_sum(c, kept[0]);
                f(c, kept[0]);
            }
        }
    };
    float squares = 0.f;
    uint32_t most = 0;
    if (live) {
        if constexpr (NV > 0) {                             // all loads first
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) read_sum(j * WPR + part, kept[j]);
            });
        }
        each([&](int chunk, const float (&s)[8]) __attribute__((always_inline)) {
            float w[8], u[8], p = 0.f;                      // short chains: the rounding error of a sum grows with its length
            times_weight(chunk, s, w, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p = fmaf(s[i], s[i], p);
                most = max(most, magnitude(u[i]));
            }
            squares += p;
        });
    }
    squares = wave_total(squares);
    most = wave_max(most);
    if constexpr (WPR > 1) {
        if (lane == 0) {
            shared.squares[wave] = squares;
            shared.most[wave] = most;
        }
        __syncthreads();
        squares = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) {
            squares += shared.squares[w0 + w];
            most = max(most, shared.most[w0 + w]);
        }
    }
    double rho = 1.f / sqrtf(squares / static_cast<float>(d) + a.eps);
    // Rows whose squares fp32 does not hold are summed again, in 64 bits.
    auto beyond = [&](float sum) { return !(sum <= 0x1p+120f) || (sum < 0x1p-80f && a.eps < 0x1p-60f); };
    const bool far = live && beyond(squares);
    bool any_far = far;
    if constexpr (WPR < WAVES) {                            // the block's other rows: all meet at the barrier below
#pragma unroll
        for (int r = 0; r < WAVES / WPR; ++r) {
            float sum = 0.f;
            if constexpr (WPR > 1) {
#pragma unroll
                for (int w = 0; w < WPR; ++w) sum += shared.squares[r * WPR + w];
                any_far |= beyond(sum);
            }
        }
    }
    if (any_far) {
        double sum = 0.0;
        if (live) {
            each([&](int chunk, const float (&s)[8]) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += static_cast<double>(s[i]) * static_cast<double>(s[i]);
            });
        }
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        if constexpr (WPR > 1) {
            if (lane == 0) shared.top[wave] = sum;
            __syncthreads();
            sum = 0.0;
#pragma unroll
            for (int w = 0; w < WPR; ++w) sum += shared.top[w0 + w];
            __syncthreads();                                // `top` is written again below
        }
        if (far) rho = 1.0 / sqrt(sum / static_cast<double>(d) + static_cast<double>(a.eps));
    }
    const float largest = __uint_as_float(most);
    // Products too large or too small for their fp32 quotients: every value from 64 bits.  (A product may pass fp32's range and the norm be
    // well within it.)
    const bool extreme = !(largest >= 0x1p-100f && largest <= 0x1p+100f);
    double top = 0.0;
    bool bad = false;
    if (live) {
        each([&](int chunk, const float (&s)[8]) __attribute__((always_inline)) {
            float w[8], u[8];
            times_weight(chunk, s, w, u);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (extreme || fabsf(u[i]) >= largest * (1.f - 0x1p-22f)) {
                    const double v = a.weight != nullptr ? static_cast<double>(s[i]) * static_cast<double>(w[i]) : static_cast<double>(s[i]);
                    bad |= !(fabs(v) < __builtin_huge_val());
                    top = fmax(top, fabs(v));
                }
        });
    }
    top = wave_top(top);
    bad = __ballot(bad) != 0;
    if constexpr (WPR > 1) {
        if (lane == 0) shared.top[wave] = bad ? __builtin_huge_val() : top;
        __syncthreads();
        top = 0.0;
#pragma unroll
        for (int w = 0; w < WPR; ++w) top = fmax(top, shared.top[w0 + w]);
    } else if (bad) {
        top = __builtin_huge_val();
    }
    if (!live) return;
    const double largest_norm = top * rho;
    bad = !(largest_norm <= static_cast<double>(FLT_MAX)) || !(rho < __builtin_huge_val());
    const bool tiny = largest_norm < 127.0 * 0x1p-126;
    const Quotient quotient{top, rho, tiny};
    const float ratio = extreme ? 0.f : kIntMax / static_cast<float>(top);
    const float scale = bad ? __uint_as_float(0x7fc00000u) : tiny ? kMinScale : static_cast<float>(largest_norm) / kIntMax;
    uint8_t* q = a.q + row * pitch;
    each([&](int chunk, const float (&s)[8]) __attribute__((always_inline)) {
        const int c = column(chunk);
        float w[8], u[8];
        times_weight(chunk, s, w, u);
        if (a.sum_out != nullptr) store8<ST, WHOLE>(static_cast<ST*>(a.sum_out) + at, c, d, s);
        if (a.norm_out != nullptr) {
            float n[8];
            const float by = static_cast<float>(rho);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] = a.weight != nullptr ? s[i] * by * w[i] : s[i] * by;
                if (far) n[i] = static_cast<float>(static_cast<double>(s[i]) * rho * (a.weight != nullptr ? static_cast<double>(w[i]) : 1.0));
            }
            store8<ST, WHOLE>(static_cast<ST*>(a.norm_out) + at, c, d, n);
        }
        Codes8 codes = codes8(u, ratio, [](int) { return kProductSlack; });
        if (extreme || tiny) codes.unsure = 0xffu;
        while (codes.unsure != 0) {
            const int i = __builtin_ctz(codes.unsure);
            codes.unsure &= codes.unsure - 1;
            const double sv = pick(s, i), wv = a.weight != nullptr ? pick(w, i) : 1.f;
            put_code(codes, i, c + i < d && !bad ? quotient(sv * wv) : 0.0);
        }
        if (bad) codes.lo = codes.hi = 0;
        if (c < static_cast<int>(pitch)) *reinterpret_cast<uint2*>(q + c) = uint2{codes.lo, codes.hi};
    });
    if (part == 0 && lane == 0) a.q_scales[row] = scale;
}

// ---- moe_act_quantize_int --------------------------------------------------------------------------------------------
template <int ACT>
__device__ __forceinline__ float act_value(float g) {
    if (ACT == MOE_ACT_RELU) return g < 0.f ? 0.f : g;      // NaN stays
    if (ACT == MOE_ACT_GELU) return gelu_exp(g);
    if (ACT == MOE_ACT_SILU) return silu(g);
    return g;
}
template <int ACT>
__device__ __forceinline__ double act_exact(double g) {
    if (ACT == MOE_ACT_RELU) return g < 0.0 ? 0.0 : g;
    if (ACT == MOE_ACT_GELU) return 0.5 * g * erfc(g * -0.70710678118654752440);
    if (ACT == MOE_ACT_SILU) return g / (1.0 + exp(-g));
    return g;
}
// Relative error of act_value * u * ratio.  GeLU: 8.4e-7 down to -4; below, its argument z^2 / 2 log2 e is |z| times that of SiLU's.
template <int ACT>
__device__ __forceinline__ float act_slack(float g) {
    if (ACT == MOE_ACT_GELU) return fmaf(g * g, 0x1p-22f, 0x1p-18f);
    if (ACT == MOE_ACT_SILU) return fmaf(fabsf(g), 0x1p-22f, 0x1p-20f);
    return kProductSlack;
}

// Where act_value has nothing left of a number that a large second factor could make the row's largest again.
template <int ACT>
__device__ __forceinline__ bool vanishing(float g) {
    return ACT == MOE_ACT_GELU ? g < -12.f : ACT == MOE_ACT_SILU ? g < -80.f : false;
}

template <typename ST, int ACT, bool GATED, int WPR, int WAVES, int NV, bool WHOLE>
__global__ __launch_bounds__(WAVES * 64) void act_int_kernel(const IntRowArgs a) {
    __shared__ RowShared<WAVES> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % WPR, w0 = wave - part;
    const int row = (blockIdx.y * gridDim.x + blockIdx.x) * (WAVES / WPR) + wave / WPR;
    bool live = row < a.rows;                               // the block meets at barriers below
    if (a.offsets != nullptr) {                             // the expert whose row this is: as many end at or before it as precede that
        int e = 0;
        for (int e0 = 0; e0 < a.E; e0 += 64) e += __popcll(__ballot(e0 + lane < a.E && a.offsets[min(e0 + lane, a.E - 1) + 1] <= row));
        live = live && e < a.E && a.offsets[min(e, a.E - 1)] <= row && (a.mask == nullptr || a.mask[min(e, a.E - 1)] != 0);
    }
    const int d = a.d;
    const ST* g_row = static_cast<const ST*>(a.x) + static_cast<size_t>(live ? row : 0) * (GATED ? 2 : 1) * d;
    const ST* u_row = g_row + d;
    const size_t pitch = quant_pitch(d);
    const int chunks = (d + kChunk - 1) / kChunk;
    auto column = [&](int chunk) { return chunk * kChunk + lane * 8; };
    struct Chunk {
        float g[8], u[GATED ? 8 : 1];
    };
    auto read = [&](int chunk, Chunk& k) {
        load8<ST, WHOLE>(g_row, column(chunk), d, k.g);
        if constexpr (GATED) load8<ST, WHOLE>(u_row, column(chunk), d, k.u);
    };
    auto value = [&](const Chunk& k, int i) __attribute__((always_inline)) {
        const float v = act_value<ACT>(k.g[i]);
        if constexpr (GATED) return v * k.u[i];
        return v;
    };
    auto exact = [&](const Chunk& k, int i) __attribute__((always_inline)) {      // i: any, or known when compiled
        const double v = act_exact<ACT>(static_cast<double>(pick(k.g, i)));
        if constexpr (GATED) return v * static_cast<double>(pick(k.u, i));
        return v;
    };
    Chunk kept[NV > 0 ? NV : 1];
    auto each = [&](auto f) __attribute__((always_inline)) {
        if constexpr (NV > 0) {
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) f(j * WPR + part, kept[j]);
            });
        } else {
            for (int c = part; c < chunks; c += WPR) {
                read(c, kept[0]);
                f(c, kept[0]);
            }
        }
    };
    uint32_t most = 0;
    if (live) {
        if constexpr (NV > 0) {
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) read(j * WPR + part, kept[j]);
            });
        }
        each([&](int chunk, const Chunk& k) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, magnitude(value(k, i)));
        });
    }
    most = wave_max(most);
    if constexpr (WPR > 1) {
        if (lane == 0) shared.most[wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WPR; ++w) most = max(most, shared.most[w0 + w]);
    }
    const float largest = __uint_as_float(most);
    const bool bad = most >= 0x7f800000u, extreme = !(largest >= 0x1p-100f);
    double top = 0.0;
    if (live && !bad) {
        each([&](int chunk, const Chunk& k) __attribute__((always_inline)) {
            uint32_t next = 0;                              // values that may be the largest
#pragma unroll
            for (int i = 0; i < 8; ++i)
                next |= extreme || (GATED && vanishing<ACT>(k.g[i])) ||
                                fabsf(value(k, i)) >= largest * (1.f - fmaf(4.f, act_slack<ACT>(k.g[i]), 0x1p-17f))
                            ? 1u << i : 0u;
            while (next != 0) {
                const int i = __builtin_ctz(next);
                next &= next - 1;
                top = fmax(top, fabs(exact(k, i)));
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
    if (!live) return;
    const bool tiny = top < 127.0 * 0x1p-126;
    const Quotient quotient{top, 1.0, tiny};
    const float ratio = extreme ? 0.f : kIntMax / static_cast<float>(top);
    const float scale = bad ? __uint_as_float(0x7fc00000u) : tiny ? kMinScale : static_cast<float>(top) / kIntMax;
    uint8_t* q = a.q + row * pitch;
    each([&](int chunk, const Chunk& k) __attribute__((always_inline)) {
        const int c = column(chunk);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = value(k, i);
        Codes8 codes = codes8(v, ratio, [&](int i) { return act_slack<ACT>(k.g[i]); });
        if (GATED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) codes.unsure |= vanishing<ACT>(k.g[i]) ? 1u << i : 0u;
        }
        if (extreme) codes.unsure = 0xffu;
        if (bad) codes = Codes8{0, 0, 0};
        while (codes.unsure != 0) {
            const int i = __builtin_ctz(codes.unsure);
            codes.unsure &= codes.unsure - 1;
            put_code(codes, i, c + i < d ? quotient(exact(k, i)) : 0.0);
        }
        if (c < static_cast<int>(pitch)) *reinterpret_cast<uint2*>(q + c) = uint2{codes.lo, codes.hi};
    });
    if (part == 0 && lane == 0) a.q_scales[row] = scale;
}

// Blocks of WAVES wavefronts, WPR for each row.
template <int WPR, int WAVES, typename Kernel>
void launch_rows(Kernel kernel, const IntRowArgs& a, hipStream_t stream) {
    // a launch counts at most 2^32 - 1 threads in one direction
    constexpr int kAcross = 1 << 21, per_block = WAVES / WPR;
    const int blocks = (a.rows + per_block - 1) / per_block;
    kernel<<<dim3(std::min(blocks, kAcross), (blocks + kAcross - 1) / kAcross), dim3(WAVES * 64), 0, stream>>>(a);
}

template <typename ST, bool WHOLE>
hipError_t launch_norm(const IntRowArgs& a, hipStream_t stream) {
    const int chunks = (a.d + kChunk - 1) / kChunk;
    if (chunks == 1) launch_rows<1, 4>(norm_int_kernel<ST, 1, 4, 1, WHOLE>, a, stream);
    else if (chunks == 2) launch_rows<2, 4>(norm_int_kernel<ST, 2, 4, 1, WHOLE>, a, stream);
    else if (chunks <= 4) launch_rows<4, 4>(norm_int_kernel<ST, 4, 4, 1, WHOLE>, a, stream);
    else if (chunks <= 8) launch_rows<4, 4>(norm_int_kernel<ST, 4, 4, 2, WHOLE>, a, stream);
    else if (chunks <= 32) launch_rows<8, 8>(norm_int_kernel<ST, 8, 8, 4, WHOLE>, a, stream);
    else launch_rows<8, 8>(norm_int_kernel<ST, 8, 8, 0, WHOLE>, a, stream);
    return hipGetLastError();
}

template <typename ST, int ACT, bool GATED, bool WHOLE>
hipError_t launch_act(const IntRowArgs& a, hipStream_t stream) {
    const int chunks = (a.d + kChunk - 1) / kChunk;
    if (chunks == 1) launch_rows<1, 4>(act_int_kernel<ST, ACT, GATED, 1, 4, 1, WHOLE>, a, stream);
    else if (chunks <= 4) launch_rows<4, 4>(act_int_kernel<ST, ACT, GATED, 4, 4, 1, WHOLE>, a, stream);
    else if (chunks <= 16) launch_rows<8, 8>(act_int_kernel<ST, ACT, GATED, 8, 8, 2, WHOLE>, a, stream);
    else launch_rows<8, 8>(act_int_kernel<ST, ACT, GATED, 8, 8, 0, WHOLE>, a, stream);
    return hipGetLastError();
}
template <typename ST, bool GATED, bool WHOLE>
hipError_t launch_act_of(const IntRowArgs& a, hipStream_t stream) {
    if (a.act == MOE_ACT_RELU) return launch_act<ST, MOE_ACT_RELU, GATED, WHOLE>(a, stream);
    if (a.act == MOE_ACT_GELU) return launch_act<ST, MOE_ACT_GELU, GATED, WHOLE>(a, stream);
    if (a.act == MOE_ACT_SILU) return launch_act<ST, MOE_ACT_SILU, GATED, WHOLE>(a, stream);
    return launch_act<ST, MOE_ACT_NONE, GATED, WHOLE>(a, stream);
}
template <typename ST>
hipError_t launch_act_type(const IntRowArgs& a, hipStream_t stream) {
    if (a.d % 8 == 0) return a.gated ? launch_act_of<ST, true, true>(a, stream) : launch_act_of<ST, false, true>(a, stream);
    return a.gated ? launch_act_of<ST, true, false>(a, stream) : launch_act_of<ST, false, false>(a, stream);
}

// ---- moe_quantize_weights_int ----------------------------------------------------------------------------------------
// A block of threads per 32 rows of a matrix, thread t columns 16 (t % 8) ... of row t / 8 in every block of 128 columns: once for the row's
// largest magnitude, once for the codes, 16 bytes at the place that the products' loads want them (moe.h, moe_quantize_weights).
typedef __attribute__((ext_vector_type(4), aligned(1))) uint32_t any_codes16;

template <typename ST>      // float, uint16_t (bf16) or uint8_t (codes)
__global__ __launch_bounds__(256) void quantize_weights_int_kernel(const ST* __restrict__ src, uint8_t* __restrict__ dst,
                                                                   float* __restrict__ scales, int N, int K) {
    const int e = blockIdx.y, n = blockIdx.x * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7, kblocks = quant_blocks(K);
    const ST* row = src + (static_cast<size_t>(e) * N + min(n, N - 1)) * K;
    uint8_t* to = dst + e * quant_matrix_bytes(N, K) + static_cast<size_t>(n >> 4) * kblocks * kFragBytes + (piece >> 2) * 1024 +
                  ((piece & 3) * 16 + (n & 15)) * 16;
    if constexpr (std::is_same_v<ST, uint8_t>) {
        for (int kb = 0; kb < kblocks; ++kb) {
            const int c = kb * kQuantBlock + piece * 16;
            uint32_t codes[4] = {0, 0, 0, 0};
            if (n < N && c + 16 <= K) {
                const any_codes16 v = *reinterpret_cast<const any_codes16*>(row + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) codes[i] = v[i];
            } else if (n < N) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c + i < K) codes[i >> 2] |= static_cast<uint32_t>(row[c + i]) << (8 * (i & 3));
            }
            *reinterpret_cast<uint4*>(to + static_cast<size_t>(kb) * kFragBytes) = uint4{codes[0], codes[1], codes[2], codes[3]};
        }
    } else {
        auto read = [&](int c, float (&v)[8]) {
            if (n < N && c + 8 <= K) {
                Eight<ST>::load(row + c, v);
                return;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = n < N && c + i < K ? Storage<ST>::load(row + c + i) : 0.f;
        };
        uint32_t most = 0;
        for (int kb = 0; kb < kblocks; ++kb) {
            float v[2][8];
#pragma unroll
            for (int h = 0; h < 2; ++h) read(kb * kQuantBlock + piece * 16 + h * 8, v[h]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[h][i]));
        }
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), o, 64)));
        const bool bad = most >= 0x7f800000u;
        const float scale = bad ? __uint_as_float(0x7fc00000u) : fmaxf(__uint_as_float(most) / kIntMax, kMinScale);
        const BlockQuotient of(scale);
        if (piece == 0 && n < N) scales[static_cast<size_t>(e) * N + n] = scale;
        for (int kb = 0; kb < kblocks; ++kb) {
            uint32_t codes[4] = {0, 0, 0, 0};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                read(kb * kQuantBlock + piece * 16 + h * 8, v);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!bad) codes[2 * h + (i >> 2)] |= (static_cast<uint32_t>(static_cast<int>(rintf(of(v[i])))) & 0xffu) << (8 * (i & 3));
            }
            *reinterpret_cast<uint4*>(to + static_cast<size_t>(kb) * kFragBytes) = uint4{codes[0], codes[1], codes[2], codes[3]};
        }
    }
}

}  // namespace

hipError_t launch_norm_quantize_int(const IntRowArgs& a, int dtype, hipStream_t stream) {
    const bool whole = a.d % 8 == 0;
    if (dtype == MOE_BF16) return whole ? launch_norm<uint16_t, true>(a, stream) : launch_norm<uint16_t, false>(a, stream);
    return whole ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream);
}

hipError_t launch_act_quantize_int(const IntRowArgs& a, int dtype, hipStream_t stream) {
    return dtype == MOE_BF16 ? launch_act_type<uint16_t>(a, stream) : launch_act_type<float>(a, stream);
}

hipError_t launch_quantize_weights_int(int E, int N, int K, int src_dtype, const void* src, uint8_t* dst, float* scales, hipStream_t stream) {
    const dim3 grid(quant_blocks(N) * 4, E), block(256);        // all rows of the padded matrix
    auto go = [&](auto* from) { quantize_weights_int_kernel<<<grid, block, 0, stream>>>(from, dst, scales, N, K); };
    if (src_dtype == MOE_F32) go(static_cast<const float*>(src));
    else if (src_dtype == MOE_BF16) go(static_cast<const uint16_t*>(src));
    else go(static_cast<const uint8_t*>(src));
    return hipGetLastError();
}

}  // namespace moe
