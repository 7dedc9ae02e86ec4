// What lies between a layer's two products: the activation, gated or not, and its values as int8 rows.
#include "int_rows.hpp"

namespace moe {

namespace {

// ACT: MOE_ACT_GELU, MOE_ACT_SILU, or MOE_ACT_RELU for it and for none, which is that with a `least` of -infinity.
template <int ACT>
__device__ __forceinline__ float act_value(float g, float least) {
    if (ACT == MOE_ACT_GELU) return gelu_exp(g);
    if (ACT == MOE_ACT_SILU) return silu(g);
    return g < least ? least : g;                           // NaN stays
}
template <int ACT>
__device__ __forceinline__ double act_exact(double g, float least) {
    if (ACT == MOE_ACT_GELU) return 0.5 * g * erfc(g * -0.70710678118654752440);
    if (ACT == MOE_ACT_SILU) return g / (1.0 + exp(-g));
    return g < static_cast<double>(least) ? static_cast<double>(least) : g;
}
// Twice the relative error of act_value * u, and of half of the quotient's roundings, for arguments up to g in magnitude.  SiLU, u = 2^-24: (1.25 |g| + 6) u (int8.hpp), the
// product and the quotient one each.  GeLU: 8.4e-7 down to -4; below, its argument z^2 / 2 log2 e is |z| times that of SiLU's.
template <int ACT>
__device__ __forceinline__ float act_slack(float g) {
    if (ACT == MOE_ACT_GELU) return fmaf(g * g, 0x1p-22f, 0x1p-18f);
    if (ACT == MOE_ACT_SILU) return fmaf(g, 0x1.4p-23f, 0x1p-20f);
    return kProductSlack;
}
// Gates below this leave nothing to act_value of a number that a large second factor could make the row's largest again.
template <int ACT>
constexpr float kTail = ACT == MOE_ACT_GELU ? -12.f : -80.f;
// And gates of which half is below fp32's normal numbers lose some of it there.  They take factors of 2^20 and more to be seen in a row whose largest value is 2^-100 and more
// (below, all of it is computed in 64 bits).
constexpr float kSmallGate = 0x1p-124f, kLargeFactor = 0x1p+20f;
constexpr float kHuge = __builtin_huge_valf();

// One pass, the row in registers from the largest value to the codes.  Bound by memory: gated SiLU of 20011 x 2048 in bf16 44.8 to 46.4 us, 4.5 TB/s read + written (a
// copy reaches 5.1; 44.6 with a divisor whose error was not counted, 47 with what fp32 does not hold looked for in the same pass); 64 x 8192 6.9 us, of which a launch is 3.5.
template <typename ST, int ACT, bool GATED, int WPR, int WAVES, int NV>
__global__ __launch_bounds__(WAVES * 64) void act_int_kernel(const IntRowArgs a) {
    static_assert(WPR == 1 || WPR == WAVES, "the block's barriers are the row's");
    constexpr bool kSmooth = ACT == MOE_ACT_GELU || ACT == MOE_ACT_SILU;
    __shared__ RowShared<WAVES> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % WPR;
    const int row = (blockIdx.y * gridDim.x + blockIdx.x) * (WAVES / WPR) + wave / WPR;
    bool live = row < a.rows;                               // the block meets at barriers below
    if (a.offsets != nullptr) {                             // the expert whose row this is: as many end at or before it as precede that
        int e = 0;
        for (int e0 = 0; e0 < a.E; e0 += 64) e += __popcll(__ballot(e0 + lane < a.E && a.offsets[min(e0 + lane, a.E - 1) + 1] <= row));
        live = live && e < a.E && a.offsets[min(e, a.E - 1)] <= row && (a.mask == nullptr || a.mask[min(e, a.E - 1)] != 0);
    }
    const float least = a.act == MOE_ACT_RELU ? 0.f : -__builtin_huge_valf();
    const int d = a.d;
    const ST* g_row = static_cast<const ST*>(a.x) + static_cast<size_t>(live ? row : 0) * (GATED ? 2 : 1) * d;
    const ST* u_row = g_row + d;
    const int chunks = (d + kChunk - 1) / kChunk;
    auto column = [&](int chunk) { return chunk * kChunk + lane * 8; };
    constexpr int kKept = NV > 0 ? NV : 1;
    float v[kKept][8], slack[kKept];
    // Values that act_value does not hold are left out of a row that has any, which is looked through again then (`apart`); their own slack says so, a negative one, and
    // before that an infinite one.
    constexpr bool kApart = GATED && kSmooth;
    bool apart = kApart && NV == 0;
    auto value = [&](const float (&g)[8], const float (&u)[GATED ? 8 : 1], float (&to)[8], float& own) __attribute__((always_inline)) {
        float size = 0.f, widest = 0.f;
        uint32_t lowest = 0;                                // bits: of negative numbers, the larger the lower
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            to[i] = act_value<ACT>(g[i], least);
            if constexpr (GATED) to[i] *= u[i];
            if constexpr (kApart) {
                lowest = max(lowest, __float_as_uint(g[i]));
                widest = fmaxf(widest, fabsf(u[i]));
            }
            if (kSmooth) size = fmaxf(size, fabsf(g[i]));
        }
        own = act_slack<ACT>(size);
        if constexpr (kApart) {
            const bool any = lowest > __builtin_bit_cast(uint32_t, kTail<ACT>) || widest >= kLargeFactor;
            if (!apart) {
                own = any ? kHuge : own;
            } else if (any) {
                size = 0.f;
                bool left = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool out = g[i] < kTail<ACT> || (fabsf(g[i]) < kSmallGate && g[i] != 0.f);
                    left |= out;
                    to[i] = out ? fmaf(g[i], 0.f, u[i] * 0.f) : to[i];      // zero, or NaN where an infinity or a NaN makes the row none
                    size = fmaxf(size, out ? 0.f : fabsf(g[i]));
                }
                own = left ? -act_slack<ACT>(size) : act_slack<ACT>(size);
            }
        }
    };
    auto each = [&](auto f) __attribute__((always_inline)) {       // f(chunk, values, slack)
        if constexpr (NV > 0) {
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) f(j * WPR + part, v[j], slack[j]);
            });
        } else {
            for (int c = part; c < chunks; c += WPR) {
                float g[8], u[GATED ? 8 : 1];
                load8<ST, false>(g_row, column(c), d, g);
                if constexpr (GATED) load8<ST, false>(u_row, column(c), d, u);
                value(g, u, v[0], slack[0]);
                f(c, v[0], slack[0]);
            }
        }
    };
    uint32_t most;
    float loosest;
#pragma unroll 1
    while (true) {
        most = 0;
        loosest = 0.f;
        if (live) {
            if constexpr (NV > 0) {                             // all loads first
                float g[NV][8], u[NV][GATED ? 8 : 1];
                unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                    if (j * WPR + part < chunks) {
                        load8<ST, false>(g_row, column(j * WPR + part), d, g[j]);
                        if constexpr (GATED) load8<ST, false>(u_row, column(j * WPR + part), d, u[j]);
                    }
                });
                unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                    if (j * WPR + part < chunks) value(g[j], u[j], v[j], slack[j]);
                });
            }
            each([&](int, const float (&values)[8], float own) __attribute__((always_inline)) {
                loosest = fmaxf(loosest, kApart && own < 0.f ? fmaxf(-own, 0x1p-17f) : own);
#pragma unroll
                for (int i = 0; i < 8; ++i) most = max(most, magnitude(values[i]));
            });
        }
        most = wave_max(most);
        if (kSmooth) loosest = __uint_as_float(wave_max(__float_as_uint(loosest)));
        if constexpr (WPR > 1) {
            if (lane == 0) {
                shared.most[wave] = most;
                shared.slack[wave] = loosest;
            }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WPR; ++w) {
                most = max(most, shared.most[w]);
                loosest = fmaxf(loosest, shared.slack[w]);
            }
        }
        if (!kApart || apart || __builtin_amdgcn_readfirstlane(__float_as_int(loosest)) < __float_as_int(kHuge)) break;
        apart = true;
        if constexpr (WPR > 1) __syncthreads();             // `shared` is written again
    }
    write_row<WPR, WAVES>(shared, live, most >= 0x7f800000u, most, loosest, 1.0, d, a.q + static_cast<size_t>(live ? row : 0) * quant_pitch(d),
                          a.q_scales + (live ? row : 0), each, [&](int chunk, int i) __attribute__((always_inline)) {
                              const double g = act_exact<ACT>(static_cast<double>(Storage<ST>::load(g_row + column(chunk) + i)), least);
                              if constexpr (GATED) return g * static_cast<double>(Storage<ST>::load(u_row + column(chunk) + i));
                              return g;
                          });
}

template <typename ST, int ACT, bool GATED>
hipError_t launch_act(const IntRowArgs& a, hipStream_t stream) {
    with_row_variant(a, [&](auto wpr, auto waves, auto nv) {
        constexpr int WPR = decltype(wpr)::value, WAVES = decltype(waves)::value, NV = decltype(nv)::value;
        launch_rows<WPR, WAVES>(act_int_kernel<ST, ACT, GATED, WPR, WAVES, NV>, a, stream);
    });
    return hipGetLastError();
}
template <typename ST, bool GATED>
hipError_t launch_act_of(const IntRowArgs& a, hipStream_t stream) {
    if (a.act == MOE_ACT_GELU) return launch_act<ST, MOE_ACT_GELU, GATED>(a, stream);
    if (a.act == MOE_ACT_SILU) return launch_act<ST, MOE_ACT_SILU, GATED>(a, stream);
    return launch_act<ST, MOE_ACT_RELU, GATED>(a, stream);
}

}  // namespace

hipError_t launch_act_quantize_int(const IntRowArgs& a, int dtype, hipStream_t stream) {
    if (dtype == MOE_BF16) return a.gated ? launch_act_of<uint16_t, true>(a, stream) : launch_act_of<uint16_t, false>(a, stream);
    return a.gated ? launch_act_of<float, true>(a, stream) : launch_act_of<float, false>(a, stream);
}

}  // namespace moe
