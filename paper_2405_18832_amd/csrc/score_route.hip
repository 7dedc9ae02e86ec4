// Router logits, and routing from logits: softmax or sigmoid scores, a bias for the choice alone, groups of experts, top-k, weights.
//
//   logits[t, e] = x[t] . w_gate[e] + bias[e]
//   p[t, e] = softmax or sigmoid of logits[t, e];   c[t, e] = p[t, e] + balance[e], in 64 bits, or logits[t, e] where there is no balance
//   a group's value: the largest of its choices, or the sum of the two largest (of p where there is no balance);  `kept` groups stay
//   the k largest choices among them, ties by lowest index;   weight = p / (sum of the chosen p) * scale
#include <algorithm>
#include <type_traits>

#include "int8.hpp"
#include "row_chunks.hpp"
#include "topk.hpp"

namespace moe {

namespace {

// ---- moe_gate_logits ---------------------------------------------------------------------------------------------------
// 16 bytes of a row, a lane's piece of a matrix instruction's operand: 8 bf16 values or 4 fp32 values.  Which values of the contraction
// an instruction takes from where does not matter as long as both operands agree.
template <typename ST> struct Piece;
template <> struct Piece<uint16_t> {
    using type = bf16x8;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(2)));
    static constexpr int kValues = 8;
    static __device__ __forceinline__ f32x4 multiply(const bf16x8& a, const bf16x8& b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Piece<float> {
    using type = f32x4;
    typedef uint32_t any __attribute__((ext_vector_type(4), aligned(4)));
    static constexpr int kValues = 4;
    static __device__ __forceinline__ f32x4 multiply(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};
// The piece from column c of a row of d values that begins at any element; values past the end are zero.
template <typename ST>
__device__ __forceinline__ typename Piece<ST>::type load_piece(const ST* row, int c, int d) {
    constexpr int V = Piece<ST>::kValues;
    if (c + V <= d) return __builtin_bit_cast(typename Piece<ST>::type, *reinterpret_cast<const typename Piece<ST>::any*>(row + c));
    ST v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = c + i < d ? row[c + i] : ST(0);
    return __builtin_bit_cast(typename Piece<ST>::type, v);
}

// 16 tokens x 16 experts per block; its wavefronts take shares of the contraction, which are added up in their order.
constexpr int kGateWaves = 16;
template <typename ST>
__global__ __launch_bounds__(kGateWaves * 64) void gate_few_kernel(const ST* __restrict__ x, const ST* __restrict__ wg, const float* __restrict__ bias,
                                                                   float* __restrict__ logits, int T, int d, int E) {
    constexpr int kStep = 4 * Piece<ST>::kValues, PF = 4;
    __shared__ f32x4 sums[kGateWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int e0 = blockIdx.x * 16, steps = (d + kStep - 1) / kStep, per = (steps + kGateWaves - 1) / kGateWaves;
    const long t0 = blockIdx.y * 16l;
    const ST* xr = x + min(t0 + r, T - 1l) * d;
    const ST* wr = wg + static_cast<size_t>(min(e0 + r, E - 1)) * d;
    const int s0 = min(steps, wave * per), s1 = min(steps, s0 + per);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s = s0; s < s1; s += PF) {
        typename Piece<ST>::type a[PF], b[PF];
#pragma unroll
        for (int p = 0; p < PF; ++p) {
            const int c = min(s + p, s1 - 1) * kStep + g * Piece<ST>::kValues;         // past the end: read again, not used
            a[p] = load_piece(wr, c, d);
            b[p] = load_piece(xr, c, d);
        }
#pragma unroll
        for (int p = 0; p < PF; ++p)
            if (s + p < s1) acc = Piece<ST>::multiply(a[p], b[p], acc);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (threadIdx.x < 256) {                   // expert e0 + e of token t0 + t: sum i of lane t + 16 (e / 4)
        const int t = threadIdx.x >> 4, e = threadIdx.x & 15;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kGateWaves; ++w) sum += sums[w][t + 16 * (e >> 2)][e & 3];
        if (t0 + t < T && e0 + e < E) logits[(t0 + t) * E + e0 + e] = bias != nullptr ? sum + bias[e0 + e] : sum;
    }
}

// ---- moe_route_logits --------------------------------------------------------------------------------------------------
// Another name than the rotations of 32 bits: declared in here, theirs would be hidden.
template <int N>
__device__ __forceinline__ double row_rot64(double v) {
    const uint64_t b = __double_as_longlong(v);
    const uint64_t lo = static_cast<uint32_t>(row_rot<N>(static_cast<int>(b))), hi = static_cast<uint32_t>(row_rot<N>(static_cast<int>(b >> 32)));
    return __longlong_as_double(static_cast<int64_t>(hi << 32 | lo));
}
template <typename V, typename Op>
__device__ __forceinline__ V row_reduce(V v, Op op) {
    auto with = [&](auto n) {
        if constexpr (std::is_same_v<V, double>) v = op(v, row_rot64<decltype(n)::value>(v));
        else v = op(v, row_rot<decltype(n)::value>(v));
    };
    with(std::integral_constant<int, 8>{});
    with(std::integral_constant<int, 4>{});
    with(std::integral_constant<int, 2>{});
    with(std::integral_constant<int, 1>{});
    return v;
}

constexpr double kNone = -__builtin_huge_val();

// One token's experts and weights, by a group of 16 lanes, in 64 bits.  `row` [E] and `group` [groups]: LDS.  Called by whole wavefronts.
template <typename ST>
__device__ void choose_exactly(const ScoreArgs& a, const ST* __restrict__ logits, double* row, double* group, int sub, bool live, long t,
                               int32_t* hist) {
    const int E = a.E, size = E / a.groups;
    // the token's largest logit, and whether there is one that is none
    float most = -__builtin_huge_valf();
    int invalid = 0;
    for (int e = sub; e < E; e += 16) {
        const float l = Storage<ST>::load(logits + e);
        invalid |= l != l || (!a.sigmoid && l == __builtin_huge_valf()) ? 1 : 0;
        most = fmaxf(most, l);
    }
    most = row_reduce(most, [](float u, float v) { return fmaxf(u, v); });
    invalid = row_reduce(invalid, [](int u, int v) { return u | v; });
    auto exponential = [&](float l) { return l == -__builtin_huge_valf() ? 0.0 : exp(static_cast<double>(l) - static_cast<double>(most)); };
    double total = 1.0;
    if (!a.sigmoid) {
        total = 0.0;
        for (int e = sub; e < E; e += 16) total += exponential(Storage<ST>::load(logits + e));
        total = row_reduce(total, [](double u, double v) { return u + v; });
    }
    auto score = [&](float l) { return a.sigmoid ? 1.0 / (1.0 + exp(-static_cast<double>(l))) : exponential(l) / total; };
    auto choice = [&](int e, float l) {
        const double c = a.balance != nullptr ? score(l) + static_cast<double>(a.balance[e]) : static_cast<double>(l);
        return l > -__builtin_huge_valf() && c == c ? c : kNone;
    };
    const bool by_score = a.groups > 1 && a.top == 2 && a.balance == nullptr;          // groups by scores, experts by logits
    for (int e = sub; e < E; e += 16) {
        const float l = Storage<ST>::load(logits + e);
        double c = choice(e, l);
        if (by_score && c != kNone) c = score(l);
        row[e] = c == c ? c : kNone;
    }
    __builtin_amdgcn_wave_barrier();
    if (a.groups > 1) {
        for (int g = sub; g < a.groups; g += 16) {
            double first = kNone, second = kNone;
            for (int i = 0; i < size; ++i) {
                const double c = row[g * size + i];
                second = fmax(second, fmin(first, c));
                first = fmax(first, c);
            }
            group[g] = a.top == 2 ? first + second : first;
        }
        __builtin_amdgcn_wave_barrier();
        for (int g = sub; g < a.groups; g += 16) {
            const double mine = group[g];
            int ahead = 0;
            for (int o = 0; o < a.groups; ++o) ahead += group[o] > mine || (group[o] == mine && o < g) ? 1 : 0;
            for (int i = 0; i < size; ++i) {
                const int e = g * size + i;
                if (ahead >= a.kept) row[e] = kNone;
                else if (by_score) row[e] = choice(e, Storage<ST>::load(logits + e));
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    int mine = 0;                              // lane j keeps the winner of round j
    double value = kNone;
    for (int j = 0; j < a.k; ++j) {
        double best = kNone;
        int at = E;
        for (int e = sub; e < E; e += 16) {
            const double c = row[e];           // NaN: taken
            if (c == c && (at == E || c > best)) {
                best = c;
                at = e;
            }
        }
        auto better = [&](double v, int e) {
            if (e < E && (at == E || v > best || (v == best && e < at))) {
                best = v;
                at = e;
            }
        };
        better(row_rot64<8>(best), row_rot<8>(at));
        better(row_rot64<4>(best), row_rot<4>(at));
        better(row_rot64<2>(best), row_rot<2>(at));
        better(row_rot64<1>(best), row_rot<1>(at));
        at = min(at, E - 1);
        if (sub == j) {
            mine = at;
            value = best;
        }
        __builtin_amdgcn_wave_barrier();
        if (sub == 0) row[at] = __builtin_nan("");
        __builtin_amdgcn_wave_barrier();
    }
    const double p = sub < a.k && value != kNone ? score(Storage<ST>::load(logits + mine)) : 0.0;
    double sum = 1.0;
    if (a.renormalize) {
        sum = 0.0;
        for (int j = 0; j < a.k; ++j) sum += __shfl(p, j, 16);
    }
    if (live && sub < a.k) {
        a.idx[t * a.k + sub] = mine;
        a.weight[t * a.k + sub] = invalid ? __uint_as_float(0x7fc00000u) : sum > 0.0 ? static_cast<float>(p / sum * static_cast<double>(a.scale)) : 0.f;
        atomicAdd(&hist[mine], 1);             // LDS, whole numbers: the order does not matter
    }
}

// Counts -> offsets and hot mask, by a block of 1024 threads, thread e with expert e's count.
__device__ __forceinline__ void finish_counts(const ScoreArgs& a, int mine, int32_t* cnt, int32_t* scan) {
    const int e = threadIdx.x;
    if (a.H >= 0) {
        if (e < a.E) cnt[e] = mine;
        __syncthreads();
        if (e < a.E) {
            int rank = 0;
            for (int o = 0; o < a.E; ++o) rank += cnt[o] > mine || (cnt[o] == mine && o < e) ? 1 : 0;
            a.hot_mask[e] = rank < a.H ? 1 : 0;
        }
    }
    const int v[1] = {mine};
    int incl[1], total[1];
    block_scan(v, incl, total, scan, (a.E + 63) >> 6);
    if (e < a.E) {
        a.counts[e] = mine;
        a.offsets[e] = incl[0] - mine;
        if (e == a.E - 1) a.offsets[a.E] = incl[0];
    }
}

// A block takes `tokens` tokens, 4 per wavefront at a time.  WHOLE: there is one block, which goes on to the outputs of the counts; else
// its counts go to the workspace.
constexpr int kRouteExactWaves = 4;
template <typename ST>
__global__ __launch_bounds__(kRouteExactWaves * 64) void route_scores_kernel(const ScoreArgs a, int tokens) {
    extern __shared__ __align__(16) unsigned char lds[];
    double* rows = reinterpret_cast<double*>(lds);                             // [16][E], then [16][groups]
    double* groups = rows + 4 * kRouteExactWaves * a.E;
    int32_t* hist = reinterpret_cast<int32_t*>(groups + 4 * kRouteExactWaves * a.groups);
    for (int e = threadIdx.x; e < a.E; e += kRouteExactWaves * 64) hist[e] = 0;
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, slot = wave * 4 + (lane >> 4);
    const long first = static_cast<long>(blockIdx.x) * tokens, last = min(first + tokens, static_cast<long>(a.T));
    for (long t0 = first + wave * 4; t0 < last; t0 += 4 * kRouteExactWaves) {
        const long t = t0 + (lane >> 4);
        const bool live = t < last;
        choose_exactly(a, static_cast<const ST*>(a.logits) + (live ? t : last - 1) * a.E, rows + slot * a.E, groups + slot * a.groups, lane & 15, live, t,
                       hist);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRouteExactWaves * 64) a.hist[static_cast<size_t>(blockIdx.x) * a.E + e] = hist[e];
}

__global__ __launch_bounds__(1024) void route_counts_kernel(const ScoreArgs a, int chunks) {
    __shared__ int32_t cnt[MOE_MAX_E], scan[kScanInts];
    int mine = 0;
    if (static_cast<int>(threadIdx.x) < a.E)
        for (int c = 0; c < chunks; ++c) mine += a.hist[static_cast<size_t>(c) * a.E + threadIdx.x];
    finish_counts(a, mine, cnt, scan);
}

}  // namespace

hipError_t launch_gate_logits(const moe_shape& s, const void* x, const void* w_gate, const float* bias, float* logits, hipStream_t stream) {
    const int tokens = (s.T + 15) / 16;
    constexpr int kMost = 65535;               // blocks of the grid's second direction
    for (int t0 = 0; t0 < tokens; t0 += kMost) {
        const long row = 16l * t0;
        const dim3 grid((s.E + 15) / 16, std::min(tokens - t0, kMost)), block(kGateWaves * 64);
        if (s.dtype == MOE_BF16)
            gate_few_kernel<<<grid, block, 0, stream>>>(static_cast<const uint16_t*>(x) + row * s.d_model, static_cast<const uint16_t*>(w_gate), bias,
                                                        logits + row * s.E, static_cast<int>(s.T - row), s.d_model, s.E);
        else
            gate_few_kernel<<<grid, block, 0, stream>>>(static_cast<const float*>(x) + row * s.d_model, static_cast<const float*>(w_gate), bias,
                                                        logits + row * s.E, static_cast<int>(s.T - row), s.d_model, s.E);
    }
    return hipGetLastError();
}

hipError_t launch_route_logits(const ScoreArgs& a, int logits_dtype, hipStream_t stream) {
    int chunks = 0;
    if (a.T > 0) {
        const int tokens = std::max(16, (a.T + 127) / 128);
        chunks = (a.T + tokens - 1) / tokens;
        const size_t lds = static_cast<size_t>(4 * kRouteExactWaves) * (a.E + a.groups) * 8 + a.E * 4;
        if (logits_dtype == MOE_BF16) route_scores_kernel<uint16_t><<<dim3(chunks), dim3(kRouteExactWaves * 64), lds, stream>>>(a, tokens);
        else route_scores_kernel<float><<<dim3(chunks), dim3(kRouteExactWaves * 64), lds, stream>>>(a, tokens);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    route_counts_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a, chunks);
    return hipGetLastError();
}

hipError_t configure_score_kernels() {
    static_assert(4 * kRouteExactWaves * (MOE_MAX_E + MOE_MAX_GROUPS) * 8 + MOE_MAX_E * 4 <= kLdsPerCu, "fits a CU");
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(route_scores_kernel<float>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsPerCu);
    if (e != hipSuccess) return e;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(route_scores_kernel<uint16_t>), hipFuncAttributeMaxDynamicSharedMemorySize, kLdsPerCu);
}

}  // namespace moe
