// Router logits, and routing from logits: softmax or sigmoid scores, a bias for the choice alone, groups of experts, top-k, weights.
//
//   logits[t, e] = x[t] . w_gate[e] + bias[e]
//   p[t, e] = softmax or sigmoid of logits[t, e];   c[t, e] = p[t, e] + balance[e], in 64 bits, or logits[t, e] where there is no balance
//   a group's value: the largest of its choices, or the sum of the two largest (of p where there is no balance);  `kept` groups stay
//   the k largest choices among them, ties by lowest index;   weight = p / (sum of the chosen p) * scale
#include <algorithm>
#include <type_traits>

#include "int8.hpp"
#include "quant_units.hpp"
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

// 16 tokens x 16 experts per block; its wavefronts take shares of the contraction, which are added up in their order.  Bound by a launch and one wait for
// memory: 32 x 256 x 2048 in bf16 takes 5.5 us, a launch that does nothing 3.5.
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

// Many tokens: 16 TF tokens x 64 NF experts per block of four wavefronts (16 NF experts each), through a ring of LDS stages of one 128-byte line of every
// row, copied by eight consecutive lanes each, the tokens' rows first.  What follows needs rows of whole 16-byte pieces; a last line that is not whole
// is copied with its first piece in place of those that do not exist, which are taken as zeros of both operands.  5003 x 256 x 2048 in bf16 take 12.8 to 13.9 us
// (16.4 with four stages, two blocks per CU and 64 tokens to a block), 16384 tokens 29.  Bound by copies out of the L2s: of the former 1.33 million lines, 170 MB, of which
// 30 MB come from memory (x is 20 MB; the weights are copied once per block of tokens), some 17 TB/s behind the launch; matrix units busy 0.18.  In 32 bits by the
// matrix units too, whose instructions take 32 clocks for four columns: 16384 tokens 147 us, 0.74 of their rate; a wavefront's 1024 of 1024 tokens 14 of 26 us.
constexpr int kGateTileWaves = 4, kGateStages = 6;
template <int TF, int NF>
struct GateTile {
    static constexpr int kTokens = 16 * TF, kExperts = 64 * NF, kRows = kTokens + kExperts;
    static constexpr int kCopies = (kRows / 8 + kGateTileWaves - 1) / kGateTileWaves, kStage = kCopies * kGateTileWaves * 1024;       // a wavefront's; bytes
    static constexpr int kLdsBytes = kGateStages * kStage;
};
template <typename ST, int TF, int NF>
__global__ __launch_bounds__(kGateTileWaves * 64) void gate_tile_kernel(const ST* __restrict__ x, const ST* __restrict__ wg, const float* __restrict__ bias,
                                                                        float* __restrict__ logits, int T, int d, int E, int groups) {
    using G = GateTile<TF, NF>;
    extern __shared__ __align__(16) unsigned char lds_rows[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int at = xcd_position(), e0 = at % groups * G::kExperts;
    const long t0 = static_cast<long>(at / groups) * G::kTokens, pitch = static_cast<long>(d) * sizeof(ST);
    const int pieces = static_cast<int>(pitch / 16), steps = (pieces + 7) / 8, last = pieces - 8 * (steps - 1);
    if (t0 >= T) return;
    const uint32_t lds = lds_address(lds_rows);
    const char* from[G::kCopies];
#pragma unroll
    for (int i = 0; i < G::kCopies; ++i) {
        const int row = (wave * G::kCopies + i) * 8 + (lane >> 3);
        const char* base = row < G::kTokens ? reinterpret_cast<const char*>(x) + min(t0 + row, T - 1l) * pitch
                                            : reinterpret_cast<const char*>(wg) + static_cast<long>(min(e0 + row - G::kTokens, E - 1)) * pitch;
        from[i] = base + piece_of_lane(lane, row);
    }
    const int own_piece = piece_of_lane(lane, lane >> 3) >> 4;             // rows of a copy are a multiple of 8: the permutation of row lane / 8 ...
    int in = 0;
    auto copy_next = [&]() __attribute__((always_inline)) {
        const uint32_t to = lds + (in % kGateStages) * G::kStage + wave * G::kCopies * 1024;
#pragma unroll
        for (int i = 0; i < G::kCopies; ++i) {
            // ... or of 8 rows on, which differs in its highest bit
            const int row = (wave * G::kCopies + i) * 8, piece = own_piece ^ (row >> 1 & 4);
            const char* p = from[i] + (in >= steps - 1 && piece >= last ? -16 * piece : 0);
            copy16_to_lds(p, to + i * 1024);
            from[i] += in < steps - 1 ? 128 : 0;       // behind the last line it is copied again, which keeps up the count that the waits go by
        }
        ++in;
        in = in >= steps + kGateStages ? in - kGateStages : in;      // by whole rings
    };
#pragma unroll 1
    for (int i = 0; i < kGateStages - 1; ++i) copy_next();
    f32x4 acc[NF][TF];
#pragma unroll
    for (int nf = 0; nf < NF; ++nf)
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) acc[nf][tf] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int at_x = row_operand(threadIdx.x, 0), at_w = (G::kTokens + wave * NF * 16) * 128 + at_x, other = row_operand_other(at_x);
    using P = typename Piece<ST>::type;
    auto step = [&](int s, auto whole) __attribute__((always_inline)) {
        copies_landed<(kGateStages - 2) * G::kCopies>();
        const unsigned char* st = lds_rows + (s % kGateStages) * G::kStage;
        P w[2][NF], v[2][TF];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int nf = 0; nf < NF; ++nf) w[h][nf] = *reinterpret_cast<const P*>(st + at_w + nf * 2048 + h * other);
#pragma unroll
            for (int tf = 0; tf < TF; ++tf) v[h][tf] = *reinterpret_cast<const P*>(st + at_x + tf * 2048 + h * other);
            if (!decltype(whole)::value && 4 * h + g >= last) {
#pragma unroll
                for (int nf = 0; nf < NF; ++nf) w[h][nf] = P{};
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) v[h][tf] = P{};
            }
        }
        copy_next();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int tf = 0; tf < TF; ++tf)
#pragma unroll
                for (int nf = 0; nf < NF; ++nf) acc[nf][tf] = Piece<ST>::multiply(w[h][nf], v[h][tf], acc[nf][tf]);
    };
#pragma unroll 1
    for (int s = 0; s < steps - 1; ++s) step(s, std::true_type{});
    step(steps - 1, std::false_type{});
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no copy may land in LDS that is another block's by then
    const bool wide = E % 4 == 0 && (reinterpret_cast<uintptr_t>(logits) & 15) == 0;
#pragma unroll
    for (int nf = 0; nf < NF; ++nf) {
        const int e = e0 + (wave * NF + nf) * 16 + g * 4;
        f32x4 b = {0.f, 0.f, 0.f, 0.f};
        if (bias != nullptr) {
#pragma unroll
            for (int i = 0; i < 4; ++i) b[i] = bias[min(e + i, E - 1)];
        }
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) {
            const long t = t0 + tf * 16 + r;
            if (t >= T) continue;
            const f32x4 v = acc[nf][tf] + b;
            if (wide) {
                if (e < E) *reinterpret_cast<f32x4*>(logits + t * E + e) = v;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e + i < E) logits[t * E + e + i] = v[i];
            }
        }
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
constexpr float kLow = -__builtin_huge_valf();

// Logit i of the call, whatever their type.
__device__ __forceinline__ float logit(const ScoreArgs& a, long i) {
    return a.bf16 ? bf16_to_f32(static_cast<const uint16_t*>(a.logits)[i]) : static_cast<const float*>(a.logits)[i];
}

template <typename V>
__device__ __forceinline__ V lane_of(V v, int lane) {
    if constexpr (sizeof(V) == 8) {
        const uint64_t b = __double_as_longlong(v);
        const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b), lane));
        const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane));
        return __longlong_as_double(static_cast<int64_t>(hi << 32 | lo));
    } else {
        return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    }
}
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V v, Op op) {
    v = row_reduce(v, op);
    return op(op(lane_of(v, 0), lane_of(v, 16)), op(lane_of(v, 32), lane_of(v, 48)));
}

// The groups that stay, from a token's choices `row` [E], by a wavefront.
__device__ __forceinline__ uint64_t groups_that_stay(const ScoreArgs& a, const double* row, double* group, int lane, int size) {
    double mine = kNone;
    if (lane < a.groups) {
        double first = kNone, second = kNone;
#pragma unroll 8
        for (int i = 0; i < size; ++i) {
            const double c = row[lane * size + i];
            second = fmax(second, fmin(first, c));
            first = fmax(first, c);
        }
        mine = a.top == 2 ? fmax(first + second, kNone) : first;        // infinity and -infinity: no sum, which is last
        group[lane] = mine;
    }
    __builtin_amdgcn_wave_barrier();
    int ahead = 0;
    if (lane < a.groups)
#pragma unroll 8
        for (int o = 0; o < a.groups; ++o) ahead += group[o] > mine || (group[o] == mine && o < lane) ? 1 : 0;
    return __ballot(lane < a.groups && ahead < a.kept);
}
// The same for finite logits and sigmoid scores.
__device__ __forceinline__ uint64_t groups_that_stay(const ScoreArgs& a, double* row, const float* values, double* group, int lane, int E) {
#pragma unroll 2
    for (int e = lane; e < E; e += 64) row[e] = 1.0 / (1.0 + exp(-static_cast<double>(values[e]))) + (a.balance != nullptr ? static_cast<double>(a.balance[e]) : 0.0);
    __builtin_amdgcn_wave_barrier();
    return groups_that_stay(a, row, group, lane, E / a.groups);
}

// One token's experts and weights, by a wavefront, in 64 bits.  `row` [E], `values` [E] (the logits, if they are `loaded`) and
// `group` [groups]: LDS.
__device__ __forceinline__ void choose_exactly(const ScoreArgs& a, double* row, float* values, bool loaded, double* group, int lane, long t, int32_t* hist) {
    int E = a.E;
    asm volatile("" : "+s"(E), "+v"(lane));    // as in choose
    const int size = E / a.groups;
    const long from = t * E;
    // the token's largest logit, and whether there is one that is none
    float most = kLow;
    int invalid = 0;
    if (!loaded) {
#pragma unroll 4
        for (int e = lane; e < E; e += 64) values[e] = logit(a, from + e);
    }
    for (int e = lane; e < E; e += 64) {
        const float l = values[e];
        invalid |= l != l || (!a.sigmoid && l == -kLow) ? 1 : 0;
        most = fmaxf(most, l);
    }
    most = wave_reduce(most, [](float u, float v) { return fmaxf(u, v); });
    invalid = wave_reduce(invalid, [](int u, int v) { return u | v; });
    auto power = [&](float l) { return l == kLow ? 0.0 : exp(a.sigmoid ? -static_cast<double>(l) : static_cast<double>(l) - static_cast<double>(most)); };
    double total = 1.0;
    if (!a.sigmoid) {
        total = 0.0;
#pragma unroll 1
        for (int e = lane; e < E; e += 64) total += power(values[e]);
        total = wave_reduce(total, [](double u, double v) { return u + v; });
    }
    auto score = [&](float l) { return l == kLow ? 0.0 : a.sigmoid ? 1.0 / (1.0 + power(l)) : power(l) / total; };
    const bool by_score = a.groups > 1 && a.top == 2 && a.balance == nullptr;          // groups by scores, experts by logits
#pragma unroll 2
    for (int e = lane; e < E; e += 64) {
        const float l = values[e];
        double c = l;
        if (a.balance != nullptr || by_score) {
            c = score(l);
            if (!by_score) c += static_cast<double>(a.balance[e]);
        }
        row[e] = l > kLow && c == c ? c : kNone;
    }
    __builtin_amdgcn_wave_barrier();
    if (a.groups > 1) {
        const uint64_t stay = groups_that_stay(a, row, group, lane, size);
#pragma unroll 1
        for (int e = lane; e < E; e += 64) {
            const float l = values[e];
            if (!(stay >> (e / size) & 1)) row[e] = __builtin_nan("");          // taken: not even where the kept groups have no other than masked experts left
            else if (by_score) row[e] = l > kLow ? static_cast<double>(l) : kNone;
        }
        __builtin_amdgcn_wave_barrier();
    }
    int mine = 0;                              // lane j keeps the winner of round j
    double value = kNone;
#pragma unroll 1
    for (int j = 0; j < a.k; ++j) {
        double best = kNone;
        int at = E;
#pragma unroll 4
        for (int e = lane; e < E; e += 64) {
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
        const double of[4] = {lane_of(best, 0), lane_of(best, 16), lane_of(best, 32), lane_of(best, 48)};
        const int is[4] = {lane_of(at, 0), lane_of(at, 16), lane_of(at, 32), lane_of(at, 48)};
#pragma unroll
        for (int r = 0; r < 4; ++r) better(of[r], is[r]);
        at = min(at, E - 1);
        if (lane == j) {
            mine = at;
            value = best;
        }
        __builtin_amdgcn_wave_barrier();
        if (lane == 0) row[at] = __builtin_nan("");
        __builtin_amdgcn_wave_barrier();
    }
    const double p = lane < a.k && value != kNone ? score(values[mine]) : 0.0;
    double sum = 1.0;
    if (a.renormalize) {
        sum = 0.0;
        for (int j = 0; j < a.k; ++j) sum += lane_of(p, j);
    }
    if (lane < a.k) {
        a.idx[t * a.k + lane] = mine;
        a.weight[t * a.k + lane] = invalid ? __uint_as_float(0x7fc00000u) : sum > 0.0 ? static_cast<float>(p / sum * static_cast<double>(a.scale)) : 0.f;
        atomicAdd(&hist[mine], 1);             // LDS, whole numbers: the order does not matter
    }
}

// The same in fp32, four tokens per wavefront, for up to 16 V experts in registers: expert 64 j + 4 sub + i is value 4 j + i of lane `sub` (of 16).
// Says whether the choice is beyond doubt (to all lanes of the token), and only then writes anything: not where two of the numbers that decide are
// so close that fp32's errors could have changed their order, and not with a logit that is no number.
//
// A lane sorts its choices once, as whole numbers of their order whose low bits are their places, and keeps the largest eight; the k rounds then
// compare the lanes' first ones and the winner's lane moves on to its next.  (Choices searched and taken out in every round: 1830 vector
// instructions per four tokens of 256 experts, k = 8.)
//
// Errors, u = 2^-24.  Sigmoid: its exponential is (|l| + 2) u of itself off, which p (1 - p) weighs (at most 0.23 |l|-fold, 0.25), the sum with one and the
// reciprocal 3 u: 4 u together.  Softmax: an exponential at x below the largest logit, whose own is exact, is (3 x + 2) u of itself off.  Their sum is added
// up in a tree, 4 + log2 V <= 10 additions deep (one after the other 64 of them would be 63 u off, one large one beside small ones); with Y for the sum of all but the
// largest, of n experts, x averages ln(n / Y) at the most, and scores of which one is the largest are ((10 + 2) (1 + Y) + Y (3 ln(n / Y) + 2)) / (1 + Y)^2 <= 14 u off
// each other (n = 1023, Y = 0.3); the smaller one's own exponential and product, 3 x e^-x <= 1.1, 2 and 1, make it 18 u.  The bias adds u |c|.
// Two numbers are in doubt up to `doubt`: that of both, and a fifth.  Logits themselves are exact.
template <bool SIGMOID>
__device__ __forceinline__ float doubt(float c) {
    return 0x1p-24f * fmaf(2.4f, fabsf(c), SIGMOID ? 10.f : 22.f);
}
// How far the value of one group may be off: the constant above, which is that of two scores; and one unit each of its choices' magnitudes for the bias, for the sum and for
// adding this to it.  Not of the sum's own magnitude: choices may cancel.
template <bool SIGMOID>
__device__ __forceinline__ float group_doubt(float size) {
    return 0x1p-24f * fmaf(3.2f, size, SIGMOID ? 10.f : 22.f);
}
typedef uint32_t any_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void load_four(const float* p, float* v) {
    const any_f32x4 w = *reinterpret_cast<const any_f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
}
__device__ __forceinline__ void load_four(const uint16_t* p, float* v) {
    const any_u32x2 w = *reinterpret_cast<const any_u32x2*>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
// The lane's values of a row of E; kLow past its end.
template <int V, typename T>
__device__ __forceinline__ void load_row(const T* from, int E, int base, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
        if (64 * j + 64 <= E) {                // the same for all lanes
            load_four(from + 64 * j + base, v + 4 * j);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 64 * j + base + i;
                const float u = Storage<T>::load(from + min(e, E - 1));
                v[4 * j + i] = e < E ? u : kLow;
            }
        }
    }
}
// Zero, or NaN if one of the row's values is no finite number.
template <int V>
__device__ __forceinline__ float finite(int E, int base, const float (&v)[V]) {
    float sum = 0.f;
#pragma unroll
    for (int q = 0; q < V; ++q) {
        const int chunk = 64 * (q / 4);
        sum = fmaf(chunk + 64 <= E || chunk + base + q % 4 < E ? v[q] : 0.f, 0.f, sum);
    }
    return sum;
}
// exp(x) of a difference of two fp32 numbers to 2 u of itself: the power of two and what is left are separated in 64 bits.
__device__ __forceinline__ float exp_of(double x) {
    const double t = x * 1.44269504088896340736, n = rint(t);
    return ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(t - n)), static_cast<int>(fmax(n, -1000.0)));
}

// The order of fp32 numbers as that of whole numbers, and back.
__device__ __forceinline__ int ordered(float v) {
    const int b = __float_as_int(v);
    return b ^ (b >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int n) { return __int_as_float(n ^ (n >> 31 & 0x7fffffff)); }

template <int CONTROL>
__device__ __forceinline__ int dpp(int v) {
    return __builtin_amdgcn_mov_dpp(v, CONTROL, 0xF, 0xF, true);
}
// Over the 16 lanes of a token.
__device__ __forceinline__ int most_of(int v) {
    v = max(v, dpp<0x128>(v));
    v = max(v, dpp<0x124>(v));
    v = max(v, dpp<0x122>(v));
    return max(v, dpp<0x121>(v));
}
__device__ __forceinline__ int least_of(int v) {
    v = min(v, dpp<0x128>(v));
    v = min(v, dpp<0x124>(v));
    v = min(v, dpp<0x122>(v));
    return min(v, dpp<0x121>(v));
}

__device__ __forceinline__ void in_order(int& a, int& b) {
    const int high = max(a, b);
    b = min(a, b);
    a = high;
}
template <int N>
__device__ __forceinline__ void merge_down(int* v) {            // a sequence that rises and falls -> descending
    if constexpr (N > 1) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) in_order(v[i], v[i + N / 2]);
        merge_down<N / 2>(v);
        merge_down<N / 2>(v + N / 2);
    }
}
template <int N>
__device__ __forceinline__ void sort_down(int* v) {             // at most eight
    if constexpr (N > 1) {
        sort_down<N / 2>(v);
        sort_down<N / 2>(v + N / 2);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) in_order(v[i], v[N - 1 - i]);       // the second half the other way round
        merge_down<N / 2>(v);
        merge_down<N / 2>(v + N / 2);
    }
}
// The largest eight of V, descending, to v[0] ... v[7].
template <int V>
__device__ __forceinline__ void largest_eight(int* v) {
    if constexpr (V <= 8) {
        sort_down<V>(v);
    } else {
        largest_eight<V / 2>(v);
        largest_eight<V / 2>(v + V / 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = max(v[i], v[V / 2 + 7 - i]);
        merge_down<8>(v);
    }
}

// Bytes of LDS of a wavefront: rows of four tokens' choices in fp32 or of one token's in 64 bits, rows of four tokens' logits, and the groups'.
__host__ __device__ constexpr int score_row_bytes(int E) { return 16 * E; }
__host__ __device__ constexpr int score_wave_bytes(int E) { return 2 * score_row_bytes(E) + MOE_MAX_GROUPS * 8; }

// Pairs, pairs of pairs, ...: log2 V additions deep.
template <int V>
__device__ __forceinline__ float tree_sum(const float* v) {
    if constexpr (V == 1) return v[0];
    else return tree_sum<V / 2>(v) + tree_sum<V / 2>(v + V / 2);
}

constexpr int kFastGroups = 16;
template <int V, bool SIGMOID, bool BALANCED>
__device__ __forceinline__ bool choose(const ScoreArgs& a, unsigned char* lds, int lane, bool live, long t, long last, int32_t* hist) {
    constexpr float kLog2e = 1.4426950408889634f;
    constexpr int kKept = V < 8 ? V : 8;
    // what follows from these is computed where it is used: kept from one turn of the caller's loop to the next, it would need 100 registers more
    int E = a.E, sub = lane & 15;
    asm volatile("" : "+s"(E), "+v"(sub));
    const int base = 4 * sub, slot = lane >> 4;
    float* row = reinterpret_cast<float*>(lds) + slot * E;
    float* all_values = reinterpret_cast<float*>(lds + score_row_bytes(E));
    float* values = all_values + slot * E;
    float* group = reinterpret_cast<float*>(lds + 2 * score_row_bytes(E)) + slot * kFastGroups;
    const long from = min(t, last - 1) * E;
    float c[V];
    if (a.bf16) load_row(static_cast<const uint16_t*>(a.logits) + from, E, base, c);
    else load_row(static_cast<const float*>(a.logits) + from, E, base, c);
    auto keep = [&](float* to, int j, const f32x4& v) __attribute__((always_inline)) {
        const int e = 64 * j + base;
        if (E % 4 == 0) {
            if (64 * j + 64 <= E || e < E) *reinterpret_cast<f32x4*>(to + e) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e + i < E) to[e + i] = v[i];
        }
    };
#pragma unroll
    for (int j = 0; j < V / 4; ++j) keep(values, j, f32x4{c[4 * j], c[4 * j + 1], c[4 * j + 2], c[4 * j + 3]});
    float none = finite(E, base, c);
    float most = 0.f, total = 1.f;
    if (!SIGMOID) {
        most = kLow;
#pragma unroll
        for (int q = 0; q < V; ++q) most = fmaxf(most, c[q]);
        most = unordered(most_of(ordered(most)));
        float e[V];
#pragma unroll
        for (int q = 0; q < V; ++q) e[q] = __builtin_amdgcn_exp2f((c[q] - most) * kLog2e);
        total = tree_sum<V>(e);
        total = row_reduce(total, [](float u, float v) { return u + v; });
    }
    const float by = SIGMOID ? 1.f : 1.f / total;
    auto score = [&](float l) __attribute__((always_inline)) {
        if (SIGMOID) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(l * -kLog2e));
        return __builtin_amdgcn_exp2f((l - most) * kLog2e) * by;
    };
    if (BALANCED) {
        float b[V];
        load_row(a.balance, E, base, b);
#pragma unroll
        for (int q = 0; q < V; ++q) c[q] = score(c[q]) + b[q];
        none += finite(E, base, c);
    }
    bool unsure = none != none;
    const bool by_score = !BALANCED && a.top == 2;      // groups by scores, experts by logits
    if (a.groups > 1) {
        const int size = E / a.groups;
#pragma unroll
        for (int j = 0; j < V / 4; ++j) {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = by_score ? score(c[4 * j + i]) : c[4 * j + i];
            keep(row, j, v);
        }
        __builtin_amdgcn_wave_barrier();
        // as many lanes for a group as there are, a power of two of them
        const int share = a.groups <= 2 ? 3 : a.groups <= 4 ? 2 : a.groups <= 8 ? 1 : 0;
        const int g = sub >> share, part = sub & ((1 << share) - 1);
        float first = kLow, second = kLow;
        auto take = [&](float v) __attribute__((always_inline)) {
            second = fmaxf(second, fminf(first, v));
            first = fmaxf(first, v);
        };
        if (g < a.groups) {
            const int n = (size + (1 << share) - 1) >> share, begin = g * size + part * n, end = min((g + 1) * size, begin + n);
            if (size % (4 << share) == 0) {    // whole pieces of 16 bytes for each
#pragma unroll 4
                for (int i = 0; i < n; i += 4) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(row + begin + i);
#pragma unroll
                    for (int u = 0; u < 4; ++u) take(v[u]);
                }
            } else {
                for (int i = begin; i < end; ++i) take(row[i]);
            }
        }
        for (int o = 1; o < 1 << share; o <<= 1) {
            const float of = __shfl_xor(first, o, 16), os = __shfl_xor(second, o, 16);
            second = fmaxf(fmaxf(second, os), fminf(first, of));
            first = fmaxf(first, of);
        }
        const float mine = a.top == 2 ? first + second : first;
        if (part == 0) group[g] = mine;
        __builtin_amdgcn_wave_barrier();
        int ahead = 0;
#pragma unroll 4
        for (int o = 0; o < a.groups; ++o) {
            const float v = group[o];
            ahead += v > mine || (v == mine && o < g) ? 1 : 0;
        }
        bool stays = g < a.groups && ahead < a.kept;
        if (BALANCED || by_score) {
            const float size = a.top == 2 ? fabsf(first) + fabsf(second) : fabsf(first), off = group_doubt<SIGMOID>(size);
            const float low = unordered(least_of(ordered(stays ? mine - off : -kLow)));
            const float high = unordered(most_of(ordered(g >= a.groups ? kLow : !(size < 0x1p+100f) ? -kLow : !stays ? mine + off : kLow)));
            const bool close = !(low > high);
            if (SIGMOID) {                     // 64 bits say which groups stay, a token at a time
                __builtin_amdgcn_wave_barrier();
                uint64_t left = __ballot(close && live && sub == 0);
#pragma unroll 1
                while (left != 0) {
                    const int n = __builtin_ctzll(left) >> 4;
                    left &= left - 1;
                    const uint64_t exact = groups_that_stay(a, reinterpret_cast<double*>(lds), all_values + n * E,
                                                            reinterpret_cast<double*>(lds + 2 * score_row_bytes(E)), lane, E);
                    if (slot == n) stays = (exact >> g & 1) != 0;
                    __builtin_amdgcn_wave_barrier();
                }
            } else {
                unsure |= close;
            }
        }
        const uint32_t stay = static_cast<uint32_t>(__ballot(stays) >> (threadIdx.x & 48)) & 0xffffu;
        const uint32_t inverse = ((1u << 20) + size - 1) / size;            // e * inverse >> 20 = e / size for e, size <= 1024
        auto out = [&](uint32_t e) { return (stay >> ((e * inverse >> 20) << share & 31u) & 1u) == 0; };
#pragma unroll
        for (int j = 0; j < V / 4; ++j) {
            const uint32_t e = 64 * j + base;
            if (size % 4 == 0) {
                const bool gone = out(e);
#pragma unroll
                for (int i = 0; i < 4; ++i) c[4 * j + i] = gone ? kLow : c[4 * j + i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) c[4 * j + i] = out(e + i) ? kLow : c[4 * j + i];
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    // Choices with a bias are multiples of 2^-24 (kUnit; an error of half of it) above their places in the lane, up to 8 (kFar) in magnitude; logits are the
    // order of their bits: of bf16 above the expert's number, so that no two are alike, else the place takes the last bits.
    constexpr float kUnit = V <= 16 ? 0x1p-24f : 0x1p-22f, kFar = 7.9f;
    static_assert(kFar / kUnit * V < 0x1p31f, "fits");
    const bool numbered = !BALANCED && a.bf16;
    int n[V];
    if (BALANCED) {
        float far = 0.f;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            far = fmaxf(far, c[q]);
            const float v = __builtin_amdgcn_fmed3f(c[q], -kFar, kFar) * (1.f / kUnit);
            n[q] = static_cast<int>(rintf(v)) * V + (V - 1 - q);
        }
        unsure |= !(far < kFar);
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int number = MOE_MAX_E - 1 - (64 * (q / 4) + base + q % 4);
            n[q] = numbered ? (ordered(c[q] + 0.f) & ~(MOE_MAX_E - 1)) | number         // -0 as 0
                            : (ordered(c[q]) & ~(V - 1)) | (V - 1 - q);
        }
    }
    largest_eight<V>(n);
    int mine = 0, taken = 0;                                    // lane j keeps the winner of round j; how many of the lane's have won
    float before = -kLow;
    // One more says whether the last was beyond doubt.  Sigmoid: two more; if the best k or k + 1 are, as a set, their order may be in doubt and is settled in 64 bits
    // below (nine differences in doubt once in 250 tokens of 256 experts, two next to each other hardly ever).
    constexpr bool kSettled = SIGMOID && BALANCED;
    const int rounds = numbered ? a.k : min(a.k + (kSettled ? 2 : 1), a.kept * (E / a.groups));
    bool in_order = true, best_k = true, best_k1 = true;
#pragma unroll 1
    for (int j = 0; j < rounds; ++j) {
        const int best = most_of(n[0]), q = V - 1 - (best & (V - 1));
        const int own = 64 * (q >> 2) + base + (q & 3);
        const int at = numbered ? MOE_MAX_E - 1 - (best & (MOE_MAX_E - 1)) : least_of(n[0] == best ? own : MOE_MAX_E);
        const bool won = numbered ? n[0] == best : n[0] == best && own == at;
#pragma unroll
        for (int i = 0; i < kKept - 1; ++i) n[i] = won ? n[i + 1] : n[i];
        if (won) n[kKept - 1] = -0x7fffffff - 1;
        taken += won ? 1 : 0;
        const float value = BALANCED ? static_cast<float>(best / V) * kUnit : unordered(best);
        if (BALANCED) {
            const bool apart = before - value > doubt<SIGMOID>(value) + 3.f * kUnit;
            // At the range's end all are alike, those that may not be chosen among them (experts of other groups, places past E).  What won there may be any of
            // them, so no winner that counts may be: none of the k, nor the next one where it is a candidate.
            const bool alike = !(value > 1.f - kFar);
            if (!kSettled) unsure |= !apart || alike;
            else if (j < a.k) {
                in_order &= apart;
                unsure |= alike;
            } else if (j == a.k) {
                best_k = apart;
                unsure |= alike && !apart;
            } else best_k1 = apart;
        } else if (!numbered) unsure |= !(before - value > fmaf(fabsf(value), V * 0x1p-23f, V * 0x1p-126f));
        before = value;
        if (sub == j) mine = min(at, E - 1);
    }
    __builtin_amdgcn_wave_barrier();
    if (kSettled) {
        unsure |= !best_k && !best_k1;
        const bool settle = !in_order || !best_k;
        if (__ballot(settle) != 0) {
            const int m = best_k ? a.k : a.k + 1;
            const double c = sub < m ? 1.0 / (1.0 + exp(-static_cast<double>(values[mine]))) + static_cast<double>(a.balance[mine]) : kNone;
            int place = 0, settled = mine;
            for (int i = 0; i <= a.k; ++i) {
                const double other = __shfl(c, i, 16);
                const int e = __shfl(mine, i, 16);
                place += i < m && (other > c || (other == c && e < mine)) ? 1 : 0;
            }
            for (int i = 0; i <= a.k; ++i) {
                const int to = __shfl(place, i, 16), e = __shfl(mine, i, 16);
                settled = i < m && to == sub ? e : settled;
            }
            if (settle) mine = settled;
        }
    }
    unsure |= V > 8 && taken >= 8;                              // what comes next in the lane is not known
    float p = 1.f;
    if (sub < a.k) {
        const double l = static_cast<double>(values[mine]);
        p = SIGMOID ? 1.f / (1.f + exp_of(-l)) : exp_of(l - static_cast<double>(most)) / total;
    }
    unsure |= !(p > 0x1p-100f);
    unsure = (__ballot(unsure) >> (threadIdx.x & 48) & 0xffffu) != 0;
    float sum = 1.f;
    if (a.renormalize) {
        sum = 0.f;
        for (int j = 0; j < a.k; ++j) sum += __shfl(p, j, 16);
    }
    if (live && !unsure && sub < a.k) {
        a.idx[t * a.k + sub] = mine;
        a.weight[t * a.k + sub] = p / sum * a.scale;
        atomicAdd(&hist[mine], 1);                              // LDS, whole numbers: the order does not matter
    }
    return !unsure;
}

// Counts -> offsets and hot mask, by a block of at least E threads, thread e with expert e's count.
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

// A block takes `tokens` tokens, 4 per wavefront at a time.  ONE: it is the only block and goes on to the outputs of the
// counts; else its counts go to the workspace, [block][E] of 16 bits.  16384 tokens of 256 experts, k = 8, take 20 us of the 24 with the counts; all of it in 64 bits
// 99; one token 7 us.  Of these 20 the vector units work 0.53 (1504 instructions per four tokens, the tokens in doubt with them, two wavefronts to a SIMD), beside half as
// many scalar instructions; a wavefront waits 0.43 of its time, for the first loads, for LDS and from one round's reductions to the next's.
template <int V>
constexpr int kRouteScoreWaves = V <= 16 ? 8 : 4;
template <int V, bool SIGMOID, bool BALANCED, bool ONE>
__global__ __launch_bounds__(kRouteScoreWaves<V> * 64) void route_scores_kernel(const ScoreArgs a, int tokens) {
    static_assert(!ONE || 16 * V <= kRouteScoreWaves<V> * 64, "a thread for each expert");
    extern __shared__ __align__(16) unsigned char lds[];
    int32_t* hist = reinterpret_cast<int32_t*>(lds);            // [E], then [E] and kScanInts ints for finish_counts
    unsigned char* rows = lds + (2 * a.E + kScanInts + 3) / 4 * 16;
    for (int e = threadIdx.x; e < a.E; e += kRouteScoreWaves<V> * 64) hist[e] = 0;
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, slot = lane >> 4;
    const long first = static_cast<long>(blockIdx.x) * tokens, last = min(first + tokens, static_cast<long>(a.T));
    unsigned char* mine = rows + wave * score_wave_bytes(a.E);
    float* values = reinterpret_cast<float*>(mine + score_row_bytes(a.E));
    unsigned char* group = mine + 2 * score_row_bytes(a.E);
#pragma unroll 1
    for (long t0 = first + wave * 4; t0 < last; t0 += 4 * kRouteScoreWaves<V>) {
        const long t = t0 + slot;
        const bool live = t < last;
        bool sure = false;
        if (a.groups <= kFastGroups)
            sure = choose<V, SIGMOID, BALANCED>(a, mine, lane, live, t, last, hist);
        uint64_t left = __ballot(!sure && live && (lane & 15) == 0);
#pragma unroll 1
        while (left != 0) {
            const int n = __builtin_ctzll(left) >> 4;
            left &= left - 1;
            __builtin_amdgcn_wave_barrier();
            choose_exactly(a, reinterpret_cast<double*>(mine), values + n * a.E, a.groups <= kFastGroups, reinterpret_cast<double*>(group), lane, t0 + n, hist);
            __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
    if constexpr (ONE) {
        finish_counts(a, static_cast<int>(threadIdx.x) < a.E ? hist[threadIdx.x] : 0, hist + a.E, hist + 2 * a.E);
    } else {
        uint16_t* out = reinterpret_cast<uint16_t*>(a.hist) + static_cast<size_t>(blockIdx.x) * ((a.E + 7) & ~7);
        for (int e = threadIdx.x; e < ((a.E + 7) & ~7); e += blockDim.x) out[e] = static_cast<uint16_t>(e < a.E ? hist[e] : 0);
    }
}

// The blocks' counts, eight experts per load.
__global__ __launch_bounds__(1024) void route_counts_kernel(const ScoreArgs a, int chunks) {
    __shared__ int32_t total[MOE_MAX_E + 8], cnt[MOE_MAX_E], scan[kScanInts];
    const int wide = (a.E + 7) / 8, groups = 1024 / wide, q = threadIdx.x / wide, at = threadIdx.x - q * wide;
    for (int e = threadIdx.x; e < 8 * wide; e += 1024) total[e] = 0;
    __syncthreads();
    if (q < groups) {
        const uint4* from = reinterpret_cast<const uint4*>(a.hist) + at;
        int sum[8] = {};
#pragma unroll 4
        for (int c = q; c < chunks; c += groups) {
            const uint4 v = from[static_cast<size_t>(c) * wide];
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[2 * i] += w[i] & 0xffffu;
                sum[2 * i + 1] += w[i] >> 16;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (sum[i] != 0) atomicAdd(&total[8 * at + i], sum[i]);
    }
    __syncthreads();
    finish_counts(a, static_cast<int>(threadIdx.x) < a.E ? total[threadIdx.x] : 0, cnt, scan);
}

}  // namespace

namespace {

template <typename ST, int TF, int NF>
hipError_t launch_gate_tile(const moe_shape& s, const ST* x, const ST* wg, const float* bias, float* logits, hipStream_t stream) {
    using G = GateTile<TF, NF>;
    constexpr long kMost = 0xffffffffl / (kGateTileWaves * 64) / 8 * 8;        // blocks of a launch, which counts at most 2^32 - 1 threads
    const int groups = (s.E + G::kExperts - 1) / G::kExperts;
    const long most = kMost / groups * G::kTokens;
    for (long t0 = 0; t0 < s.T; t0 += most) {
        const int tokens = static_cast<int>(std::min(s.T - t0, most));
        const long blocks = (tokens + G::kTokens - 1l) / G::kTokens * groups;
        gate_tile_kernel<ST, TF, NF><<<dim3(static_cast<unsigned>((blocks + 7) / 8 * 8)), dim3(kGateTileWaves * 64), G::kLdsBytes, stream>>>(
            x + t0 * s.d_model, wg, bias, logits + t0 * s.E, tokens, s.d_model, s.E, groups);
    }
    return hipGetLastError();
}
template <typename ST>
hipError_t launch_gate(const moe_shape& s, const ST* x, const ST* wg, const float* bias, float* logits, hipStream_t stream) {
    const int tokens = (s.T + 15) / 16;
    const bool pieces = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(wg)) & 15) == 0 && s.d_model % Piece<ST>::kValues == 0;
    // Of the first kernel a block per CU (two in 32 bits) at the most, and the second from there on; at the next power of two of tokens, the first and the
    // second, d_model 2048: bf16, 512 tokens x 256 experts 9.3 and 8.6 us, 1024 tokens 16.4 and 8.9; f32, 512 tokens 16.7 and 25.6, 1024 tokens 31.6 and 25.8.
    // Up to 16 experts leave three quarters of the second's products unused, which counts in 32 bits: 16384 tokens x 8 experts 28.1 and 42.2 (bf16 17.3 and 12.5).
    constexpr bool kWide = sizeof(ST) == 4;
    if (pieces && static_cast<long>(tokens) * ((s.E + 15) / 16) > (kWide ? 512 : 256) && !(kWide && s.E <= 16)) {
        // As few tokens per block as make one round of the CUs, a block each, or the most: 5003 tokens x 256 experts x 2048 in blocks of 16, 32, 48 and
        // 64 tokens 26.1, 20.9, 13.9 and 15.4 us.
        const int columns = s.E <= 64 ? 1 : (s.E + 127) / 128, cus = device_cu_count();
        const int tf = static_cast<int>(std::min(4l, (static_cast<long>(tokens) * columns + cus - 1) / cus));
        if (s.E <= 64) {
            if (tf == 4) return launch_gate_tile<ST, 4, 1>(s, x, wg, bias, logits, stream);
            if (tf == 3) return launch_gate_tile<ST, 3, 1>(s, x, wg, bias, logits, stream);
            if (tf == 2) return launch_gate_tile<ST, 2, 1>(s, x, wg, bias, logits, stream);
            return launch_gate_tile<ST, 1, 1>(s, x, wg, bias, logits, stream);
        }
        if (tf == 4) return launch_gate_tile<ST, 4, 2>(s, x, wg, bias, logits, stream);
        if (tf == 3) return launch_gate_tile<ST, 3, 2>(s, x, wg, bias, logits, stream);
        if (tf == 2) return launch_gate_tile<ST, 2, 2>(s, x, wg, bias, logits, stream);
        return launch_gate_tile<ST, 1, 2>(s, x, wg, bias, logits, stream);
    }
    constexpr int kMost = 65535;               // blocks of the grid's second direction
    for (int t0 = 0; t0 < tokens; t0 += kMost) {
        const long row = 16l * t0;
        const dim3 grid((s.E + 15) / 16, std::min(tokens - t0, kMost)), block(kGateWaves * 64);
        gate_few_kernel<<<grid, block, 0, stream>>>(x + row * s.d_model, wg, bias, logits + row * s.E, static_cast<int>(s.T - row), s.d_model, s.E);
    }
    return hipGetLastError();
}
template <typename ST>
hipError_t configure_gate() {
    auto allow = [](const void* kernel, int bytes) { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
    hipError_t e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 4, 1>), GateTile<4, 1>::kLdsBytes)) != hipSuccess) return e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 4, 2>), GateTile<4, 2>::kLdsBytes)) != hipSuccess) return e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 3, 1>), GateTile<3, 1>::kLdsBytes)) != hipSuccess) return e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 2, 1>), GateTile<2, 1>::kLdsBytes)) != hipSuccess) return e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 3, 2>), GateTile<3, 2>::kLdsBytes)) != hipSuccess) return e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 2, 2>), GateTile<2, 2>::kLdsBytes)) != hipSuccess) return e;
    if ((e = allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 1, 1>), GateTile<1, 1>::kLdsBytes)) != hipSuccess) return e;
    return allow(reinterpret_cast<const void*>(gate_tile_kernel<ST, 1, 2>), GateTile<1, 2>::kLdsBytes);
}

}  // namespace

hipError_t launch_gate_logits(const moe_shape& s, const void* x, const void* w_gate, const float* bias, float* logits, hipStream_t stream) {
    if (s.dtype == MOE_BF16) return launch_gate(s, static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(w_gate), bias, logits, stream);
    return launch_gate(s, static_cast<const float*>(x), static_cast<const float*>(w_gate), bias, logits, stream);
}

// Tokens up to which one block does all, instead of several and a second launch that adds up their counts: 32 tokens x 256 experts 9.6 and 11.8 us
// (x 8 experts 3.7 and 5.9), 64 tokens 16.9 and 11.8 (5.3 and 6.1).
constexpr int kOneBlockTokens = 32;
constexpr long kRouteBlocks = 256;         // 512, which two to a CU would do: 24.0 for 25.1 us of 16384 tokens x 256 experts, and 0.4 us more for the counts

template <int V, bool SIGMOID, bool BALANCED>
static hipError_t launch_scores(const ScoreArgs& a, hipStream_t stream) {
    constexpr int kPass = 4 * kRouteScoreWaves<V>;
    const dim3 threads(64 * kRouteScoreWaves<V>);
    const size_t lds = (2 * a.E + kScanInts + 3) / 4 * 16 + kRouteScoreWaves<V> * score_wave_bytes(a.E);
    if constexpr (V <= 16) {
        if (a.T <= kOneBlockTokens) {
            route_scores_kernel<V, SIGMOID, BALANCED, true><<<dim3(1), threads, lds, stream>>>(a, a.T);
            return hipGetLastError();
        }
    }
    // a block for each CU, of as few tokens as that gives, as far as there is place for the blocks' counts, but no more than 16 bits count
    const long place = (static_cast<long>(a.T + 15) / 16 + 1) * a.E * 4, most = std::min(kRouteBlocks, std::max(1l, place / (2 * ((a.E + 7) & ~7))));
    const long tokens = std::min((a.T + most - 1) / most + kPass - 1, 0xffffl) / kPass * kPass;
    const int chunks = static_cast<int>((a.T + tokens - 1) / tokens);
    route_scores_kernel<V, SIGMOID, BALANCED, false><<<dim3(chunks), threads, lds, stream>>>(a, static_cast<int>(tokens));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    route_counts_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a, chunks);
    return hipGetLastError();
}
// go(V, SIGMOID, BALANCED) of the variant for a call.
template <typename Go>
static hipError_t with_score_variant(int E, bool sigmoid, bool balanced, Go go) {
    auto of = [&](auto v) {
        if (sigmoid) return balanced ? go(v, std::true_type{}, std::true_type{}) : go(v, std::true_type{}, std::false_type{});
        return balanced ? go(v, std::false_type{}, std::true_type{}) : go(v, std::false_type{}, std::false_type{});
    };
    if (E <= 64) return of(std::integral_constant<int, 4>{});
    if (E <= 128) return of(std::integral_constant<int, 8>{});
    if (E <= 256) return of(std::integral_constant<int, 16>{});
    return of(std::integral_constant<int, 64>{});
}

hipError_t launch_route_logits(const ScoreArgs& a, hipStream_t stream) {
    if (a.T == 0) {
        route_counts_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a, 0);
        return hipGetLastError();
    }
    return with_score_variant(a.E, a.sigmoid, a.balance != nullptr, [&](auto v, auto sigmoid, auto balanced) {
        return launch_scores<decltype(v)::value, decltype(sigmoid)::value, decltype(balanced)::value>(a, stream);
    });
}

static hipError_t allow_lds(const void* kernel) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kLdsPerCu));
}
hipError_t configure_score_kernels() {
    static_assert((2 * MOE_MAX_E + kScanInts + 3) / 4 * 16 + kRouteScoreWaves<64> * score_wave_bytes(MOE_MAX_E) <= static_cast<int>(kLdsPerCu), "fits a CU");
    hipError_t e = configure_gate<uint16_t>();
    if (e == hipSuccess) e = configure_gate<float>();
    if (e != hipSuccess) return e;
    for (int E : {64, 128, 256, MOE_MAX_E})
        for (int sigmoid = 0; sigmoid < 2; ++sigmoid)
            for (int balanced = 0; balanced < 2; ++balanced) {
                e = with_score_variant(E, sigmoid != 0, balanced != 0, [](auto v, auto s, auto b) {
                    constexpr int V = decltype(v)::value;
                    if constexpr (V <= 16) {
                        const hipError_t e = allow_lds(reinterpret_cast<const void*>(route_scores_kernel<V, decltype(s)::value, decltype(b)::value, true>));
                        if (e != hipSuccess) return e;
                    }
                    return allow_lds(reinterpret_cast<const void*>(route_scores_kernel<V, decltype(s)::value, decltype(b)::value, false>));
                });
                if (e != hipSuccess) return e;
            }
    return hipSuccess;
}

}  // namespace moe
