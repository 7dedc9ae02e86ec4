// Products on int8 rows with a scale per row and per output channel, for one weight matrix and grouped by expert:
//
//   out[p, n] = act( sa[row(p)] * sw[e, n] * sum_c a[row(p), c] * w[e, n, c] + bias[e, n] )
//
// Sums are int32 and exact (K <= 131071), however the contraction is cut and in whatever order it is added up; scales, bias and activation are
// fp32.  The weights are the matrix instruction's first operand, so that a lane's results are four columns of one row.
#include <algorithm>
#include <type_traits>

#include "int8.hpp"
#include "quant_units.hpp"

namespace moe {

namespace {

// Lane l holds 16 codes of row l % 16 of each operand, for each half of a block of 128 columns; which columns they are does not matter as long
// as both operands agree.  Result i of lane l: weight row 4 (l / 16) + i, token row l % 16.
__device__ __forceinline__ i32x4 multiply(const i32x8& w, const i32x8& x, i32x4 sum) {
    sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_shufflevector(w, w, 0, 1, 2, 3), __builtin_shufflevector(x, x, 0, 1, 2, 3), sum, 0, 0, 0);
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_shufflevector(w, w, 4, 5, 6, 7), __builtin_shufflevector(x, x, 4, 5, 6, 7), sum, 0, 0, 0);
}

// SMOOTH: GeLU or SiLU, else none or ReLU, the kernels' variants (every one in each of a kernel's many epilogues is more code than its cache holds).
bool is_smooth(int act) { return act == MOE_ACT_GELU || act == MOE_ACT_SILU; }
template <bool SMOOTH>
__device__ __forceinline__ float int_activate(float v, int act) {
    if constexpr (SMOOTH) return act == MOE_ACT_GELU ? gelu_exp(v) : silu(v);
    const float least = act == MOE_ACT_RELU ? 0.f : -__builtin_huge_valf();
    return v < least ? least : v;                           // NaN stays
}
// A lane's sums of a fragment of 16 columns x 16 rows as values: sx of its row, sw and bias of its four columns.
template <bool SMOOTH>
__device__ __forceinline__ f32x4 finish_fragment(int act, float sx, const f32x4& w, const f32x4& b, const i32x4& sums) {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = int_activate<SMOOTH>(fmaf(static_cast<float>(sums[i]), sx * w[i], b[i]), act);
    return v;
}
// The same for NF fragments of columns x TF of rows; sw and bias (or NULL): the lane's columns' in LDS.
template <bool SMOOTH, int NF, int TF>
__device__ __forceinline__ void finish(int act, const float (&sx)[TF], const unsigned char* sw, const unsigned char* bias, const i32x4 (&sums)[NF][TF],
                                       f32x4 (&v)[NF][TF]) {
#pragma unroll
    for (int nf = 0; nf < NF; ++nf) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(sw + nf * 64);
        f32x4 b = {0.f, 0.f, 0.f, 0.f};
        if (bias != nullptr) b = *reinterpret_cast<const f32x4*>(bias + nf * 64);
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) {
            v[nf][tf] = finish_fragment<SMOOTH>(act, sx[tf], w, b, sums[nf][tf]);
            if (NF * TF > 4) __builtin_amdgcn_sched_barrier(0);        // many values at once would need registers that there are not
        }
    }
}

// ---- few rows per matrix: the weights are streamed -------------------------------------------------------------------
// Unit: an expert's rows, at most 64, x 16 NF columns for each of W wavefronts, a block of 128 columns of the contraction per step: 8 wavefronts, or 4
// where units of 128 columns leave half of the CUs without one.  Bound by memory: what matters is that copies never stop.  Weights and rows go to LDS directly,
// through a ring of stages that runs on across units; a unit's scales and bias go before its first stage to a place of their own: one more than there are
// stages, for units of one step.
// Two experts of 8192 x 2048, a row each, 8.3 us (34 MB), of which a launch is 3.5.
constexpr int kStreamRows = 64, kStreamWaves = 8;
template <int NF, int W>
struct Streams {
    static constexpr int kStages = NF * W == 4 ? 8 : NF == 1 ? 6 : 3, kCols = NF * W * 16, kRowCopies = 8 / W;
    static constexpr int kX = kCols * kQuantBlock, kStage = kX + kStreamRows * kQuantBlock;
    static constexpr int kUnits = kStages * kStage, kPlaces = kStages + 1, kSw = 256, kBias = kSw + kCols * 4, kUnit = kBias + kCols * 4;       // of a unit: scales of rows, columns, bias
    static constexpr int kList = kUnits + kPlaces * kUnit, kLdsBytes = kList + MOE_MAX_E * 2 + W * 4;
    static constexpr int kCopies = 2 * NF + kRowCopies;          // a wavefront's, per stage
    static_assert(kLdsBytes <= 160 * 1024, "fits a CU");
};

// OUT = kOutParts: the contraction is cut into `split` parts, whose sums go to a.out as [split][rows][pitch of N] int32.
constexpr int kOutParts = 3;

template <int OUT, int NF, bool SMOOTH, int W = kStreamWaves>
__device__ __forceinline__ void stream_units(const QuantArgs& a, const uint16_t* list, int tiles, int parts_wanted, int b, int G, unsigned char* smem) {
    using S = Streams<NF, W>;
    constexpr int kStages = S::kStages, kStage = S::kStage;
    const int split = OUT == kOutParts ? parts_wanted : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int KB = quant_blocks(a.K), blocks = quant_blocks(a.N), groups = (blocks * 8 + NF * W - 1) / (NF * W);
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const int per_tile = groups * split, units = tiles * per_tile;

    // Block b of G.  Every block gets the same number of units, as few as the grid allows: a CU can pull more than its share of the memory's rate, so
    // that a quarter of them idle costs nothing, but a last round of a few units does.  The runs are dealt to the XCDs evenly.
    const int rounds = (units + G - 1) / G, runs = rounds > 0 ? (units + rounds - 1) / rounds : 0;
    const int per_xcd = (runs + 7) >> 3;
    const int run = G % 8 == 0 ? (b >> 3 < per_xcd ? (b & 7) * per_xcd + (b >> 3) : runs) : b;
    const int first = run * rounds, last = min(units, first + rounds);
    if (first >= last) return;

    struct Unit {
        int tile, rest, e, row0, rows, group, kb, kb1, part;    // number `rest` of row tile `tile`
    };
    auto unit_at = [&](int t, int rest) __attribute__((always_inline)) {
        Unit w;
        w.tile = t;
        w.rest = rest;
        w.e = __builtin_amdgcn_readfirstlane(static_cast<int>(list[t]));
        const Segment seg = segment_of_unit(a, w.e);
        w.row0 = seg.row0;
        w.rows = seg.rows;
        w.group = rest / split;
        w.part = rest - w.group * split;
        w.kb = KB * w.part / split;
        w.kb1 = KB * (w.part + 1) / split;
        return w;
    };
    // the next unit of the run, in the same row tile: nothing is looked up
    auto along = [&](Unit w) __attribute__((always_inline)) {
        const int part = w.part + 1, over = part == split ? 1 : 0;
        w.part = over ? 0 : part;
        w.group += over;
        w.rest += 1;
        w.kb = KB * w.part / split;
        w.kb1 = KB * (w.part + 1) / split;
        return w;
    };

    // copies: wavefront w brings rows 8 w ... 8 w + 7 (and 8 (w + W) ...), weight fragments NF w ..., and of a unit 64 of its columns' scales or biases and
    // (all the same) the rows' scales
    const uint32_t lds = lds_address(smem);
    const uint32_t to_weights = lds + wave * NF * kFragBytes, to_rows = lds + S::kX + wave * 1024;
    constexpr int kPieces = S::kCols / 64;
    const int piece = wave % (2 * kPieces);
    const uint8_t *tile_row[S::kRowCopies], *weights_from;
    size_t in_row = 0;
    const float* tile_scale;
    int unit_in = 0;                        // place of the next unit's scales
    auto point_at_tile = [&](const Unit& w) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::kRowCopies; ++i) {
            const int in_tile = (wave + i * W) * 8 + (lane >> 3);
            tile_row[i] = a.a + source_row(a, w.row0 + min(in_tile, w.rows - 1)) * pitch + piece_of_lane(lane, in_tile);
        }
        tile_scale = a.a_scales + source_row(a, w.row0 + min(lane, w.rows - 1));
    };
    auto point_at = [&](const Unit& w) __attribute__((always_inline)) {
        in_row = static_cast<size_t>(w.kb) * kQuantBlock;
        // columns of the last unit that do not exist are read as the last ones that do, and not stored
        const int fragment = min((w.group * W + wave) * NF, blocks * 8 - NF);
        weights_from = a.w + static_cast<size_t>(w.e) * quant_matrix_bytes(a.N, a.K) + (static_cast<size_t>(fragment) * KB + w.kb) * kFragBytes + lane * 16;
        if constexpr (OUT != kOutParts) {
            const float* from = piece < kPieces || a.bias == nullptr ? a.w_scales : a.bias;
            const uint32_t to = lds + S::kUnits + unit_in * S::kUnit;
            copy4_to_lds(from + static_cast<size_t>(w.e) * a.N + min(w.group * S::kCols + (piece % kPieces) * 64 + lane, a.N - 1), to + S::kSw + piece * 256);
            copy4_to_lds(tile_scale, to);
            unit_in = unit_in == S::kPlaces - 1 ? 0 : unit_in + 1;
        }
    };
    auto stage_in = [&](int slot) {
        const int at = slot * kStage;
        auto weights = [&](auto copy) __attribute__((always_inline)) {
#pragma unroll
            for (int nf = 0; nf < NF; ++nf) {
                const uint8_t* from = weights_from + static_cast<size_t>(nf) * KB * kFragBytes;
                copy(from, to_weights + at + nf * kFragBytes);
                copy(from + 1024, to_weights + at + nf * kFragBytes + 1024);
            }
        };
        if (a.once) weights([](const void* from, uint32_t to) __attribute__((always_inline)) { copy16_once_to_lds(from, to); });
        else weights([](const void* from, uint32_t to) __attribute__((always_inline)) { copy16_to_lds(from, to); });
#pragma unroll
        for (int i = 0; i < S::kRowCopies; ++i) copy16_to_lds(tile_row[i] + in_row, to_rows + at + i * W * 1024);
        weights_from += kFragBytes;
        in_row += kQuantBlock;
    };

    const int tile0 = first / per_tile;
    Unit ahead = unit_at(tile0, first - tile0 * per_tile);      // the unit that is being copied
    int units_in = last - first, units_out = units_in;
    point_at_tile(ahead);
    point_at(ahead);
    int slot_in = 0;
    bool copying = true;
    auto copy_next = [&]() __attribute__((always_inline)) {
        if (copying) {
            stage_in(slot_in);
        } else {
            // nothing left to copy: copies of some row to the slot that has fallen free keep up the count that the waits go by
#pragma unroll
            for (int i = 0; i < S::kCopies; ++i) copy16_to_lds(tile_row[0], to_rows + slot_in * kStage);
        }
        slot_in = slot_in == kStages - 1 ? 0 : slot_in + 1;
        ++ahead.kb;
        if (ahead.kb == ahead.kb1) {
            if (--units_in > 0) {
                if (ahead.rest + 1 == per_tile) {
                    ahead = unit_at(ahead.tile + 1, 0);
                    point_at_tile(ahead);
                } else {
                    ahead = along(ahead);
                }
                point_at(ahead);
            } else {
                copying = false;
            }
        }
    };
#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) copy_next();

    Unit cur = unit_at(tile0, first - tile0 * per_tile);
    const int at_w = wave * NF * kFragBytes + lane * 16, at_x = S::kX + row_operand(threadIdx.x, 0), x_other = row_operand_other(at_x);
    const int at_columns = (wave * NF * 16 + (lane >> 4) * 4) * 4;
    int slot = 0, unit = 0;
    while (true) {
        auto run_unit = [&](auto tf_const) __attribute__((always_inline)) {
            constexpr int TF = decltype(tf_const)::value;
            i32x4 acc[NF][TF];
#pragma unroll
            for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) acc[nf][tf] = i32x4{0, 0, 0, 0};
            for (; cur.kb < cur.kb1; ++cur.kb) {
                copies_landed<(kStages - 2) * S::kCopies>();
                const unsigned char* st = smem + slot * kStage;
                i32x8 w[NF], x[TF];
#pragma unroll
                for (int nf = 0; nf < NF; ++nf) w[nf] = read_codes(st + at_w + nf * kFragBytes, 1024);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) x[tf] = read_codes(st + at_x + tf * kFragBytes, x_other);
                copy_next();
#pragma unroll
                for (int tf = 0; tf < TF; ++tf)
#pragma unroll
                    for (int nf = 0; nf < NF; ++nf) acc[nf][tf] = multiply(w[nf], x[tf], acc[nf][tf]);
                slot = slot == kStages - 1 ? 0 : slot + 1;
            }
            const int n0 = cur.group * S::kCols + wave * NF * 16;
            if constexpr (OUT == kOutParts) {
                static_assert(NF == 1, "calls of few rows are cut, which have few columns per unit");
                int32_t* parts = static_cast<int32_t*>(a.out) + static_cast<size_t>(cur.part) * a.rows * quant_pitch(a.N);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf)
                    if (tf * 16 + r < cur.rows)
                        *reinterpret_cast<i32x4*>(parts + static_cast<size_t>(cur.row0 + tf * 16 + r) * quant_pitch(a.N) + n0 + (lane >> 4) * 4) =
                            acc[0][tf];
            } else {
                // they came before the unit's first stage, which has been waited for
                const unsigned char* of = smem + S::kUnits + unit * S::kUnit;
                float sx[TF];
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) sx[tf] = *reinterpret_cast<const float*>(of + (tf * 16 + r) * 4);
                f32x4 v[NF][TF];
                finish<SMOOTH>(a.act, sx, of + S::kSw + at_columns, a.bias != nullptr ? of + S::kBias + at_columns : nullptr, acc, v);
                store_values<OUT, 16>(a, n0, cur.row0, cur.rows, v);
                unit = unit == S::kPlaces - 1 ? 0 : unit + 1;
            }
        };
        const int tf = (cur.rows + 15) >> 4;
        if (tf == 1) run_unit(std::integral_constant<int, 1>{});
        else if (tf == 2) run_unit(std::integral_constant<int, 2>{});
        else if (tf == 3) run_unit(std::integral_constant<int, 3>{});
        else run_unit(std::integral_constant<int, 4>{});
        if (--units_out == 0) break;
        cur = cur.rest + 1 == per_tile ? unit_at(cur.tile + 1, 0) : along(cur);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no copy may land in LDS that is another block's by then
}

constexpr int kListAt = std::max({Streams<1, 4>::kList, Streams<1, kStreamWaves>::kList, Streams<2, kStreamWaves>::kList});       // behind every ring
constexpr int kStreamLds = kListAt + MOE_MAX_E * 2 + kStreamWaves * 4;
static_assert(kStreamLds <= 160 * 1024, "fits a CU");

template <int OUT, bool SMOOTH, int W>
__global__ __launch_bounds__(W * 64) void int_stream_kernel(const QuantArgs a, int max_rows, int parts_wanted) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* list = reinterpret_cast<uint16_t*>(smem + kListAt);
    const int tiles = list_experts<W * 64>(a, max_rows, list, reinterpret_cast<int32_t*>(list + MOE_MAX_E));
    stream_units<OUT, 1, SMOOTH, W>(a, list, tiles, parts_wanted, blockIdx.x, gridDim.x, smem);
}

// Adds up the parts of a split contraction and finishes the rows.  A block of threads per row and 1024 columns, four per thread.
template <int OUT, bool SMOOTH>
__global__ __launch_bounds__(256) void int_join_kernel(const QuantArgs a, const int32_t* __restrict__ parts, int split) {
    const int row = blockIdx.x, n0 = (blockIdx.y * 256 + threadIdx.x) * 4;
    const size_t pitch = quant_pitch(a.N);
    i32x4 sum = {0, 0, 0, 0};
    if (n0 < a.N) {
        const int32_t* p = parts + static_cast<size_t>(row) * pitch + n0;
        const size_t stride = static_cast<size_t>(a.rows) * pitch;
#pragma unroll 4
        for (int s = 0; s < split; ++s) sum += *reinterpret_cast<const i32x4*>(p + s * stride);
    }
    int e = 0;
    if (a.offsets != nullptr) {            // the expert whose rows this one is among: as many end at or before it as precede that
        for (int e0 = 0; e0 < a.E; e0 += 256) e += __syncthreads_count(e0 + static_cast<int>(threadIdx.x) < a.E && a.offsets[e0 + threadIdx.x + 1] <= row);
        if (e >= a.E) return;
        const Segment seg = segment_of(a, e);
        if (row < seg.row0 || row >= seg.row0 + seg.rows) return;
    }
    const float sx = a.a_scales[source_row(a, row)];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n0 + i < a.N) {
            const size_t of = static_cast<size_t>(e) * a.N + n0 + i, at = static_cast<size_t>(row) * a.N + n0 + i;
            const float v = int_activate<SMOOTH>(fmaf(static_cast<float>(sum[i]), sx * a.w_scales[of], a.bias != nullptr ? a.bias[of] : 0.f), a.act);
            if constexpr (OUT == kOutF32) static_cast<float*>(a.out)[at] = v;
            else static_cast<uint16_t*>(a.out)[at] = f32_to_bf16(v);
        }
}

// ---- many rows per matrix: tiles in LDS -----------------------------------------------------------------------------
// Unit: 64 R rows (R = 1, 2, 4) x 128 columns by 8 wavefronts, a block of 128 columns of the contraction per step, through a ring of
// LDS stages that runs on across units.  Everything goes from memory to LDS directly, 16 bytes per lane; a stage holds
//   rows     [64 RMAX][128 bytes]
//   weights  8 fragments of 2 KiB as they are packed, 16 rows each
// and a unit's scales and biases go before its first stage to a place of their own, one more than there are stages.
// Wavefront (wm, wn) of the 4 x 2 multiplies row fragments wm, wm + 4, ... (R of them) and the columns 64 wn ... 64 wn + 63.
// Bound by a step's copies and its barrier: 16384 x 8192 x 2048, bf16 out, 276 to 287 us (1920 to 1990 TOP/s, matrix units busy 0.41 at 1.9 GHz), 2048 x 4096 x 4096
// 37 (1840), 1501 x 1024 x 4096 15.2.  The sums of a tile of 256 rows wait in registers until the next tile's steps finish and store them (299 us without).
constexpr int kTileWaves = 8;
template <int RMAX>
struct Tiles {
    static constexpr int kRows = 64 * RMAX, kStages = RMAX == 4 ? 3 : RMAX == 2 ? 4 : 6;
    static constexpr int kStageW = kRows * kQuantBlock, kStage = kStageW + kQuantBlock * kQuantBlock;
    static constexpr int kUnits = kStages * kStage, kPlaces = kStages + 1, kSw = kRows * 4, kBias = kSw + 512, kUnit = kBias + 512;
    static constexpr int kStarts = kUnits + kPlaces * kUnit;
    static constexpr int kLdsBytes = kStarts + kTileWaves * 16 + (MOE_MAX_E + 1) * 4 + MOE_MAX_E * 2;
    static constexpr int kCopies = RMAX + 2;            // a wavefront's, per stage
    static_assert(kLdsBytes <= 160 * 1024, "fits a CU");
};

// What there is to do of a grouped product, counted by every block for itself (a list in memory would cost a launch): experts of at least min_rows rows run in
// tiles of tile_rows rows.  whole[e] is the number of whole tiles that the experts before e have, whole[E] that of all (at most as many as the rows have, so
// that offsets that are none do not overflow what follows); `rest` lists the experts with a shorter last tile, those of more than 128 rows first, then of more
// than 64, then the others.  `tmp`: four ints per wavefront.  One matrix: all rows are its.
struct Work {
    int whole, last[3], streamed;          // tiles; last tiles by length; experts of fewer rows
};
template <int THREADS>
__device__ __forceinline__ Work count_work(const QuantArgs& a, int tile_rows, int min_rows, int32_t* whole, uint16_t* rest, int4* tmp) {
    constexpr int W = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, most = a.rows / tile_rows;
    const int least = a.offsets == nullptr ? 1 : min_rows;
    int4 before = {0, 0, 0, 0};            // whole tiles; last tiles by length, streamed experts: 16 bits each hold 1024
    int base1 = 0, base2 = 0;
    // the lengths' totals are needed before the first expert's place is known: first pass counts, second one places
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1) {
            base1 = before.y & 0xffff;
            base2 = base1 + (before.y >> 16);
            if (threadIdx.x == 0) whole[a.E] = before.x;
            before = int4{0, 0, 0, 0};
        }
        for (int e0 = 0; e0 < a.E; e0 += THREADS) {
            const int e = e0 + threadIdx.x;
            const int rows = e < a.E ? segment_of(a, e).rows : 0, m = rows < least ? 0 : rows;
            const int n = m / tile_rows, left = m - n * tile_rows;
            const int kind = left == 0 ? -1 : left > 128 ? 0 : left > 64 ? 1 : 2;
            const int incl = wave_scan(n);
            const uint64_t k0 = __ballot(kind == 0), k1 = __ballot(kind == 1), k2 = __ballot(kind == 2), few = __ballot(rows > 0 && m == 0);
            if (lane == 63) tmp[wave] = int4{incl, __popcll(k0) | __popcll(k1) << 16, __popcll(k2) | __popcll(few) << 16, 0};
            __syncthreads();
            int4 mine = before;
            for (int w = 0; w < W; ++w) {
                const int4 t = tmp[w];
                if (w < wave) mine = int4{min(mine.x + t.x, most), mine.y + t.y, mine.z + t.z, 0};
                before = int4{min(before.x + t.x, most), before.y + t.y, before.z + t.z, 0};
            }
            if (pass == 1) {
                if (e < a.E) whole[e] = min(mine.x + incl - n, most);
                const uint64_t below = (1ull << lane) - 1;
                const int at = kind == 0 ? (mine.y & 0xffff) + __popcll(k0 & below)
                             : kind == 1 ? base1 + (mine.y >> 16) + __popcll(k1 & below)
                                         : base2 + (mine.z & 0xffff) + __popcll(k2 & below);
                if (kind >= 0) rest[at] = static_cast<uint16_t>(e);
            }
            __syncthreads();
        }
    }
    return Work{uniform(before.x), {uniform(before.y & 0xffff), uniform(before.y >> 16), uniform(before.z & 0xffff)}, uniform(before.z >> 16)};
}

template <int RMAX>
__device__ __forceinline__ int32_t* tile_starts(unsigned char* smem) {
    return reinterpret_cast<int32_t*>(smem + Tiles<RMAX>::kStarts + kTileWaves * 16);
}
template <int RMAX>
__device__ __forceinline__ Work count_work(const QuantArgs& a, int min_rows, unsigned char* smem) {
    int32_t* whole = tile_starts<RMAX>(smem);
    return count_work<kTileWaves * 64>(a, Tiles<RMAX>::kRows, min_rows, whole, reinterpret_cast<uint16_t*>(whole + MOE_MAX_E + 1),
                                       reinterpret_cast<int4*>(smem + Tiles<RMAX>::kStarts));
}

// Units first, first + stride, ... before `end`, of the whole tiles' and then the last tiles' (see count_work, which has left their lists).
// PASS: the output passes by the caches.
template <int OUT, int RMAX, bool SMOOTH, bool PASS>
__device__ __forceinline__ void tile_units(const QuantArgs& a, int whole_tiles, int first, int end, int stride, unsigned char* smem) {
    using T = Tiles<RMAX>;
    constexpr int kStages = T::kStages, kStageW = T::kStageW, kStage = T::kStage, tile_rows = T::kRows;
    const int32_t* whole = tile_starts<RMAX>(smem);
    const uint16_t* rest = reinterpret_cast<const uint16_t*>(whole + MOE_MAX_E + 1);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int wm = wave >> 1, wn = wave & 1;
    const int KB = quant_blocks(a.K), groups = quant_blocks(a.N);
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const int whole_units = whole_tiles * groups, units = end;
    int u = first, u_in = u;                // the unit that is computed, and the one that is copied
    if (u >= units) return;

    struct Unit {
        int e, row0, rows, group;
    };
    auto unit_at = [&](int n) __attribute__((always_inline)) {
        Unit w;
        int tile;
        if (n < whole_units) {
            w.e = __builtin_amdgcn_readfirstlane(expert_of(whole, a.E, n / groups));
            const int before = __builtin_amdgcn_readfirstlane(whole[w.e]);
            const int tiles = __builtin_amdgcn_readfirstlane(whole[w.e + 1]) - before, local = n - before * groups;
            // eight column groups of a tile, then the next tile's: 32 neighbours share four tiles' rows and eight groups' weights
            const int band = local / (tiles * 8), width = min(8, groups - band * 8), in_band = local - band * tiles * 8;
            tile = in_band / width;
            w.group = __builtin_amdgcn_readfirstlane(band * 8 + in_band - tile * width);
        } else {
            const int v = n - whole_units, t = v / groups;
            w.e = __builtin_amdgcn_readfirstlane(static_cast<int>(rest[t]));
            tile = __builtin_amdgcn_readfirstlane(whole[w.e + 1] - whole[w.e]);
            w.group = __builtin_amdgcn_readfirstlane(v - t * groups);
        }
        const Segment seg = segment_of_unit(a, w.e);
        w.row0 = seg.row0 + __builtin_amdgcn_readfirstlane(tile * tile_rows);
        w.rows = min(tile_rows, seg.rows - __builtin_amdgcn_readfirstlane(tile * tile_rows));
        return w;
    };

    // copies: wavefront w brings rows 64 i + 8 w ... + 7, weight fragment w, and of a unit 64 rows' or columns' scales or biases
    const uint32_t lds = lds_address(smem);
    const uint32_t to_rows = lds + wave * 1024, to_weights = lds + kStageW + wave * 2048;
    const int piece = wave % (RMAX + 4);
    // Of a stage: the row pieces' offsets from `rows_base` (tiles of 256 rows have no registers for whole addresses; see tile_fragments for
    // operands of more than 4 GiB), the weights' base.
    constexpr bool OFFSETS = RMAX == 4;
    uint32_t row_offset[OFFSETS ? RMAX : 1];
    const uint8_t* row_from[OFFSETS ? 1 : RMAX];
    const uint8_t *rows_base = a.a, *weights_base = a.w;
    const uint32_t lane16 = lane * 16;
    int unit_in = 0;
    auto point_at = [&](const Unit& w) __attribute__((always_inline)) {
        const int lane = here(threadIdx.x) & 63;
#pragma unroll
        for (int i = 0; i < RMAX; ++i) {
            const int in_tile = i * 64 + wave * 8 + (lane >> 3);
            const int row = source_row(a, w.row0 + min(in_tile, w.rows - 1));
            if constexpr (OFFSETS) row_offset[i] = static_cast<uint32_t>(row) * static_cast<uint32_t>(pitch) + piece_of_lane(lane, in_tile);
            else row_from[i] = a.a + row * pitch + piece_of_lane(lane, in_tile);
        }
        rows_base = a.a;
        weights_base = a.w + static_cast<size_t>(w.e) * quant_matrix_bytes(a.N, a.K) + static_cast<size_t>(w.group * 8 + wave) * KB * kFragBytes;
        const float* from;
        if (piece < RMAX) {
            from = a.a_scales + source_row(a, w.row0 + min(piece * 64 + lane, w.rows - 1));
        } else {
            const float* base = piece < RMAX + 2 || a.bias == nullptr ? a.w_scales : a.bias;
            from = base + static_cast<size_t>(w.e) * a.N + min(w.group * kQuantBlock + ((piece - RMAX) & 1) * 64 + lane, a.N - 1);
        }
        copy4_to_lds(from, lds + T::kUnits + unit_in * T::kUnit + piece * 256);
        unit_in = unit_in == T::kPlaces - 1 ? 0 : unit_in + 1;
    };
    Unit ahead = unit_at(u_in);
    point_at(ahead);
    int kb_in = 0, slot_in = 0;
    // The ring runs on across units: the next unit's first stages go out during the last steps of this one.  Behind the last unit the
    // last stage is copied again, which keeps up the count that the waits go by.
    auto copy_piece = [&](int n) __attribute__((always_inline)) {
        const int at = slot_in * kStage;
        if (n < RMAX) {
            if constexpr (OFFSETS) copy16_to_lds(rows_base, row_offset[n < RMAX ? n : 0], to_rows + at + n * 8192);
            else copy16_to_lds(row_from[n < RMAX ? n : 0], to_rows + at + n * 8192);
        } else if (n < RMAX + 2) {
            copy16_to_lds(weights_base + (n - RMAX) * 1024, lane16, to_weights + at + (n - RMAX) * 1024);
        }
    };
    uint32_t stage_step = 1;               // 0 behind the last unit
    auto next_stage = [&]() __attribute__((always_inline)) {
        slot_in = slot_in == kStages - 1 ? 0 : slot_in + 1;
        weights_base += stage_step * kFragBytes;
        if constexpr (OFFSETS) {
            rows_base += stage_step * kQuantBlock;
        } else {
#pragma unroll
            for (int i = 0; i < RMAX; ++i) row_from[i] += stage_step * kQuantBlock;
        }
    };
    // when all of a unit's stages have been sent for (kb_in == KB)
    auto next_unit = [&]() __attribute__((always_inline)) {
        kb_in = 0;
        if (u_in + stride < units) {
            u_in += stride;
            ahead = unit_at(u_in);
            point_at(ahead);
        } else if (stage_step != 0) {      // back to the last stage, which is copied from now on
            weights_base -= kFragBytes;
            if constexpr (OFFSETS) {
                rows_base -= kQuantBlock;
            } else {
#pragma unroll
                for (int i = 0; i < RMAX; ++i) row_from[i] -= kQuantBlock;
            }
            stage_step = 0;
        }
    };
    Unit cur = ahead;
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) {
        if (kb_in == KB) next_unit();
#pragma unroll
        for (int n = 0; n < T::kCopies; ++n) copy_piece(n);
        next_stage();
        ++kb_in;
    }
    copies_landed<(kStages - 1) * T::kCopies>();

    int slot = 0, unit = 0;
    uint32_t landed = 0;                    // steps from here on whose next stage is known to have landed
    // The sums of a unit of all row fragments are finished and stored during the next one's steps, a row fragment at a time (so that no two units' results
    // go to memory at once and the matrix units need not wait for the vector unit), where that has all fragments too and enough steps.
    constexpr int kSpread = 2;              // steps per row fragment
    i32x4 old[4][RMAX];
    Unit done{0, 0, 0, 0};
    int done_place = 0;                     // of its scales
    bool left = false;                      // whether it is still to be finished
    auto columns_of = [&](int place) { return smem + T::kUnits + place * T::kUnit + T::kSw + (wn * 64 + ((here(threadIdx.x) & 63) >> 4) * 4) * 4; };
    auto row_scale = [&](int place, int i) {
        return *reinterpret_cast<const float*>(smem + T::kUnits + place * T::kUnit + (wm * 16 + i * 64 + (here(threadIdx.x) & 15)) * 4);
    };
    auto store_fragments = [&](const Unit& w, int i, const f32x4 (&v)[4][1]) __attribute__((always_inline)) {
        store_values<OUT, 64>(a, w.group * kQuantBlock + wn * 64, w.row0 + wm * 16 + i * 64, w.rows - wm * 16 - i * 64, v);
    };
    // Whether every store of this wavefront's part of a unit is to 16 bytes that exist, so that it takes kStores of them for a row fragment: the steps count
    // on that number.
    constexpr int kStores = OUT == kOutF32 ? 4 : 2;
    auto all_exist = [&](const Unit& w) {
        return a.N % (OUT == kOutF32 ? 4 : 8) == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && w.group * kQuantBlock + wn * 64 + 64 <= a.N &&
               w.rows >= wm * 16 + (RMAX - 1) * 64 + 16;
    };
    auto store_all = [&](const Unit& w, int i, const f32x4 (&v)[4][1]) __attribute__((always_inline)) {
        const int lane = here(threadIdx.x) & 63, g = lane >> 4;
        const size_t at = static_cast<size_t>(w.row0 + wm * 16 + i * 64 + (lane & 15)) * a.N + w.group * kQuantBlock + wn * 64;
        if constexpr (OUT == kOutF32) {
#pragma unroll
            for (int nf = 0; nf < 4; ++nf) {
                f32x4* out = reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at + nf * 16 + g * 4);
                if constexpr (PASS) __builtin_nontemporal_store(v[nf][0], out);
                else *out = v[nf][0];
            }
        } else {
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int nf = 0; nf < 4; ++nf) {
                lo[nf] = pack_bf16x2(v[nf][0][0], v[nf][0][1]);
                hi[nf] = pack_bf16x2(v[nf][0][2], v[nf][0][3]);
            }
#pragma unroll
            for (int t = 0; t < 4; t += 2) {
                gather_pair(lo[t], lo[t + 1]);
                gather_pair(hi[t], hi[t + 1]);
            }
            i32x4* out = reinterpret_cast<i32x4*>(static_cast<uint16_t*>(a.out) + at + g * 8);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const i32x4 piece = {static_cast<int>(lo[2 * t]), static_cast<int>(hi[2 * t]), static_cast<int>(lo[2 * t + 1]), static_cast<int>(hi[2 * t + 1])};
                if constexpr (PASS) __builtin_nontemporal_store(piece, out + 4 * t);
                else out[4 * t] = piece;
            }
        }
    };
    auto finish_now = [&](const Unit& w, int place, const auto& sums, auto fragments) __attribute__((always_inline)) {
        // The stores are counted behind the copies in flight, which have landed when they go out; so the next unit's first steps need not wait
        // for stores.
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        landed = kStages - 1;
        const unsigned char* sw = columns_of(place);
#pragma unroll
        for (int i = 0; i < decltype(fragments)::value; ++i) {
            const float sx = row_scale(place, i);
            f32x4 v[4][1];
#pragma unroll
            for (int nf = 0; nf < 4; ++nf) {
                f32x4 b = {0.f, 0.f, 0.f, 0.f};
                if (a.bias != nullptr) b = *reinterpret_cast<const f32x4*>(sw + T::kBias - T::kSw + nf * 64);
                v[nf][0] = finish_fragment<SMOOTH>(a.act, sx, *reinterpret_cast<const f32x4*>(sw + nf * 64), b, sums[nf][i]);
                __builtin_amdgcn_sched_barrier(0);         // many values at once would need registers that there are not
            }
            store_fragments(w, i, v);
        }
    };
    auto run_unit = [&](auto fragments) __attribute__((always_inline)) {
        constexpr int R = decltype(fragments)::value;
        const int tid = here(threadIdx.x);
        const int at_x = row_operand(tid, wm * 16), x_other = row_operand_other(at_x), at_w = kStageW + wn * 4 * kFragBytes;
        auto row_codes = [&](const unsigned char* st, int i) { return read_codes(st + at_x + i * 64 * kQuantBlock, x_other); };
        auto weight_codes = [&](const unsigned char* st, int nf) { return read_codes(st + at_w + lane16 + nf * kFragBytes, 1024); };
        i32x4 acc[4][R];
#pragma unroll
        for (int nf = 0; nf < 4; ++nf)
#pragma unroll
            for (int i = 0; i < R; ++i) acc[nf][i] = i32x4{0, 0, 0, 0};
        // A step is 4 R pairs of matrix instructions: the first two weight fragments x every row fragment, then the other two.  Operands are
        // read from the next stage into the registers of those that were used last, at least 2 R + 1 pairs (2 of one row fragment) before
        // their use; a stage's slot is free again in the middle of its own step.  The order is held by the scheduling barriers.
        i32x8 w[4], x[R];
        const unsigned char* st0 = smem + slot * kStage;
#pragma unroll
        for (int nf = 0; nf < 4; ++nf) w[nf] = weight_codes(st0, nf);
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = row_codes(st0, i);
        // `more`: stores that went out since the copies that are waited for
        auto step = [&](auto what, auto more) __attribute__((always_inline)) {
            constexpr int M = 4 * R, kFirst = R == 1 ? 0 : M / 2;       // from where on the next stage is read and copies go out
            constexpr int F = decltype(what)::value, kEvery = R == 4 ? 2 : 1;   // row fragment of the unit before that is finished; pairs between its columns
            f32x4 v[4][1], sw, bias = {0.f, 0.f, 0.f, 0.f};
            float sx = 0.f;
            if constexpr (F >= 0) {
                sx = row_scale(done_place, F);
                sw = *reinterpret_cast<const f32x4*>(columns_of(done_place));
                if (a.bias != nullptr) bias = *reinterpret_cast<const f32x4*>(columns_of(done_place) + T::kBias - T::kSw);
            }
            slot = slot == kStages - 1 ? 0 : slot + 1;
            const unsigned char* st = smem + slot * kStage;
#pragma unroll
            for (int n = 0; n < M; ++n) {
                const int half = n / (2 * R), i = n % (2 * R) >> 1, nf = 2 * half + (n & 1);
                if (n == kFirst) {
                    __builtin_amdgcn_sched_barrier(0);
                    copies_landed_unless<(kStages - 2) * T::kCopies + decltype(more)::value>(landed);
                    landed = landed > 0 ? landed - 1 : 0;
                    if (R > 1) {
                        w[0] = weight_codes(st, 0);
                        w[1] = weight_codes(st, 1);
                    }
                }
                acc[nf][i] = multiply(w[nf], x[i], acc[nf][i]);
                __builtin_amdgcn_sched_barrier(0);
                if (R == 1 && n < 2) w[n] = weight_codes(st, n);
                if (half == 1 && i == R - 1) w[nf] = weight_codes(st, nf);
                if (half == 1 && (n & 1)) x[i] = row_codes(st, i);
                if constexpr (F >= 0) {
                    if (n % kEvery == 0 && n / kEvery < 4) {
                        const int c = n / kEvery;
                        v[c][0] = finish_fragment<SMOOTH>(a.act, sx, sw, bias, old[c][F < 0 ? 0 : F]);
                        if (c < 3) {
                            sw = *reinterpret_cast<const f32x4*>(columns_of(done_place) + (c + 1) * 64);
                            if (a.bias != nullptr) bias = *reinterpret_cast<const f32x4*>(columns_of(done_place) + T::kBias - T::kSw + (c + 1) * 64);
                        }
                    }
                    if (n == (R == 1 ? 3 : M / 2)) store_all(done, F, v);
                }
                constexpr int kPer = (T::kCopies + M - kFirst - 1) / (M - kFirst);
#pragma unroll
                for (int c = 0; c < kPer; ++c)
                    if (n >= kFirst) copy_piece((n - kFirst) * kPer + c);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto before_steps = [&]() __attribute__((always_inline)) {
            // behind branches that not every lane takes, such as the stores of the unit before
            u_in = uniform(u_in);
            kb_in = uniform(kb_in);
            slot_in = uniform(slot_in);
            slot = uniform(slot);
            landed = uniform(landed);
            stage_step = uniform(stage_step);
            weights_base = uniform(weights_base);
            if constexpr (OFFSETS) rows_base = uniform(rows_base);
            if (kb_in == KB) {
                // Units of one step: the place that the next unit's scales go to is that of the unit before this one, which every wavefront
                // has to be done with.  Longer units meet in their steps in between.
                if (KB == 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                next_unit();
            }
            // nothing pending on the way in (lgkmcnt(0), the compiler counts with it): the steps wait only for what they read themselves
            __builtin_amdgcn_s_waitcnt(0xc07f);
        };
        int j = 0;
        if constexpr (R == RMAX) if (left) {
            auto with_old = [&](auto f) __attribute__((always_inline)) {
                before_steps();
                step(f, std::integral_constant<int, 0>{});
                next_stage();
                ++kb_in;
                before_steps();
                step(std::integral_constant<int, -1>{}, std::integral_constant<int, R == 1 ? 0 : kStores>{});     // R == 1: they are behind the copies
                next_stage();
                ++kb_in;
            };
            with_old(std::integral_constant<int, 0>{});
            if constexpr (R > 1) with_old(std::integral_constant<int, 1>{});
            if constexpr (R > 2) {
                with_old(std::integral_constant<int, 2>{});
                with_old(std::integral_constant<int, 3>{});
            }
            left = false;
            j = kSpread * R;
        }
        // the steps to the end of the unit or to where the copies go on to the next one: without a branch, so that the order stays
#pragma unroll 1
        while (j < KB) {
            before_steps();
            const int steps = min(KB - j, KB - kb_in);
            j += steps;
            kb_in += steps;
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                step(std::integral_constant<int, -1>{}, std::integral_constant<int, 0>{});
                next_stage();
            }
        }
        if constexpr (R == RMAX) {
#pragma unroll
            for (int nf = 0; nf < 4; ++nf)
#pragma unroll
                for (int i = 0; i < R; ++i) old[nf][i] = acc[nf][i];
            done = cur;
            done_place = unit;
            left = true;
        } else {
            finish_now(cur, unit, acc, fragments);
        }
        unit = unit == T::kPlaces - 1 ? 0 : unit + 1;
    };
    auto all_fragments = [&](const Unit& w) { return RMAX == 1 || w.rows > 32 * RMAX; };
    while (true) {
        if (all_fragments(cur)) run_unit(std::integral_constant<int, RMAX>{});
        else if (RMAX < 4 || cur.rows <= 64) run_unit(std::integral_constant<int, (RMAX > 1 ? 1 : RMAX)>{});
        else run_unit(std::integral_constant<int, (RMAX > 2 ? 2 : RMAX)>{});
        u = uniform(u + stride);
        const bool more = u < units;
        if (more) cur = unit_at(u);
        if (left && !(more && all_fragments(cur) && all_exist(done) && KB >= kSpread * RMAX)) {
            finish_now(done, done_place, old, std::integral_constant<int, RMAX>{});
            left = false;
        }
        if (!more) break;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no copy may land in LDS that is used for something else by then
}

// All of a grouped product as one kernel: where one kind of unit does not occur, a launch of its own would cost 4 to 5 us all the same.
// Long tiles are bound by the matrix units, short last tiles and streamed experts by memory, of which a CU alone gets 35 GB/s and 256 of them 20 each.  So
// where there are rounds of the former, some CUs of every XCD (as many as the two kinds' times give, see memory_blocks) do the latter while the others
// do the tiles; else all do the tiles first, then the streamed units, which are dealt from the last block number down.
// 16384 tokens to 128 experts of 8192 x 2048, top-2, skewed: none apart 917 us, as many as the rule gives 847 to 875, 0.6, 0.8 and 1.3 of them 1100, 930 and 875.
template <int RMAX>
__device__ __forceinline__ int memory_blocks(int grid, int long_units, int short_units, int streamed_units) {       // a multiple of 8
    if (grid % 8 != 0 || long_units < grid) return 0;
    // us per step: of a long tile where the others do something else, of what a CU takes from memory
    const float l = long_units * (RMAX == 4 ? 1.1f : RMAX == 2 ? 0.7f : 0.6f), m = short_units * 0.6f + streamed_units * 0.5f;
    const int per_xcd = grid / 8, n = static_cast<int>(static_cast<float>(per_xcd) * m / (l + m) + 0.5f);
    return 8 * min(n, per_xcd - 1);
}
template <int OUT, int RMAX, bool SMOOTH, bool PASS>
__global__ __launch_bounds__(kTileWaves * 64) void int_product_kernel(const QuantArgs a, int tiled_min_rows) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int groups = quant_blocks(a.N), grid = gridDim.x, at = xcd_position();
    Work work = count_work<RMAX>(a, tiled_min_rows, smem);
    const int long_units = (work.whole + work.last[0]) * groups, units = long_units + (work.last[1] + work.last[2]) * groups;
    const int streamed = work.streamed * groups, apart = uniform(memory_blocks<RMAX>(grid, long_units, units - long_units, streamed));
    auto stream = [&](int b, int blocks) __attribute__((always_inline)) {
        uint16_t* list = reinterpret_cast<uint16_t*>(smem + kListAt);
        const int tiles = list_experts<kTileWaves * 64>(a, tiled_min_rows - 1, list, reinterpret_cast<int32_t*>(list + MOE_MAX_E));
        // Units of 256 columns read each row fragment for twice the columns; but where those of 128 are at most one per block they use more of the CUs.
        if (tiles * groups > blocks) stream_units<OUT, 2, SMOOTH>(a, list, tiles, 1, b, blocks, smem);
        else stream_units<OUT, 1, SMOOTH>(a, list, tiles, 1, b, blocks, smem);
    };
    int first = at, end = units, stride = grid;
    if (apart != 0) {
        const int per_xcd = grid / 8, mine = per_xcd - apart / 8, xcd = at / per_xcd, n = at - xcd * per_xcd;
        if (n < mine) {
            first = xcd * mine + n;
            end = long_units;
            stride = 8 * mine;
        } else {
            if (streamed > 0) {
                __syncthreads();               // everybody has read the counts
                stream((n - mine) * 8 + xcd, apart);
                __syncthreads();
                work = count_work<RMAX>(a, tiled_min_rows, smem);
            }
            first = long_units + xcd * (apart / 8) + n - mine;
            stride = apart;
        }
    }
    tile_units<OUT, RMAX, SMOOTH, PASS>(a, work.whole, uniform(first), uniform(end), uniform(stride), smem);
    if (apart == 0 && streamed > 0) {
        __syncthreads();
        stream(grid - 1 - static_cast<int>(blockIdx.x), grid);
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------
// Experts with at least this many rows run in tiles, the others are streamed, which are the rows that a streamed unit holds: from 33 rows on in tiles, us,
// 64 x 2048 x 8192 (rows x N x K) 22.4 for 13.8, 64 x 8192 x 8192 32.5 for 21.9, 33 x 2048 x 2048 10.3 for 9.0.
constexpr int kTiledMinRows = 65;

// Units of 128 columns up to which a call of at most 64 rows takes units of half as many, which are then no more than the CUs.  Of 128 and of 64 columns, us:
// 1 x 16384 x 2048 (rows x N x K) 8.1 and 6.8, 16 x 8192 x 2048 7.9 and 6.6, 64 x 8192 x 2048 10.3 and 8.8, 64 x 16384 x 2048 10.8 and 9.7.
constexpr int kNarrowUnits = 128;

// Parts that the contraction of a streamed product is cut into: calls of at most 64 rows whose units would leave half of the CUs without one.  A unit takes
// about 0.2 us per block of its contraction, more with its rows, a part's, of twice the columns, 0.25; the second launch 3.5 us and what the parts' sums take on their
// way to memory and back, 8 bytes of each.  Never cut and cut so, us: 1 x 1024 x 4096 8.8 and 8.1, 1 x 1024 x 14336 21.8 and 9.9, 16 x 2048 x 8192 14.0 and 9.9,
// 64 x 2048 x 4096 12.7 and 11.2; not cut, and in four parts: 16 x 8192 x 2048 6.4 and 9.0, 64 x 8192 x 2048 8.7 and 13.5.
int stream_split(int rows, int N, int K, int E) {
    if (rows == 0 || rows >= kTiledMinRows) return 1;
    const int KB = quant_blocks(K), most = std::min(256 / std::min(256, std::min(rows, E) * quant_blocks(N)), KB / 2);
    int best = 1;
    float least = KB * (0.2f + 0.002f * rows);
    for (int parts = 2; parts <= most; ++parts) {
        const float us = (KB + parts - 1) / parts * 0.25f + 3.5f + static_cast<float>(parts) * rows * N * 2e-6f;
        if (us < least) best = parts, least = us;
    }
    return best;
}

// Row fragments per wavefront of the tiled kernel, so rows per tile / 64: large tiles do more per byte, small ones occupy more CUs.
// Tiles of 256 rows address the rows by 32-bit offsets.  The costs are of a step of a tile, relative; of tiles of 64, 128 and 256 rows, us: 1501 x 1024 x 4096
// (rows x N x K) 17.1, 22.5 and 32.0, 1024 x 4096 x 4096 29.6, 24.1 and 36.2, 2048 x 4096 x 4096 54.4, 42.4 and 37.4, 8192 x 2048 x 2048 61.3, 47.8 and 42.1.
int tile_fragments(int rows, int N, size_t operand_bytes) {
    auto cost = [&](int r, float step) {
        const long long units = static_cast<long long>((rows + 64 * r - 1) / (64 * r)) * quant_blocks(N);
        return static_cast<float>((units + 255) / 256) * step;
    };
    const float c4 = cost(4, 0.95f), c2 = cost(2, 0.7f), c1 = cost(1, 0.6f);
    if (c1 < c2 && c1 < c4) return 1;
    return c2 < 0.9f * c4 || operand_bytes > 0xffffffffull ? 2 : 4;
}

// dynamic LDS of the kernel with both kinds of units
template <int RMAX>
constexpr int kProductLds = Tiles<RMAX>::kLdsBytes > kStreamLds ? Tiles<RMAX>::kLdsBytes : kStreamLds;

// Outputs that no L2 holds pass by it, so that the operands stay there: 16384 x 8192 x 2048, fp32 out (537 MB), 367 -> 333 us, bf16 342 -> 334; but 4096 x 4096 x
// 1024, bf16 out (34 MB), 27.1 -> 28.2, 1501 x 1024 x 4096 (3 MB) 16.9 -> 17.8.
constexpr size_t kCachedOutput = size_t{64} << 20;

template <int OUT, bool SMOOTH>
hipError_t launch_out(const QuantArgs& a, void* ws, hipStream_t stream) {
    const int cus = device_cu_count();
    const dim3 grid(cus), threads(kStreamWaves * 64);
    const int split = stream_split(a.rows, a.N, a.K, a.E);
    if (split > 1) {
        QuantArgs parts = a;
        parts.out = ws;
        int_stream_kernel<kOutParts, false, kStreamWaves><<<grid, threads, kStreamLds, stream>>>(parts, a.rows, split);
        int_join_kernel<OUT, SMOOTH><<<dim3(a.rows, (a.N + 1023) / 1024), dim3(256), 0, stream>>>(a, static_cast<const int32_t*>(ws), split);
    } else if (a.rows < kTiledMinRows) {
        if (std::min(a.rows, a.E) * quant_blocks(a.N) <= kNarrowUnits) int_stream_kernel<OUT, SMOOTH, 4><<<grid, dim3(256), kStreamLds, stream>>>(a, a.rows, 1);
        else int_stream_kernel<OUT, SMOOTH, kStreamWaves><<<grid, threads, kStreamLds, stream>>>(a, a.rows, 1);
    } else {
        const size_t out_bytes = static_cast<size_t>(a.rows) * a.N * elem_size(a.out_dtype);
        const int r = tile_fragments(a.rows, a.N, a.rows / a.k * quant_pitch(a.K));
        if (r == 4 && out_bytes > kCachedOutput) int_product_kernel<OUT, 4, SMOOTH, true><<<grid, threads, kProductLds<4>, stream>>>(a, kTiledMinRows);
        else if (r == 4) int_product_kernel<OUT, 4, SMOOTH, false><<<grid, threads, kProductLds<4>, stream>>>(a, kTiledMinRows);
        else if (r == 2) int_product_kernel<OUT, 2, SMOOTH, false><<<grid, threads, kProductLds<2>, stream>>>(a, kTiledMinRows);
        else int_product_kernel<OUT, 1, SMOOTH, false><<<grid, threads, kProductLds<1>, stream>>>(a, kTiledMinRows);
    }
    return hipGetLastError();
}

hipError_t allow_lds(const void* kernel, int bytes) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int OUT, bool SMOOTH>
hipError_t configure_out() {
    hipError_t e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 4, SMOOTH, true>), kProductLds<4>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 4, SMOOTH, false>), kProductLds<4>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 2, SMOOTH, false>), kProductLds<2>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 1, SMOOTH, false>), kProductLds<1>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_stream_kernel<OUT, SMOOTH, 4>), kStreamLds)) != hipSuccess) return e;
    return allow_lds(reinterpret_cast<const void*>(int_stream_kernel<OUT, SMOOTH, kStreamWaves>), kStreamLds);
}

// Weights that do not fit the L2s (8 x 4 MiB) are gone before the next call reads them, or have pushed out the rows: streamed units then read
// them as what is read once.
constexpr size_t kCachedWeights = size_t{32} << 20;

}  // namespace

size_t int_product_workspace(const moe_quant_shape& s) {
    const int split = stream_split(s.rows, s.N, s.K, s.E);
    const size_t parts = split > 1 ? static_cast<size_t>(split) * s.rows * quant_pitch(s.N) * sizeof(int32_t) : 0;
    return (std::max<size_t>(parts, 1) + 255) / 256 * 256;
}

hipError_t configure_int_kernels() {
    hipError_t e;
    if ((e = configure_out<kOutF32, false>()) != hipSuccess) return e;
    if ((e = configure_out<kOutF32, true>()) != hipSuccess) return e;
    if ((e = configure_out<kOutBf16, false>()) != hipSuccess) return e;
    if ((e = configure_out<kOutBf16, true>()) != hipSuccess) return e;
    return allow_lds(reinterpret_cast<const void*>(int_stream_kernel<kOutParts, false, kStreamWaves>), kStreamLds);
}

hipError_t launch_int_product(const QuantArgs& args, void* ws, hipStream_t stream) {
    QuantArgs a = args;
    a.once = a.E * quant_matrix_bytes(a.N, a.K) > kCachedWeights;
    if (is_smooth(a.act)) return a.out_dtype == MOE_F32 ? launch_out<kOutF32, true>(a, ws, stream) : launch_out<kOutBf16, true>(a, ws, stream);
    return a.out_dtype == MOE_F32 ? launch_out<kOutF32, false>(a, ws, stream) : launch_out<kOutBf16, false>(a, ws, stream);
}

}  // namespace moe
