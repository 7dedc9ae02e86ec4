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

__device__ __forceinline__ float int_activate(float v, int act) {
    if (act == MOE_ACT_RELU) return v < 0.f ? 0.f : v;      // NaN stays
    if (act == MOE_ACT_GELU) return gelu_exp(v);
    if (act == MOE_ACT_SILU) return silu(v);
    return v;
}
// A lane's sums of NF fragments of columns x TF of rows as values: sx of its rows, sw and bias of its columns (four of each fragment), in LDS.
template <int NF, int TF>
__device__ __forceinline__ void finish(int act, const float (&sx)[TF], const unsigned char* sw, const unsigned char* bias, const i32x4 (&sums)[NF][TF],
                                       f32x4 (&v)[NF][TF]) {
#pragma unroll
    for (int nf = 0; nf < NF; ++nf) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(sw + nf * 64);
        f32x4 b = {0.f, 0.f, 0.f, 0.f};
        if (bias != nullptr) b = *reinterpret_cast<const f32x4*>(bias + nf * 64);
#pragma unroll
        for (int tf = 0; tf < TF; ++tf)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[nf][tf][i] = fmaf(static_cast<float>(sums[nf][tf][i]), sx[tf] * w[i], b[i]);
    }
    if (act == MOE_ACT_NONE) return;
#pragma unroll
    for (int nf = 0; nf < NF; ++nf)
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[nf][tf][i] = int_activate(v[nf][tf][i], act);
            if (NF * TF > 4) __builtin_amdgcn_sched_barrier(0);        // many values at once would need registers that there are not
        }
}

// ---- few rows per matrix: the weights are streamed -------------------------------------------------------------------
// Unit: an expert's rows, at most 64, x 128 NF columns, by 8 wavefronts of 16 NF columns each, a block of 128 columns of the contraction
// per step.  Bound by memory: what matters is that copies never stop.  Weights and rows go to LDS directly, through a ring of stages that
// runs on across units; a unit's scales and bias go before its first stage to a place of their own: one more than there are stages, for units of one step.
constexpr int kStreamRows = 64, kStreamWaves = 8;
template <int NF>
struct Streams {
    static constexpr int kStages = NF == 1 ? 6 : 3, kCols = NF * kQuantBlock;
    static constexpr int kX = kCols * kQuantBlock, kStage = kX + kStreamRows * kQuantBlock;
    static constexpr int kUnits = kStages * kStage, kPlaces = kStages + 1, kSw = 256, kBias = kSw + kCols * 4, kUnit = kBias + kCols * 4;       // of a unit: scales of rows, columns, bias
    static constexpr int kList = kUnits + kPlaces * kUnit, kLdsBytes = kList + MOE_MAX_E * 2 + kStreamWaves * 4;
    static constexpr int kCopies = 2 * NF + 1;          // a wavefront's, per stage
    static_assert(kLdsBytes <= 160 * 1024, "fits a CU");
};

// OUT = kOutParts: the contraction is cut into `split` parts, whose sums go to a.out as [split][rows][pitch of N] int32.
constexpr int kOutParts = 3;

template <int OUT, int NF>
__device__ __forceinline__ void stream_units(const QuantArgs& a, const uint16_t* list, int tiles, int parts_wanted, int b, unsigned char* smem) {
    using S = Streams<NF>;
    constexpr int kStages = S::kStages, kStage = S::kStage;
    const int split = OUT == kOutParts ? parts_wanted : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int KB = quant_blocks(a.K), blocks = quant_blocks(a.N), groups = (blocks + NF - 1) / NF;
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const int per_tile = groups * split, units = tiles * per_tile;

    // Every block gets the same number of units, as few as the grid allows: a CU can pull more than its share of the memory's rate, so
    // that a quarter of them idle costs nothing, but a last round of a few units does.  The runs are dealt to the XCDs evenly.
    const int G = gridDim.x, rounds = (units + G - 1) / G, runs = rounds > 0 ? (units + rounds - 1) / rounds : 0;
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

    // copies: wavefront w brings rows 8 w ... 8 w + 7, weight fragments NF w ..., and of a unit 64 of its columns' scales or biases and
    // (all the same) the rows' scales
    const uint32_t lds = lds_address(smem);
    const uint32_t to_weights = lds + wave * NF * kFragBytes, to_rows = lds + S::kX + wave * 1024;
    const int piece = wave % (4 * NF);
    const uint8_t *tile_row, *row_from, *weights_from;
    const float* tile_scale;
    int unit_in = 0;                        // place of the next unit's scales
    auto point_at_tile = [&](const Unit& w) __attribute__((always_inline)) {
        const int in_tile = wave * 8 + (lane >> 3);
        tile_row = a.a + source_row(a, w.row0 + min(in_tile, w.rows - 1)) * pitch + piece_of_lane(lane, in_tile);
        tile_scale = a.a_scales + source_row(a, w.row0 + min(lane, w.rows - 1));
    };
    auto point_at = [&](const Unit& w) __attribute__((always_inline)) {
        row_from = tile_row + static_cast<size_t>(w.kb) * kQuantBlock;
        // columns of the last unit that do not exist are read as the last ones that do, and not stored
        const int fragment = min(w.group * 8 * NF + wave * NF, blocks * 8 - NF);
        weights_from = a.w + static_cast<size_t>(w.e) * quant_matrix_bytes(a.N, a.K) + (static_cast<size_t>(fragment) * KB + w.kb) * kFragBytes + lane * 16;
        if constexpr (OUT != kOutParts) {
            const float* from = piece < 2 * NF || a.bias == nullptr ? a.w_scales : a.bias;
            const uint32_t to = lds + S::kUnits + unit_in * S::kUnit;
            copy4_to_lds(from + static_cast<size_t>(w.e) * a.N + min(w.group * S::kCols + (piece % (2 * NF)) * 64 + lane, a.N - 1), to + S::kSw + piece * 256);
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
        copy16_to_lds(row_from, to_rows + at);
        weights_from += kFragBytes;
        row_from += kQuantBlock;
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
            for (int i = 0; i < S::kCopies; ++i) copy16_to_lds(tile_row, to_rows + slot_in * kStage);
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
                finish(a.act, sx, of + S::kSw + at_columns, a.bias != nullptr ? of + S::kBias + at_columns : nullptr, acc, v);
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

constexpr int kListAt = Streams<1>::kList > Streams<2>::kList ? Streams<1>::kList : Streams<2>::kList;      // behind both rings
constexpr int kStreamLds = kListAt + MOE_MAX_E * 2 + kStreamWaves * 4;

template <int OUT>
__global__ __launch_bounds__(kStreamWaves * 64) void int_stream_kernel(const QuantArgs a, int max_rows, int parts_wanted) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* list = reinterpret_cast<uint16_t*>(smem + kListAt);
    const int tiles = list_experts<kStreamWaves * 64>(a, max_rows, list, reinterpret_cast<int32_t*>(list + MOE_MAX_E));
    stream_units<OUT, 1>(a, list, tiles, parts_wanted, blockIdx.x, smem);
}

// Adds up the parts of a split contraction and finishes the rows.  A block of threads per row and 1024 columns, four per thread.
template <int OUT>
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
            const float v = int_activate(fmaf(static_cast<float>(sum[i]), sx * a.w_scales[of], a.bias != nullptr ? a.bias[of] : 0.f), a.act);
            if constexpr (OUT == kOutF32) static_cast<float*>(a.out)[at] = v;
            else static_cast<uint16_t*>(a.out)[at] = f32_to_bf16(v);
        }
}

// ---- many rows per matrix: tiles in LDS -----------------------------------------------------------------------------
// Unit: 64 R rows (R = 1, 2, 4) x 128 columns by 8 wavefronts, a block of 128 columns of the contraction per step, through a ring of
// LDS stages that runs on across units.  Everything goes from memory to LDS directly, 16 bytes per lane; a stage holds
//   rows     [64 RMAX][128 bytes]
//   weights  8 fragments of 2 KiB as they are packed, 16 rows each
// and a unit's scales and biases go before its first stage to a place of their own, one more than there are stages, for units of one step.
// Wavefront (wm, wn) of the 4 x 2 multiplies row fragments wm, wm + 4, ... (R of them) and the columns 64 wn ... 64 wn + 63.
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

template <int OUT, int RMAX>
__device__ __forceinline__ void tile_units(const QuantArgs& a, int min_rows, unsigned char* smem) {
    using T = Tiles<RMAX>;
    constexpr int kStages = T::kStages, kStageW = T::kStageW, kStage = T::kStage, tile_rows = T::kRows;
    int4* counts = reinterpret_cast<int4*>(smem + T::kStarts);
    int32_t* whole = reinterpret_cast<int32_t*>(counts + kTileWaves);
    uint16_t* rest = reinterpret_cast<uint16_t*>(whole + MOE_MAX_E + 1);
    const int last_tiles = count_tiles<kTileWaves * 64>(a, tile_rows, min_rows, whole, rest, counts);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int wm = wave >> 1, wn = wave & 1;
    const int KB = quant_blocks(a.K), groups = quant_blocks(a.N);
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const int whole_units = __builtin_amdgcn_readfirstlane(whole[a.E]) * groups, units = whole_units + last_tiles * groups;
    int u = xcd_position(), u_in = u;       // the unit that is computed, and the one that is copied
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
    bool copying = true;
    auto copy_next = [&]() __attribute__((always_inline)) {
        const int at = slot_in * kStage;
#pragma unroll
        for (int i = 0; i < RMAX; ++i) {
            if constexpr (OFFSETS) copy16_to_lds(rows_base, row_offset[i], to_rows + at + i * 8192);
            else copy16_to_lds(row_from[i], to_rows + at + i * 8192);
        }
        copy16_to_lds(weights_base, lane16, to_weights + at);
        copy16_to_lds(weights_base + 1024, lane16, to_weights + at + 1024);
        slot_in = slot_in == kStages - 1 ? 0 : slot_in + 1;
        if (copying) {                     // behind the last unit its last stage is copied again, which keeps up the count that the waits go by
            if (++kb_in == KB) {
                kb_in = 0;
                if (u_in + static_cast<int>(gridDim.x) < units) {
                    u_in += gridDim.x;
                    ahead = unit_at(u_in);
                    point_at(ahead);
                } else {
                    copying = false;
                }
            } else {
                weights_base += kFragBytes;
                if constexpr (OFFSETS) {
                    rows_base += kQuantBlock;
                } else {
#pragma unroll
                    for (int i = 0; i < RMAX; ++i) row_from[i] += kQuantBlock;
                }
            }
        }
    };
    Unit cur = ahead;
#pragma unroll 1
    for (int i = 0; i < kStages - 1; ++i) copy_next();

    int slot = 0, unit = 0;
    auto run_unit = [&](auto fragments) __attribute__((always_inline)) {
        constexpr int R = decltype(fragments)::value;
        const int tid = here(threadIdx.x);
        const int at_x = row_operand(tid, wm * 16), x_other = row_operand_other(at_x), at_w = kStageW + wn * 4 * kFragBytes;
        i32x4 acc[4][R];
#pragma unroll
        for (int nf = 0; nf < 4; ++nf)
#pragma unroll
            for (int i = 0; i < R; ++i) acc[nf][i] = i32x4{0, 0, 0, 0};
#pragma unroll 1
        for (int kb = 0; kb < KB; ++kb) {
            copies_landed<(kStages - 2) * T::kCopies>();
            const unsigned char* st = smem + slot * kStage;
            i32x8 w[4], x[R];
#pragma unroll
            for (int nf = 0; nf < 4; ++nf) w[nf] = read_codes(st + at_w + lane16 + nf * kFragBytes, 1024);
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = read_codes(st + at_x + i * 64 * kQuantBlock, x_other);
            copy_next();
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int nf = 0; nf < 4; ++nf) acc[nf][i] = multiply(w[nf], x[i], acc[nf][i]);
            slot = slot == kStages - 1 ? 0 : slot + 1;
        }
        const int lane = here(threadIdx.x) & 63, r = lane & 15;
        const int col0 = cur.group * kQuantBlock + wn * 64, first = wm * 16;            // this wavefront's columns and rows
        const unsigned char* of = smem + T::kUnits + unit * T::kUnit;
        const int at_columns = (wn * 64 + (lane >> 4) * 4) * 4;
        float sx[R];
#pragma unroll
        for (int i = 0; i < R; ++i) sx[i] = *reinterpret_cast<const float*>(of + (first + i * 64 + r) * 4);
        f32x4 v[4][R];
        finish(a.act, sx, of + T::kSw + at_columns, a.bias != nullptr ? of + T::kBias + at_columns : nullptr, acc, v);
        store_values<OUT, 64>(a, col0, cur.row0 + first, cur.rows - first, v);
        unit = unit == T::kPlaces - 1 ? 0 : unit + 1;
    };
    while (true) {
        if (RMAX == 1 || cur.rows <= 64) run_unit(std::integral_constant<int, 1>{});
        else if (RMAX == 2 || cur.rows <= 128) run_unit(std::integral_constant<int, (RMAX < 2 ? RMAX : 2)>{});
        else run_unit(std::integral_constant<int, RMAX>{});
        u = uniform(u + static_cast<int>(gridDim.x));
        if (u >= units) break;
        cur = unit_at(u);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no copy may land in LDS that is used for something else by then
}

// Both kinds of units of a grouped product as one kernel, the tiles first: where one kind does not occur, a launch of its own would
// cost 4 to 5 us all the same.  Streamed units are dealt from the last block number down, evenly over the XCDs.
template <int OUT, int RMAX>
__global__ __launch_bounds__(kTileWaves * 64) void int_product_kernel(const QuantArgs a, int tiled_min_rows) {
    extern __shared__ __align__(16) unsigned char smem[];
    tile_units<OUT, RMAX>(a, tiled_min_rows, smem);
    if (a.offsets == nullptr) return;
    __syncthreads();
    uint16_t* list = reinterpret_cast<uint16_t*>(smem + kListAt);
    const int tiles = list_experts<kTileWaves * 64>(a, tiled_min_rows - 1, list, reinterpret_cast<int32_t*>(list + MOE_MAX_E));
    const int b = gridDim.x - 1 - blockIdx.x;
    if (tiles * quant_blocks(a.N) > static_cast<int>(gridDim.x)) stream_units<OUT, 2>(a, list, tiles, 1, b, smem);
    else stream_units<OUT, 1>(a, list, tiles, 1, b, smem);
}

// ---- launches -------------------------------------------------------------------------------------------------------
// Experts with at least this many rows run in tiles, the others are streamed.
constexpr int kTiledMinRows = 65;

// Parts that the contraction of a streamed product is cut into: calls of at most 64 rows whose units would leave most CUs without one.
int stream_split(int rows, int N, int K, int E) {
    if (rows == 0 || rows >= kTiledMinRows) return 1;
    const int units = std::min(rows, E) * quant_blocks(N);
    return units <= 96 ? std::max(1, std::min(256 / units, quant_blocks(K) / 2)) : 1;
}

// Row fragments per wavefront of the tiled kernel, so rows per tile / 64: large tiles do more per byte, small ones occupy more CUs.
// Tiles of 256 rows address the rows by 32-bit offsets.
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

template <int OUT>
hipError_t launch_out(const QuantArgs& a, void* ws, hipStream_t stream) {
    const int cus = device_cu_count();
    const dim3 grid(cus), threads(kStreamWaves * 64);
    const int split = stream_split(a.rows, a.N, a.K, a.E);
    if (split > 1) {
        QuantArgs parts = a;
        parts.out = ws;
        int_stream_kernel<kOutParts><<<grid, threads, kStreamLds, stream>>>(parts, a.rows, split);
        int_join_kernel<OUT><<<dim3(a.rows, (a.N + 1023) / 1024), dim3(256), 0, stream>>>(a, static_cast<const int32_t*>(ws), split);
    } else if (a.rows < kTiledMinRows) {
        int_stream_kernel<OUT><<<grid, threads, kStreamLds, stream>>>(a, a.rows, 1);
    } else {
        const int r = tile_fragments(a.rows, a.N, a.rows / a.k * quant_pitch(a.K));
        if (r == 4) int_product_kernel<OUT, 4><<<grid, threads, kProductLds<4>, stream>>>(a, kTiledMinRows);
        else if (r == 2) int_product_kernel<OUT, 2><<<grid, threads, kProductLds<2>, stream>>>(a, kTiledMinRows);
        else int_product_kernel<OUT, 1><<<grid, threads, kProductLds<1>, stream>>>(a, kTiledMinRows);
    }
    return hipGetLastError();
}

hipError_t allow_lds(const void* kernel, int bytes) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int OUT>
hipError_t configure_out() {
    hipError_t e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 4>), kProductLds<4>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 2>), kProductLds<2>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(int_product_kernel<OUT, 1>), kProductLds<1>)) != hipSuccess) return e;
    return allow_lds(reinterpret_cast<const void*>(int_stream_kernel<OUT>), kStreamLds);
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
    if ((e = configure_out<kOutF32>()) != hipSuccess) return e;
    if ((e = configure_out<kOutBf16>()) != hipSuccess) return e;
    return allow_lds(reinterpret_cast<const void*>(int_stream_kernel<kOutParts>), kStreamLds);
}

hipError_t launch_int_product(const QuantArgs& args, void* ws, hipStream_t stream) {
    QuantArgs a = args;
    a.once = a.E * quant_matrix_bytes(a.N, a.K) > kCachedWeights;
    return a.out_dtype == MOE_F32 ? launch_out<kOutF32>(a, ws, stream) : launch_out<kOutBf16>(a, ws, stream);
}

}  // namespace moe
