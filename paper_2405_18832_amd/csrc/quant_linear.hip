// Products on quantised rows, for one weight matrix and grouped by expert:
//
//   out[p, n] = act( sum_b sa[row(p), b] * sw[e, n / 128, b] * sum_{c in block b} a[row(p), c] * w[e, n, c] + bias[e, n] )
//
// A product of codes starts from zero in every block of 128 columns and is added to the fp32 accumulators by one multiply-add per
// value, scaled with the block's two scales: the weights' is the same for the whole wavefront, the rows' one value per lane, because
// the weights are the matrix instruction's first operand and a lane's results are four columns of one row.
#include <algorithm>
#include <type_traits>

#include "quant.hpp"

namespace moe {

enum OutKind { kOutF32 = 0, kOutBf16 = 1, kOutE4m3 = 2 };

// 32 codes of a lane as bf16 values, which hold them exactly.
struct Widened {
    bf16x8 v[4];
};
__device__ __forceinline__ Widened widen(const i32x8& codes) {
    Widened r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        union {
            bf16x2_t two[4];
            bf16x8 eight;
        } u;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            u.two[2 * j] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * i + j], 1.f, false);
            u.two[2 * j + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[2 * i + j], 1.f, true);
        }
        r.v[i] = u.eight;
    }
    return r;
}

// 16 x 16 results of one block of 128 columns: first operand 16 weight rows, second 16 token rows.  Lane l holds 32 codes of row
// l % 16 of each; which columns they are does not matter as long as both operands agree (moe.h: 64 h + 16 (l / 16), h = 0, 1).
// Result i of lane l: weight row 4 (l / 16) + i, token row l % 16.
// On the bf16 units: those for 8-bit operands (v_mfma_f32_16x16x128_f8f6f4) add up groups of products after aligning them to the largest
// and drop what lies below about 2^-14 of it, which is 1.5e-5 of the rms of a sum of 128 products of normal values.
__device__ __forceinline__ f32x4 mfma_block(const Widened& w, const Widened& x) {
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.v[i], x.v[i], p, 0, 0, 0);
    return p;
}

__device__ __forceinline__ float quant_activate(float v, int act) {
    if (act == MOE_ACT_GELU) return gelu_exp(v);
    if (act == MOE_ACT_RELU) return v < 0.f ? 0.f : v;      // NaN stays
    return v;
}

// ---- which rows are whose -------------------------------------------------------------------------------------------
struct Segment {
    int row0, rows;
};
// Rows of expert e; none where it is masked out.  Clamped to the buffers, whatever the offsets hold.
__device__ __forceinline__ Segment segment_of(const QuantArgs& a, int e) {
    if (a.offsets == nullptr) return Segment{0, a.rows};
    if (a.mask != nullptr && a.mask[e] == 0) return Segment{0, 0};
    const int lo = min(max(a.offsets[e], 0), a.rows), hi = min(max(a.offsets[e + 1], lo), a.rows);
    return Segment{lo, hi - lo};
}
// Row of `a` that row p of the product reads.
__device__ __forceinline__ int source_row(const QuantArgs& a, int p) {
    if (a.perm == nullptr) return p;
    return min(max(a.perm[p], 0), a.rows - 1) / a.k;
}

// Row tiles before each expert, starts[0 ... E], counted by every block for itself: E is at most 1024, a list in memory would cost
// a launch.  Experts outside [min_rows, max_rows] have none.  `tmp`: 17 ints.
template <int THREADS>
__device__ __forceinline__ void count_tiles(const QuantArgs& a, int tile_rows, int min_rows, int max_rows, int32_t* starts, int32_t* tmp) {
    constexpr int W = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += THREADS) {
        const int e = e0 + threadIdx.x;
        int n = 0;
        if (e < a.E) {
            const int m = segment_of(a, e).rows;
            if (m >= min_rows && m <= max_rows) n = (m + tile_rows - 1) / tile_rows;
        }
        const int incl = wave_scan(n);
        if (lane == 63) tmp[wave] = incl;
        __syncthreads();
        int mine = before;
        for (int w = 0; w < W; ++w) {
            if (w < wave) mine += tmp[w];
            before += tmp[w];
        }
        if (e < a.E) starts[e] = mine + incl - n;
        __syncthreads();
    }
    if (threadIdx.x == 0) starts[a.E] = before;
    __syncthreads();
}
// The expert that tile t belongs to: the last whose tiles begin at or before t.  By whole wavefronts.
__device__ __forceinline__ int expert_of(const int32_t* starts, int E, int t) {
    if (E == 1) return 0;
    const int lane = threadIdx.x & 63;
    static_assert(MOE_MAX_E <= 64 * 16, "16 experts per lane");
    const int coarse = lane * 16;
    const int group = (__popcll(__ballot(coarse < E && starts[min(coarse, E)] <= t)) - 1) * 16;
    const int fine = group + lane;
    return group + __popcll(__ballot(lane < 16 && fine < E && starts[min(fine, E)] <= t)) - 1;
}

// Blocks go to the 8 XCDs in turn; position of this one such that an XCD's blocks hold neighbouring units, which share rows or weights
// in its L2.
__device__ __forceinline__ int xcd_position() {
    const int G = gridDim.x, b = blockIdx.x;
    return G % 8 == 0 ? (b & 7) * (G >> 3) + (b >> 3) : b;
}

// ---- what becomes of a tile's sums ----------------------------------------------------------------------------------
// A wavefront's NF x TF results of 16 columns x 16 rows: columns n0 + 16 nf + 4 (lane / 16) + i, rows row0 + 16 tf + lane % 16, the first
// `rows` of which exist.
template <int NF, int TF>
__device__ __forceinline__ void activate_values(int act, f32x4 (&acc)[NF][TF]) {
#pragma unroll
    for (int nf = 0; nf < NF; ++nf)
#pragma unroll
        for (int tf = 0; tf < TF; ++tf)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nf][tf][i] = quant_activate(acc[nf][tf][i], act);
}
template <int NF, int TF>
__device__ __forceinline__ void finish_values(const QuantArgs& a, int e, int n0, f32x4 (&acc)[NF][TF]) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int nf = 0; nf < NF; ++nf) {
        const int n = n0 + nf * 16 + g * 4;
        if (a.bias != nullptr) {
            const float* bias = a.bias + static_cast<size_t>(e) * a.N;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float b = n + i < a.N ? bias[n + i] : 0.f;
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) acc[nf][tf][i] += b;
            }
        }
    }
    activate_values(a.act, acc);
}

template <int OUT, int NF, int TF>
__device__ __forceinline__ void store_values(const QuantArgs& a, int n0, int row0, int rows, const f32x4 (&acc)[NF][TF]) {
    static_assert(OUT != kOutE4m3, "");
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    // four columns at once where every row begins on a boundary of four
    const bool wide = a.N % 4 == 0 && reinterpret_cast<uintptr_t>(a.out) % (OUT == kOutF32 ? 16 : 8) == 0;
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        if (tf * 16 + r >= rows) continue;
        const size_t at = static_cast<size_t>(row0 + tf * 16 + r) * a.N;
#pragma unroll
        for (int nf = 0; nf < NF; ++nf) {
            const int n = n0 + nf * 16 + g * 4;
            const f32x4 v = acc[nf][tf];
            if (wide) {
                if (n >= a.N) continue;
                if constexpr (OUT == kOutF32) *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at + n) = v;
                else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at + n) = uint2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n + i < a.N) {
                        if constexpr (OUT == kOutF32) static_cast<float*>(a.out)[at + n + i] = v[i];
                        else static_cast<uint16_t*>(a.out)[at + n + i] = f32_to_bf16(v[i]);
                    }
            }
        }
    }
}

// Largest magnitude of each row over the wavefront's columns that exist, for lane l of row 16 tf + l % 16.
template <int NF, int TF>
__device__ __forceinline__ void row_magnitudes(int N, int n0, f32x4 (&acc)[NF][TF], uint32_t (&most)[TF]) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        uint32_t m = 0;
#pragma unroll
        for (int nf = 0; nf < NF; ++nf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (n0 + nf * 16 + g * 4 + i >= N) acc[nf][tf][i] = 0.f;
                m = max(m, magnitude(acc[nf][tf][i]));
            }
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, 64)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, 64)));
        most[tf] = m;
    }
}

// Codes of a block of 128 columns whose rows' largest magnitudes are known; the wavefront with `scales` also stores the scales.
template <int NF, int TF>
__device__ __forceinline__ void store_codes(const QuantArgs& a, int n0, int row0, int rows, const f32x4 (&acc)[NF][TF],
                                            const uint32_t (&most)[TF], bool scales) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const size_t pitch = quant_pitch(a.N);
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        if (tf * 16 + r >= rows) continue;
        const size_t row = static_cast<size_t>(row0 + tf * 16 + r);
        const float scale = block_scale(most[tf]), inv = __builtin_amdgcn_rcpf(scale);
        uint8_t* out = static_cast<uint8_t*>(a.out) + row * pitch;
#pragma unroll
        for (int nf = 0; nf < NF; ++nf) {
            const int n = n0 + nf * 16 + g * 4;
            const f32x4 v = acc[nf][tf];
            uint32_t codes = pack_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            if (n + 4 > a.N) codes = n >= a.N ? 0u : codes & (0xffffffffu >> (8 * (n + 4 - a.N)));     // zeros past the end
            *reinterpret_cast<uint32_t*>(out + n) = codes;
        }
        if (scales && g == 0) a.out_scales[row * quant_blocks(a.N) + n0 / kQuantBlock] = scale;
    }
}

// ---- copies into LDS ------------------------------------------------------------------------------------------------
// 4 bytes per lane into LDS, as copy16_to_lds
__device__ __forceinline__ void copy4_to_lds(const void* src, uint32_t lds_base) {
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(dst) : "memory");
}
// The wavefront's copies up to the newest `left` have landed, and with the barrier everybody's; every LDS read before it is done too.
template <int LEFT>
__device__ __forceinline__ void copies_landed() {
    static_assert(LEFT < 64, "vmcnt has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory");
}
__device__ __forceinline__ i32x8 read_codes(const unsigned char* p, int other) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(p), hi = *reinterpret_cast<const i32x4*>(p + other);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Rows in LDS: 128 bytes each, the 16-byte pieces of a row permuted by its number, so that an operand read (16 rows x one piece) meets no
// bank twice: piece c of row r lies at c ^ (r / 2 % 8).  A copy brings 8 rows, each a whole line by eight lanes.
__device__ __forceinline__ int piece_of_lane(int row) { return ((threadIdx.x & 7) ^ (row >> 1 & 7)) << 4; }
// Where lane l reads piece l / 16 of row `first` + l % 16 (`first` a multiple of 16), and how far from there piece 4 + l / 16 lies.
__device__ __forceinline__ int row_operand(int first) {
    const int lane = threadIdx.x & 63, r = lane & 15;
    return (first + r) * kQuantBlock + (((lane >> 4) ^ (r >> 1)) << 4);
}
__device__ __forceinline__ int row_operand_other(int at) { return at & 64 ? -64 : 64; }

// ---- few rows per matrix: the weights are streamed -------------------------------------------------------------------
// Unit: up to 64 rows of an expert x 128 columns, by 8 wavefronts of 16 columns each, a block of 128 columns of the contraction per
// step.  Bound by memory, so what matters is that copies never stop: weights (16 KiB a step), rows and scales go to LDS directly, through
// a ring of six stages that runs on across units.  A block's units follow each other in one row tile, where nothing needs to be looked up
// (a load that the compiler sees would make it wait for every copy in flight).
constexpr int kStreamRows = 64, kStreamWaves = 8, kStreamStages = 6, kStreamCopies = 4;
constexpr int kStreamX = kQuantBlock * kQuantBlock, kStreamS = kStreamX + kStreamRows * kQuantBlock;
constexpr int kStreamStage = kStreamS + 4 * 256;            // scales of the rows, of the weights (64 times), bias of the 128 columns
constexpr int kStreamMost = kStreamStages * kStreamStage, kStreamStarts = kStreamMost + kStreamWaves * kStreamRows * 4;
constexpr int kStreamLdsBytes = kStreamStarts + (MOE_MAX_E + 1 + kStreamWaves) * 4;
static_assert(kStreamLdsBytes <= 160 * 1024, "fits a CU");

// OUT = kOutParts: the contraction is cut into `split` parts, whose sums go to a.out as [split][rows][pitch of N] fp32.
constexpr int kOutParts = 3;

template <int OUT>
__global__ __launch_bounds__(kStreamWaves * 64) void quant_stream_kernel(const QuantArgs a, int max_rows, int parts_wanted) {
    const int split = OUT == kOutParts ? parts_wanted : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* mosts = reinterpret_cast<uint32_t*>(smem + kStreamMost);         // [64][8]
    int32_t* starts = reinterpret_cast<int32_t*>(smem + kStreamStarts);
    count_tiles<kStreamWaves * 64>(a, kStreamRows, 1, max_rows, starts, starts + MOE_MAX_E + 1);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15;
    const int KB = quant_blocks(a.K), groups = quant_blocks(a.N);
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const int per_tile = groups * split, units = starts[a.E] * per_tile;

    // Every block gets the same number of units, as few as the grid allows: a CU can pull more than its share of the memory's rate, so
    // that a quarter of them idle costs nothing, but a last round of a few units does.  The runs are dealt to the XCDs evenly.
    const int G = gridDim.x, rounds = (units + G - 1) / G, runs = rounds > 0 ? (units + rounds - 1) / rounds : 0;
    const int per_xcd = (runs + 7) >> 3, b = blockIdx.x;
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
        w.e = __builtin_amdgcn_readfirstlane(expert_of(starts, a.E, t));
        const Segment seg = segment_of(a, w.e);
        const int tile = __builtin_amdgcn_readfirstlane(t - starts[w.e]);
        w.row0 = __builtin_amdgcn_readfirstlane(seg.row0 + tile * kStreamRows);
        w.rows = __builtin_amdgcn_readfirstlane(min(kStreamRows, seg.rows - tile * kStreamRows));
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

    // copies: wavefront w brings rows 8 w ... 8 w + 7, weight fragment w, and a quarter of the scales and bias (two wavefronts each)
    const uint32_t lds = lds_address(smem);
    const uint32_t to_weights = lds + wave * kFragBytes, to_rows = lds + kStreamX + wave * 1024, to_scales = lds + kStreamS + (wave & 3) * 256;
    const uint8_t *tile_row, *row_from, *weights_from;
    const float *tile_scale, *scales_from;
    int scales_step;
    auto point_at_tile = [&](const Unit& w) __attribute__((always_inline)) {
        const int in_tile = wave * 8 + (lane >> 3);
        tile_row = a.a + source_row(a, w.row0 + min(in_tile, w.rows - 1)) * pitch + piece_of_lane(in_tile);
        tile_scale = a.a_scales + static_cast<size_t>(source_row(a, w.row0 + min(lane, w.rows - 1))) * KB;
    };
    auto point_at = [&](const Unit& w) __attribute__((always_inline)) {
        row_from = tile_row + static_cast<size_t>(w.kb) * kQuantBlock;
        weights_from = a.w + static_cast<size_t>(w.e) * quant_matrix_bytes(a.N, a.K) +
                       (static_cast<size_t>(w.group * 8 + wave) * KB + w.kb) * kFragBytes + lane * 16;
        const int quarter = wave & 3;
        scales_step = 1;
        if (quarter == 0) scales_from = tile_scale + w.kb;
        else if (quarter == 1 || a.bias == nullptr) scales_from = a.w_scales + (static_cast<size_t>(w.e) * groups + w.group) * KB + w.kb;
        else {
            scales_from = a.bias + static_cast<size_t>(w.e) * a.N + min(w.group * kQuantBlock + (quarter - 2) * 64 + lane, a.N - 1);
            scales_step = 0;
        }
    };
    auto stage_in = [&](int slot) {
        const int at = slot * kStreamStage;
        copy16_to_lds(weights_from, to_weights + at);
        copy16_to_lds(weights_from + 1024, to_weights + at + 1024);
        copy16_to_lds(row_from, to_rows + at);
        copy4_to_lds(scales_from, to_scales + at);
        weights_from += kFragBytes;
        row_from += kQuantBlock;
        scales_from += scales_step;
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
            // nothing left to copy: copies of some scale to the slot that has fallen free keep up the count that the waits go by
#pragma unroll
            for (int i = 0; i < kStreamCopies; ++i) copy4_to_lds(tile_scale, to_scales + slot_in * kStreamStage);
        }
        slot_in = slot_in == kStreamStages - 1 ? 0 : slot_in + 1;
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
    for (int i = 0; i < kStreamStages - 1; ++i) copy_next();

    Unit cur = unit_at(tile0, first - tile0 * per_tile);
    const int at_w = wave * kFragBytes + lane * 16, at_x = kStreamX + row_operand(0), x_other = row_operand_other(at_x);
    const int at_sx = kStreamS + r * 4, at_sw = kStreamS + 256, at_bias = kStreamS + 512 + (wave * 16 + (lane >> 4) * 4) * 4;
    int slot = 0;
    while (true) {
        auto run_unit = [&](auto tf_const) __attribute__((always_inline)) {
            constexpr int TF = decltype(tf_const)::value;
            f32x4 acc[1][TF];
#pragma unroll
            for (int tf = 0; tf < TF; ++tf) acc[0][tf] = f32x4{0.f, 0.f, 0.f, 0.f};
            f32x4 bias = {0.f, 0.f, 0.f, 0.f};
            for (; cur.kb < cur.kb1; ++cur.kb) {
                copies_landed<(kStreamStages - 2) * kStreamCopies>();
                copy_next();
                const unsigned char* st = smem + slot * kStreamStage;
                const float sw = *reinterpret_cast<const float*>(st + at_sw);
                const Widened w = widen(read_codes(st + at_w, 1024));
                i32x8 x[TF];
                float sx[TF];
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) {
                    x[tf] = read_codes(st + at_x + tf * kFragBytes, x_other);
                    sx[tf] = *reinterpret_cast<const float*>(st + at_sx + tf * 64);
                }
                if (cur.kb + 1 == cur.kb1) bias = *reinterpret_cast<const f32x4*>(st + at_bias);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) {
                    const f32x4 p = mfma_block(w, widen(x[tf]));
                    const float scale = sx[tf] * sw;
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[0][tf][i] = fmaf(scale, p[i], acc[0][tf][i]);
                }
                slot = slot == kStreamStages - 1 ? 0 : slot + 1;
            }
            const int n0 = cur.group * kQuantBlock + wave * 16;
            if constexpr (OUT == kOutParts) {
                float* parts = static_cast<float*>(a.out) + static_cast<size_t>(cur.part) * a.rows * quant_pitch(a.N);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf)
                    if (tf * 16 + r < cur.rows)
                        *reinterpret_cast<f32x4*>(parts + static_cast<size_t>(cur.row0 + tf * 16 + r) * quant_pitch(a.N) + n0 + (lane >> 4) * 4) =
                            acc[0][tf];
            } else {
                if (a.bias != nullptr) {
#pragma unroll
                    for (int tf = 0; tf < TF; ++tf) acc[0][tf] += bias;
                }
                activate_values(a.act, acc);
                if constexpr (OUT == kOutE4m3) {
                    uint32_t most[TF];
                    row_magnitudes(a.N, n0, acc, most);
                    if (lane < 16) {
#pragma unroll
                        for (int tf = 0; tf < TF; ++tf) mosts[(tf * 16 + lane) * kStreamWaves + wave] = most[tf];
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
                    for (int tf = 0; tf < TF; ++tf)
#pragma unroll
                        for (int v = 0; v < kStreamWaves; v += 4) {
                            const uint4 m = *reinterpret_cast<const uint4*>(mosts + (tf * 16 + r) * kStreamWaves + v);
                            most[tf] = max(most[tf], max(max(m.x, m.y), max(m.z, m.w)));
                        }
                    store_codes(a, n0, cur.row0, cur.rows, acc, most, wave == 0);
                } else {
                    store_values<OUT>(a, n0, cur.row0, cur.rows, acc);
                }
            }
        };
        const int tf = (cur.rows + 15) >> 4;
        if (tf == 1) run_unit(std::integral_constant<int, 1>{});
        else if (tf == 2) run_unit(std::integral_constant<int, 2>{});
        else run_unit(std::integral_constant<int, 4>{});
        if (--units_out == 0) break;
        cur = cur.rest + 1 == per_tile ? unit_at(cur.tile + 1, 0) : along(cur);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no copy may land in LDS that is another block's by then
}

// Adds up the parts of a split contraction, in their order, and finishes the rows.  A block of threads per row and 8 groups of 128
// columns; four columns per thread.
template <int OUT>
__global__ __launch_bounds__(256) void quant_join_kernel(const QuantArgs a, const float* __restrict__ parts, int split) {
    const int row = blockIdx.x, lane = threadIdx.x & 63;
    __shared__ int32_t before;
    int e = 0;
    if (a.offsets != nullptr) {            // the expert whose rows this one is among
        if (threadIdx.x == 0) before = 0;
        __syncthreads();
        int n = 0;
        for (int i = threadIdx.x; i < a.E; i += 256) n += a.offsets[i + 1] <= row ? 1 : 0;
        atomicAdd(&before, n);
        __syncthreads();
        e = before;
        if (e >= a.E) return;
        const Segment seg = segment_of(a, e);
        if (row < seg.row0 || row >= seg.row0 + seg.rows) return;
    }
    const int n0 = (blockIdx.y * 256 + threadIdx.x) * 4;
    const size_t pitch = quant_pitch(a.N);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n0 < static_cast<int>(pitch)) {
        const float* p = parts + static_cast<size_t>(row) * pitch + n0;
        for (int s = 0; s < split; ++s) v += *reinterpret_cast<const f32x4*>(p + static_cast<size_t>(s) * a.rows * pitch);
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n0 + i >= a.N) v[i] = 0.f;
        else v[i] = quant_activate(a.bias != nullptr ? v[i] + a.bias[static_cast<size_t>(e) * a.N + n0 + i] : v[i], a.act);
        most = max(most, magnitude(v[i]));
    }
    if constexpr (OUT == kOutE4m3) {
        most = row16_max(most);
        most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 16, 64)));       // 32 lanes are a block of 128
        const float scale = block_scale(most), inv = 1.f / scale;
        if (n0 < static_cast<int>(pitch)) {
            uint32_t codes = pack_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            if (n0 + 4 > a.N) codes = n0 >= a.N ? 0u : codes & (0xffffffffu >> (8 * (n0 + 4 - a.N)));
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.out) + row * pitch + n0) = codes;
            if ((lane & 31) == 0) a.out_scales[static_cast<size_t>(row) * quant_blocks(a.N) + n0 / kQuantBlock] = scale;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n0 + i < a.N) {
                const size_t at = static_cast<size_t>(row) * a.N + n0 + i;
                if constexpr (OUT == kOutF32) static_cast<float*>(a.out)[at] = v[i];
                else static_cast<uint16_t*>(a.out)[at] = f32_to_bf16(v[i]);
            }
    }
}

// ---- many rows per matrix: tiles in LDS -----------------------------------------------------------------------------
// Unit: 256 rows x 128 columns by 8 wavefronts (4 x 2, 64 x 64 each), a block of 128 columns of the contraction per step, through a
// ring of three LDS stages: one being read, one that has landed (its first fragments are read ahead), one in flight.  Everything goes from
// memory to LDS directly, 16 bytes per lane; a stage holds
//   rows     [256][128 bytes]
//   weights  8 fragments of 2 KiB as they are packed, 16 rows each
//   scales   of the 256 rows, and the weights' (one for the unit's 128 columns)
constexpr int kTileRows = 256, kTileCols = kQuantBlock, kTileWaves = 8, kTileStages = 3;
constexpr int kStageW = kTileRows * kQuantBlock, kStageS = kStageW + kTileCols * kQuantBlock, kStage = kStageS + kTileRows * 4 + 256;
constexpr int kTileMost = kTileStages * kStage, kTileStarts = kTileMost + 2 * kTileRows * 4;
constexpr int kTileLdsBytes = kTileStarts + (MOE_MAX_E + 1 + kTileWaves) * 4;
static_assert(kTileLdsBytes <= 160 * 1024, "fits a CU");

template <int OUT>
__global__ __launch_bounds__(kTileWaves * 64) void quant_tile_kernel(const QuantArgs a, int min_rows) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* mosts = reinterpret_cast<uint32_t*>(smem + kTileMost);           // [2][256]
    int32_t* starts = reinterpret_cast<int32_t*>(smem + kTileStarts);
    count_tiles<kTileWaves * 64>(a, kTileRows, min_rows, a.rows, starts, starts + MOE_MAX_E + 1);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int wm = wave >> 1, wn = wave & 1;
    const int KB = quant_blocks(a.K), groups = quant_blocks(a.N);
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const int units = starts[a.E] * groups;
    const uint32_t lds = lds_address(smem);
    // copies: wavefront w brings rows 32 w ... 32 w + 31, weight fragment w, and the scales of rows 64 (w % 4) ... or of the weights
    const uint32_t to_rows = lds + wave * 4096, to_weights = lds + kStageW + wave * 2048;
    const uint32_t to_scales = lds + kStageS + (wave < 4 ? wave * 256 : kTileRows * 4);
    const int at_x = row_operand(wm * 64), x_other = row_operand_other(at_x), at_w = kStageW + wn * 4 * kFragBytes + lane * 16;
    const int at_sx = kStageS + (wm * 64 + r) * 4, at_sw = kStageS + kTileRows * 4;

    for (int u = xcd_position(); u < units; u += gridDim.x) {
        const int e = __builtin_amdgcn_readfirstlane(expert_of(starts, a.E, u / groups));
        const int tiles = starts[e + 1] - starts[e], local = u - starts[e] * groups;
        // eight column groups of a tile, then the next tile's: 32 neighbours share four tiles' rows and eight groups' weights
        const int band = local / (tiles * 8), width = min(8, groups - band * 8), rest = local - band * tiles * 8;
        const int tile = rest / width, group = band * 8 + rest % width;
        const Segment seg = segment_of(a, e);
        const int row0 = __builtin_amdgcn_readfirstlane(seg.row0 + tile * kTileRows);
        const int rows = __builtin_amdgcn_readfirstlane(min(kTileRows, seg.rows - tile * kTileRows));
        const int n0 = group * kTileCols;

        const uint8_t* from_rows[4];
        const uint8_t* from_weights = a.w + static_cast<size_t>(e) * quant_matrix_bytes(a.N, a.K) +
                                      static_cast<size_t>(n0 / 16 + wave) * KB * kFragBytes + lane * 16;
        const float* from_scales;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int in_tile = wave * 32 + i * 8 + (lane >> 3);
            const size_t row = source_row(a, row0 + min(in_tile, rows - 1));
            from_rows[i] = a.a + row * pitch + piece_of_lane(in_tile);
        }
        if (wave < 4) from_scales = a.a_scales + static_cast<size_t>(source_row(a, row0 + min(wave * 64 + lane, rows - 1))) * KB;
        else from_scales = a.w_scales + (static_cast<size_t>(e) * groups + group) * KB;
        auto stage_in = [&](int slot) {
            const int at = slot * kStage;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                copy16_to_lds(from_rows[i], to_rows + at + i * 1024);
                from_rows[i] += kQuantBlock;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) copy16_to_lds(from_weights + i * 1024, to_weights + at + i * 1024);
            from_weights += kFragBytes;
            copy4_to_lds(from_scales, to_scales + at);
            ++from_scales;
        };
        f32x4 acc[4][4];
#pragma unroll
        for (int nf = 0; nf < 4; ++nf)
#pragma unroll
            for (int tf = 0; tf < 4; ++tf) acc[nf][tf] = f32x4{0.f, 0.f, 0.f, 0.f};

        copies_landed<0>();         // the ring is free
        stage_in(0);
        if (KB > 1) stage_in(1);
        if (KB > 1) copies_landed<7>();
        else copies_landed<0>();
        Widened w[4];
#pragma unroll
        for (int nf = 0; nf < 4; ++nf) w[nf] = widen(read_codes(smem + at_w + nf * kFragBytes, 1024));
        i32x8 x = read_codes(smem + at_x, x_other);
        int slot = 0;
        for (int j = 0; j < KB; ++j) {
            const int next = slot == kTileStages - 1 ? 0 : slot + 1, after = next == kTileStages - 1 ? 0 : next + 1;
            const unsigned char* st = smem + slot * kStage;
            const unsigned char* st_next = smem + next * kStage;
            const bool more = j + 1 < KB;
            if (more) copies_landed<0>();
            if (j + 2 < KB) stage_in(after);
            const float sw = *reinterpret_cast<const float*>(st + at_sw);
#pragma unroll
            for (int tf = 0; tf < 4; ++tf) {
                const float scale = *reinterpret_cast<const float*>(st + at_sx + tf * 64) * sw;
                const Widened wx = widen(x);
                if (tf < 3) x = read_codes(st + at_x + (tf + 1) * kFragBytes, x_other);
                else if (more) x = read_codes(st_next + at_x, x_other);
#pragma unroll
                for (int nf = 0; nf < 4; ++nf) {
                    const f32x4 p = mfma_block(w[nf], wx);
                    if (tf == 3 && more) w[nf] = widen(read_codes(st_next + at_w + nf * kFragBytes, 1024));
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nf][tf][i] = fmaf(scale, p[i], acc[nf][tf][i]);
                }
            }
            slot = next;
        }
        const int col0 = n0 + wn * 64, first = wm * 64;            // this wavefront's columns and rows
        finish_values(a, e, col0, acc);
        if constexpr (OUT == kOutE4m3) {
            uint32_t most[4];
            row_magnitudes(a.N, col0, acc, most);
            if (lane < 16) {
#pragma unroll
                for (int tf = 0; tf < 4; ++tf) mosts[wn * kTileRows + first + tf * 16 + lane] = most[tf];
            }
            __syncthreads();
#pragma unroll
            for (int tf = 0; tf < 4; ++tf) most[tf] = max(most[tf], mosts[(wn ^ 1) * kTileRows + first + tf * 16 + r]);
            store_codes(a, col0, row0 + first, rows - first, acc, most, wn == 0);
        } else {
            store_values<OUT>(a, col0, row0 + first, rows - first, acc);
        }
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------
// Experts with at least this many rows run in tiles, the others are streamed.
constexpr int kTiledMinRows = 65;

// Parts that the contraction of a streamed product is cut into: calls of at most 64 rows whose units would leave most CUs without one.
// A grouped call's number of row tiles is not known here; half of the most it can be is taken.
static int stream_split(int rows, int N, int K, int E) {
    if (rows >= kTiledMinRows) return 1;
    const int tiles = E == 1 ? 1 : (std::min(rows, E) + 1) / 2;
    const int units = tiles * quant_blocks(N);
    return std::max(1, std::min(256 / units, quant_blocks(K) / 2));
}

size_t quant_product_workspace(const moe_quant_shape& s) {
    const int split = stream_split(s.rows, s.N, s.K, s.E);
    const size_t parts = split > 1 ? static_cast<size_t>(split) * s.rows * quant_pitch(s.N) * sizeof(float) : 0;
    return (std::max<size_t>(parts, 1) + 255) / 256 * 256;
}

template <int OUT>
static hipError_t launch_out(const QuantArgs& a, void* ws, hipStream_t stream) {
    const dim3 grid(device_cu_count()), threads(kStreamWaves * 64);
    const int split = stream_split(a.rows, a.N, a.K, a.E);
    if (split > 1) {
        QuantArgs parts = a;
        parts.out = ws;
        quant_stream_kernel<kOutParts><<<grid, threads, kStreamLdsBytes, stream>>>(parts, a.rows, split);
        quant_join_kernel<OUT><<<dim3(a.rows, (quant_blocks(a.N) + 7) / 8), dim3(256), 0, stream>>>(a, static_cast<const float*>(ws), split);
        return hipGetLastError();
    }
    if (a.rows >= kTiledMinRows) quant_tile_kernel<OUT><<<grid, dim3(kTileWaves * 64), kTileLdsBytes, stream>>>(a, kTiledMinRows);
    if (a.offsets != nullptr || a.rows < kTiledMinRows)
        quant_stream_kernel<OUT><<<grid, threads, kStreamLdsBytes, stream>>>(a, std::min(a.rows, kTiledMinRows - 1), 1);
    return hipGetLastError();
}

hipError_t configure_quant_kernels() {
    const struct {
        const void* kernel;
        int lds;
    } all[] = {{reinterpret_cast<const void*>(quant_tile_kernel<kOutF32>), kTileLdsBytes},
               {reinterpret_cast<const void*>(quant_tile_kernel<kOutBf16>), kTileLdsBytes},
               {reinterpret_cast<const void*>(quant_tile_kernel<kOutE4m3>), kTileLdsBytes},
               {reinterpret_cast<const void*>(quant_stream_kernel<kOutF32>), kStreamLdsBytes},
               {reinterpret_cast<const void*>(quant_stream_kernel<kOutBf16>), kStreamLdsBytes},
               {reinterpret_cast<const void*>(quant_stream_kernel<kOutE4m3>), kStreamLdsBytes},
               {reinterpret_cast<const void*>(quant_stream_kernel<kOutParts>), kStreamLdsBytes}};
    for (const auto& k : all) {
        const hipError_t e = hipFuncSetAttribute(k.kernel, hipFuncAttributeMaxDynamicSharedMemorySize, k.lds);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_quant_product(const QuantArgs& a, void* ws, hipStream_t stream) {
    if (a.out_dtype == MOE_F32) return launch_out<kOutF32>(a, ws, stream);
    if (a.out_dtype == MOE_BF16) return launch_out<kOutBf16>(a, ws, stream);
    return launch_out<kOutE4m3>(a, ws, stream);
}

}  // namespace moe
