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
#pragma unroll
        for (int tf = 0; tf < TF; ++tf)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nf][tf][i] = quant_activate(acc[nf][tf][i], a.act);
    }
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
        const float scale = block_scale(most[tf]), inv = 1.f / scale;
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

// ---- few rows per matrix: the weights are streamed -------------------------------------------------------------------
// Unit: up to 16 TFMAX rows of an expert x 16 NF WN columns.  WN wavefronts side by side, KS of them share the contraction and add up in
// LDS in a fixed order.  The weights come from memory straight into registers, a fragment of 2 KiB as two contiguous KiB, D blocks
// ahead; token rows come through L2.
template <int TF, int NF, int D>
__device__ __forceinline__ void stream_sums(const QuantArgs& a, int row0, int rows, const uint8_t* w, const float* sw, int kb0, int kb1,
                                            f32x4 (&acc)[NF][TF]) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int KB = quant_blocks(a.K);
    const size_t pitch = static_cast<size_t>(KB) * kQuantBlock;
    const uint8_t* x[TF];
    const float* sx[TF];
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        const size_t row = source_row(a, row0 + min(tf * 16 + r, rows - 1));
        x[tf] = a.a + row * pitch + g * 16;
        sx[tf] = a.a_scales + row * KB;
    }
    w += lane * 16;
    struct Step {
        i32x8 w[NF], x[TF];
        float sx[TF], sw;
    } ring[D];
    auto load = [&](Step& s, int kb) {
#pragma unroll
        for (int nf = 0; nf < NF; ++nf) {
            const uint8_t* p = w + (static_cast<size_t>(nf) * KB + kb) * kFragBytes;
            const i32x4 lo = *reinterpret_cast<const i32x4*>(p), hi = *reinterpret_cast<const i32x4*>(p + 1024);
            s.w[nf] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) {
            const uint8_t* p = x[tf] + static_cast<size_t>(kb) * kQuantBlock;
            const i32x4 lo = *reinterpret_cast<const i32x4*>(p), hi = *reinterpret_cast<const i32x4*>(p + 64);
            s.x[tf] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            s.sx[tf] = sx[tf][kb];
        }
        s.sw = sw[kb];
    };
    auto add = [&](const Step& s) {
        Widened wide[NF];
#pragma unroll
        for (int nf = 0; nf < NF; ++nf) wide[nf] = widen(s.w[nf]);
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) {
            const Widened x = widen(s.x[tf]);
            const float scale = s.sx[tf] * s.sw;
#pragma unroll
            for (int nf = 0; nf < NF; ++nf) {
                const f32x4 p = mfma_block(wide[nf], x);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nf][tf][i] = fmaf(scale, p[i], acc[nf][tf][i]);
            }
        }
    };
    if (kb0 >= kb1) return;
    // loads past the end repeat the last block: no load is conditional, so that the loop waits for the oldest ones only
#pragma unroll
    for (int i = 0; i < D; ++i) load(ring[i], min(kb0 + i, kb1 - 1));
    int kb = kb0;
    for (; kb + D <= kb1; kb += D) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            add(ring[i]);
            load(ring[i], min(kb + i + D, kb1 - 1));
        }
    }
#pragma unroll
    for (int i = 0; i < D; ++i)
        if (kb + i < kb1) add(ring[i]);
}

template <int TFMAX, int WN, int NF, int KS, int OUT>
__global__ __launch_bounds__(64 * WN * KS) void quant_stream_kernel(const QuantArgs a, int min_rows, int max_rows) {
    constexpr int kThreads = 64 * WN * KS, kCols = 16 * NF * WN;
    static_assert(OUT != kOutE4m3 || kCols == kQuantBlock, "a unit holds the columns that share a scale");
    __shared__ int32_t starts[MOE_MAX_E + 1], tmp[kThreads / 64];
    __shared__ f32x4 parts[KS > 1 ? (KS - 1) * WN * NF * TFMAX * 64 : 1];
    __shared__ uint32_t mosts[OUT == kOutE4m3 ? WN * TFMAX * 16 : 1];
    count_tiles<kThreads>(a, 16 * TFMAX, min_rows, max_rows, starts, tmp);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wn = wave % WN, ks = wave / WN;
    const int KB = quant_blocks(a.K), groups = (a.N + kCols - 1) / kCols;
    const int units = starts[a.E] * groups;
    const int kb0 = KB * ks / KS, kb1 = KB * (ks + 1) / KS;
    for (int u = xcd_position(); u < units; u += gridDim.x) {
        const int e = __builtin_amdgcn_readfirstlane(expert_of(starts, a.E, u / groups));
        const int tiles = starts[e + 1] - starts[e], local = u - starts[e] * groups;
        // the tiles of one column group follow each other: they read the same weights
        const int group = local / tiles, tile = local % tiles;
        const Segment seg = segment_of(a, e);
        const int row0 = __builtin_amdgcn_readfirstlane(seg.row0 + tile * 16 * TFMAX);
        const int rows = __builtin_amdgcn_readfirstlane(min(16 * TFMAX, seg.rows - tile * 16 * TFMAX));
        const int n0 = __builtin_amdgcn_readfirstlane(group * kCols + wn * 16 * NF);
        const uint8_t* w = a.w + static_cast<size_t>(e) * quant_matrix_bytes(a.N, a.K) + static_cast<size_t>(n0 / 16) * KB * kFragBytes;
        const float* sw = a.w_scales + (static_cast<size_t>(e) * quant_blocks(a.N) + n0 / kQuantBlock) * KB;
        auto run = [&](auto tf_const) {
            constexpr int TF = decltype(tf_const)::value;
            f32x4 acc[NF][TF];
#pragma unroll
            for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) acc[nf][tf] = f32x4{0.f, 0.f, 0.f, 0.f};
            stream_sums<TF, NF, (TF <= 2 ? 4 : 3)>(a, row0, rows, w, sw, kb0, kb1, acc);
            if constexpr (KS > 1) {
                f32x4* part = parts + (wn * NF * TF) * 64 + lane;
                if (ks > 0) {
#pragma unroll
                    for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                        for (int tf = 0; tf < TF; ++tf) part[((ks - 1) * WN * NF * TF + nf * TF + tf) * 64] = acc[nf][tf];
                }
                __syncthreads();
                if (ks == 0) {
#pragma unroll
                    for (int s = 1; s < KS; ++s)
#pragma unroll
                        for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                            for (int tf = 0; tf < TF; ++tf) acc[nf][tf] += part[((s - 1) * WN * NF * TF + nf * TF + tf) * 64];
                }
            }
            if (ks == 0) finish_values(a, e, n0, acc);
            if constexpr (OUT == kOutE4m3) {
                uint32_t most[TF];
                if (ks == 0) {
                    row_magnitudes(a.N, n0, acc, most);
                    if (lane < 16) {
#pragma unroll
                        for (int tf = 0; tf < TF; ++tf) mosts[wn * TFMAX * 16 + tf * 16 + lane] = most[tf];
                    }
                }
                __syncthreads();
                if (ks == 0) {
#pragma unroll
                    for (int tf = 0; tf < TF; ++tf)
#pragma unroll
                        for (int v = 0; v < WN; ++v) most[tf] = max(most[tf], mosts[v * TFMAX * 16 + tf * 16 + (lane & 15)]);
                    store_codes(a, n0, row0, rows, acc, most, wn == 0);
                }
            } else {
                if (ks == 0) store_values<OUT>(a, n0, row0, rows, acc);
            }
        };
        const int tf = (rows + 15) >> 4;
        if (TFMAX == 1 || tf == 1) run(std::integral_constant<int, 1>{});
        else if (TFMAX == 2 || tf == 2) run(std::integral_constant<int, (TFMAX < 2 ? TFMAX : 2)>{});
        else run(std::integral_constant<int, TFMAX>{});
        if constexpr (KS > 1 || OUT == kOutE4m3) __syncthreads();       // the LDS is the next unit's
    }
}

// ---- many rows per matrix: tiles in LDS -----------------------------------------------------------------------------
// Unit: 256 rows x 128 columns by 8 wavefronts (4 x 2, 64 x 64 each), a block of 128 columns of the contraction per step, through a
// ring of three LDS stages: one being read, one that has landed (its first fragments are read ahead), one in flight.  Everything goes from
// memory to LDS directly, 16 bytes per lane; a stage holds
//   rows     [256][128 bytes], copied a whole line per eight lanes; the 16-byte pieces of a row are permuted by its number so that the
//            operand reads (16 rows x one piece) meet no bank twice: piece c of row r lies at c ^ (r / 2 % 8)
//   weights  8 fragments of 2 KiB as they are packed, 16 rows each
//   scales   of the 256 rows, and the weights' (one for the unit's 128 columns)
constexpr int kTileRows = 256, kTileCols = kQuantBlock, kTileWaves = 8, kTileStages = 3;
constexpr int kStageW = kTileRows * kQuantBlock, kStageS = kStageW + kTileCols * kQuantBlock, kStage = kStageS + kTileRows * 4 + 256;
constexpr int kTileMost = kTileStages * kStage, kTileStarts = kTileMost + 2 * kTileRows * 4;
constexpr int kTileLdsBytes = kTileStarts + (MOE_MAX_E + 1 + kTileWaves) * 4;
static_assert(kTileLdsBytes <= 160 * 1024, "fits a CU");

// 4 bytes per lane into LDS, as copy16_to_lds
__device__ __forceinline__ void copy4_to_lds(const void* src, uint32_t lds_base) {
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(dst) : "memory");
}

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
    // operand reads: piece g of row r, the other half's piece 4 + g is 64 bytes away by exclusive or
    const int at_x = (wm * 64 + r) * kQuantBlock + ((g ^ (r >> 1)) << 4), at_w = kStageW + wn * 4 * kFragBytes + lane * 16;
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
            from_rows[i] = a.a + row * pitch + (((lane & 7) ^ (in_tile >> 1 & 7)) << 4);
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

        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");       // the ring is free
        stage_in(0);
        if (KB > 1) stage_in(1);
        if (KB > 1) asm volatile("s_waitcnt vmcnt(7)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        auto read_codes = [&](const unsigned char* p, int other) {
            const i32x4 lo = *reinterpret_cast<const i32x4*>(p), hi = *reinterpret_cast<const i32x4*>(p + other);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        const int x_other = (at_x & 64) ? -64 : 64;
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
            if (more) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
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
size_t quant_product_workspace(const moe_quant_shape&) { return 256; }

// Experts with at least this many rows run in tiles, the others are streamed.
constexpr int kTiledMinRows = 65;

template <int OUT>
static hipError_t launch_out(const QuantArgs& a, hipStream_t stream) {
    const int cus = device_cu_count();
    const int grid = 2 * cus, stream_max = std::min(a.rows, kTiledMinRows - 1);
    if (a.rows >= kTiledMinRows) quant_tile_kernel<OUT><<<dim3(cus), dim3(kTileWaves * 64), kTileLdsBytes, stream>>>(a, kTiledMinRows);
    if (a.offsets == nullptr && a.rows >= kTiledMinRows) return hipGetLastError();
    if (a.rows <= 16) quant_stream_kernel<1, 4, 2, 2, OUT><<<dim3(grid), dim3(512), 0, stream>>>(a, 1, stream_max);
    else if (a.rows <= 32) quant_stream_kernel<2, 4, 2, 2, OUT><<<dim3(grid), dim3(512), 0, stream>>>(a, 1, stream_max);
    else quant_stream_kernel<4, 4, 2, 2, OUT><<<dim3(grid), dim3(512), 0, stream>>>(a, 1, stream_max);
    return hipGetLastError();
}

hipError_t configure_quant_kernels() {
    for (const void* f : {reinterpret_cast<const void*>(quant_tile_kernel<kOutF32>), reinterpret_cast<const void*>(quant_tile_kernel<kOutBf16>),
                          reinterpret_cast<const void*>(quant_tile_kernel<kOutE4m3>)}) {
        const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, kTileLdsBytes);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_quant_product(const QuantArgs& a, void*, hipStream_t stream) {
    if (a.out_dtype == MOE_F32) return launch_out<kOutF32>(a, stream);
    if (a.out_dtype == MOE_BF16) return launch_out<kOutBf16>(a, stream);
    return launch_out<kOutE4m3>(a, stream);
}

}  // namespace moe
