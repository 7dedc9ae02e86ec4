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
    i32x4 v[4];
    __device__ __forceinline__ bf16x8 eight(int i) const { return __builtin_bit_cast(bf16x8, v[i]); }
    // the values of codes 2 n, 2 n + 1, in the four bytes that hold them
    __device__ __forceinline__ void widen_two(int32_t codes, int n) {
        v[n >> 2][n & 3] = __builtin_bit_cast(int32_t, n & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, true)
                                                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, false));
    }
};
// the values of codes 8 k ... 8 k + 7
__device__ __forceinline__ bf16x8 widen8(const i32x8& codes, int k) {
    Widened r;
#pragma unroll
    for (int n = 4 * k; n < 4 * k + 4; ++n) r.widen_two(codes[n >> 1], n);
    return r.eight(k);
}
__device__ __forceinline__ Widened widen(const i32x8& codes) {
    Widened r;
#pragma unroll
    for (int n = 0; n < 16; ++n) r.widen_two(codes[n >> 1], n);
    return r;
}

// The matrix instruction's first operand is 16 weight rows, the second one 16 token rows.  Lane l holds 32 codes of row l % 16 of each;
// which columns they are does not matter as long as both operands agree (moe.h: 64 h + 16 (l / 16), h = 0, 1).  Result i of lane l: weight
// row 4 (l / 16) + i, token row l % 16.
//
// Which matrix units (EIGHT): those for 8-bit operands (v_mfma_f32_16x16x128_f8f6f4) take twice the products per cycle and need no widened
// codes, but add products in groups of eight neighbours, cut at 2^-13 of the power of two of the group's largest; the groups' sums are fp32.
// Measured: 1.5e-5 of the rms of a sum of 128 products of normal values, 5e-5 where one column of a block is 50 times the others, and where
// large products cancel, all of what they leave.  The bf16 units' sums of widened codes are exact to 1e-8 of the rms.  So the bf16 units are
// used, and the 8-bit ones where the caller asks for them (MOE_QUANT_UNIT_SUMS); the parts of a cut contraction are fp32 sums either way.
__device__ __forceinline__ f32x4 multiply_codes(const i32x8& w, const i32x8& x) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);     // e4m3 both, scales of one
}

__device__ __forceinline__ float quant_activate(float v, int act) {
    if (act == MOE_ACT_GELU) return gelu_exp(v);
    if (act == MOE_ACT_RELU) return v < 0.f ? 0.f : v;      // NaN stays
    return v;
}

// A value whose uses are computed where they stand: what is needed once per unit is not to be kept in registers through the steps.
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// The same value for the whole wavefront, told to the compiler where it cannot see it.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <typename P>
__device__ __forceinline__ const P* uniform(const P* p) {
    const uint64_t v = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const P*>(static_cast<uint64_t>(static_cast<uint32_t>(uniform(static_cast<int>(v)))) |
                                      static_cast<uint64_t>(static_cast<uint32_t>(uniform(static_cast<int>(v >> 32)))) << 32);
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
// The same for an expert that runs, its number the same for the whole wavefront, by scalar loads: they are not counted with the copies into LDS.
__device__ __forceinline__ Segment segment_of_unit(const QuantArgs& a, int e) {
    if (a.offsets == nullptr) return Segment{0, a.rows};
    const auto* offsets = (const __attribute__((address_space(4))) int32_t*)a.offsets;
    const int lo = min(max(offsets[e], 0), a.rows), hi = min(max(offsets[e + 1], lo), a.rows);
    return Segment{lo, hi - lo};
}
// Row of `a` that row p of the product reads.
__device__ __forceinline__ int source_row(const QuantArgs& a, int p) {
    if (a.perm == nullptr) return p;
    return min(max(a.perm[p], 0), a.rows - 1) / a.k;
}

// Row tiles of the experts of at least min_rows rows, counted by every block for itself: E is at most 1024, a list in memory would cost
// a launch.  whole[e] is the number of tiles of `tile_rows` rows that the experts before e have, whole[E] that of all; `rest` lists the
// experts with a shorter last tile, those of more than 128 rows first, then of more than 64, then the others, so that units of one length
// are handed out together.  Returns how many of these there are.  `tmp`: four ints per wavefront.
// Offsets that are none (0, rows, 0, rows, ...) may give every other expert all rows: the whole tiles end at as many as the rows have, which
// keeps their number times the column groups within 32 bits.
template <int THREADS>
__device__ __forceinline__ int count_tiles(const QuantArgs& a, int tile_rows, int min_rows, int32_t* whole, uint16_t* rest, int4* tmp) {
    constexpr int W = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, most = a.rows / tile_rows;
    int4 before = {0, 0, 0, 0};            // whole tiles, and last tiles by length
    int kind_base[3] = {0, 0, 0};
    // the lengths' totals are needed before the first expert's place is known: first pass counts, second one places
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 1) {
            if (before.x + before.y + before.z + before.w == 0) break;         // the same for every thread
            kind_base[1] = before.y;
            kind_base[2] = before.y + before.z;
            if (threadIdx.x == 0) whole[a.E] = before.x;
            before = int4{0, 0, 0, 0};
        }
        for (int e0 = 0; e0 < a.E; e0 += THREADS) {
            const int e = e0 + threadIdx.x;
            int m = e < a.E ? segment_of(a, e).rows : 0;
            if (m < min_rows) m = 0;
            const int n = m / tile_rows, left = m - n * tile_rows;
            const int kind = left == 0 ? -1 : left > 128 ? 0 : left > 64 ? 1 : 2;
            const int incl = wave_scan(n);
            const uint64_t k0 = __ballot(kind == 0), k1 = __ballot(kind == 1), k2 = __ballot(kind == 2);
            if (lane == 63) tmp[wave] = int4{incl, __popcll(k0), __popcll(k1), __popcll(k2)};
            __syncthreads();
            int4 mine = before;
            for (int w = 0; w < W; ++w) {
                const int4 t = tmp[w];
                if (w < wave) mine = int4{min(mine.x + t.x, most), mine.y + t.y, mine.z + t.z, mine.w + t.w};
                before = int4{min(before.x + t.x, most), before.y + t.y, before.z + t.z, before.w + t.w};
            }
            if (pass == 1) {
                if (e < a.E) whole[e] = min(mine.x + incl - n, most);
                const uint64_t below = (1ull << lane) - 1;
                const int at = kind == 0 ? mine.y + __popcll(k0 & below)
                             : kind == 1 ? kind_base[1] + mine.z + __popcll(k1 & below)
                                         : kind_base[2] + mine.w + __popcll(k2 & below);
                if (kind >= 0) rest[at] = static_cast<uint16_t>(e);
            }
            __syncthreads();
        }
    }
    if (before.x + before.y + before.z + before.w == 0 && threadIdx.x == 0) whole[a.E] = 0;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(before.y + before.z + before.w);
}
// The expert that tile t of a list belongs to: the last whose tiles begin at or before t.  By whole wavefronts.
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
// A wavefront's NF x TF results of 16 columns x 16 rows: columns n0 + 16 nf + 4 (lane / 16) + i, rows row0 + STRIDE tf + lane % 16; of the
// rows from row0 on, `rows` exist.
template <int NF, int TF>
__device__ __forceinline__ void activate_values(int act, f32x4 (&acc)[NF][TF]) {
    if (act == MOE_ACT_GELU) {
#pragma unroll
        for (int nf = 0; nf < NF; ++nf)
#pragma unroll
            for (int tf = 0; tf < TF; ++tf) {
                acc[nf][tf] = activate4<MOE_ACT_GELU>(acc[nf][tf]);
                if (NF * TF > 4) __builtin_amdgcn_sched_barrier(0);        // many values at once would need registers that there are not
            }
    } else if (act == MOE_ACT_RELU) {
#pragma unroll
        for (int nf = 0; nf < NF; ++nf)
#pragma unroll
            for (int tf = 0; tf < TF; ++tf)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[nf][tf][i] = acc[nf][tf][i] < 0.f ? 0.f : acc[nf][tf][i];        // NaN stays
    }
}
template <int NF, int TF>
__device__ __forceinline__ void finish_values(const QuantArgs& a, int e, int n0, f32x4 (&acc)[NF][TF]) {
    const int g = (here(threadIdx.x) & 63) >> 4;
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

// Lane group g (of 16) holds v[nf] = columns 16 nf + 4 g ...; afterwards v[i] = columns 16 g + 4 i ...: a lane's four pieces are
// neighbours, so that it stores 16 bytes instead of four times 4 (a store of 4 bytes per lane to 16 rows costs the memory path as much
// as one of 16).
__device__ __forceinline__ void gather_columns(uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto s = __builtin_amdgcn_permlane32_swap(v[i], v[i + 2], false, false);
        v[i] = s[0];
        v[i + 2] = s[1];
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const auto s = __builtin_amdgcn_permlane16_swap(v[i], v[i + 1], false, false);
        v[i] = s[0];
        v[i + 1] = s[1];
    }
}

// Lane group g holds u = piece g of 32 columns' first half, v = of their second half (4 columns a piece); afterwards pieces 2 g, 2 g + 1 of
// all 32, so that a store of 8 columns per lane covers 64 bytes of each row.
__device__ __forceinline__ void gather_pair(uint32_t& u, uint32_t& v) {
    const auto s = __builtin_amdgcn_permlane32_swap(u, v, false, false);
    const auto t = __builtin_amdgcn_permlane16_swap(s[0], s[1], false, false);
    u = t[0];
    v = t[1];
}

template <int OUT, int STRIDE, int NF, int TF>
__device__ __forceinline__ void store_values(const QuantArgs& a, int n0, int row0, int rows, const f32x4 (&acc)[NF][TF]) {
    static_assert(OUT != kOutE4m3, "");
    const int lane = here(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
    // four columns at once where every row begins on a boundary of four
    const bool wide = a.N % 4 == 0 && reinterpret_cast<uintptr_t>(a.out) % (OUT == kOutF32 ? 16 : 8) == 0;
    if (OUT == kOutBf16 && NF == 4 && a.N % 8 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0) {
#pragma unroll
        for (int tf = 0; tf < TF; ++tf) {
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int nf = 0; nf < 4; ++nf) {
                lo[nf] = pack_bf16x2(acc[nf % NF][tf][0], acc[nf % NF][tf][1]);
                hi[nf] = pack_bf16x2(acc[nf % NF][tf][2], acc[nf % NF][tf][3]);
            }
#pragma unroll
            for (int t = 0; t < 4; t += 2) {
                gather_pair(lo[t], lo[t + 1]);
                gather_pair(hi[t], hi[t + 1]);
            }
            if (tf * STRIDE + r >= rows) continue;
            const int n = n0 + g * 8;
            uint16_t* out = static_cast<uint16_t*>(a.out) + static_cast<size_t>(row0 + tf * STRIDE + r) * a.N + n;
            if (n < a.N) *reinterpret_cast<uint4*>(out) = uint4{lo[0], hi[0], lo[1], hi[1]};
            if (n + 32 < a.N) *reinterpret_cast<uint4*>(out + 32) = uint4{lo[2], hi[2], lo[3], hi[3]};
        }
        return;
    }
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        if (tf * STRIDE + r >= rows) continue;
        const size_t at = static_cast<size_t>(row0 + tf * STRIDE + r) * a.N;
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
    if (n0 + NF * 16 > N) {                 // some do not exist
        const int g = (here(threadIdx.x) & 63) >> 4;
#pragma unroll
        for (int tf = 0; tf < TF; ++tf)
#pragma unroll
            for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n0 + nf * 16 + g * 4 + i >= N) acc[nf][tf][i] = 0.f;
    }
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        uint32_t m = 0;
#pragma unroll
        for (int nf = 0; nf < NF; ++nf)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m = max(m, magnitude(acc[nf][tf][i]));
            }
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, 64)));
        m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, 64)));
        most[tf] = m;
    }
}

// Codes of a block of 128 columns whose rows' largest magnitudes are known; the wavefront with `scales` also stores the scales.
template <int STRIDE, int NF, int TF>
__device__ __forceinline__ void store_codes(const QuantArgs& a, int n0, int row0, int rows, const f32x4 (&acc)[NF][TF],
                                            const uint32_t (&most)[TF], bool scales) {
    const int lane = here(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
    const size_t pitch = quant_pitch(a.N);
#pragma unroll
    for (int tf = 0; tf < TF; ++tf) {
        const size_t row = static_cast<size_t>(row0 + tf * STRIDE + r);
        const float scale = block_scale(most[tf]);
        const BlockQuotient of(scale);
        uint32_t codes[NF];
#pragma unroll
        for (int nf = 0; nf < NF; ++nf) {
            const int n = n0 + nf * 16 + g * 4;
            const f32x4 v = acc[nf][tf];
            codes[nf] = pack_e4m3x4(of(v[0]), of(v[1]), of(v[2]), of(v[3]));
            if (n + 4 > a.N) codes[nf] = n >= a.N ? 0u : codes[nf] & (0xffffffffu >> (8 * (n + 4 - a.N)));     // zeros past the end
        }
        if constexpr (NF == 4) gather_columns(codes);
        if (tf * STRIDE + r >= rows) continue;
        uint8_t* out = static_cast<uint8_t*>(a.out) + row * pitch + n0;
        if constexpr (NF == 4) {
            *reinterpret_cast<uint4*>(out + g * 16) = uint4{codes[0], codes[1], codes[2], codes[3]};
        } else {
#pragma unroll
            for (int nf = 0; nf < NF; ++nf) *reinterpret_cast<uint32_t*>(out + nf * 16 + g * 4) = codes[nf];
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
// copy16_to_lds of what is read once: the lines are the first to leave the caches
__device__ __forceinline__ void copy16_once_to_lds(const void* src, uint32_t lds_base) {
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt" : : "v"(src), "s"(dst) : "memory");
}
// The same from 32-bit offsets to a base that is the same for the whole wavefront: half the registers, and the base moves on for free
__device__ __forceinline__ void copy16_to_lds(const void* base, uint32_t offset, uint32_t lds_base) {
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(uniform(static_cast<const char*>(base))), "s"(dst) : "memory");
}
__device__ __forceinline__ void copy4_to_lds(const void* base, uint32_t offset, uint32_t lds_base) {
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(offset), "s"(uniform(static_cast<const char*>(base))), "s"(dst) : "memory");
}
// The wavefront's copies up to the newest `left` have landed, and with the barrier everybody's; every LDS read before it is done too.
template <int LEFT>
__device__ __forceinline__ void copies_landed() {
    static_assert(LEFT < 64, "vmcnt has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory");
}
// The same where `known` says (to the whole wavefront) that they have landed: no wait for what was issued since.  One block, so that no branch
// of the compiler's divides a step.
template <int LEFT>
__device__ __forceinline__ void copies_landed_unless(uint32_t known) {
    static_assert(LEFT < 64, "vmcnt has six bits");
    asm volatile("s_cmp_lg_u32 %0, 0\n\ts_cbranch_scc1 .Lknown%=\n\ts_waitcnt vmcnt(%1)\n.Lknown%=:\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier"
                 : : "s"(uniform(static_cast<int>(known))), "n"(LEFT) : "memory", "scc");
}
__device__ __forceinline__ i32x8 read_codes(const unsigned char* p, int other) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(p), hi = *reinterpret_cast<const i32x4*>(p + other);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Rows in LDS: 128 bytes each, the 16-byte pieces of a row permuted by its number, so that an operand read (16 rows x one piece) meets no
// bank twice: piece c of row r lies at c ^ (r / 2 % 8).  A copy brings 8 rows, each a whole line by eight lanes.
__device__ __forceinline__ int piece_of_lane(int lane, int row) { return ((lane & 7) ^ (row >> 1 & 7)) << 4; }
// Where lane l reads piece l / 16 of row `first` + l % 16 (`first` a multiple of 16), and how far from there piece 4 + l / 16 lies.
__device__ __forceinline__ int row_operand(int tid, int first) {
    const int lane = tid & 63, r = lane & 15;
    return (first + r) * kQuantBlock + (((lane >> 4) ^ (r >> 1)) << 4);
}
__device__ __forceinline__ int row_operand_other(int at) { return at & 64 ? -64 : 64; }

// ---- few rows per matrix: the weights are streamed -------------------------------------------------------------------
// Unit: an expert's rows, at most 64, x 128 NF columns, by 8 wavefronts of 16 NF columns each, a block of 128 columns of the contraction
// per step.  Bound by memory (49 experts of one to three rows, 2048 x 8192: 131 to 140 us = 6.1 to 6.5 TB/s; 64 experts of 32 rows, 3072 x
// 768, e4m3 out: 39 us = 3.9 TB/s, 34 with the 8-bit units, 3 of them for the launch), so what matters is that copies never stop: weights (16 NF KiB a step), rows and scales go to LDS directly,
// through a ring of stages that runs on across units.  A block's units follow each other in one expert, where nothing needs to be looked
// up (a load that the compiler sees would make it wait for every copy in flight).
constexpr int kStreamRows = 64, kStreamWaves = 8;
template <int NF>
struct Streams {
    static constexpr int kStages = NF == 1 ? 6 : 3, kCols = NF * kQuantBlock;
    static constexpr int kX = kCols * kQuantBlock, kS = kX + kStreamRows * kQuantBlock;
    // pieces of 256 bytes: scales of the rows, scale of each 128 columns (64 times), bias of the columns
    static constexpr int kPieces = 1 + 3 * NF, kSw = kS + 256, kBias = kSw + NF * 256, kStage = kS + kPieces * 256;
    static constexpr int kMost = kStages * kStage, kList = kMost + kStreamWaves * kStreamRows * 4;
    static constexpr int kLdsBytes = kList + MOE_MAX_E * 2 + kStreamWaves * 4;
    static constexpr int kCopies = 2 * NF + 2;          // a wavefront's, per stage
    static_assert(kLdsBytes <= 160 * 1024 && kPieces <= kStreamWaves, "fits a CU");
};

// The experts of 1 ... max_rows rows, in order, counted by every block for itself; returns how many.  `tmp`: an int per wavefront.
template <int THREADS>
__device__ __forceinline__ int list_experts(const QuantArgs& a, int max_rows, uint16_t* list, int32_t* tmp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += THREADS) {
        const int e = e0 + threadIdx.x;
        const int rows = e < a.E ? segment_of(a, e).rows : 0;
        const bool in = rows > 0 && rows <= max_rows;
        const uint64_t ins = __ballot(in);
        if (lane == 0) tmp[wave] = __popcll(ins);
        __syncthreads();
        int at = before + __popcll(ins & ((1ull << lane) - 1));
        for (int w = 0; w < THREADS / 64; ++w) {
            const int n = tmp[w];
            if (w < wave) at += n;
            before += n;
        }
        if (in) list[at] = static_cast<uint16_t>(e);
        __syncthreads();
    }
    return __builtin_amdgcn_readfirstlane(before);
}

// OUT = kOutParts: the contraction is cut into `split` parts, whose sums go to a.out as [split][rows][pitch of N] fp32.
constexpr int kOutParts = 3;

template <int OUT, int NF, bool EIGHT>
__device__ __forceinline__ void stream_units(const QuantArgs& a, int tiles, int parts_wanted, int b, unsigned char* smem) {
    using S = Streams<NF>;
    constexpr int kStages = S::kStages, kStage = S::kStage;
    const int split = OUT == kOutParts ? parts_wanted : 1;
    uint32_t* mosts = reinterpret_cast<uint32_t*>(smem + S::kMost);         // [64][8]
    const uint16_t* list = reinterpret_cast<const uint16_t*>(smem + Streams<1>::kList);
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

    // copies: wavefront w brings rows 8 w ... 8 w + 7, weight fragments NF w ..., and one of the pieces of scales and bias (some twice)
    const uint32_t lds = lds_address(smem);
    const int piece = NF == 1 ? wave & 3 : min(wave, S::kPieces - 1);
    const uint32_t to_weights = lds + wave * NF * kFragBytes, to_rows = lds + S::kX + wave * 1024, to_scales = lds + S::kS + piece * 256;
    const uint8_t *tile_row, *row_from, *weights_from;
    const float *tile_scale, *scales_from;
    int scales_step;
    auto point_at_tile = [&](const Unit& w) __attribute__((always_inline)) {
        const int in_tile = wave * 8 + (lane >> 3);
        tile_row = a.a + source_row(a, w.row0 + min(in_tile, w.rows - 1)) * pitch + piece_of_lane(lane, in_tile);
        tile_scale = a.a_scales + static_cast<size_t>(source_row(a, w.row0 + min(lane, w.rows - 1))) * KB;
    };
    auto point_at = [&](const Unit& w) __attribute__((always_inline)) {
        row_from = tile_row + static_cast<size_t>(w.kb) * kQuantBlock;
        // columns of the last unit that do not exist are read as the last ones that do, and not stored
        const int fragment = min(w.group * 8 * NF + wave * NF, blocks * 8 - NF);
        weights_from = a.w + static_cast<size_t>(w.e) * quant_matrix_bytes(a.N, a.K) + (static_cast<size_t>(fragment) * KB + w.kb) * kFragBytes + lane * 16;
        scales_step = 1;
        if (piece == 0) scales_from = tile_scale + w.kb;
        else if (piece <= NF || a.bias == nullptr) scales_from = a.w_scales + (static_cast<size_t>(w.e) * blocks + min(w.group * NF + min(piece, NF) - 1, blocks - 1)) * KB + w.kb;
        else {
            scales_from = a.bias + static_cast<size_t>(w.e) * a.N + min(w.group * S::kCols + (piece - 1 - NF) * 64 + lane, a.N - 1);
            scales_step = 0;
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
            for (int i = 0; i < S::kCopies; ++i) copy4_to_lds(tile_scale, to_scales + slot_in * kStage);
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
    const int at_sx = S::kS + r * 4, at_sw = S::kSw + wave * NF / 8 * 256, at_bias = S::kBias + (wave * NF * 16 + (lane >> 4) * 4) * 4;
    int slot = 0;
    while (true) {
        auto run_unit = [&](auto tf_const) __attribute__((always_inline)) {
            constexpr int TF = decltype(tf_const)::value;
            f32x4 acc[NF][TF], bias[NF];
#pragma unroll
            for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) acc[nf][tf] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (; cur.kb < cur.kb1; ++cur.kb) {
                copies_landed<(kStages - 2) * S::kCopies>();
                const unsigned char* st = smem + slot * kStage;
                i32x8 w[NF], x[TF];
                float sx[TF];
#pragma unroll
                for (int nf = 0; nf < NF; ++nf) w[nf] = read_codes(st + at_w + nf * kFragBytes, 1024);
                const float sw = *reinterpret_cast<const float*>(st + at_sw);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) x[tf] = read_codes(st + at_x + tf * kFragBytes, x_other);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) sx[tf] = *reinterpret_cast<const float*>(st + at_sx + tf * 64);
                if constexpr (OUT != kOutParts) {
#pragma unroll
                    for (int nf = 0; nf < NF; ++nf) bias[nf] = *reinterpret_cast<const f32x4*>(st + at_bias + nf * 64);
                }
                copy_next();
                f32x4 p[NF][TF];
                if constexpr (EIGHT) {
#pragma unroll
                    for (int tf = 0; tf < TF; ++tf)
#pragma unroll
                        for (int nf = 0; nf < NF; ++nf) p[nf][tf] = multiply_codes(w[nf], x[tf]);
                } else {
                    // a quarter of the block after the other, so that the fragments' sums are independent of each other and codes are
                    // widened while others are multiplied
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        bf16x8 wide[NF];
#pragma unroll
                        for (int nf = 0; nf < NF; ++nf) wide[nf] = widen8(w[nf], k);
#pragma unroll
                        for (int tf = 0; tf < TF; ++tf) {
                            const bf16x8 row = widen8(x[tf], k);
#pragma unroll
                            for (int nf = 0; nf < NF; ++nf)
                                p[nf][tf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[nf], row, k == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : p[nf][tf], 0, 0, 0);
                        }
                    }
                }
#pragma unroll
                for (int tf = 0; tf < TF; ++tf) {
                    const float scale = sx[tf] * sw;
#pragma unroll
                    for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[nf][tf][i] = fmaf(scale, p[nf][tf][i], acc[nf][tf][i]);
                }
                slot = slot == kStages - 1 ? 0 : slot + 1;
            }
            const int n0 = cur.group * S::kCols + wave * NF * 16;
            if constexpr (OUT == kOutParts) {
                static_assert(NF == 1, "calls of few rows are cut, which have few columns per unit");
                float* parts = static_cast<float*>(a.out) + static_cast<size_t>(cur.part) * a.rows * quant_pitch(a.N);
#pragma unroll
                for (int tf = 0; tf < TF; ++tf)
                    if (tf * 16 + r < cur.rows)
                        *reinterpret_cast<f32x4*>(parts + static_cast<size_t>(cur.row0 + tf * 16 + r) * quant_pitch(a.N) + n0 + (lane >> 4) * 4) =
                            acc[0][tf];
            } else {
                if (a.bias != nullptr) {
#pragma unroll
                    for (int nf = 0; nf < NF; ++nf)
#pragma unroll
                        for (int tf = 0; tf < TF; ++tf) acc[nf][tf] += bias[nf];
                }
                activate_values(a.act, acc);
                if constexpr (OUT == kOutE4m3) {
                    constexpr int kSharing = kStreamWaves / NF;         // wavefronts whose columns share a scale
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
                        for (int v = 0; v < kSharing; v += 4) {
                            const uint4 m = *reinterpret_cast<const uint4*>(mosts + (tf * 16 + r) * kStreamWaves + wave / kSharing * kSharing + v);
                            most[tf] = max(most[tf], max(max(m.x, m.y), max(m.z, m.w)));
                        }
                    if (n0 < blocks * kQuantBlock) store_codes<16>(a, n0, cur.row0, cur.rows, acc, most, wave % kSharing == 0);
                } else {
                    store_values<OUT, 16>(a, n0, cur.row0, cur.rows, acc);
                }
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

template <int OUT, bool EIGHT>
__global__ __launch_bounds__(kStreamWaves * 64) void quant_stream_kernel(const QuantArgs a, int max_rows, int parts_wanted) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t* list = reinterpret_cast<uint16_t*>(smem + Streams<1>::kList);
    const int tiles = list_experts<kStreamWaves * 64>(a, max_rows, list, reinterpret_cast<int32_t*>(list + MOE_MAX_E));
    stream_units<OUT, 1, EIGHT>(a, tiles, parts_wanted, blockIdx.x, smem);
}

// Adds up the parts of a split contraction, in their order, and finishes the rows.  A block of threads per row and 8 groups of 128
// columns; four columns per thread.
template <int OUT>
__global__ __launch_bounds__(256) void quant_join_kernel(const QuantArgs a, const float* __restrict__ parts, int split) {
    const int row = blockIdx.x, lane = threadIdx.x & 63;
    const int n0 = (blockIdx.y * 256 + threadIdx.x) * 4;
    const size_t pitch = quant_pitch(a.N);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n0 < static_cast<int>(pitch)) {
        const float* p = parts + static_cast<size_t>(row) * pitch + n0;
        const size_t stride = static_cast<size_t>(a.rows) * pitch;
        int s = 0;
        for (; s + 4 <= split; s += 4) {
            f32x4 part[4];                 // four loads in flight, added in the parts' order
#pragma unroll
            for (int i = 0; i < 4; ++i) part[i] = *reinterpret_cast<const f32x4*>(p + (s + i) * stride);
#pragma unroll
            for (int i = 0; i < 4; ++i) v += part[i];
        }
        for (; s < split; ++s) v += *reinterpret_cast<const f32x4*>(p + s * stride);
    }
    int e = 0;
    if (a.offsets != nullptr) {            // the expert whose rows this one is among: as many end at or before it as precede that
        for (int e0 = 0; e0 < a.E; e0 += 256) e += __syncthreads_count(e0 + static_cast<int>(threadIdx.x) < a.E && a.offsets[e0 + threadIdx.x + 1] <= row);
        if (e >= a.E) return;
        const Segment seg = segment_of(a, e);
        if (row < seg.row0 || row >= seg.row0 + seg.rows) return;
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
        const float scale = block_scale(most);
        const BlockQuotient of(scale);
        if (n0 < static_cast<int>(pitch)) {
            uint32_t codes = pack_e4m3x4(of(v[0]), of(v[1]), of(v[2]), of(v[3]));
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
// Unit: 64 R rows (R = 1, 2, 4) x 128 columns by 8 wavefronts, a block of 128 columns of the contraction per step, through a ring of
// LDS stages: one being read, one that has landed (its first fragments are read ahead), the others in flight.  Everything goes from memory
// to LDS directly, 16 bytes per lane; a stage holds
//   rows     [64 RMAX][128 bytes]
//   weights  8 fragments of 2 KiB as they are packed, 16 rows each
//   scales   of the rows, and the weights' (one for the unit's 128 columns)
// Wavefront (wm, wn) of the 4 x 2 multiplies row fragments wm, wm + 4, ... (R of them) and the columns 64 wn ... 64 wn + 63.
//
// What bounds it: with the bf16 units the vector unit, which widens 128 x 64 codes per matrix unit and step (16384 x 8192 x 8192, bf16 out: 1776
// us = 1240 TFLOP/s; x 2048: 483 us = 1140; with GeLU to e4m3 568; 16384 x 2048 x 8192, fp32 out: 460 us = 1200).  With the 8-bit units (1050 us =
// 2090 TFLOP/s; 296 = 1860; 363; a library product with one scale per operand, 16384 x 8192 x 2048: 254 us) the power limit, under which the
// clock falls to 1.4 to 1.8 GHz, and the copies: of 1054 us a copy of this kernel without the copies took 771, without the LDS reads 1045, with
// neither 698, without the multiply-adds 1058, copying one stage over and over 1043, so that it is not the distance to the memory.  Units of
// 256 x 256, which copy a third less per product, took 1064 us where this kernel took 1095 on the same card, but 349 against 307 for 2048
// columns of contraction: the next unit's copies have half the time, twice the sums are finished at once and registers run out there.
constexpr int kTileWaves = 8;
template <int RMAX>
struct Tiles {
    static constexpr int kRows = 64 * RMAX, kStages = RMAX == 4 ? 3 : RMAX == 2 ? 4 : 6;
    static constexpr int kStageW = kRows * kQuantBlock, kStageS = kStageW + kQuantBlock * kQuantBlock, kStage = kStageS + kRows * 4 + 256;
    static constexpr int kMost = kStages * kStage, kStarts = kMost + 2 * kRows * 4;
    static constexpr int kLdsBytes = kStarts + kTileWaves * 16 + (MOE_MAX_E + 1) * 4 + MOE_MAX_E * 2;
    static constexpr int kCopies = RMAX + 3;            // a wavefront's, per stage
    static_assert(kLdsBytes <= 160 * 1024, "fits a CU");
};

template <int OUT, int RMAX, bool EIGHT>
__device__ __forceinline__ void tile_units(const QuantArgs& a, int min_rows, unsigned char* smem) {
    using T = Tiles<RMAX>;
    constexpr int kStages = T::kStages, kStageW = T::kStageW, kStageS = T::kStageS, kStage = T::kStage, tile_rows = T::kRows;
    uint32_t* mosts = reinterpret_cast<uint32_t*>(smem + T::kMost);           // [2][rows]
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

    // copies: wavefront w brings rows 64 i + 8 w ... + 7, weight fragment w, and scales: of rows 64 w ... or of the weights
    const uint32_t lds = lds_address(smem);
    const uint32_t to_rows = lds + wave * 1024, to_weights = lds + kStageW + wave * 2048;
    const int scale_part = wave < RMAX ? wave : RMAX;       // of 64 rows, or the weights'
    const uint32_t to_scales = lds + kStageS + scale_part * 256;
    // Of a stage: the row pieces' offsets from `rows_base` (tiles of 256 rows have no registers for whole addresses; see tile_fragments for
    // operands of more than 4 GiB), the weights' and scales' base.
    constexpr bool OFFSETS = RMAX == 4;
    uint32_t row_offset[OFFSETS ? RMAX : 1], scale_offset = 0;
    const uint8_t* row_from[OFFSETS ? 1 : RMAX];
    const uint8_t *rows_base = a.a, *weights_base = a.w;
    const float *scales_base = a.a_scales, *scales_from = nullptr;
    const uint32_t lane16 = lane * 16;
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
        const int scale_row = scale_part < RMAX ? source_row(a, w.row0 + min(wave * 64 + lane, w.rows - 1)) : 0;
        const float* base = scale_part < RMAX ? a.a_scales : a.w_scales + (static_cast<size_t>(w.e) * groups + w.group) * KB;
        if constexpr (OFFSETS) {
            scales_base = base;
            scale_offset = static_cast<uint32_t>(scale_row) * static_cast<uint32_t>(KB * 4);
        } else {
            scales_from = base + static_cast<size_t>(scale_row) * KB;
        }
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
        } else if (n == RMAX + 2) {
            if constexpr (OFFSETS) copy4_to_lds(scales_base, scale_offset, to_scales + at);
            else copy4_to_lds(scales_from, to_scales + at);
        }
    };
    uint32_t stage_step = 1;               // 0 behind the last unit
    auto next_stage = [&]() __attribute__((always_inline)) {
        slot_in = slot_in == kStages - 1 ? 0 : slot_in + 1;
        weights_base += stage_step * kFragBytes;
        if constexpr (OFFSETS) {
            rows_base += stage_step * kQuantBlock;
            scales_base += stage_step;
        } else {
#pragma unroll
            for (int i = 0; i < RMAX; ++i) row_from[i] += stage_step * kQuantBlock;
            scales_from += stage_step;
        }
    };
    // when all of a unit's stages have been sent for (kb_in == KB)
    auto next_unit = [&]() __attribute__((always_inline)) {
        kb_in = 0;
        if (u_in + static_cast<int>(gridDim.x) < units) {
            u_in += gridDim.x;
            ahead = unit_at(u_in);
            point_at(ahead);
        } else if (stage_step != 0) {      // back to the last stage, which is copied from now on
            weights_base -= kFragBytes;
            if constexpr (OFFSETS) {
                rows_base -= kQuantBlock;
                --scales_base;
            } else {
#pragma unroll
                for (int i = 0; i < RMAX; ++i) row_from[i] -= kQuantBlock;
                --scales_from;
            }
            stage_step = 0;
        }
    };
    auto copy_next = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < T::kCopies; ++n) copy_piece(n);
        next_stage();
        if (++kb_in == KB) next_unit();
    };
    Unit cur = ahead;
    if constexpr (EIGHT) {
#pragma unroll 1
        for (int i = 0; i < kStages; ++i) copy_next();
        copies_landed<(kStages - 1) * T::kCopies>();
    } else {
        copy_next();
        copies_landed<0>();
#pragma unroll 1
        for (int i = 0; i < kStages - 2; ++i) copy_next();
    }

    int slot = 0;
    uint32_t landed = 0;                    // steps from here on whose next stage is known to have landed
    auto run_unit = [&](auto fragments) __attribute__((always_inline)) {
        constexpr int R = decltype(fragments)::value;
        const int tid = here(threadIdx.x);
        const int at_x = row_operand(tid, wm * 16), x_other = row_operand_other(at_x), at_w = kStageW + wn * 4 * kFragBytes;
        const int at_sx = kStageS + (wm * 16 + (tid & 15)) * 4, at_sw = kStageS + tile_rows * 4;
        auto row_codes = [&](const unsigned char* st, int i) { return read_codes(st + at_x + i * 64 * kQuantBlock, x_other); };
        auto row_codes_half = [&](const unsigned char* st, int i, int half) {
            return *reinterpret_cast<const i32x4*>(st + at_x + i * 64 * kQuantBlock + (half ? x_other : 0));
        };
        auto weight_codes = [&](const unsigned char* st, int nf) { return read_codes(st + at_w + lane16 + nf * kFragBytes, 1024); };
        f32x4 acc[4][R];
#pragma unroll
        for (int nf = 0; nf < 4; ++nf)
#pragma unroll
            for (int i = 0; i < R; ++i) acc[nf][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        // the steps to the end of the unit or to where the copies go on to the next one: without a branch, so that the order stays
        auto all_steps = [&](auto step) __attribute__((always_inline)) {
#pragma unroll 1
            for (int j = 0; j < KB;) {
                // behind branches that not every lane takes, such as the stores of the unit before
                u_in = uniform(u_in);
                kb_in = uniform(kb_in);
                slot_in = uniform(slot_in);
                slot = uniform(slot);
                landed = uniform(landed);
                stage_step = uniform(stage_step);
                weights_base = uniform(weights_base);
                if constexpr (OFFSETS) {
                    rows_base = uniform(rows_base);
                    scales_base = uniform(scales_base);
                }
                const int steps = min(KB - j, KB - kb_in);
                j += steps;
                kb_in += steps;
                // nothing pending on the way in (lgkmcnt(0), the compiler counts with it): the steps wait only for what they read themselves
                __builtin_amdgcn_s_waitcnt(0xc07f);
#pragma unroll 1
                for (int s = 0; s < steps; ++s) {
                    step();
                    next_stage();
                }
                if (kb_in == KB) next_unit();
            }
        };
        if constexpr (EIGHT) {
            // A step is 4 R matrix instructions: the first two weight fragments x every row fragment, then the other two.  Operands are
            // read from the next stage into the registers of those that were used last, at least 2 R + 1 instructions (2 of one row
            // fragment) before their use; a stage's slot is free again in the middle of its own step, so that a copy has two steps to
            // land in.  A sum is added to its accumulator three instructions after its own.  The order is held by the scheduling barriers.
            i32x8 w[4], x[R];
            f32x4 sums[4] = {};
            float by[R], last[R] = {};
            const unsigned char* st0 = smem + slot * kStage;
#pragma unroll
            for (int nf = 0; nf < 4; ++nf) w[nf] = weight_codes(st0, nf);
#pragma unroll
            for (int i = 0; i < R; ++i) x[i] = row_codes(st0, i);
#pragma unroll
            for (int i = 0; i < R; ++i) by[i] = *reinterpret_cast<const float*>(st0 + at_sx + i * 256) * *reinterpret_cast<const float*>(st0 + at_sw);
            all_steps([&]() __attribute__((always_inline)) {
                constexpr int M = 4 * R, kFirst = R == 1 ? 0 : M / 2;       // from where on the next stage is read and copies go out
                slot = slot == kStages - 1 ? 0 : slot + 1;
                const unsigned char* st = smem + slot * kStage;
                float next_sx[R], next_sw = 0.f;
#pragma unroll
                for (int n = 0; n < M; ++n) {
                    const int half = n / (2 * R), i = n % (2 * R) >> 1, nf = 2 * half + (n & 1);
                    if (n == kFirst) {
                        __builtin_amdgcn_sched_barrier(0);
                        copies_landed_unless<(kStages - 2) * T::kCopies>(landed);
                        landed = landed > 0 ? landed - 1 : 0;
                        next_sw = *reinterpret_cast<const float*>(st + at_sw);
#pragma unroll
                        for (int f = 0; f < R; ++f) next_sx[f] = *reinterpret_cast<const float*>(st + at_sx + f * 256);
                        if (R > 1) {
                            w[0] = weight_codes(st, 0);
                            w[1] = weight_codes(st, 1);
                        }
                    }
                    sums[n & 3] = multiply_codes(w[nf], x[i]);
                    __builtin_amdgcn_sched_barrier(0);
                    if (R == 1 && n < 2) w[n] = weight_codes(st, n);
                    if (half == 1 && i == R - 1) w[nf] = weight_codes(st, nf);
                    if (half == 1 && (n & 1)) x[i] = row_codes(st, i);
                    constexpr int kPer = (T::kCopies + M - kFirst - 1) / (M - kFirst);
#pragma unroll
                    for (int c = 0; c < kPer; ++c)
                        if (n >= kFirst) copy_piece((n - kFirst) * kPer + c);
                    const int m = (n + M - 3) % M, m_half = m / (2 * R), m_i = m % (2 * R) >> 1;
                    f32x4& sum = acc[2 * m_half + (m & 1)][m_i];
                    const float scale = n < 3 ? last[m_i] : by[m_i];
#pragma unroll
                    for (int c = 0; c < 4; ++c) sum[c] = fmaf(scale, sums[m & 3][c], sum[c]);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    last[i] = by[i];
                    by[i] = next_sx[i] * next_sw;
                }
            });
#pragma unroll
            for (int m = 4 * R - 3; m < 4 * R; ++m) {
                const int i = m % (2 * R) >> 1;
                f32x4& sum = acc[2 * (m / (2 * R)) + (m & 1)][i];
#pragma unroll
                for (int c = 0; c < 4; ++c) sum[c] = fmaf(last[i], sums[m & 3][c], sum[c]);
            }
            // The stores below are counted behind the copies in flight, which have landed when they go out; so the next unit's first steps need
            // not wait for stores.
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            landed = kStages - 1;
        } else {
            // A step is 2 R rounds of eight matrix instructions, two weight fragments x one row fragment.  What the vector unit has to do
            // is spread between them, one piece after each: the codes of the next row fragment are widened, the sums of the round before
            // are added to the accumulators; in the last round and in the next step's first one also the next stage's weights are widened,
            // two fragments each, as their registers fall free.  The order is held by the scheduling barriers.
            // At the beginning of a step: w[0], w[1] and the first row fragment widened, the codes of w[2], w[3] and half of the
            // second row fragment's (if there is one), and the sums of the last round before it.
            Widened w[4], x[2];
            i32x8 codes_w[2], next_w[2];
            i32x4 codes_x[2];                   // halves of the fragment that is widened next
            f32x4 sums[2][2] = {};
            float last_scale = 0.f;
            const unsigned char* st0 = smem + slot * kStage;
            w[0] = widen(weight_codes(st0, 0));
            w[1] = widen(weight_codes(st0, 1));
            codes_w[0] = weight_codes(st0, 2);
            codes_w[1] = weight_codes(st0, 3);
            x[0] = widen(row_codes(st0, 0));
            codes_x[0] = row_codes_half(st0, 1, 0);
            all_steps([&]() __attribute__((always_inline)) {
                const unsigned char* st = smem + slot * kStage;
                slot = slot == kStages - 1 ? 0 : slot + 1;
                const unsigned char* st_next = smem + slot * kStage;
                float scale[R];
                const float sw = *reinterpret_cast<const float*>(st + at_sw);
#pragma unroll
                for (int i = 0; i < R; ++i) scale[i] = *reinterpret_cast<const float*>(st + at_sx + i * 256);
#pragma unroll
                for (int round = 0; round < 2 * R; ++round) {
                    const int i = round >> 1, half = round & 1;
                    if (round == (R > 2 ? 2 * R - 4 : 0)) {     // the next stage has landed, the one after it goes out
                        __builtin_amdgcn_sched_barrier(0);
                        copies_landed<(kStages - 3) * T::kCopies>();
                        if (R == 1) codes_x[0] = row_codes_half(st_next, 0, 0);
                    }
                    // A round ahead of its use: the second half of the fragment that is widened now, the first half of the one after it.
                    // Behind the last row fragment comes the next stage's first.
                    if (half == 0) codes_x[1] = i + 1 < R ? row_codes_half(st, i + 1, 1) : row_codes_half(st_next, 0, 1);
                    else if (R > 1) codes_x[0] = i + 2 < R ? row_codes_half(st, i + 2, 0) : row_codes_half(st_next, i + 2 - R, 0);
                    if (half == 0 && i == R - 1) {
                        next_w[0] = weight_codes(st_next, 0);
                        next_w[1] = weight_codes(st_next, 1);
                    }
                    if (R == 1 && round == 1) {                 // one row fragment: their last use was a round ago
                        w[2] = widen(codes_w[0]);
                        w[3] = widen(codes_w[1]);
                    }
                    Widened& x_now = x[R > 1 ? i & 1 : 0];
                    Widened& x_later = x[R > 1 ? (i & 1) ^ 1 : 1];
                    const int before = round == 0 ? 2 * R - 1 : round - 1;      // the round whose sums are added
                    const float by = round == 0 ? last_scale : scale[before >> 1] * sw;
#pragma unroll
                    for (int m = 0; m < 8; ++m) {
                        const int k = m >> 1, q = m & 1;
                        f32x4& p = sums[round & 1][q];
                        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[2 * half + q].eight(k), x_now.eight(k),
                                                                    k == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : p, 0, 0, 0);
                        // one copy at a time: issued together they would hold up every wavefront
                        constexpr int kFirst = R > 2 ? 8 * (2 * R - 4) : 0, kEvery = R == 1 ? 2 : 4;
                        const int at = 8 * round + m - kFirst;
                        if (at >= 0 && at % kEvery == 0) copy_piece(at / kEvery);
                        x_later.widen_two(codes_x[half][m >> 1], half * 8 + m);
                        f32x4& sum = acc[2 * (before & 1) + (m >> 2)][before >> 1];
                        sum[m & 3] = fmaf(by, sums[(round & 1) ^ 1][m >> 2][m & 3], sum[m & 3]);
                        if (R > 1 && round == 0) {
#pragma unroll
                            for (int c = 4 * m; c < 4 * m + 4; ++c) w[2 + (c >> 4)].widen_two(codes_w[c >> 4][(c & 15) >> 1], c & 15);
                        }
                        if (round == 2 * R - 1) {
#pragma unroll
                            for (int c = 4 * m; c < 4 * m + 4; ++c) w[c >> 4].widen_two(next_w[c >> 4][(c & 15) >> 1], c & 15);
                            if (m == 4) codes_w[0] = weight_codes(st_next, 2);
                            if (m == 7) codes_w[1] = weight_codes(st_next, 3);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                last_scale = scale[R - 1] * sw;
                if (R == 1) x[0] = x[1];
            });
#pragma unroll
            for (int m = 0; m < 8; ++m)
                acc[2 + (m >> 2)][R - 1][m & 3] = fmaf(last_scale, sums[1][m >> 2][m & 3], acc[2 + (m >> 2)][R - 1][m & 3]);
        }
        const int lane = here(threadIdx.x) & 63, r = lane & 15;
        const int col0 = cur.group * kQuantBlock + wn * 64, first = wm * 16;            // this wavefront's columns and rows
        finish_values(a, cur.e, col0, acc);
        if constexpr (OUT == kOutE4m3) {
            uint32_t most[R];
            row_magnitudes(a.N, col0, acc, most);
            if (lane < 16) {
#pragma unroll
                for (int i = 0; i < R; ++i) mosts[wn * tile_rows + first + i * 64 + lane] = most[i];
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
            for (int i = 0; i < R; ++i) most[i] = max(most[i], mosts[(wn ^ 1) * tile_rows + first + i * 64 + r]);
            store_codes<64>(a, col0, cur.row0 + first, cur.rows - first, acc, most, wn == 0);
        } else {
            store_values<OUT, 64>(a, col0, cur.row0 + first, cur.rows - first, acc);
        }
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
// cost 4 to 5 us all the same.  Streamed units are dealt from the last block number down, evenly over the XCDs; the blocks that have a tile more
// than others are whole XCDs, so that some of those get streamed units too while others have neither (128 of each: 64 blocks have both).
template <int OUT, int RMAX, bool EIGHT>
__global__ __launch_bounds__(kTileWaves * 64) void quant_product_kernel(const QuantArgs a, int tiled_min_rows) {
    extern __shared__ __align__(16) unsigned char smem[];
    tile_units<OUT, RMAX, EIGHT>(a, tiled_min_rows, smem);
    if (a.offsets == nullptr) return;
    __syncthreads();
    static_assert(Streams<1>::kList >= Streams<2>::kList, "the list lies behind both rings");
    uint16_t* list = reinterpret_cast<uint16_t*>(smem + Streams<1>::kList);
    const int tiles = list_experts<kTileWaves * 64>(a, tiled_min_rows - 1, list, reinterpret_cast<int32_t*>(list + MOE_MAX_E));
    const int b = gridDim.x - 1 - blockIdx.x;
    // Units of 256 columns widen each row fragment for twice the columns; but where those of 128 are at most one per block they use
    // more of the CUs.
    if (tiles * quant_blocks(a.N) > static_cast<int>(gridDim.x)) stream_units<OUT, 2, EIGHT>(a, tiles, 1, b, smem);
    else stream_units<OUT, 1, EIGHT>(a, tiles, 1, b, smem);
}

// ---- launches -------------------------------------------------------------------------------------------------------
// Experts with at least this many rows run in tiles, the others are streamed.
constexpr int kTiledMinRows = 65;

// Parts that the contraction of a streamed product is cut into: calls of at most 64 rows whose units would leave most CUs without one.
// It costs a second launch: one to four parts of 64 units 14.7 -> 12.4 us (32 x 8192 x 2048), of 16 units to sixteen 13.7 -> 11.3 us
// (1 x 2048 x 8192); but 128 units 13.3 -> 14.5 us with two (the experts of one token, 8192 x 2048).  Tiles are not cut, however few: 65 rows x
// 2048 x 8192 take 51 us (26 with the 8-bit units), 64 rows 16.
// A grouped call's number of experts with rows is not known here; a row each is taken, the most it can be.
static int stream_split(int rows, int N, int K, int E) {
    if (rows == 0 || rows >= kTiledMinRows) return 1;
    const int units = std::min(rows, E) * quant_blocks(N);
    return units <= 96 ? std::max(1, std::min(256 / units, quant_blocks(K) / 2)) : 1;
}

size_t quant_product_workspace(const moe_quant_shape& s) {
    const int split = stream_split(s.rows, s.N, s.K, s.E);
    const size_t parts = split > 1 ? static_cast<size_t>(split) * s.rows * quant_pitch(s.N) * sizeof(float) : 0;
    return (std::max<size_t>(parts, 1) + 255) / 256 * 256;
}

// Row fragments per wavefront of the tiled kernel, so rows per tile / 64: large tiles do more per byte and per conversion, small ones
// occupy more CUs.  A step of 256, 128 and 64 rows takes 1.95, 1.2 and 0.8 us on a CU with the bf16 units, 0.95, 0.7 and 0.6 with the 8-bit
// ones; a unit of each kind has as many steps as the other, so what counts is rounds of 256 units times that.  The ratios of the first three are
// taken for both: with each kind forced, the choice was the fastest one or within 5 % of it for each of 22 shapes of 200 to 8000 rows
// (64, 128, 256 rows, us; by the 8-bit units, bf16 out: 1501 x 768 x 3072 16.0, 21.3, 30.1; 4096 x 1024 x 4096 31.8, 26.9, 41.0; 2048 x 8192 x 2048 65.4,
// 53.0, 45.5; by the bf16 units, fp32 out: 25.4, 33.4, 46.9; 54.1, 41.7, 64.5; 109, 84, 74).  A grouped call's last tiles are not known here and left out.
// Tiles of 256 rows address the rows by 32-bit offsets.
static int tile_fragments(int rows, int N, size_t operand_bytes) {
    auto cost = [&](int r, float step) {
        const long long units = static_cast<long long>((rows + 64 * r - 1) / (64 * r)) * quant_blocks(N);
        return static_cast<float>((units + 255) / 256) * step;
    };
    const float c4 = cost(4, 1.95f), c2 = cost(2, 1.2f), c1 = cost(1, 0.8f);
    if (c1 < c2 && c1 < c4) return 1;
    return c2 < 0.9f * c4 || operand_bytes > 0xffffffffull ? 2 : 4;
}

// dynamic LDS of the kernel with both kinds of units
template <int RMAX>
constexpr int kProductLds = Tiles<RMAX>::kLdsBytes > Streams<1>::kLdsBytes ? Tiles<RMAX>::kLdsBytes : Streams<1>::kLdsBytes;

template <int OUT, int RMAX, bool EIGHT>
static void launch_tiles(const QuantArgs& a, int grid, hipStream_t stream) {
    quant_product_kernel<OUT, RMAX, EIGHT><<<dim3(grid), dim3(kTileWaves * 64), kProductLds<RMAX>, stream>>>(a, kTiledMinRows);
}

template <int OUT, bool EIGHT>
static hipError_t launch_out(const QuantArgs& a, void* ws, hipStream_t stream) {
    const int cus = device_cu_count();
    const dim3 grid(cus), threads(kStreamWaves * 64);
    const int split = stream_split(a.rows, a.N, a.K, a.E);
    if (split > 1) {
        QuantArgs parts = a;
        parts.out = ws;
        quant_stream_kernel<kOutParts, false><<<grid, threads, Streams<1>::kLdsBytes, stream>>>(parts, a.rows, split);
        quant_join_kernel<OUT><<<dim3(a.rows, (quant_blocks(a.N) + 7) / 8), dim3(256), 0, stream>>>(a, static_cast<const float*>(ws), split);
        return hipGetLastError();
    }
    if (a.rows >= kTiledMinRows) {
        const int r = tile_fragments(a.rows, a.N, a.rows / a.k * quant_pitch(a.K));
        if (r == 4) launch_tiles<OUT, 4, EIGHT>(a, cus, stream);
        else if (r == 2) launch_tiles<OUT, 2, EIGHT>(a, cus, stream);
        else launch_tiles<OUT, 1, EIGHT>(a, cus, stream);
    } else {
        quant_stream_kernel<OUT, EIGHT><<<grid, threads, Streams<1>::kLdsBytes, stream>>>(a, a.rows, 1);
    }
    return hipGetLastError();
}

static hipError_t allow_lds(const void* kernel, int bytes) {
    return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <int OUT, bool EIGHT>
static hipError_t configure_out() {
    hipError_t e;
    if ((e = allow_lds(reinterpret_cast<const void*>(quant_product_kernel<OUT, 4, EIGHT>), kProductLds<4>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(quant_product_kernel<OUT, 2, EIGHT>), kProductLds<2>)) != hipSuccess) return e;
    if ((e = allow_lds(reinterpret_cast<const void*>(quant_product_kernel<OUT, 1, EIGHT>), kProductLds<1>)) != hipSuccess) return e;
    return allow_lds(reinterpret_cast<const void*>(quant_stream_kernel<OUT, EIGHT>), Streams<1>::kLdsBytes);
}
hipError_t configure_quant_kernels() {
    hipError_t e;
    if ((e = configure_out<kOutF32, false>()) != hipSuccess) return e;
    if ((e = configure_out<kOutBf16, false>()) != hipSuccess) return e;
    if ((e = configure_out<kOutBf16, true>()) != hipSuccess) return e;
    if ((e = configure_out<kOutE4m3, false>()) != hipSuccess) return e;
    if ((e = configure_out<kOutE4m3, true>()) != hipSuccess) return e;
    return allow_lds(reinterpret_cast<const void*>(quant_stream_kernel<kOutParts, false>), Streams<1>::kLdsBytes);
}

// Weights that do not fit the L2s (8 x 4 MiB) are gone before the next call reads them, or have pushed out the rows: streamed units then read
// them as what is read once.  Kept and read once, us, the same weights again and others in turn (bf16 out): 32 rows x 8192 x 2048, 17 MB, 11.1 and
// 11.1, 12.4 and 12.3 (e4m3 out, again: 10.9 and 12.1); 26 MB 12.9 and 13.2, 14.5 and 14.2; 50 MB 16.4 and 16.5, 17.3 and 17.7; 67 MB 19.5 and 18.9,
// 23.3 and 21.6; 134 MB 38.2 and 37.7, 39.2 and 38.0; 400 MB 110 and 106 both ways.  Grouped: 40 experts, 42 MB, 11.2 and 10.2, 12.5 and 11.7; 64 experts
// of 32 rows, 151 MB, 29.2 and 32.6 (the memory-side cache holds them), 37.2 and 34.6; 49 of 128 experts, 2 GB of which 822 MB are read, 141 and 131.
constexpr size_t kCachedWeights = size_t{32} << 20;

hipError_t launch_quant_product(const QuantArgs& args, void* ws, hipStream_t stream) {
    QuantArgs a = args;
    a.once = a.E * quant_matrix_bytes(a.N, a.K) > kCachedWeights;
    if (a.out_dtype == MOE_F32) return launch_out<kOutF32, false>(a, ws, stream);
    if (a.out_dtype == MOE_BF16) return a.unit_sums ? launch_out<kOutBf16, true>(a, ws, stream) : launch_out<kOutBf16, false>(a, ws, stream);
    return a.unit_sums ? launch_out<kOutE4m3, true>(a, ws, stream) : launch_out<kOutE4m3, false>(a, ws, stream);
}

}  // namespace moe
