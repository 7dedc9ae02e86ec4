// Parts that the products on 8-bit rows share: which rows are whose, copies into LDS, operands in LDS, stores of a tile's sums.
#pragma once

#include "quant.hpp"

namespace moe {

enum OutKind { kOutF32 = 0, kOutBf16 = 1, kOutE4m3 = 2 };

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

// ---- stores of a tile's sums -----------------------------------------------------------------------------------------
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

// ---- which experts are streamed --------------------------------------------------------------------------------------
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

}  // namespace moe
