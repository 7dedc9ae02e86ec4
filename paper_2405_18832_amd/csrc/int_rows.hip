// The norm in front of a layer with int8 rows, and the weights' layout.
#include "int_rows.hpp"

namespace moe {

namespace {

// ---- moe_norm_quantize_int -------------------------------------------------------------------------------------------
// One pass, bound by memory: 16384 x 2048 in bf16 with a residual and both outputs 59.0 us, 5.1 TB/s read + written, which is what a copy reaches.
// NV: chunks that a wavefront keeps in registers; 0: rows longer than any variant keeps, which are read again.
template <typename ST, int WPR, int WAVES, int NV>
__global__ __launch_bounds__(WAVES * 64) void norm_int_kernel(const IntRowArgs a) {
    static_assert(WPR == 1 || WPR == WAVES, "what all of a row's wavefronts know, all that meet at a barrier know");
    __shared__ RowShared<WAVES> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % WPR;
    const int row = (blockIdx.y * gridDim.x + blockIdx.x) * (WAVES / WPR) + wave / WPR;
    const bool live = row < a.rows;
    const int d = a.d;
    const size_t at = static_cast<size_t>(live ? row : 0) * d;
    const ST* x = static_cast<const ST*>(a.x) + at;
    const ST* res = a.residual ? static_cast<const ST*>(a.residual) + at : nullptr;
    ST* sum_out = a.sum_out ? static_cast<ST*>(a.sum_out) + at : nullptr;
    const int chunks = (d + kChunk - 1) / kChunk;
    auto column = [&](int chunk) { return chunk * kChunk + lane * 8; };
    auto read_sum = [&](int chunk, float (&s)[8]) {
        load8<ST, false>(x, column(chunk), d, s);
        if (res != nullptr) {
            float r[8];
            load8<ST, false>(res, column(chunk), d, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] = Eight<ST>::round(s[i] + r[i]);
        }
    };
    // What the lane has read once: sum_out may be x or residual, and has been written then (the longest rows' at the very end).
    auto sum_again = [&](int c) {
        if (NV > 0 && sum_out != nullptr) return Storage<ST>::load(sum_out + c);
        const float s = Storage<ST>::load(x + c);
        return res != nullptr ? Eight<ST>::round(s + Storage<ST>::load(res + c)) : s;
    };
    auto weight_at = [&](int c) { return a.weight != nullptr ? a.weight[c] : 1.f; };
    auto times_weight = [&](int chunk, float (&s)[8]) {
        if (a.weight == nullptr) return;
        float w[8];
        load8<float, false>(a.weight, column(chunk), d, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] *= w[i];
    };

    float u[NV > 0 ? NV : 1][8];                            // sum * weight
    float squares = 0.f;
    uint32_t most = 0;
    auto add_squares = [&](const float (&s)[8]) {
        float p = 0.f;                                      // short chains: the rounding error of a sum grows with its length
#pragma unroll
        for (int i = 0; i < 8; ++i) p = fmaf(s[i], s[i], p);
        squares += p;
    };
    auto each = [&](auto f) __attribute__((always_inline)) {       // f(chunk, products)
        if constexpr (NV > 0) {
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) f(j * WPR + part, u[j]);
            });
        } else {
            for (int c = part; c < chunks; c += WPR) {
                read_sum(c, u[0]);
                times_weight(c, u[0]);
                f(c, u[0]);
            }
        }
    };
    if (live) {
        if constexpr (NV > 0) {
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {       // all loads first
                if (j * WPR + part < chunks) read_sum(j * WPR + part, u[j]);
            });
            unrolled<NV>([&](auto j) __attribute__((always_inline)) {
                if (j * WPR + part < chunks) {
                    add_squares(u[j]);
                    if (sum_out != nullptr) store8<ST, false>(sum_out, column(j * WPR + part), d, u[j]);
                    times_weight(j * WPR + part, u[j]);
                }
            });
        } else {
            for (int c = part; c < chunks; c += WPR) {
                read_sum(c, u[0]);
                add_squares(u[0]);
            }
        }
        each([&](int, const float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
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
            squares += shared.squares[w];
            most = max(most, shared.most[w]);
        }
    }
    double rho = 1.f / sqrtf(squares / static_cast<float>(d) + a.eps);
    // Rows whose squares fp32 does not hold are summed again, in 64 bits.
    const bool far = live && (!(squares <= 0x1p+120f) || (squares < 0x1p-80f && a.eps < 0x1p-60f));
    auto each_column = [&](auto f) {                        // f(column) of the lane's
        for (int chunk = part; chunk < chunks; chunk += WPR)
            for (int c = column(chunk); c < min(column(chunk) + 8, d); ++c) f(c);
    };
    auto row_sum = [&](double v) {
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        if constexpr (WPR > 1) {
            if (lane == 0) shared.top[wave] = v;
            __syncthreads();
            v = 0.0;
#pragma unroll
            for (int w = 0; w < WPR; ++w) v += shared.top[w];
            __syncthreads();                                // `top` is written again
        }
        return v;
    };
    if (far) {
        double sum = 0.0;
        each_column([&](int c) {
            const double v = static_cast<double>(sum_again(c));
            sum += v * v;
        });
        rho = 1.0 / sqrt(row_sum(sum) / static_cast<double>(d) + static_cast<double>(a.eps));
    }
    // A NaN or an infinity among sums and weights; products of finite numbers may be infinite without one.
    bool bad = !(rho < __builtin_huge_val());
    if (live && most >= 0x7f800000u) {
        double none = 0.0;
        each_column([&](int c) { none += fabsf(sum_again(c)) < __builtin_huge_valf() && fabsf(weight_at(c)) < __builtin_huge_valf() ? 0.0 : 1.0; });
        bad = row_sum(none) != 0.0 || bad;
    }
    if (live && a.norm_out != nullptr) {
        ST* norm_out = static_cast<ST*>(a.norm_out) + at;
        if (far || !(__uint_as_float(most) <= 0x1p+100f)) {       // a factor or products that fp32 does not hold
            each_column([&](int c) {
                Storage<ST>::store(norm_out + c, static_cast<float>(static_cast<double>(sum_again(c)) * rho * static_cast<double>(weight_at(c))));
            });
        } else {
            const float by = static_cast<float>(rho);
            each([&](int chunk, const float (&v)[8]) __attribute__((always_inline)) {
                float n[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) n[i] = v[i] * by;
                store8<ST, false>(norm_out, column(chunk), d, n);
            });
        }
    }
    write_row<WPR, WAVES>(
        shared, live, bad, most, kProductSlack, rho, d, a.q + static_cast<size_t>(live ? row : 0) * quant_pitch(d), a.q_scales + (live ? row : 0),
        [&](auto f) __attribute__((always_inline)) {
            each([&](int chunk, const float (&v)[8]) __attribute__((always_inline)) { f(chunk, v, kProductSlack); });
        },
        [&](int chunk, int i) __attribute__((always_inline)) {
            return static_cast<double>(sum_again(column(chunk) + i)) * static_cast<double>(weight_at(column(chunk) + i));
        });
    if constexpr (NV == 0) {
        if (live && sum_out != nullptr)
            for (int c = part; c < chunks; c += WPR) {
                float s[8];
                read_sum(c, s);
                store8<ST, false>(sum_out, column(c), d, s);
            }
    }
}

template <typename ST>
hipError_t launch_norm(const IntRowArgs& a, hipStream_t stream) {
    with_row_variant(a, [&](auto wpr, auto waves, auto nv) {
        constexpr int WPR = decltype(wpr)::value, WAVES = decltype(waves)::value, NV = decltype(nv)::value;
        launch_rows<WPR, WAVES>(norm_int_kernel<ST, WPR, WAVES, NV>, a, stream);
    });
    return hipGetLastError();
}

// ---- moe_quantize_weights_int ----------------------------------------------------------------------------------------
// A block of threads per 32 rows of a matrix, thread t columns 16 (t % 8) ... of row t / 8 in every block of 128 columns: once for the row's
// largest magnitude, once for the codes, 16 bytes at the place that the products' loads want them (moe.h, moe_quantize_weights).
// Once per layer: 32 matrices of 8192 x 2048 in fp32 935 us, bf16 556 (the second time they are read counts, 2.9 TB/s without it), codes 201 (5.3 TB/s).
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
    return dtype == MOE_BF16 ? launch_norm<uint16_t>(a, stream) : launch_norm<float>(a, stream);
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
