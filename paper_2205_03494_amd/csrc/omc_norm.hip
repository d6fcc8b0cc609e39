// omc_layer_norm and omc_layer_norm_backward.
//
// y = (x - mean) rstd gamma + beta; backward, with h = (x - mean) rstd and u = dy gamma: dx = rstd (u - mean(u) - h mean(u h)), dgamma = sum over rows of dy h, dbeta of dy.
//
// Bound by memory: a row is read once and stays in registers, eight neighbours a lane and piece, between the sum of its values, the sum of their squared distances from the mean, and
// the result.  Forward, 32768 x 4096 in bf16 93 - 99 us, 5.6 TB/s; 8192 x 1024, fp32 to bf16, 9.5 us, 5.3 TB/s; 1 x 512 2.1 us.  Backward, 32768 x 4096
// 143 us and 5 for the sums of partial sums, 5.6 TB/s; 8192 x 1024 with x in fp32 20 us; 1 x 512 2.5 us.  8, 16, 32 or 64 lanes take a row of up to 64, 128, 256 or 1024 values, 2, 4, 8 or 16 waves up to 16384; longer rows are read
// again for every sum.
// Backward, a thread keeps the same columns of all rows that its workgroup takes, so that the sums over the rows (dgamma, dbeta) stay in registers too; every workgroup leaves one row of
// partial sums, which a second kernel adds up in order.
#include <type_traits>

#include "omc_mx4.h"

namespace omc {

template <int CONTROL>
__device__ __forceinline__ float from_lane(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ float add_row_pairs(float x) {      // over the two rows of 16 lanes in each half of the wave
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float add_halves(float x) {
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Sum over the LANES neighbours that share a row, in all of them; a fixed tree.
template <int LANES>
__device__ __forceinline__ float row_lanes_sum(float x) {
    x += from_lane<0xb1>(x);                   // lanes 1 0 3 2
    x += from_lane<0x4e>(x);                   // lanes 2 3 0 1
    x += from_lane<0x141>(x);                  // eight lanes mirrored
    if constexpr (LANES >= 16) x += from_lane<0x140>(x);   // sixteen lanes mirrored
    if constexpr (LANES >= 32) x = add_row_pairs(x);
    if constexpr (LANES >= 64) x = add_halves(x);
    return x;
}
// Sum over the lanes of a wave that have the same columns of different rows.
template <int LANES>
__device__ __forceinline__ float same_columns_sum(float x) {
    if constexpr (LANES <= 32) x = add_halves(x);
    if constexpr (LANES <= 16) x = add_row_pairs(x);
    if constexpr (LANES <= 8) x += from_lane<0x128>(x);    // eight lanes on
    return x;
}

// Sums over the lanes and the WAVES waves that share a row.  Every call takes the next of two places in LDS, so that one barrier a call is enough: who writes a place again has passed
// the barrier of the call between, which nobody does before having read it.
template <int LANES, int WAVES, int COUNT>
struct RowSum {
    float (*places)[16][COUNT];                // [2]
    uint32_t wave, next;
    __device__ __forceinline__ void operator()(float (&x)[COUNT]) {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) x[c] = row_lanes_sum<LANES>(x[c]);
        if constexpr (WAVES > 1) {
            auto &place = places[next];
            next ^= 1;
            if ((threadIdx.x & 63u) == 0) {
#pragma unroll
                for (int c = 0; c < COUNT; ++c) place[wave][c] = x[c];
            }
            __syncthreads();
            const uint32_t first = wave / WAVES * WAVES;
#pragma unroll
            for (int c = 0; c < COUNT; ++c) {
                x[c] = place[first][c];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) x[c] += place[first + w][c];
            }
        }
    }
};

// Eight of gamma or beta from column `col` on, like a row's values; all `otherwise` if there is none.
template <bool SHORT>
__device__ __forceinline__ void fetch_weights(Eight<F32> &w, const float *row, uint32_t col, uint32_t cols, float otherwise) {
    if (row) {
        w.fetch<SHORT>(row, col, cols);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w.w[i] = __float_as_uint(otherwise);
    }
}

__device__ __forceinline__ float reciprocal_deviation(float variance, float eps) { return 1.0f / __builtin_sqrtf(variance + eps); }

// How a workgroup's threads are dealt out to rows and columns: LANES lanes (64 if WAVES > 1) of WAVES waves a row, kRows rows at a time; at least four waves.
// With kAhead a row's values are asked for before the row before it is worked on.  That takes registers, so that fewer waves are there, and pays where a row has many waves, which wait for
// each other: 8192 x 8192 in bf16 takes 50 us with it, 55 without, 8192 x 1024 8.2 and 7.6.  Backward (kGradAhead) it pays without many waves too, since a wave's sums over the rows
// leave no room for others: 8192 x 1024 with x in fp32 20 us, 22 without, 8192 x 8192 80 and 90; not at four waves (32768 x 4096: 152 and 147), nor at sixteen, whose registers it exceeds.
template <int LANES, int WAVES>
struct Deal {
    static_assert(LANES == 64 || WAVES == 1, "whole waves share a row");
    static constexpr int kWaves = WAVES < 4 ? 4 : WAVES, kThreads = 64 * kWaves, kWidth = LANES * WAVES, kRows = kThreads / kWidth;
    static constexpr bool kAhead = WAVES >= 4, kGradAhead = WAVES <= 2 || WAVES == 8;
    static constexpr uint32_t kGroups = kAhead ? 512 : 1024, kGradGroups = kGradAhead || WAVES == 16 ? 256 : 512;   // at most
    static __device__ __forceinline__ uint32_t row() { return threadIdx.x / kWidth; }
    static __device__ __forceinline__ uint32_t lane() { return threadIdx.x % kWidth; }
};

template <typename X, typename Y, int LANES, int WAVES, int PIECES, bool SHORT>
__global__ __launch_bounds__((Deal<LANES, WAVES>::kThreads)) void norm_kernel(NormArgs na) {
    typedef Deal<LANES, WAVES> D;
    __shared__ float places[2][16][1];
    const uint32_t cols = na.cols, t = D::lane(), mine = D::row();
    RowSum<LANES, WAVES, 1> row_sum{places, threadIdx.x >> 6, 0};
    uint32_t left[PIECES], missing[PIECES];
    Eight<F32> gamma[PIECES], beta[PIECES];
    Eight<X> next[PIECES];
    auto load = [&](uint32_t row) {            // (the last row once more past the end)
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + min(row, na.rows - 1) * na.ldx;
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) next[p].template fetch<SHORT>(x, 8 * (t + D::kWidth * p), cols);
    };
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        const uint32_t col = 8 * (t + D::kWidth * p);
        left[p] = col < cols ? cols - col : 0u;
        missing[p] = Eight<X>::missing(col, cols);
    }
    load(blockIdx.x * D::kRows + mine);
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        const uint32_t col = 8 * (t + D::kWidth * p);
        fetch_weights<SHORT>(gamma[p], na.gamma, col, cols, 1.0f);
        fetch_weights<SHORT>(beta[p], na.beta, col, cols, 0.0f);
    }
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        if (na.gamma) gamma[p].settle(missing[p]);
        if (na.beta) beta[p].settle(missing[p]);
    }
    const float count = static_cast<float>(cols);
    for (uint32_t base = blockIdx.x * D::kRows; base < na.rows; base += gridDim.x * D::kRows) {
        const uint32_t row = base + mine;
        if (!D::kAhead) load(row);
        Eight<X> v[PIECES];
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            v[p] = next[p];
            v[p].settle(missing[p]);
        }
        if (D::kAhead) load(row + gridDim.x * D::kRows);
        float sum[1] = {0.0f};
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v[p].value(i);
        row_sum(sum);
        const float mean = sum[0] / count;
        float squares[1] = {0.0f};
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p)
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const float d = v[p].value(i) - mean;
                squares[0] = __builtin_fmaf(i < left[p] ? d : 0.0f, d, squares[0]);
            }
        row_sum(squares);
        const float rstd = reciprocal_deviation(squares[0] / count, na.eps);
        if (row >= na.rows) continue;          // (no barrier follows in this turn)
        typename Y::type *y = static_cast<typename Y::type *>(na.y) + row * na.ldy + 8 * t;
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            float out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = __builtin_fmaf((v[p].value(i) - mean) * rstd, gamma[p].value(i), beta[p].value(i));
            store_run<Y, 8>(y + 8 * D::kWidth * p, out, left[p]);
        }
        if (t == 0) {
            if (na.mean) na.mean[row] = mean;
            if (na.rstd) na.rstd[row] = rstd;
        }
    }
}

// Longer rows, a workgroup of sixteen waves each: one pass for the mean, one for the deviation, one for the result, of which the last two find most of the row in the caches.
// 2048 x 20000 in bf16: 55 us.
template <typename X, typename Y>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs na) {
    __shared__ float places[2][16][1];
    const uint32_t cols = na.cols;
    const float count = static_cast<float>(cols);
    RowSum<64, 16, 1> row_sum{places, threadIdx.x >> 6, 0};
    for (uint32_t row = blockIdx.x; row < na.rows; row += gridDim.x) {
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + row * na.ldx;
        typename Y::type *y = static_cast<typename Y::type *>(na.y) + row * na.ldy;
        float sum[1] = {0.0f}, squares[1] = {0.0f};
        Eight<X> v;
        for (uint32_t c = 8 * threadIdx.x; c < cols; c += 8192) {
            v.template load<false>(x, c, cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v.value(i);
        }
        row_sum(sum);
        const float mean = sum[0] / count;
        for (uint32_t c = 8 * threadIdx.x; c < cols; c += 8192) {
            v.template load<false>(x, c, cols);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const float d = v.value(i) - mean;
                squares[0] = __builtin_fmaf(c + i < cols ? d : 0.0f, d, squares[0]);
            }
        }
        row_sum(squares);
        const float rstd = reciprocal_deviation(squares[0] / count, na.eps);
        for (uint32_t c = 8 * threadIdx.x; c < cols; c += 8192) {
            Eight<F32> gamma, beta;
            fetch_weights<false>(gamma, na.gamma, c, cols, 1.0f);
            fetch_weights<false>(beta, na.beta, c, cols, 0.0f);
            v.template load<false>(x, c, cols);
            const uint32_t missing = Eight<X>::missing(c, cols);
            if (na.gamma) gamma.settle(missing);
            if (na.beta) beta.settle(missing);
            float out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = __builtin_fmaf((v.value(i) - mean) * rstd, gamma.value(i), beta.value(i));
            store_run<Y, 8>(y + c, out, cols - c);
        }
        if (threadIdx.x == 0) {
            if (na.mean) na.mean[row] = mean;
            if (na.rstd) na.rstd[row] = rstd;
        }
    }
}

// ---- backward

// The partial sums of a workgroup: a row of 2 * cols floats, dgamma's then dbeta's; of the only workgroup: dgamma and dbeta.
template <typename X, typename Y, int LANES, int WAVES, int PIECES, bool SHORT>
__global__ __launch_bounds__((Deal<LANES, WAVES>::kThreads)) void norm_grad_kernel(NormGradArgs na) {
    typedef Deal<LANES, WAVES> D;
    constexpr int kSets = D::kWaves / WAVES;   // of waves: as many threads have the same columns, after those of a wave are added
    __shared__ float places[2][16][2];
    __shared__ float joined[kSets > 1 ? kSets - 1 : 1][kSets > 1 ? 64 * WAVES * 16 : 1];
    const uint32_t wave = threadIdx.x >> 6, cols = na.cols, t = D::lane(), mine = D::row();
    RowSum<LANES, WAVES, 2> row_sum{places, wave, 0};
    uint32_t left[PIECES], missing[PIECES];
    Eight<F32> gamma[PIECES];
    float dgamma[PIECES][8], dbeta[PIECES][8];
    Eight<X> next_x[PIECES];
    Eight<Y> next_dy[PIECES];
    float next_mean, next_rstd;
    auto load = [&](uint32_t row) {            // (the last row once more past the end)
        const uint32_t from = min(row, na.rows - 1);
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + from * na.ldx;
        const typename Y::type *dy = static_cast<const typename Y::type *>(na.dy) + from * na.lddy;
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            next_x[p].template fetch<SHORT>(x, 8 * (t + D::kWidth * p), cols);
            next_dy[p].template fetch<SHORT>(dy, 8 * (t + D::kWidth * p), cols);
        }
        next_mean = na.mean[from];
        next_rstd = na.rstd[from];
    };
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        const uint32_t col = 8 * (t + D::kWidth * p);
        left[p] = col < cols ? cols - col : 0u;
        missing[p] = Eight<X>::missing(col, cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) dgamma[p][i] = dbeta[p][i] = 0.0f;
    }
    if (D::kGradAhead) load(blockIdx.x * D::kRows + mine);
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) fetch_weights<SHORT>(gamma[p], na.gamma, 8 * (t + D::kWidth * p), cols, 1.0f);
    if (na.gamma) {
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) gamma[p].settle(missing[p]);
    }
    const float count = static_cast<float>(cols);
    for (uint32_t base = blockIdx.x * D::kRows; base < na.rows; base += gridDim.x * D::kRows) {
        const uint32_t row = base + mine;
        if (!D::kGradAhead) load(row);
        Eight<X> v[PIECES];
        Eight<Y> g[PIECES];
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            v[p] = next_x[p];
            g[p] = next_dy[p];
            v[p].settle(missing[p]);
            g[p].settle(row < na.rows ? missing[p] : 8u);
        }
        const float mean = next_mean, rstd = next_rstd;
        if (D::kGradAhead) load(row + gridDim.x * D::kRows);
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) {      // (past the end dy is zero, and x finite)
                const float hat = (v[p].value(i) - mean) * rstd, d = g[p].value(i), u = d * gamma[p].value(i);
                sums[0] += u;
                sums[1] = __builtin_fmaf(u, hat, sums[1]);
                dgamma[p][i] = __builtin_fmaf(d, hat, dgamma[p][i]);
                dbeta[p][i] += d;
            }
        if (!na.dx) continue;
        row_sum(sums);
        if (row >= na.rows) continue;
        const float mean_u = sums[0] / count, mean_uh = sums[1] / count;
        typename X::type *dx = static_cast<typename X::type *>(na.dx) + row * na.lddx + 8 * t;
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            float out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hat = (v[p].value(i) - mean) * rstd;
                out[i] = rstd * ((__builtin_fmaf(g[p].value(i), gamma[p].value(i), -mean_u)) - hat * mean_uh);
            }
            store_run<X, 8>(dx + 8 * D::kWidth * p, out, left[p]);
        }
    }
    if (!na.parts) return;
    const bool only = gridDim.x == 1;
    float *to_gamma = only ? na.dgamma : na.parts + static_cast<uint64_t>(blockIdx.x) * 2 * cols;
    float *to_beta = only ? na.dbeta : na.parts + (static_cast<uint64_t>(blockIdx.x) * 2 + 1) * cols;
    const uint32_t set = wave / WAVES, at = threadIdx.x % (64 * WAVES);
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dgamma[p][i] = same_columns_sum<LANES>(dgamma[p][i]);
            dbeta[p][i] = same_columns_sum<LANES>(dbeta[p][i]);
        }
        if constexpr (kSets > 1) {
            if (p > 0) __syncthreads();
            if (set > 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    joined[set - 1][i * (64 * WAVES) + at] = dgamma[p][i];
                    joined[set - 1][(8 + i) * (64 * WAVES) + at] = dbeta[p][i];
                }
            }
            __syncthreads();
            if (set == 0) {
#pragma unroll 1
                for (int w = 0; w < kSets - 1; ++w)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dgamma[p][i] += joined[w][i * (64 * WAVES) + at];
                        dbeta[p][i] += joined[w][(8 + i) * (64 * WAVES) + at];
                    }
            }
        }
        if (threadIdx.x < D::kWidth && left[p] > 0) {
            const uint32_t col = 8 * (t + D::kWidth * p);
            if (to_gamma) store_run<F32, 8>(to_gamma + col, dgamma[p], left[p]);
            if (to_beta) store_run<F32, 8>(to_beta + col, dbeta[p], left[p]);
        }
    }
}

// Longer rows: dx by a workgroup a row, in two passes of which the second finds most in the caches, the columns' sums by another kernel.  2048 x 20000 in bf16: 64 and 41 us.
template <typename X, typename Y>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs na) {
    __shared__ float places[2][16][2];
    const uint32_t cols = na.cols;
    const float count = static_cast<float>(cols);
    RowSum<64, 16, 2> row_sum{places, threadIdx.x >> 6, 0};
    for (uint32_t row = blockIdx.x; row < na.rows; row += gridDim.x) {
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + row * na.ldx;
        const typename Y::type *dy = static_cast<const typename Y::type *>(na.dy) + row * na.lddy;
        typename X::type *dx = static_cast<typename X::type *>(na.dx) + row * na.lddx;
        const float mean = na.mean[row], rstd = na.rstd[row];
        Eight<X> v;
        Eight<Y> g;
        Eight<F32> gamma;
        auto load = [&](uint32_t c) {          // (past the end dy is zero)
            const uint32_t missing = Eight<X>::missing(c, cols);
            v.template fetch<false>(x, c, cols);
            g.template fetch<false>(dy, c, cols);
            fetch_weights<false>(gamma, na.gamma, c, cols, 1.0f);
            v.settle(missing);
            g.settle(missing);
            if (na.gamma) gamma.settle(missing);
        };
        float sums[2] = {0.0f, 0.0f};
        for (uint32_t c = 8 * threadIdx.x; c < cols; c += 8192) {
            load(c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = g.value(i) * gamma.value(i);
                sums[0] += u;
                sums[1] = __builtin_fmaf(u, (v.value(i) - mean) * rstd, sums[1]);
            }
        }
        row_sum(sums);
        const float mean_u = sums[0] / count, mean_uh = sums[1] / count;
        for (uint32_t c = 8 * threadIdx.x; c < cols; c += 8192) {
            load(c);
            float out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hat = (v.value(i) - mean) * rstd;
                out[i] = rstd * (__builtin_fmaf(g.value(i), gamma.value(i), -mean_u) - hat * mean_uh);
            }
            store_run<X, 8>(dx + c, out, cols - c);
        }
    }
}
template <typename X, typename Y>
__global__ __launch_bounds__(256) void norm_grad_columns_kernel(NormGradArgs na) {
    const uint32_t col = blockIdx.x * 256 + threadIdx.x, part = blockIdx.y;
    if (col >= na.cols) return;
    float dgamma = 0.0f, dbeta = 0.0f;
    for (uint32_t row = part; row < na.rows; row += gridDim.y) {
        const float d = load_f32(static_cast<const typename Y::type *>(na.dy) + row * na.lddy + col);
        const float hat = (load_f32(static_cast<const typename X::type *>(na.x) + row * na.ldx + col) - na.mean[row]) * na.rstd[row];
        dgamma = __builtin_fmaf(d, hat, dgamma);
        dbeta += d;
    }
    float *to = na.parts + static_cast<uint64_t>(part) * 2 * na.cols + col;
    to[0] = dgamma;
    to[na.cols] = dbeta;
}

constexpr uint32_t kLongest = 16384;           // values of a row that stays in registers
// call(lanes, waves, pieces, short) of the kernel that rows of this length take.
template <int V>
using Int = std::integral_constant<int, V>;
template <typename F>
static void by_length(uint32_t cols, F &&call) {
    if (cols < 8) call(Int<8>{}, Int<1>{}, Int<1>{}, std::true_type{});
    else if (cols <= 64) call(Int<8>{}, Int<1>{}, Int<1>{}, std::false_type{});
    else if (cols <= 128) call(Int<16>{}, Int<1>{}, Int<1>{}, std::false_type{});
    else if (cols <= 256) call(Int<32>{}, Int<1>{}, Int<1>{}, std::false_type{});
    else if (cols <= 512) call(Int<64>{}, Int<1>{}, Int<1>{}, std::false_type{});
    else if (cols <= 1024) call(Int<64>{}, Int<1>{}, Int<2>{}, std::false_type{});
    else if (cols <= 2048) call(Int<64>{}, Int<2>{}, Int<2>{}, std::false_type{});
    else if (cols <= 4096) call(Int<64>{}, Int<4>{}, Int<2>{}, std::false_type{});
    else if (cols <= 8192) call(Int<64>{}, Int<8>{}, Int<2>{}, std::false_type{});
    else call(Int<64>{}, Int<16>{}, Int<2>{}, std::false_type{});
}

template <typename X, typename Y>
static int launch_norm(const NormArgs &na, hipStream_t st) {
    if (na.cols > kLongest) {
        norm_long_kernel<X, Y><<<dim3(na.rows < 4096 ? na.rows : 4096), dim3(1024), 0, st>>>(na);
        return static_cast<int>(hipGetLastError());
    }
    by_length(na.cols, [&](auto lanes, auto waves, auto pieces, auto few) {
        constexpr int L = decltype(lanes)::value, W = decltype(waves)::value, P = decltype(pieces)::value;
        constexpr bool S = decltype(few)::value;
        const uint32_t groups = (na.rows + Deal<L, W>::kRows - 1) / Deal<L, W>::kRows;
        norm_kernel<X, Y, L, W, P, S><<<dim3(groups < Deal<L, W>::kGroups ? groups : Deal<L, W>::kGroups), dim3(Deal<L, W>::kThreads), 0, st>>>(na);
    });
    return static_cast<int>(hipGetLastError());
}
int launch_layer_norm(const NormArgs &na, bool x_bf16, bool y_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_bf16) return y_bf16 ? launch_norm<BF16, BF16>(na, st) : launch_norm<BF16, F32>(na, st);
    return y_bf16 ? launch_norm<F32, BF16>(na, st) : launch_norm<F32, F32>(na, st);
}

// Rows of partial sums, as many as workgroups.  Each costs 16 bytes a column through memory, as much as two to four rows of x, dy and dx: a workgroup has at least four rows.
static uint32_t grad_groups(uint32_t rows, uint32_t cols) {
    if (cols > kLongest) return rows < 64 ? rows : 64;
    uint32_t groups = 0;
    by_length(cols, [&](auto lanes, auto waves, auto, auto) {
        typedef Deal<decltype(lanes)::value, decltype(waves)::value> D;
        const uint32_t each = D::kRows < 4 ? 4 : D::kRows;
        groups = (rows + each - 1) / each;
        if (groups > D::kGradGroups) groups = D::kGradGroups;
    });
    return groups;
}
size_t layer_norm_backward_workspace(uint32_t rows, uint32_t cols) { return 8ull * grad_groups(rows, cols) * cols; }

template <typename X, typename Y>
static int launch_grad(const NormGradArgs &given, hipStream_t st) {
    NormGradArgs na = given;
    if (!na.dgamma && !na.dbeta) na.parts = nullptr;
    const uint32_t groups = grad_groups(na.rows, na.cols);
    if (na.cols > kLongest) {
        if (na.dx) norm_grad_long_kernel<X, Y><<<dim3(na.rows < 4096 ? na.rows : 4096), dim3(1024), 0, st>>>(na);
        if (na.parts) norm_grad_columns_kernel<X, Y><<<dim3((na.cols + 255) / 256, groups), dim3(256), 0, st>>>(na);
    } else {
        by_length(na.cols, [&](auto lanes, auto waves, auto pieces, auto few) {
            constexpr int L = decltype(lanes)::value, W = decltype(waves)::value, P = decltype(pieces)::value;
        constexpr bool S = decltype(few)::value;
            norm_grad_kernel<X, Y, L, W, P, S><<<dim3(groups), dim3(Deal<L, W>::kThreads), 0, st>>>(na);
        });
        if (groups == 1) na.parts = nullptr;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !na.parts) return static_cast<int>(e);
    return launch_column_sums(na.parts, groups, false, na.cols, 2 * na.cols, na.dgamma, na.dbeta, st);
}
int launch_layer_norm_backward(const NormGradArgs &na, bool x_bf16, bool dy_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_bf16) return dy_bf16 ? launch_grad<BF16, BF16>(na, st) : launch_grad<BF16, F32>(na, st);
    return dy_bf16 ? launch_grad<F32, BF16>(na, st) : launch_grad<F32, F32>(na, st);
}

}  // namespace omc
