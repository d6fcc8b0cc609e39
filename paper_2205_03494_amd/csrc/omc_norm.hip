// omc_layer_norm and omc_layer_norm_backward.
//
// Bound by memory: a row is read once and stays in registers, eight neighbours a lane and piece, between the sum of its values, the sum of their squared distances from the mean, and
// the result.  A wave takes a row of up to 2048 values, four waves up to 8192, sixteen up to 16384; longer rows are read again for every sum.
// Backward, a thread keeps the same columns of all rows that its workgroup takes, so that the sums over the rows (dgamma, dbeta) stay in registers too; every workgroup leaves one row of
// partial sums, which a second kernel adds up in order.
#include <type_traits>

#include "omc_mx4.h"

namespace omc {

// Sum over the 64 lanes, in all of them; a fixed tree.
__device__ __forceinline__ float wave_sum(float x) {
    auto dpp = [](float v, auto control) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true)); };
    x += dpp(x, std::integral_constant<int, 0xb1>{});    // lanes 1 0 3 2
    x += dpp(x, std::integral_constant<int, 0x4e>{});    // lanes 2 3 0 1
    x += dpp(x, std::integral_constant<int, 0x141>{});   // eight lanes mirrored
    x += dpp(x, std::integral_constant<int, 0x140>{});   // sixteen lanes mirrored
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Sums over the WAVES waves that share a row.  Every call takes the next of two places in LDS, so that one barrier a call is enough: who writes a place again has passed
// the barrier of the call between, which nobody does before having read it.
template <int WAVES, int COUNT>
struct RowSum {
    float (*places)[WAVES][COUNT];             // [2]
    uint32_t wave, next;
    __device__ __forceinline__ void operator()(float (&x)[COUNT]) {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) x[c] = wave_sum(x[c]);
        if constexpr (WAVES > 1) {
            auto &place = places[next];
            next ^= 1;
            if ((threadIdx.x & 63u) == 0) {
#pragma unroll
                for (int c = 0; c < COUNT; ++c) place[wave][c] = x[c];
            }
            __syncthreads();
#pragma unroll
            for (int c = 0; c < COUNT; ++c) {
                x[c] = place[0][c];
#pragma unroll
                for (int w = 1; w < WAVES; ++w) x[c] += place[w][c];
            }
        }
    }
};

__device__ __forceinline__ void load_weights(float (&w)[8], const float *p, uint32_t left, float otherwise) {
    if (p && left >= 8) {
        __builtin_memcpy(w, p, 32);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) w[i] = p && i < left ? p[i] : otherwise;
    }
}

__device__ __forceinline__ float reciprocal_deviation(float variance, float eps) { return 1.0f / __builtin_sqrtf(variance + eps); }

// WAVES waves a row, PIECES pieces of eight values a lane; a workgroup of 4 waves (WAVES <= 4) or of WAVES takes rows blockIdx.x, + gridDim.x, ... of its groups.
template <typename X, typename Y, int WAVES, int PIECES>
__global__ __launch_bounds__(WAVES < 4 ? 256 : 64 * WAVES) void norm_kernel(NormArgs na) {
    constexpr int kTogether = WAVES < 4 ? 4 / WAVES : 1;
    __shared__ float places[2][WAVES][1];
    const uint32_t wave = threadIdx.x >> 6, cols = na.cols, t = threadIdx.x % (64 * WAVES);
    RowSum<WAVES, 1> row_sum{places, wave, 0};
    uint32_t left[PIECES];
    float gamma[PIECES][8], beta[PIECES][8];
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        const uint32_t col = 8 * (t + 64 * WAVES * p);
        left[p] = col < cols ? cols - col : 0u;
        load_weights(gamma[p], na.gamma ? na.gamma + col : nullptr, left[p], 1.0f);
        load_weights(beta[p], na.beta ? na.beta + col : nullptr, left[p], 0.0f);
    }
    const float count = static_cast<float>(cols);
    for (uint32_t row = blockIdx.x * kTogether + (WAVES < 4 ? wave / WAVES : 0u); row < na.rows; row += gridDim.x * kTogether) {
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + row * na.ldx + 8 * t;
        Eight<X> v[PIECES];
        float sum[1] = {0.0f};
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) v[p].load(x + 512 * WAVES * p, left[p]);
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
        typename Y::type *y = static_cast<typename Y::type *>(na.y) + row * na.ldy + 8 * t;
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            float out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = __builtin_fmaf((v[p].value(i) - mean) * rstd, gamma[p][i], beta[p][i]);
            store_run<Y, 8>(y + 512 * WAVES * p, out, left[p]);
        }
        if (t == 0) {
            if (na.mean) na.mean[row] = mean;
            if (na.rstd) na.rstd[row] = rstd;
        }
    }
}

// Rows of any length, a workgroup of sixteen waves each: one pass for the mean, one for the deviation, one for the result.
template <typename X, typename Y>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs na) {
    __shared__ float places[2][16][1];
    const uint32_t cols = na.cols;
    const float count = static_cast<float>(cols);
    RowSum<16, 1> row_sum{places, threadIdx.x >> 6, 0};
    for (uint32_t row = blockIdx.x; row < na.rows; row += gridDim.x) {
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + row * na.ldx;
        typename Y::type *y = static_cast<typename Y::type *>(na.y) + row * na.ldy;
        float sum[1] = {0.0f}, squares[1] = {0.0f};
        for (uint32_t c = threadIdx.x; c < cols; c += 1024) sum[0] += load_f32(x + c);
        row_sum(sum);
        const float mean = sum[0] / count;
        for (uint32_t c = threadIdx.x; c < cols; c += 1024) {
            const float d = load_f32(x + c) - mean;
            squares[0] = __builtin_fmaf(d, d, squares[0]);
        }
        row_sum(squares);
        const float rstd = reciprocal_deviation(squares[0] / count, na.eps);
        for (uint32_t c = threadIdx.x; c < cols; c += 1024) {
            const float out[1] = {__builtin_fmaf((load_f32(x + c) - mean) * rstd, na.gamma ? na.gamma[c] : 1.0f, na.beta ? na.beta[c] : 0.0f)};
            if constexpr (Y::kBytes == 4) y[c] = out[0];
            else y[c] = to_bf16(out[0]);
        }
        if (threadIdx.x == 0) {
            if (na.mean) na.mean[row] = mean;
            if (na.rstd) na.rstd[row] = rstd;
        }
    }
}

// ---- backward

// The partial sums of a workgroup: a row of 2 * cols floats, dgamma's then dbeta's.
template <typename X, typename Y, int WAVES, int PIECES>
__global__ __launch_bounds__(WAVES < 4 ? 256 : 64 * WAVES) void norm_grad_kernel(NormGradArgs na) {
    constexpr int kTogether = WAVES < 4 ? 4 / WAVES : 1;
    __shared__ float places[2][WAVES][2];
    __shared__ float joined[kTogether > 1 ? kTogether - 1 : 1][kTogether > 1 ? 64 * WAVES * 16 : 1];
    const uint32_t wave = threadIdx.x >> 6, cols = na.cols, t = threadIdx.x % (64 * WAVES), mine = WAVES < 4 ? wave / WAVES : 0u;
    RowSum<WAVES, 2> row_sum{places, wave, 0};
    uint32_t left[PIECES];
    float gamma[PIECES][8], dgamma[PIECES][8], dbeta[PIECES][8];
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        const uint32_t col = 8 * (t + 64 * WAVES * p);
        left[p] = col < cols ? cols - col : 0u;
        load_weights(gamma[p], na.gamma ? na.gamma + col : nullptr, left[p], 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) dgamma[p][i] = dbeta[p][i] = 0.0f;
    }
    const float count = static_cast<float>(cols);
    for (uint32_t row = blockIdx.x * kTogether + mine; row < na.rows; row += gridDim.x * kTogether) {
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + row * na.ldx + 8 * t;
        const typename Y::type *dy = static_cast<const typename Y::type *>(na.dy) + row * na.lddy + 8 * t;
        Eight<X> v[PIECES];
        Eight<Y> g[PIECES];
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p) {
            v[p].load(x + 512 * WAVES * p, left[p]);
            g[p].load(dy + 512 * WAVES * p, left[p]);
        }
        const float mean = na.mean[row], rstd = na.rstd[row];
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (uint32_t p = 0; p < PIECES; ++p)
#pragma unroll
            for (int i = 0; i < 8; ++i) {      // (past the end dy is zero, and x finite)
                const float hat = (v[p].value(i) - mean) * rstd, d = g[p].value(i), u = d * gamma[p][i];
                sums[0] += u;
                sums[1] = __builtin_fmaf(u, hat, sums[1]);
                dgamma[p][i] = __builtin_fmaf(d, hat, dgamma[p][i]);
                dbeta[p][i] += d;
            }
        if (na.dx) {
            row_sum(sums);
            const float mean_u = sums[0] / count, mean_uh = sums[1] / count;
            typename X::type *dx = static_cast<typename X::type *>(na.dx) + row * na.lddx + 8 * t;
#pragma unroll
            for (uint32_t p = 0; p < PIECES; ++p) {
                float out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float hat = (v[p].value(i) - mean) * rstd;
                    out[i] = rstd * ((__builtin_fmaf(g[p].value(i), gamma[p][i], -mean_u)) - hat * mean_uh);
                }
                store_run<X, 8>(dx + 512 * WAVES * p, out, left[p]);
            }
        }
    }
    if (!na.parts) return;
    float *to = na.parts + static_cast<uint64_t>(blockIdx.x) * 2 * cols;
#pragma unroll
    for (uint32_t p = 0; p < PIECES; ++p) {
        if constexpr (kTogether > 1) {
            if (p > 0) __syncthreads();
            if (mine > 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    joined[mine - 1][i * (64 * WAVES) + t] = dgamma[p][i];
                    joined[mine - 1][(8 + i) * (64 * WAVES) + t] = dbeta[p][i];
                }
            }
            __syncthreads();
            if (mine == 0) {
#pragma unroll
                for (int w = 0; w < kTogether - 1; ++w)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dgamma[p][i] += joined[w][i * (64 * WAVES) + t];
                        dbeta[p][i] += joined[w][(8 + i) * (64 * WAVES) + t];
                    }
            }
        }
        if (mine == 0 && left[p] > 0) {
            const uint32_t col = 8 * (t + 64 * WAVES * p);
            store_run<F32, 8>(to + col, dgamma[p], left[p]);
            store_run<F32, 8>(to + cols + col, dbeta[p], left[p]);
        }
    }
}

// Rows of any length: dx by a workgroup a row, the columns' sums by another kernel.
template <typename X, typename Y>
__global__ __launch_bounds__(1024) void norm_grad_long_kernel(NormGradArgs na) {
    __shared__ float places[2][16][2];
    const uint32_t cols = na.cols;
    const float count = static_cast<float>(cols);
    RowSum<16, 2> row_sum{places, threadIdx.x >> 6, 0};
    for (uint32_t row = blockIdx.x; row < na.rows; row += gridDim.x) {
        const typename X::type *x = static_cast<const typename X::type *>(na.x) + row * na.ldx;
        const typename Y::type *dy = static_cast<const typename Y::type *>(na.dy) + row * na.lddy;
        typename X::type *dx = static_cast<typename X::type *>(na.dx) + row * na.lddx;
        const float mean = na.mean[row], rstd = na.rstd[row];
        float sums[2] = {0.0f, 0.0f};
        for (uint32_t c = threadIdx.x; c < cols; c += 1024) {
            const float u = load_f32(dy + c) * (na.gamma ? na.gamma[c] : 1.0f);
            sums[0] += u;
            sums[1] = __builtin_fmaf(u, (load_f32(x + c) - mean) * rstd, sums[1]);
        }
        row_sum(sums);
        const float mean_u = sums[0] / count, mean_uh = sums[1] / count;
        for (uint32_t c = threadIdx.x; c < cols; c += 1024) {
            const float u = load_f32(dy + c) * (na.gamma ? na.gamma[c] : 1.0f), hat = (load_f32(x + c) - mean) * rstd;
            const float out = rstd * ((u - mean_u) - hat * mean_uh);
            if constexpr (X::kBytes == 4) dx[c] = out;
            else dx[c] = to_bf16(out);
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
static uint32_t waves_of(uint32_t cols) { return cols <= 2048 ? 1 : cols <= 8192 ? 4 : 16; }

template <typename X, typename Y>
static int launch_norm(const NormArgs &na, hipStream_t st) {
    if (na.cols > kLongest) {
        norm_long_kernel<X, Y><<<dim3(na.rows < 4096 ? na.rows : 4096), dim3(1024), 0, st>>>(na);
        return static_cast<int>(hipGetLastError());
    }
    const uint32_t waves = waves_of(na.cols), together = waves < 4 ? 4 / waves : 1, groups = (na.rows + together - 1) / together;
    const dim3 grid(groups < 2048 ? groups : 2048), block(waves < 4 ? 256 : 64 * waves);
    if (na.cols <= 512) norm_kernel<X, Y, 1, 1><<<grid, block, 0, st>>>(na);
    else if (na.cols <= 1024) norm_kernel<X, Y, 1, 2><<<grid, block, 0, st>>>(na);
    else if (na.cols <= 2048) norm_kernel<X, Y, 1, 4><<<grid, block, 0, st>>>(na);
    else if (na.cols <= 4096) norm_kernel<X, Y, 4, 2><<<grid, block, 0, st>>>(na);
    else if (na.cols <= 8192) norm_kernel<X, Y, 4, 4><<<grid, block, 0, st>>>(na);
    else norm_kernel<X, Y, 16, 2><<<grid, block, 0, st>>>(na);
    return static_cast<int>(hipGetLastError());
}
int launch_layer_norm(const NormArgs &na, bool x_bf16, bool y_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_bf16) return y_bf16 ? launch_norm<BF16, BF16>(na, st) : launch_norm<BF16, F32>(na, st);
    return y_bf16 ? launch_norm<F32, BF16>(na, st) : launch_norm<F32, F32>(na, st);
}

// Rows of partial sums: as many as workgroups.
static uint32_t grad_groups(uint32_t rows, uint32_t cols) {
    if (cols > kLongest) return rows < 64 ? rows : 64;
    const uint32_t waves = waves_of(cols), together = waves < 4 ? 4 / waves : 1, groups = (rows + together - 1) / together;
    const uint32_t most = waves == 16 ? 256 : 512;
    return groups < most ? groups : most;
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
        const uint32_t waves = waves_of(na.cols);
        const dim3 grid(groups), block(waves < 4 ? 256 : 64 * waves);
        if (na.cols <= 512) norm_grad_kernel<X, Y, 1, 1><<<grid, block, 0, st>>>(na);
        else if (na.cols <= 1024) norm_grad_kernel<X, Y, 1, 2><<<grid, block, 0, st>>>(na);
        else if (na.cols <= 2048) norm_grad_kernel<X, Y, 1, 4><<<grid, block, 0, st>>>(na);
        else if (na.cols <= 4096) norm_grad_kernel<X, Y, 4, 2><<<grid, block, 0, st>>>(na);
        else if (na.cols <= 8192) norm_grad_kernel<X, Y, 4, 4><<<grid, block, 0, st>>>(na);
        else norm_grad_kernel<X, Y, 16, 2><<<grid, block, 0, st>>>(na);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !na.parts) return static_cast<int>(e);
    return launch_column_sums(na.parts, groups, na.cols, 2 * na.cols, na.dgamma, na.dbeta, st);
}
int launch_layer_norm_backward(const NormGradArgs &na, bool x_bf16, bool dy_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_bf16) return dy_bf16 ? launch_grad<BF16, BF16>(na, st) : launch_grad<BF16, F32>(na, st);
    return dy_bf16 ? launch_grad<F32, BF16>(na, st) : launch_grad<F32, F32>(na, st);
}

}  // namespace omc
