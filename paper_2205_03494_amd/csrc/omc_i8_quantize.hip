// omc_i8_quantize: a matrix in fp32 or bf16 to 8-bit integers, a scale for every row or for every column.
//
//   a = max |x_i|,  s = a / 127 rounded to fp32,  code_i = the whole number nearest to x_i / s, ties to even.
// The quotient is never formed exactly: r = rint(x * (1 / s)) is off by at most one, and d = x - r s, which fp32 holds exactly (r = 0: x itself; r = 1: both are within a factor of two; otherwise x > s, and d is a
// multiple of s' last place below s / 2 and a little), says whether the neighbour is nearer.  Scales below 2^-100 are handled times 2^100, which is exact.
#include "omc_mx4.h"
#include "omc_product.h"

namespace omc {

struct Rounding {
    float scale, up, s, inverse;
    bool nan;
    __device__ __forceinline__ void of(float top, bool is_nan) {
        nan = is_nan;
        scale = is_nan ? __builtin_nanf("") : top / 127.0f;
        up = scale < 0x1p-100f ? 0x1p100f : 1.0f;
        s = is_nan || scale == 0.0f ? 1.0f : scale * up;
        inverse = is_nan || scale == 0.0f ? 0.0f : 1.0f / s;         // 0: all codes are 0
    }
    __device__ __forceinline__ float code(float x) const {
        if (inverse == 0.0f) return 0.0f;
        const float v = x * up;
        float r = rintf(v * inverse);
        const float d = fmaf(-r, s, v), twice = fabsf(d + d);
        const bool odd = static_cast<int>(r) & 1;
        if (twice > s || (twice == s && odd)) r += copysignf(1.0f, d);
        return fminf(fmaxf(r, -127.0f), 127.0f);                     // (a scale below 2^-126 is coarser than its largest value's 127th part)
    }
    __device__ __forceinline__ float value(float r) const { return r * scale; }
};
__device__ __forceinline__ uint32_t four_bytes(const float *r) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (static_cast<uint32_t>(static_cast<int>(r[i])) & 255u) << (8 * i);
    return w;
}
template <typename T>
__device__ __forceinline__ float from_top(uint32_t top) {
    return __uint_as_float(T::kBytes == 4 ? top : top << 16);
}

// LANES lanes (64, or the workgroup's 256) take a row, R pieces of eight values each; PIECES in registers.  REREAD: the row is longer, and is read twice.
template <typename T, int LANES, int R, bool REREAD>
__global__ __launch_bounds__(256) void i8_rows_kernel(I8Args ia) {
    __shared__ uint32_t tops[4];
    const uint32_t row = LANES == 64 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x, lane = LANES == 64 ? threadIdx.x & 63u : threadIdx.x;
    if (row >= ia.rows) return;                // (LANES == 256: the whole workgroup)
    const typename T::type *x = static_cast<const typename T::type *>(ia.x) + row * ia.ldx;
    const uint32_t pitch = static_cast<uint32_t>(i8_pitch(ia.cols)), run = 8 * LANES * R;
    Eight<T> v[R];
    uint32_t top = 0;
    for (uint32_t from = 0; from < (REREAD ? ia.cols : 1u); from += run) {
#pragma unroll
        for (uint32_t k = 0; k < R; ++k) {
            const uint32_t col = from + 8 * (lane + LANES * k);
            v[k].clear();
            if (col < ia.cols) v[k].load(x, col, ia.cols);
        }
#pragma unroll
        for (uint32_t k = 0; k < R; ++k) top = max(top, v[k].top());
    }
#pragma unroll
    for (int by = 1; by < 64; by *= 2) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), by)));
    if constexpr (LANES == 256) {
        if ((threadIdx.x & 63u) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
        top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    Rounding to;
    to.of(from_top<T>(top), top > T::kFinite);
    if (lane == 0) ia.scales[row] = to.scale;
    uint8_t *codes = ia.codes + row * static_cast<uint64_t>(pitch);
    for (uint32_t from = 0; from < (REREAD ? pitch : 1u); from += run) {
        if constexpr (REREAD) {
#pragma unroll
            for (uint32_t k = 0; k < R; ++k) {
                const uint32_t col = from + 8 * (lane + LANES * k);
                v[k].clear();
                if (col < ia.cols) v[k].load(x, col, ia.cols);
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < R; ++k) {
            const uint32_t col = from + 8 * (lane + LANES * k);
            if (col >= pitch) continue;
            float r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = to.code(v[k].value(i));
            const uint64_t w = four_bytes(r) | static_cast<uint64_t>(four_bytes(r + 4)) << 32;
            *reinterpret_cast<uint64_t *>(codes + col) = w;
            if (ia.values && col < ia.cols) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = to.value(r[i]);
                store_run<T, 8>(static_cast<typename T::type *>(ia.values) + row * ia.ldv + col, r, ia.cols - col);
            }
        }
    }
}

// A workgroup takes 32 columns, twice: for their largest magnitudes, and for the codes, which go through LDS so that runs of a column are written together.
template <typename T>
__global__ __launch_bounds__(1024) void i8_columns_kernel(I8Args ia) {
    constexpr uint32_t kRows = 512, kPitch = kRows + 16;
    __shared__ __attribute__((aligned(16))) uint8_t turned[32 * kPitch];
    __shared__ uint32_t tops[16][32];
    const uint32_t col0 = blockIdx.x * 32, col = col0 + 4 * (threadIdx.x & 7u), line = threadIdx.x >> 3;
    const uint32_t inside = col < ia.cols ? min(4u, ia.cols - col) : 0u;
    const typename T::type *x = static_cast<const typename T::type *>(ia.x) + col;
    auto load = [&](uint32_t row, float (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0.0f;
        if (row >= ia.rows) return;
        const typename T::type *from = x + row * ia.ldx;
        if (inside == 4) {
            typename T::type w[4];
            __builtin_memcpy(w, from, sizeof(w));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = load_f32(w + i);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                if (i < inside) v[i] = load_f32(from + i);
        }
    };
    uint32_t top[4] = {0, 0, 0, 0};
    for (uint32_t first = 0; first < ia.rows; first += kRows) {
        float v[4][4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) load(first + 128 * k + line, v[k]);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[i] = max(top[i], __float_as_uint(v[k][i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int by = 8; by < 64; by *= 2) top[i] = max(top[i], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[i]), by)));
        if ((threadIdx.x & 63u) < 8) tops[threadIdx.x >> 6][4 * (threadIdx.x & 7u) + i] = top[i];
    }
    __syncthreads();
    Rounding to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t t = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) t = max(t, tops[w][4 * (threadIdx.x & 7u) + i]);
        to[i].of(__uint_as_float(t), t > 0x7f7fffffu);
        if (line == 0 && static_cast<uint32_t>(i) < inside) ia.scales[col + i] = to[i].scale;
    }
    const uint64_t pitch = i8_pitch(ia.rows);
    for (uint32_t first = 0; first < ia.rows; first += kRows) {
        float v[4][4];
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) load(first + 128 * k + line, v[k]);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t row = first + 128 * k + line;
            float r[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                r[i] = to[i].code(v[k][i]);
                turned[(4 * (threadIdx.x & 7u) + i) * kPitch + 128 * k + line] = static_cast<uint8_t>(static_cast<int>(r[i]));
                r[i] = to[i].value(r[i]);
            }
            if (ia.values && row < ia.rows && inside > 0) store_run<T, 4>(static_cast<typename T::type *>(ia.values) + row * ia.ldv + col, r, inside);
        }
        __syncthreads();
        const uint32_t c = threadIdx.x / 32, at = 16 * (threadIdx.x % 32);
        if (col0 + c < ia.cols && first + at < pitch) *reinterpret_cast<u32x4 *>(ia.codes + (col0 + c) * pitch + first + at) = *reinterpret_cast<const u32x4 *>(turned + c * kPitch + at);
        __syncthreads();
    }
}

template <typename T>
static int launch_rows(const I8Args &ia, hipStream_t st) {
    const dim3 by_wave((ia.rows + 3) / 4), by_group(ia.rows), block(256);
    if (ia.cols <= 512) i8_rows_kernel<T, 64, 1, false><<<by_wave, block, 0, st>>>(ia);
    else if (ia.cols <= 1024) i8_rows_kernel<T, 64, 2, false><<<by_wave, block, 0, st>>>(ia);
    else if (ia.cols <= 2048) i8_rows_kernel<T, 256, 1, false><<<by_group, block, 0, st>>>(ia);
    else if (ia.cols <= 4096) i8_rows_kernel<T, 256, 2, false><<<by_group, block, 0, st>>>(ia);
    else if (ia.cols <= 8192) i8_rows_kernel<T, 256, 4, false><<<by_group, block, 0, st>>>(ia);
    else i8_rows_kernel<T, 256, 4, true><<<by_group, block, 0, st>>>(ia);
    return static_cast<int>(hipGetLastError());
}
int launch_i8_rows(const I8Args &ia, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch_rows<BF16>(ia, st) : launch_rows<F32>(ia, st);
}
int launch_i8_columns(const I8Args &ia, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((ia.cols + 31) / 32), block(1024);
    if (bf16) i8_columns_kernel<BF16><<<grid, block, 0, st>>>(ia);
    else i8_columns_kernel<F32><<<grid, block, 0, st>>>(ia);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
