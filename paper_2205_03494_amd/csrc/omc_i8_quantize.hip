// omc_i8_quantize: a matrix in fp32 or bf16 to 8-bit integers, a scale for every row or for every column (see omc_i8.h).
//
// Bound by memory.  Along rows a wave takes a row of up to 1024 values, a workgroup one of up to 8192, eight neighbours to a lane, and holds it in registers between the largest magnitude and the codes; longer ones are read
// twice.  16384 x 8192 in bf16: 75 us, 5.4 TB/s, and 118 with the rounded values, 5.7; 8192 x 8192 in fp32 57 us, 5.9 TB/s.
#include "omc_i8.h"
#include "omc_product.h"

namespace omc {

// LANES lanes (64, or the workgroup's 256) take a row, R pieces of eight values each; PIECES in registers.  REREAD: the row is longer, and is read twice.
template <typename T, int LANES, int R, bool REREAD, bool SHORT = false>
__global__ __launch_bounds__(256) void i8_rows_kernel(I8Args ia) {
    __shared__ uint32_t tops[4];
    const uint32_t lane = LANES == 64 ? threadIdx.x & 63u : threadIdx.x, stride = LANES == 64 ? 4 * gridDim.x : gridDim.x;
    for (uint32_t row = LANES == 64 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x; row < ia.rows; row += stride) {   // (LANES == 256: the whole workgroup)
        const typename T::type *x = static_cast<const typename T::type *>(ia.x) + row * ia.ldx;
        const uint32_t pitch = static_cast<uint32_t>(i8_pitch(ia.cols)), run = 8 * LANES * R;
        Eight<T> v[R];
        auto load_run = [&](uint32_t from) {       // nothing waits between the loads
#pragma unroll
            for (uint32_t k = 0; k < R; ++k) {
                const uint32_t col = from + 8 * (lane + LANES * k);
                v[k].clear();
                if (col < ia.cols) v[k].template fetch<SHORT>(x, col, ia.cols);
            }
#pragma unroll
            for (uint32_t k = 0; k < R; ++k) {
                const uint32_t col = from + 8 * (lane + LANES * k);
                if (col < ia.cols) v[k].settle(Eight<T>::missing(col, ia.cols));
            }
        };
        uint32_t top = 0;
        for (uint32_t from = 0; from < (REREAD ? ia.cols : 1u); from += run) {
            load_run(from);
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
            if constexpr (REREAD) load_run(from);
#pragma unroll
            for (uint32_t k = 0; k < R; ++k) {
                const uint32_t col = from + 8 * (lane + LANES * k);
                if (col >= pitch) continue;
                float x8[8], r[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x8[i] = v[k].value(i);
                to.eight(x8, r);
                const uint64_t w = four_bytes(r) | static_cast<uint64_t>(four_bytes(r + 4)) << 32;
                *reinterpret_cast<uint64_t *>(codes + col) = w;
                if (ia.values && col < ia.cols) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[i] = to.value(r[i]);
                    store_run<T, 8>(static_cast<typename T::type *>(ia.values) + row * ia.ldv + col, r, ia.cols - col);
                }
            }
        }
        if constexpr (LANES == 256) __syncthreads();   // tops again
    }
}

// Along columns, of few values: a workgroup takes COLS columns, twice (up to 2048 rows from registers the second time): for their largest magnitudes, and for the codes, which go through LDS so that runs of a column are written together.
template <typename T>
__global__ __launch_bounds__(1024) void i8_columns_kernel(I8Args ia) {
    constexpr uint32_t COLS = 8, kAcross = COLS / 4, kLines = 1024 / kAcross, kRows = 4 * kLines, kPitch = kRows + 16;   // lanes of a row, rows at a time
    __shared__ __attribute__((aligned(16))) uint8_t turned[COLS * kPitch];
    __shared__ uint32_t tops[16][COLS];
    const uint32_t across = threadIdx.x % kAcross, line = threadIdx.x / kAcross, col0 = blockIdx.x * COLS, col = col0 + 4 * across;
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
    float v[4][4];
    for (uint32_t first = 0; first < ia.rows; first += kRows) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) load(first + kLines * k + line, v[k]);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[i] = max(top[i], __float_as_uint(v[k][i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int by = kAcross; by < 64; by *= 2) top[i] = max(top[i], static_cast<uint32_t>(__shfl_xor(static_cast<int>(top[i]), by)));
        if ((threadIdx.x & 63u) < kAcross) tops[threadIdx.x >> 6][4 * across + i] = top[i];
    }
    __syncthreads();
    Rounding to[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t t = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) t = max(t, tops[w][4 * across + i]);
        to[i].of(__uint_as_float(t), t > 0x7f7fffffu);
        if (line == 0 && static_cast<uint32_t>(i) < inside) ia.scales[col + i] = to[i].scale;
    }
    const bool special = to[0].special() || to[1].special() || to[2].special() || to[3].special();
    const uint64_t pitch = i8_pitch(ia.rows);
    for (uint32_t first = 0; first < ia.rows; first += kRows) {
        if (ia.rows > kRows) {                 // (otherwise they are there)
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) load(first + kLines * k + line, v[k]);
        }
        float r[4][4], far = 0.0f;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            if (first + kLines * k >= ia.rows) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[k][i] = to[i].near(v[k][i], far);
        }
        if (far > Rounding::kFar || special) {
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) r[k][i] = to[i].code(v[k][i]);
        }
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            if (first + kLines * k >= ia.rows) break;   // (kLines is whole 128s: no codes there either)
            const uint32_t row = first + kLines * k + line;
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                turned[(4 * across + i) * kPitch + kLines * k + line] = static_cast<uint8_t>(static_cast<int>(r[k][i]));
                r[k][i] = to[i].value(r[k][i]);
            }
            if (ia.values && row < ia.rows && inside > 0) store_run<T, 4>(static_cast<typename T::type *>(ia.values) + row * ia.ldv + col, r[k], inside);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t c = threadIdx.x / (kRows / 16); c < COLS; c += 1024 / (kRows / 16)) {
            const uint32_t at = 16 * (threadIdx.x % (kRows / 16));
            if (col0 + c < ia.cols && first + at < pitch)
                *reinterpret_cast<u32x4 *>(ia.codes + (col0 + c) * pitch + first + at) = *reinterpret_cast<const u32x4 *>(turned + c * kPitch + at);
        }
        __syncthreads();
    }
}

// Of many: three launches.  The largest magnitudes of every kMaximaRows rows, a row of bits for each, which lie where the codes will;
constexpr uint32_t kMaximaRows = 128;
template <typename T>
__global__ __launch_bounds__(256) void i8_maxima_kernel(I8Args ia, uint32_t *parts) {
    __shared__ uint32_t tops[4][512];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, across = (ia.cols + 511) / 512, down = blockIdx.x / across, col0 = (blockIdx.x - down * across) * 512, col = col0 + 8 * lane, row0 = down * kMaximaRows;
    uint32_t top[8] = {};
    if (col < ia.cols) {
        const typename T::type *x = static_cast<const typename T::type *>(ia.x);
        const uint32_t missing = Eight<T>::missing(col, ia.cols);
        for (uint32_t first = 0; first < kMaximaRows / 4 && row0 + 4 * first < ia.rows; first += 4) {
            Eight<T> v[4];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) v[k].template fetch<false>(x + min(row0 + 4 * (first + k) + wave, ia.rows - 1) * ia.ldx, col, ia.cols);   // (the last row more than once)
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                v[k].settle(missing);
#pragma unroll
                for (int i = 0; i < 8; ++i) top[i] = max(top[i], __float_as_uint(v[k].value(i)) & 0x7fffffffu);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) tops[wave][8 * lane + i] = top[i];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 512; c += 256)
        if (col0 + c < ia.cols) parts[static_cast<uint64_t>(down) * ia.cols + col0 + c] = max(max(tops[0][c], tops[1][c]), max(tops[2][c], tops[3][c]));
}
// the scales;
__global__ __launch_bounds__(64) void i8_scales_kernel(const uint32_t *parts, uint32_t count, uint32_t cols, float *scales) {
    const uint32_t col = blockIdx.x * 64 + threadIdx.x;
    if (col >= cols) return;
    uint32_t top = 0;
    for (uint32_t first = 0; first < count; first += 8) {
        uint32_t v[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) v[k] = parts[static_cast<uint64_t>(min(first + k, count - 1)) * cols + col];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) top = max(top, v[k]);
    }
    Rounding to;
    to.of(__uint_as_float(top), top > 0x7f7fffffu);
    scales[col] = to.scale;
}
// and the codes, a workgroup of 128 rows x 64 columns.
template <typename T>
__global__ __launch_bounds__(256) void i8_turn_kernel(I8Args ia) {
    constexpr uint32_t kPitch = 132;           // (eight columns apart, lanes write to different banks)
    __shared__ uint32_t turned[64 * kPitch / 4];
    uint8_t *bytes = reinterpret_cast<uint8_t *>(turned);
    const uint32_t across = threadIdx.x & 7u, line = threadIdx.x >> 3, tiles_across = (ia.cols + 63) / 64, tiles = tiles_across * ((ia.rows + 127) / 128);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t down = tile / tiles_across, col0 = (tile - down * tiles_across) * 64, col = col0 + 8 * across, row0 = down * 128;
        if (col < ia.cols) {
            const typename T::type *x = static_cast<const typename T::type *>(ia.x);
            const uint32_t missing = Eight<T>::missing(col, ia.cols);
            Eight<T> v[4];
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) v[k].template fetch<false>(x + min(row0 + 32 * k + line, ia.rows - 1) * ia.ldx, col, ia.cols);
            Rounding to[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) to[i].with(ia.scales[min(col + i, ia.cols - 1)]);
            bool special = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) special |= to[i].special();
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) {
                const uint32_t row = row0 + 32 * k + line;
                v[k].settle(missing);
                float r[8], far = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = to[i].near(v[k].value(i), far);
                if (far > Rounding::kFar || special) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[i] = to[i].code(v[k].value(i));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) bytes[(8 * across + i) * kPitch + 32 * k + line] = row < ia.rows ? static_cast<uint8_t>(static_cast<int>(r[i])) : 0;
                if (ia.values && row < ia.rows) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[i] = to[i].value(r[i]);
                    store_run<T, 8>(static_cast<typename T::type *>(ia.values) + row * ia.ldv + col, r, ia.cols - col);
                }
            }
        }
        __syncthreads();
        const uint64_t pitch = i8_pitch(ia.rows);
#pragma unroll
        for (uint32_t t = threadIdx.x; t < 512; t += 256) {
            const uint32_t c = t / 8, at = 16 * (t % 8);
            if (col0 + c >= ia.cols) continue;
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = turned[(c * kPitch + at) / 4 + i];
            *reinterpret_cast<u32x4 *>(ia.codes + (col0 + c) * pitch + row0 + at) = w;
        }
        __syncthreads();
    }
}

constexpr uint32_t kMostGroups = 1u << 22;    // a launch's work-items within 32 bits; what is more is taken in turn
template <typename T>
static int launch_rows(const I8Args &ia, hipStream_t st) {
    const dim3 by_wave((ia.rows + 3) / 4), by_group(ia.rows < kMostGroups ? ia.rows : kMostGroups), block(256);
    if (ia.cols < 8) i8_rows_kernel<T, 64, 1, false, true><<<by_wave, block, 0, st>>>(ia);
    else if (ia.cols <= 512) i8_rows_kernel<T, 64, 1, false><<<by_wave, block, 0, st>>>(ia);
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
// In a graph, fp32 / bf16, in one launch and in three.  Up to the limits, without values: 971 x 243 7.4 / 7.8 us and 15.5 / 15.4, 1024 x 1024 10.2 / 10.1 and 13.8 / 12.5, 1024 x 2048 12.1 / 12.1 and 15.5 / 14.7, 2048 x 1024 14.3 / 13.4
// and 15.8 / 14.7, 2048 x 1536 17.0 / 15.5 and 16.9 / 16.4, 2048 x 2048 18.4 / 17.6 and 18.4 / 16.7.  With values three win in the far corner, by 3 us at most: 2048 x 1024 18.5 / 15.1 and 16.9 / 15.4, 2048 x 1536 21.4 / 17.3 and 18.7 / 17.4,
// 2048 x 2048 23.6 / 20.2 and 20.7 / 18.0 (1024 x 2048: 14.5 / 13.9 and 16.7 / 15.7); one rule for both.  Beyond: 1024 x 4096 21.8 / 21.6 and 17.0 / 16.4, 4096 x 1024 36.5 / 32.0 and 18.2 / 17.4; 8192 x 8192 in fp32 362 and 113;
// 16384 x 8192 in bf16 593 and 158, which reads the matrix twice: 4.3 TB/s.  Strips of four columns instead of eight: 971 x 243 in fp32 with values 8.3 -> 9.3 us, 2048 x 2048 23.6 -> 42.
// Fewer than eight columns go in one launch whatever their length, since the others' loads are of eight: all in one workgroup, 0.23 ms for 65536 x 7 in fp32, 4.4 for 2^20 x 7, 90 for 2^24 x 7 (of eight columns, in three launches, 0.4 and 7.1).
constexpr uint32_t kStripRows = 2048, kStripCols = 2048;
template <typename T>
static int launch_columns(const I8Args &ia, hipStream_t st) {
    if (ia.cols < 8 || (ia.rows <= kStripRows && ia.cols <= kStripCols)) {
        i8_columns_kernel<T><<<dim3((ia.cols + 7) / 8), dim3(1024), 0, st>>>(ia);
        return static_cast<int>(hipGetLastError());
    }
    const uint32_t count = (ia.rows + kMaximaRows - 1) / kMaximaRows;
    uint32_t *parts = reinterpret_cast<uint32_t *>(ia.codes);    // (4 bytes for every kMaximaRows rows)
    i8_maxima_kernel<T><<<dim3((ia.cols + 511) / 512 * count), dim3(256), 0, st>>>(ia, parts);
    i8_scales_kernel<<<dim3((ia.cols + 63) / 64), dim3(64), 0, st>>>(parts, count, ia.cols, ia.scales);
    const uint32_t tiles = (ia.cols + 63) / 64 * count;
    static_assert(kMaximaRows == 128, "a row of tiles");
    i8_turn_kernel<T><<<dim3(tiles < kMostGroups ? tiles : kMostGroups), dim3(256), 0, st>>>(ia);
    return static_cast<int>(hipGetLastError());
}
int launch_i8_columns(const I8Args &ia, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch_columns<BF16>(ia, st) : launch_columns<F32>(ia, st);
}

}  // namespace omc
