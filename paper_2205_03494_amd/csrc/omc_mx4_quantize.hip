// omc_mx4_quantize: a matrix in fp32 or bf16 to MX4 codes and scales, blocks along its rows, its columns, or both from one read.
//
// Bound by memory: 2 or 4 bytes read and 17/32 written a value and direction, some ten instructions a value between them.
//
// Along rows alone a lane takes eight neighbours, 16 or 32 bytes and one dword of codes, and the four lanes of a block compare their largest magnitudes.
// Along columns a wave takes 32 rows x 128 columns, a lane two columns of them, so that a lane holds two whole blocks and no lane needs another's
// values; the codes of a workgroup's 256 rows go through LDS, so that 128 bytes of a column are written together.  Where both directions are asked for, 16 lanes compare
// their largest magnitudes of a row, from the same registers.
#include "omc_mx4.h"

namespace omc {

template <typename T>
__device__ __forceinline__ void store_values(const QuantArgs &qa, uint32_t row, uint32_t col, uint32_t codes, uint32_t byte) {
    typename T::type *to = static_cast<typename T::type *>(qa.values) + row * qa.ldv + col;
    const float unit = mx4_unit(byte);
    const bool nan = byte == kMx4NaN;
    uint32_t w[2 * T::kBytes];
    if constexpr (T::kBytes == 4) {
        const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3)};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = nan ? 0x7fc00000u : __float_as_uint(v[i / 2][i % 2]);
    } else {
        const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1),
                             __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3)};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = nan ? 0x7fc07fc0u : __builtin_bit_cast(uint32_t, v[i]);
    }
    if (col + 8 <= qa.cols) {
        __builtin_memcpy(to, w, 8 * T::kBytes);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (col + i < qa.cols) {
                if constexpr (T::kBytes == 4) to[i] = __builtin_bit_cast(float, w[i]);
                else to[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
            }
    }
}

// The eight values of a row from `col` on (four lanes hold a block, all of them take part): codes, scale and values.
template <typename T>
__device__ __forceinline__ void quantize_eight(const QuantArgs &qa, const Eight<T> &v, uint32_t row, uint32_t col, uint32_t padded, bool mine) {
    uint32_t top = v.top();
    top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0xb1, 0xf, 0xf, true)));   // lanes 1 0 3 2
    top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x4e, 0xf, 0xf, true)));   // lanes 2 3 0 1
    const uint32_t byte = mx4_scale<T>(top);
    const uint32_t codes = byte == kMx4NaN ? 0u : v.codes(mx4_unit(byte));
    if (!mine) return;
    if (qa.codes) {
        *reinterpret_cast<uint32_t *>(qa.codes + static_cast<uint64_t>(row) * (padded / 2) + col / 2) = codes;
        if (col % 32 == 0) {
            const uint32_t block = col / 32;
            if (!qa.images) {
                qa.scales[static_cast<uint64_t>(row) * (padded / 32) + block] = static_cast<uint8_t>(byte);
            } else {
                uint8_t *to = qa.scales + (block / 8) * mx4_image_pitch(qa.rows) + 8ull * row;
                to[mx4_image_byte(block % 8)] = static_cast<uint8_t>(byte);
                if (block % 8 == 0 && col + 128 == padded) {
                    *reinterpret_cast<uint16_t *>(to + mx4_image_byte(4)) = 0;
                    *reinterpret_cast<uint16_t *>(to + mx4_image_byte(6)) = 0;
                }
            }
        }
    }
    if (qa.values && col < qa.cols) store_values<T>(qa, row, col, codes, byte);
}

// 8 bytes of scales of a row, a thread.
__device__ __forceinline__ void reorder_scales(const Mx4Reorder &re, uint32_t block) {
    const uint32_t k128 = mx4_padded(re.cols) / 128, stages = (k128 + 1) / 2, groups = (re.rows + 255) / 256;
    const uint32_t stage = block / groups, row = block % groups * 256 + threadIdx.x;
    if (stage >= stages || row >= re.rows || threadIdx.x >= 256) return;
    const uint32_t *from = reinterpret_cast<const uint32_t *>(re.scales) + static_cast<uint64_t>(row) * k128 + 2 * stage;
    const uint32_t lower = from[0], upper = 2 * stage + 1 < k128 ? from[1] : 0u;
    uint32_t *to = reinterpret_cast<uint32_t *>(re.image + stage * mx4_image_pitch(re.rows)) + 2 * row;
    to[0] = (lower & 0xffffu) | upper << 16;
    to[1] = lower >> 16 | (upper & 0xffff0000u);
}
static uint32_t reorder_blocks(const Mx4Reorder &re) { return re.image ? (re.rows + 255) / 256 * ((mx4_padded(re.cols) + 255) / 256) : 0u; }

__global__ __launch_bounds__(256) void mx4_reorder_kernel(Mx4Reorder a, Mx4Reorder b, uint32_t blocks_a) {
    if (blockIdx.x < blocks_a) reorder_scales(a, blockIdx.x);
    else reorder_scales(b, blockIdx.x - blocks_a);
}
int launch_mx4_reorder(const Mx4Reorder &a, const Mx4Reorder &b, void *stream) {
    const uint32_t blocks_a = reorder_blocks(a), blocks = blocks_a + reorder_blocks(b);
    mx4_reorder_kernel<<<dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(a, b, blocks_a);
    return static_cast<int>(hipGetLastError());
}

// `first`: row of the launch's first item (a launch has less than 2^32 items).  The workgroups behind the items reorder the other matrix' scales.
template <typename T>
__global__ __launch_bounds__(256) void mx4_rows_kernel(QuantArgs qa, uint32_t first, uint32_t items) {
    if (qa.also.image && blockIdx.x >= (items + 255) / 256) {
        reorder_scales(qa.also, blockIdx.x - (items + 255) / 256);
        return;
    }
    const uint32_t padded = mx4_padded(qa.cols), eights = padded / 8, item = blockIdx.x * 256 + threadIdx.x;
    const bool mine = item < items;            // (whole blocks: padded / 8 is a multiple of 16)
    const uint32_t row = first + item / eights, col = 8 * (item % eights);
    Eight<T> v;
    v.clear();
    if (mine && col < qa.cols) v.load(static_cast<const typename T::type *>(qa.x) + row * qa.ldx + col, qa.cols - col);
    quantize_eight<T>(qa, v, row, col, padded, mine);
}

constexpr uint32_t kHigh = 256, kWide = 128;   // a tile; a wave takes 32 rows of it

// Two columns of 32 rows in a lane (bf16: both in lo): their blocks' codes and scale bytes.
template <typename T>
__device__ __forceinline__ void quantize_columns(const uint32_t (&lo)[32], const uint32_t (&hi)[32], u32x4 (&codes)[2], uint32_t (&byte)[2]) {
    uint32_t top[2] = {0, 0};
    if constexpr (T::kBytes == 4) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            top[0] = max(top[0], lo[i] & 0x7fffffffu);
            top[1] = max(top[1], hi[i] & 0x7fffffffu);
        }
    } else {
        u16x2 m = {0, 0};
#pragma unroll
        for (int i = 0; i < 32; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, lo[i] & 0x7fff7fffu));
        top[0] = m[0];
        top[1] = m[1];
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        byte[c] = mx4_scale<T>(top[c]);
        const float unit = mx4_unit(byte[c]);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            Eight<T> v;
            if constexpr (T::kBytes == 4) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v.w[i] = c == 0 ? lo[8 * d + i] : hi[8 * d + i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)   // the lower or upper halves of two rows
                    v.w[i] = __builtin_amdgcn_perm(lo[8 * d + 2 * i + 1], lo[8 * d + 2 * i], c == 0 ? 0x05040100u : 0x07060302u);
            }
            codes[c][d] = byte[c] == kMx4NaN ? 0u : v.codes(unit);
        }
    }
}

// Largest of 16 lanes' values, in all of them.
template <typename M>
__device__ __forceinline__ uint32_t largest_of_16(uint32_t x, M &&larger) {
    x = larger(x, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0xb1, 0xf, 0xf, true)));    // lanes 1 0 3 2
    x = larger(x, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x4e, 0xf, 0xf, true)));    // lanes 2 3 0 1
    x = larger(x, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x141, 0xf, 0xf, true)));   // eight lanes mirrored
    return larger(x, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x140, 0xf, 0xf, true)));   // sixteen lanes mirrored
}

// The same registers along the rows, of which 16 lanes hold a block: a lane's two codes of row i go to codes[i * 64 + lane], the scale of row i and block b to scales[i * 4 + b].
template <typename T>
__device__ __forceinline__ void quantize_rows(const uint32_t (&lo)[32], const uint32_t (&hi)[32], uint8_t *codes, uint8_t *scales, uint32_t lane) {
    auto one = [&](uint32_t i, uint32_t top) {
        const uint32_t byte = mx4_scale<T>(top);
        const float unit = mx4_unit(byte);
        uint32_t c;
        if constexpr (T::kBytes == 4) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, __uint_as_float(lo[i]), __uint_as_float(hi[i]), unit, 0);
        else c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, lo[i]), unit, 0);
        codes[i * 64 + lane] = static_cast<uint8_t>(byte == kMx4NaN ? 0u : c);
        if ((lane & 15u) == 0) scales[i * 4 + (lane >> 4)] = static_cast<uint8_t>(byte);
    };
    if constexpr (T::kBytes == 4) {
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) one(i, largest_of_16(max(lo[i] & 0x7fffffffu, hi[i] & 0x7fffffffu), [](uint32_t x, uint32_t y) { return max(x, y); }));
    } else {
        auto larger = [](uint32_t x, uint32_t y) { return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y))); };
#pragma unroll
        for (uint32_t i = 0; i < 32; i += 2) {   // two rows' largest in a register
            const uint32_t x = lo[i] & 0x7fff7fffu, y = lo[i + 1] & 0x7fff7fffu;
            const uint32_t top = largest_of_16(larger(__builtin_amdgcn_perm(y, x, 0x05040100u), __builtin_amdgcn_perm(y, x, 0x07060302u)), larger);
            one(i, top & 0xffffu);
            one(i + 1, top >> 16);
        }
    }
}

// Tiles of 256 x 128: blocks along the columns, along the rows, the columns' sums.
template <typename T>
__global__ __launch_bounds__(512) void mx4_tiles_kernel(QuantArgs qa, uint32_t tiles_r, uint32_t tiles_c) {
    typedef typename T::type E;
    constexpr uint32_t kPitch = 144;           // bytes of a column's codes in LDS, 128 and padding
    __shared__ __attribute__((aligned(16))) uint8_t codes_lds[kWide * kPitch];
    __shared__ __attribute__((aligned(16))) uint8_t rows_lds[8][32 * 64];
    __shared__ __attribute__((aligned(16))) uint8_t scales_lds[kWide * 8];
    __shared__ __attribute__((aligned(16))) uint8_t row_scales_lds[8][32 * 4];
    __shared__ float sums_lds[8][kWide];
    if (qa.also.image && blockIdx.x >= tiles_r * tiles_c) {
        reorder_scales(qa.also, blockIdx.x - tiles_r * tiles_c);
        return;
    }
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
    const uint32_t r0 = tr * kHigh + 32 * wave, c0 = tc * kWide, col = c0 + 2 * lane;
    const uint32_t height = r0 < qa.rows ? min(32u, qa.rows - r0) : 0u;
    const E *x = static_cast<const E *>(qa.x);

    uint32_t lo[32], hi[32];
#pragma unroll
    for (uint32_t i = 0; i < 32; ++i) lo[i] = hi[i] = 0;
    auto put = [&](uint32_t i, const E *from) {   // both columns, from any address
        uint32_t w[T::kBytes / 2];
        __builtin_memcpy(w, from, 2 * T::kBytes);
        lo[i] = w[0];
        if constexpr (T::kBytes == 4) hi[i] = w[1];
    };
    if (height == 32 && c0 + kWide <= qa.cols) {
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) put(i, x + (r0 + i) * qa.ldx + col);
    } else if (height > 0 && qa.cols > 1) {    // at the edges: what lies outside is read in the last row or the last two columns, and is zero
        const uint32_t at = min(col, qa.cols - 2);
        const bool in0 = col < qa.cols, in1 = col + 1 < qa.cols, shifted = col + 1 == qa.cols;
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) put(i, x + (r0 + min(i, height - 1)) * qa.ldx + at);
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) {
            const bool in = i < height;
            if constexpr (T::kBytes == 4) {
                lo[i] = in && in0 ? (shifted ? hi[i] : lo[i]) : 0u;
                hi[i] = in && in1 ? hi[i] : 0u;
            } else {
                lo[i] = in && in0 ? (shifted ? lo[i] >> 16 : lo[i]) : 0u;
            }
        }
    } else if (height > 0 && lane == 0) {
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i)
            if (i < height) {
                const E v = x[(r0 + i) * qa.ldx];
                if constexpr (T::kBytes == 4) lo[i] = __float_as_uint(v);
                else lo[i] = v;
            }
    }
    if (qa.codes_t) {
        u32x4 codes[2];
        uint32_t byte[2];
        quantize_columns<T>(lo, hi, codes, byte);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            *reinterpret_cast<u32x4 *>(codes_lds + (2 * lane + c) * kPitch + 16 * wave) = codes[c];
            scales_lds[(2 * lane + c) * 8 + (qa.images ? mx4_image_byte(wave) : wave)] = static_cast<uint8_t>(byte[c]);
        }
    }
    if (qa.codes) quantize_rows<T>(lo, hi, rows_lds[wave], row_scales_lds[wave], lane);
    if (qa.colsum) {
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            s0 += T::kBytes == 4 ? __uint_as_float(lo[i]) : bf16_low(lo[i]);
            s1 += T::kBytes == 4 ? __uint_as_float(hi[i]) : bf16_high(lo[i]);
        }
        sums_lds[wave][2 * lane] = s0;
        sums_lds[wave][2 * lane + 1] = s1;
    }
    __syncthreads();
    if (qa.codes_t) {
        const uint32_t pitch = mx4_padded(qa.rows) / 2, begin = tr * (kHigh / 2), there = min(pitch - begin, kHigh / 2);   // bytes of a column, of those in this tile
#pragma unroll
        for (uint32_t p = threadIdx.x; p < 8 * kWide; p += 512) {
            const uint32_t c = p / 8, at = 16 * (p % 8);
            if (c0 + c < qa.cols && at < there)
                *reinterpret_cast<u32x4 *>(qa.codes_t + static_cast<uint64_t>(c0 + c) * pitch + begin + at) = *reinterpret_cast<const u32x4 *>(codes_lds + c * kPitch + at);
        }
        const uint32_t c = threadIdx.x / 2, half = threadIdx.x % 2;
        if (threadIdx.x < 2 * kWide && c0 + c < qa.cols) {
            const uint32_t bytes = reinterpret_cast<const uint32_t *>(scales_lds)[threadIdx.x];
            if (qa.images) reinterpret_cast<uint32_t *>(qa.scales_t + tr * mx4_image_pitch(qa.cols))[2 * (c0 + c) + half] = bytes;
            else if (64 * half < there) reinterpret_cast<uint32_t *>(qa.scales_t + static_cast<uint64_t>(c0 + c) * (pitch / 16))[2 * tr + half] = bytes;
        }
    }
    if (qa.codes) {                            // 64 bytes of a row (all of them: rows are padded to 128 values)
        const uint32_t pitch = mx4_padded(qa.cols) / 2;
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            const uint32_t i = 16 * k + lane / 4, at = 16 * (lane % 4);
            if (i < height) *reinterpret_cast<u32x4 *>(qa.codes + static_cast<uint64_t>(r0 + i) * pitch + 64 * tc + at) = *reinterpret_cast<const u32x4 *>(rows_lds[wave] + 64 * i + at);
        }
        if (lane < height) {
            const uint32_t bytes = reinterpret_cast<const uint32_t *>(row_scales_lds[wave])[lane];
            if (!qa.images) {
                reinterpret_cast<uint32_t *>(qa.scales + static_cast<uint64_t>(r0 + lane) * (pitch / 16))[tc] = bytes;
            } else {                           // blocks 0, 1 and 2, 3 of a first or second half
                uint16_t *to = reinterpret_cast<uint16_t *>(qa.scales + (tc / 2) * mx4_image_pitch(qa.rows) + 8ull * (r0 + lane));
                to[tc % 2] = static_cast<uint16_t>(bytes);
                to[2 + tc % 2] = static_cast<uint16_t>(bytes >> 16);
                if (tc % 2 == 0 && tc + 1 == tiles_c) to[1] = to[3] = 0;
            }
        }
    }
    if (qa.colsum) {
        const uint32_t c = threadIdx.x;
        if (c < kWide && c0 + c < qa.cols) {
            float s = sums_lds[0][c];
#pragma unroll
            for (int w = 1; w < 8; ++w) s += sums_lds[w][c];
            qa.colsum[static_cast<uint64_t>(tr) * qa.cols + c0 + c] = s;
        }
    }
}

template <typename T>
static int launch(QuantArgs qa, hipStream_t st) {
    if (qa.codes_t || qa.colsum) {
        QuantArgs ta = qa;
        if (qa.values) ta.codes = ta.scales = nullptr;   // these along the rows, with the values
        const uint32_t tiles_r = (qa.rows + kHigh - 1) / kHigh, tiles_c = (qa.cols + kWide - 1) / kWide;
        mx4_tiles_kernel<T><<<dim3(tiles_r * tiles_c + reorder_blocks(qa.also)), dim3(512), 0, st>>>(ta, tiles_r, tiles_c);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || !qa.values) return static_cast<int>(e);
        qa.also.image = nullptr;
    }
    const uint32_t eights = mx4_padded(qa.cols) / 8, most = (1u << 30) / eights;   // rows of one launch
    for (uint32_t first = 0; first < qa.rows; first += most) {
        const uint32_t items = (qa.rows - first < most ? qa.rows - first : most) * eights;
        mx4_rows_kernel<T><<<dim3((items + 255) / 256 + reorder_blocks(qa.also)), dim3(256), 0, st>>>(qa, first, items);
        qa.also.image = nullptr;
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || qa.rows - first <= most) return static_cast<int>(e);
    }
    return 0;
}

int launch_mx4_quantize(const QuantArgs &qa, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch<BF16>(qa, st) : launch<F32>(qa, st);
}

}  // namespace omc
