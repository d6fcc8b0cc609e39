// omc_mx4_quantize: a matrix in fp32 or bf16 to MX4 codes and scales, blocks along its rows, its columns, or both from one read.
//
// Bound by memory: 2 or 4 bytes read and 17/32 written a value and direction, some ten instructions a value between them.
//
// Along rows a lane takes eight neighbours, 16 or 32 bytes and one dword of codes, and the four lanes of a block compare their largest magnitudes.
// Along columns a wave takes 32 rows x 128 columns, a lane two columns of them, so that a lane holds two whole blocks and no lane needs another's
// values; the codes of a workgroup's 128 rows go through LDS, so that 64 bytes of a column are written together.  Where both
// directions are asked for, the tile is read a second time, row-wise, from the cache.
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
    if (stage >= stages || row >= re.rows) return;
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

constexpr uint32_t kTile = 128;

// Two columns of 32 rows in a lane: their blocks' codes and scale bytes.
template <typename T>
__device__ __forceinline__ void quantize_pair(const uint32_t (&lo)[32], const uint32_t (&hi)[32], u32x4 (&codes)[2], uint32_t (&byte)[2]) {
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

// Tiles of 128 x 128: blocks along the columns, the columns' sums, and on a second read blocks along the rows.
template <typename T>
__global__ __launch_bounds__(256) void mx4_tiles_kernel(QuantArgs qa, uint32_t tiles_r, uint32_t tiles_c) {
    typedef typename T::type E;
    constexpr uint32_t kPitch = 80;            // bytes of a column's codes in LDS, 64 and padding
    __shared__ __attribute__((aligned(16))) uint8_t codes_lds[kTile * kPitch];
    __shared__ uint8_t scales_lds[kTile * 4];
    __shared__ float sums_lds[4][kTile];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // neighbours down a column, whose codes share a cache line, one after the other on the same die
    if (qa.also.image && blockIdx.x >= tiles_r * tiles_c) {
        reorder_scales(qa.also, blockIdx.x - tiles_r * tiles_c);
        return;
    }
    const uint32_t total = tiles_r * tiles_c, q = total / 8, rest = total % 8, die = blockIdx.x % 8;
    const uint32_t id = die * q + min(die, rest) + blockIdx.x / 8;
    const uint32_t tr = id % tiles_r, tc = id / tiles_r;
    const uint32_t r0 = tr * kTile + 32 * wave, c0 = tc * kTile, col = c0 + 2 * lane;
    const uint32_t height = r0 < qa.rows ? min(32u, qa.rows - r0) : 0u;
    const E *x = static_cast<const E *>(qa.x);
    const uint32_t padded_t = mx4_padded(qa.rows);

    uint32_t lo[32], hi[32];                   // bf16: both columns in lo
    if (height == 32 && c0 + kTile <= qa.cols) {
        const E *from = x + r0 * qa.ldx + col;
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) {
            uint32_t w[T::kBytes / 2];
            __builtin_memcpy(w, from + i * qa.ldx, 2 * T::kBytes);
            lo[i] = w[0];
            if constexpr (T::kBytes == 4) hi[i] = w[1];
        }
    } else if (height > 0) {                   // at the edges: what lies outside is read at the last row or column, and is zero
        const E *from0 = x + r0 * qa.ldx + min(col, qa.cols - 1), *from1 = x + r0 * qa.ldx + min(col + 1, qa.cols - 1);
        const bool in0 = col < qa.cols, in1 = col + 1 < qa.cols;
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) {
            const uint64_t at = min(i, height - 1) * qa.ldx;
            const E v0 = from0[at], v1 = from1[at];
            if constexpr (T::kBytes == 4) {
                lo[i] = in0 && i < height ? __builtin_bit_cast(uint32_t, v0) : 0u;
                hi[i] = in1 && i < height ? __builtin_bit_cast(uint32_t, v1) : 0u;
            } else {
                lo[i] = (in0 && i < height ? v0 : 0u) | (in1 && i < height ? static_cast<uint32_t>(v1) << 16 : 0u);
            }
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 32; ++i) lo[i] = hi[i] = 0;
    }
    if (qa.codes_t) {
        u32x4 codes[2];
        uint32_t byte[2];
        quantize_pair<T>(lo, hi, codes, byte);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            *reinterpret_cast<u32x4 *>(codes_lds + (2 * lane + c) * kPitch + 16 * wave) = codes[c];
            scales_lds[(2 * lane + c) * 4 + wave] = static_cast<uint8_t>(byte[c]);
        }
    }
    if (qa.colsum) {
        float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            s0 += T::kBytes == 4 ? __builtin_bit_cast(float, lo[i]) : bf16_low(lo[i]);
            s1 += T::kBytes == 4 ? __builtin_bit_cast(float, hi[i]) : bf16_high(lo[i]);
        }
        sums_lds[wave][2 * lane] = s0;
        sums_lds[wave][2 * lane + 1] = s1;
    }
    __syncthreads();
    if (qa.codes_t) {
#pragma unroll
        for (uint32_t p = threadIdx.x; p < 4 * kTile; p += 256) {
            const uint32_t c = p / 4;
            if (c0 + c < qa.cols)
                *reinterpret_cast<u32x4 *>(qa.codes_t + static_cast<uint64_t>(c0 + c) * (padded_t / 2) + tr * (kTile / 2) + 16 * (p % 4)) =
                    *reinterpret_cast<const u32x4 *>(codes_lds + c * kPitch + 16 * (p % 4));
        }
        const uint32_t c = threadIdx.x;
        if (c < kTile && c0 + c < qa.cols) {
            const uint32_t bytes = *reinterpret_cast<const uint32_t *>(scales_lds + 4 * c);
            if (!qa.images) {
                *reinterpret_cast<uint32_t *>(qa.scales_t + static_cast<uint64_t>(c0 + c) * (padded_t / 32) + 4 * tr) = bytes;
            } else {
                uint16_t *to = reinterpret_cast<uint16_t *>(qa.scales_t + (tr / 2) * mx4_image_pitch(qa.cols) + 8ull * (c0 + c));
                to[tr % 2] = static_cast<uint16_t>(bytes);
                to[2 + tr % 2] = static_cast<uint16_t>(bytes >> 16);
                if (tr % 2 == 0 && tr + 1 == tiles_r) to[1] = to[3] = 0;
            }
        }
    }
    if (qa.colsum) {
        const uint32_t c = threadIdx.x;
        if (c < kTile && c0 + c < qa.cols)
            qa.colsum[static_cast<uint64_t>(tr) * qa.cols + c0 + c] = (sums_lds[0][c] + sums_lds[1][c]) + (sums_lds[2][c] + sums_lds[3][c]);
    }
    if (qa.codes || qa.values) {
        const uint32_t at = c0 + 8 * (lane & 15u);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t r = 4 * i + (lane >> 4);
            Eight<T> v;
            v.clear();
            if (r < height && at < qa.cols) v.load(x + (r0 + r) * qa.ldx + at, qa.cols - at);
            quantize_eight<T>(qa, v, r0 + r, at, mx4_padded(qa.cols), r < height);
        }
    }
}

template <typename T>
static int launch(QuantArgs qa, hipStream_t st) {
    if (qa.codes_t || qa.colsum) {
        const uint32_t tiles_r = (qa.rows + kTile - 1) / kTile, tiles_c = (qa.cols + kTile - 1) / kTile;
        mx4_tiles_kernel<T><<<dim3(tiles_r * tiles_c + reorder_blocks(qa.also)), dim3(256), 0, st>>>(qa, tiles_r, tiles_c);
        return static_cast<int>(hipGetLastError());
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
