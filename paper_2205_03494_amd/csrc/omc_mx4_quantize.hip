// omc_mx4_quantize: a matrix in fp32 or bf16 to MX4 codes and scales, blocks along its rows, its columns, or both from one read.
//
// Bound by memory: 2 or 4 bytes read and 17/32 written a value and direction, some ten instructions a value between them.
//
// Along rows alone a lane takes eight neighbours, 16 or 32 bytes and one dword of codes, and the four lanes of a block compare their largest magnitudes.
// Along columns a wave takes 32 rows x 128 columns, a lane two columns of them, so that a lane holds two whole blocks and no lane needs another's
// values; the codes of a workgroup's 256 rows go through LDS, so that 128 bytes of a column are written together.  Where both directions are asked for, 16 lanes compare
// their largest magnitudes of a row, from the same registers.
// 8192 x 4096 from memory: along rows 28 us in fp32 (5.4 TB/s), 18.5 in bf16 (4.6); along columns 32 and 21; both 37 and 30 (3.4 TB/s; memory sees every byte once, although codes of 64
// and scales of 2 bytes a row and tile are parts of cache lines; waves wait 42 % of their time, and an LDS instruction has four clocks of bank conflicts; tiles of 128 x 256 take as long).  16384 x 8192 in bf16 along rows, with the rounded values: 100 us, 6.1 TB/s.
#include <type_traits>

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
template <uint32_t ROWS>
__device__ __forceinline__ void reorder_scales(const Mx4Reorder &re, uint32_t block) {
    const uint32_t k128 = mx4_padded(re.cols) / 128, stages = (k128 + 1) / 2, groups = (re.rows + ROWS - 1) / ROWS;
    const uint32_t stage = block / groups, row = block % groups * ROWS + threadIdx.x;
    if (stage >= stages || row >= re.rows || threadIdx.x >= ROWS) return;
    const uint32_t *from = reinterpret_cast<const uint32_t *>(re.scales) + static_cast<uint64_t>(row) * k128 + 2 * stage;
    const uint32_t lower = from[0], upper = 2 * stage + 1 < k128 ? from[1] : 0u;
    uint32_t *to = reinterpret_cast<uint32_t *>(re.image + stage * mx4_image_pitch(re.rows)) + 2 * row;
    to[0] = (lower & 0xffffu) | upper << 16;
    to[1] = lower >> 16 | (upper & 0xffff0000u);
}
static uint32_t reorder_blocks(const Mx4Reorder &re, uint32_t rows) { return re.image ? (re.rows + rows - 1) / rows * ((mx4_padded(re.cols) + 255) / 256) : 0u; }

// 24576 rows of 8192 values: 8.8 us, as a launch of its own (omc_mx4_gemm); elsewhere it is part of a rounding's.
__global__ __launch_bounds__(256) void mx4_reorder_kernel(Mx4Reorder a, Mx4Reorder b, uint32_t blocks_a) {
    if (blockIdx.x < blocks_a) reorder_scales<256>(a, blockIdx.x);
    else reorder_scales<256>(b, blockIdx.x - blocks_a);
}
int launch_mx4_reorder(const Mx4Reorder &a, const Mx4Reorder &b, void *stream) {
    const uint32_t blocks_a = reorder_blocks(a, 256), blocks = blocks_a + reorder_blocks(b, 256);
    mx4_reorder_kernel<<<dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(a, b, blocks_a);
    return static_cast<int>(hipGetLastError());
}

// `first`: row of the launch's first item (a launch has less than 2^32 items).  The workgroups behind the items reorder the other matrix' scales.
template <typename T>
__global__ __launch_bounds__(256) void mx4_rows_kernel(QuantArgs qa, uint32_t first, uint32_t items) {
    if (qa.also.image && blockIdx.x >= (items + 255) / 256) {
        reorder_scales<256>(qa.also, blockIdx.x - (items + 255) / 256);
        return;
    }
    const uint32_t padded = mx4_padded(qa.cols), eights = padded / 8, item = blockIdx.x * 256 + threadIdx.x;
    const bool mine = item < items;            // (whole blocks: padded / 8 is a multiple of 16)
    const uint32_t row = first + item / eights, col = 8 * (item % eights);
    Eight<T> v;
    v.clear();
    if (mine && col < qa.cols) v.load(static_cast<const typename T::type *>(qa.x) + row * qa.ldx, col, qa.cols);
    quantize_eight<T>(qa, v, row, col, padded, mine);
}

constexpr uint32_t kWide = 128;                // columns of a tile; a wave takes 32 rows of it

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

// Largest magnitudes of 16 lanes' columns, two rows (halves) in each of 16 registers: lane l of the 16 gets those of rows 2 l and 2 l + 1.  Every exchange halves the registers: a lane keeps the
// half that its bit of the lane number names, and its partner, which has the same bits above that one, gets the other.
__device__ __forceinline__ uint32_t largest_of_16(uint32_t (&x)[16], uint32_t lane) {
    auto exchange = [&](auto count, auto control, uint32_t bit) {
        constexpr int N = decltype(count)::value;
        const bool upper = (lane & bit) != 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t keep = upper ? x[i + N] : x[i], give = upper ? x[i] : x[i + N];
            const uint32_t got = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(give), decltype(control)::value, 0xf, 0xf, true));
            x[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, keep), __builtin_bit_cast(u16x2, got)));
        }
    };
    typedef std::integral_constant<int, 0x140> Mirror16;     // lane ^ 15
    typedef std::integral_constant<int, 0x141> Mirror8;      // lane ^ 7
    typedef std::integral_constant<int, 0x1b> Mirror4;       // lane ^ 3
    typedef std::integral_constant<int, 0xb1> Mirror2;       // lane ^ 1
    exchange(std::integral_constant<int, 8>{}, Mirror16{}, 8u);
    exchange(std::integral_constant<int, 4>{}, Mirror8{}, 4u);
    exchange(std::integral_constant<int, 2>{}, Mirror4{}, 2u);
    exchange(std::integral_constant<int, 1>{}, Mirror2{}, 1u);
    return x[0];
}

template <int J>
__device__ __forceinline__ uint32_t of_lane(uint32_t x) {   // lane J's of the 16
    return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x150 + J, 0xf, 0xf, true));
}
template <int FROM, int TO, typename F>
__device__ __forceinline__ void for_each(F &&f) {
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>{});
        for_each<FROM + 1, TO>(f);
    }
}

// The same registers along the rows, of which 16 lanes hold a block.  A lane's codes, two columns of four rows a dword, go to codes[(row / 4) * 64 + lane], the scale of row i and block b to
// scales[i * 4 + b].  (Of fp32 values the upper halves do for the largest magnitude: its exponent is all that is asked for.)
template <typename T>
__device__ __forceinline__ void quantize_rows(const uint32_t (&lo)[32], const uint32_t (&hi)[32], uint32_t *codes, uint8_t *scales, uint32_t lane) {
    uint32_t tops[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        uint32_t x, y;                         // rows 2 i and 2 i + 1 of either column
        if constexpr (T::kBytes == 4) {
            x = __builtin_amdgcn_perm(lo[2 * i + 1], lo[2 * i], 0x07060302u);
            y = __builtin_amdgcn_perm(hi[2 * i + 1], hi[2 * i], 0x07060302u);
        } else {
            x = __builtin_amdgcn_perm(lo[2 * i + 1], lo[2 * i], 0x05040100u);
            y = __builtin_amdgcn_perm(lo[2 * i + 1], lo[2 * i], 0x07060302u);
        }
        tops[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x & 0x7fff7fffu), __builtin_bit_cast(u16x2, y & 0x7fff7fffu)));
    }
    const uint32_t mine = largest_of_16(tops, lane);
    const uint32_t first = mx4_scale<BF16>(mine & 0xffffu), second = mx4_scale<BF16>(mine >> 16);
    scales[8 * (lane & 15u) + (lane >> 4)] = static_cast<uint8_t>(first);
    scales[8 * (lane & 15u) + 4 + (lane >> 4)] = static_cast<uint8_t>(second);
    const uint32_t both = second << 23 | first;
    const bool any_nan = __any(first == kMx4NaN || second == kMx4NaN);
    for_each<0, 8>([&](auto four) {            // of four rows
        constexpr int G = decltype(four)::value;
        uint32_t c = 0;
        for_each<0, 4>([&](auto in) {
            constexpr int J = decltype(in)::value, I = 4 * G + J;
            const uint32_t scale = of_lane<I / 2>(both);
            const float unit = __uint_as_float(I % 2 == 0 ? scale << 23 : scale & 0xff800000u);
            if constexpr (T::kBytes == 4) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(lo[I]), __uint_as_float(hi[I]), unit, J);
            else c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, lo[I]), unit, J);
            if (any_nan && __float_as_uint(unit) == kMx4NaN << 23) c &= ~(0xffu << (8 * J));
        });
        codes[64 * G + lane] = c;
    });
}

// Several matrices' tiles in one launch, then another one's scales.
struct TileJobs {
    QuantArgs job[kMostJobs];
    uint32_t tiles_c[kMostJobs], end[kMostJobs];   // tiles across; the job's workgroups end here
    Mx4Reorder also;
};

// Tiles of HIGH x 128: blocks along the columns, along the rows, the columns' sums.
template <typename T, uint32_t HIGH>
__global__ __launch_bounds__(2 * HIGH) void mx4_tiles_kernel(TileJobs jobs) {
    typedef typename T::type E;
    static_assert(HIGH == 64 || HIGH == 256, "two blocks along a column, or all of a stage's");
    constexpr uint32_t kWaves = HIGH / 32, kPitch = HIGH / 2 + 16;   // bytes of a column's codes in LDS, with padding
    __shared__ __attribute__((aligned(16))) uint8_t codes_lds[kWide * kPitch];
    __shared__ __attribute__((aligned(16))) uint32_t rows_lds[kWaves][8 * 64];
    __shared__ __attribute__((aligned(16))) uint8_t scales_lds[kWide * kWaves];
    __shared__ __attribute__((aligned(16))) uint8_t row_scales_lds[kWaves][32 * 4];
    __shared__ float sums_lds[kWaves][kWide];
    uint32_t begin = 0, which = 0;
#pragma unroll
    for (uint32_t j = 0; j < kMostJobs; ++j)
        if (blockIdx.x >= jobs.end[j]) {
            begin = jobs.end[j];
            which = j + 1;
        }
    if (which == kMostJobs) {
        reorder_scales<(HIGH < 256 ? 128 : 256)>(jobs.also, blockIdx.x - begin);
        return;
    }
    const QuantArgs &qa = jobs.job[which];
    const uint32_t tiles_c = jobs.tiles_c[which], total = jobs.end[which] - begin, block = blockIdx.x - begin;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a run of the tiles to every die: 64 bytes of a row's codes are half a cache line, whose other half the next tile has (4096 x 4095 along columns 9.5 us, dealt out one by one 10.9)
    const uint32_t q = total / 8, rest = total % 8, die = block % 8, id = die * q + min(die, rest) + block / 8;
    const uint32_t tr = id / tiles_c, tc = id % tiles_c;
    const uint32_t r0 = tr * HIGH + 32 * wave, c0 = tc * kWide, col = c0 + 2 * lane;
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
            scales_lds[(2 * lane + c) * kWaves + (qa.images ? mx4_image_byte(wave) : wave)] = static_cast<uint8_t>(byte[c]);
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
        const uint32_t pitch = mx4_padded(qa.rows) / 2, from = tr * (HIGH / 2), there = from < pitch ? min(pitch - from, HIGH / 2) : 0u;   // bytes of a column, of those in this tile
#pragma unroll
        for (uint32_t p = threadIdx.x; p < kWaves * kWide; p += 2 * HIGH) {
            const uint32_t c = p / kWaves, at = 16 * (p % kWaves);
            if (c0 + c < qa.cols && at < there)
                *reinterpret_cast<u32x4 *>(qa.codes_t + static_cast<uint64_t>(c0 + c) * pitch + from + at) = *reinterpret_cast<const u32x4 *>(codes_lds + c * kPitch + at);
        }
        if constexpr (HIGH == 256) {
            const uint32_t c = threadIdx.x / 2, half = threadIdx.x % 2;
            if (threadIdx.x < 2 * kWide && c0 + c < qa.cols) {
                const uint32_t bytes = reinterpret_cast<const uint32_t *>(scales_lds)[threadIdx.x];
                if (qa.images) reinterpret_cast<uint32_t *>(qa.scales_t + tr * mx4_image_pitch(qa.cols))[2 * (c0 + c) + half] = bytes;
                else if (64 * half < there) reinterpret_cast<uint32_t *>(qa.scales_t + static_cast<uint64_t>(c0 + c) * (pitch / 16))[2 * tr + half] = bytes;
            }
        } else {
            const uint32_t c = threadIdx.x;
            if (c0 + c < qa.cols) {
                const uint16_t bytes = reinterpret_cast<const uint16_t *>(scales_lds)[c];
                if (qa.images) reinterpret_cast<uint16_t *>(qa.scales_t + (tr / 4) * mx4_image_pitch(qa.cols) + 8ull * (c0 + c))[mx4_image_byte(2 * (tr % 4)) / 2] = bytes;
                else if (there > 0) reinterpret_cast<uint16_t *>(qa.scales_t + static_cast<uint64_t>(c0 + c) * (pitch / 16))[tr] = bytes;
            }
        }
    }
    if (qa.codes) {                            // 64 bytes of a row (all of them: rows are padded to 128 values)
        const uint32_t pitch = mx4_padded(qa.cols) / 2;
#pragma unroll
        for (uint32_t k = 0; k < 2; ++k) {
            const uint32_t group = 4 * k + (lane >> 4), at = 4 * (lane & 15u);   // four lanes' codes of four rows, to four rows' of eight columns
            const u32x4 d = *reinterpret_cast<const u32x4 *>(rows_lds[wave] + 64 * group + at);
            const uint32_t x0 = __builtin_amdgcn_perm(d[1], d[0], 0x05010400u), x1 = __builtin_amdgcn_perm(d[3], d[2], 0x05010400u);
            const uint32_t x2 = __builtin_amdgcn_perm(d[1], d[0], 0x07030602u), x3 = __builtin_amdgcn_perm(d[3], d[2], 0x07030602u);
            const uint32_t row[4] = {__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x05040100u),
                                     __builtin_amdgcn_perm(x3, x2, 0x07060302u)};
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                if (4 * group + j < height) *reinterpret_cast<uint32_t *>(qa.codes + static_cast<uint64_t>(r0 + 4 * group + j) * pitch + 64 * tc + at) = row[j];
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
        // of two waves, then of such pairs in order: here all of a tile's 256 rows, or a row of the four that column_sums adds the same way
        const uint32_t c = threadIdx.x;
        if (c < kWide && c0 + c < qa.cols) {
            float s = sums_lds[0][c] + sums_lds[1][c];
#pragma unroll
            for (uint32_t w = 2; w < kWaves; w += 2) s += sums_lds[w][c] + sums_lds[w + 1][c];
            qa.colsum[static_cast<uint64_t>(tr) * qa.cols + c0 + c] = s;
        }
    }
}

// Fewer tiles of 256 rows than compute units: tiles of 64 (1000 x 777, both directions: 6.9 -> 5.5 us; 2048 x 2048 in fp32: 7.0 -> 6.4).  Of many these would store quarters of cache lines along the
// columns (512 x 16384: 8.7 us, 10.1 with them).
uint32_t mx4_tile_height(const QuantArgs *args, uint32_t count) {
    uint64_t tiles = 0;
    for (uint32_t j = 0; j < count; ++j) tiles += static_cast<uint64_t>((args[j].rows + 255) / 256) * ((args[j].cols + kWide - 1) / kWide);
    return tiles < 256 ? 64 : 256;
}
// Whole stages of 256 rows in either tile's height, so that an image is written whole.
template <typename T, uint32_t HIGH>
static int launch_tiles_of(const QuantArgs *args, uint32_t count, const Mx4Reorder &also, hipStream_t st) {
    TileJobs jobs{};
    uint32_t end = 0;
    for (uint32_t j = 0; j < kMostJobs; ++j) {
        if (j < count) {
            jobs.job[j] = args[j];
            jobs.tiles_c[j] = (args[j].cols + kWide - 1) / kWide;
            end += (args[j].rows + 255) / 256 * (256 / HIGH) * jobs.tiles_c[j];
        }
        jobs.end[j] = end;
    }
    jobs.also = also;
    mx4_tiles_kernel<T, HIGH><<<dim3(end + reorder_blocks(also, HIGH < 256 ? 128 : 256)), dim3(2 * HIGH), 0, st>>>(jobs);
    return static_cast<int>(hipGetLastError());
}
template <typename T>
static int launch_tiles(const QuantArgs *args, uint32_t count, const Mx4Reorder &also, hipStream_t st) {
    return mx4_tile_height(args, count) == 64 ? launch_tiles_of<T, 64>(args, count, also, st) : launch_tiles_of<T, 256>(args, count, also, st);
}
int launch_mx4_tiles(const QuantArgs *args, uint32_t count, const Mx4Reorder &also, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch_tiles<BF16>(args, count, also, st) : launch_tiles<F32>(args, count, also, st);
}

template <typename T>
static int launch(QuantArgs qa, hipStream_t st) {
    if (qa.codes_t) {
        QuantArgs ta = qa;
        if (qa.values) ta.codes = ta.scales = nullptr;   // these along the rows, with the values
        const int rc = launch_tiles<T>(&ta, 1, Mx4Reorder{}, st);
        if (rc != 0 || !qa.values) return rc;
    }
    const uint32_t eights = mx4_padded(qa.cols) / 8, most = (1u << 30) / eights;   // rows of one launch
    for (uint32_t first = 0; first < qa.rows; first += most) {
        const uint32_t items = (qa.rows - first < most ? qa.rows - first : most) * eights;
        mx4_rows_kernel<T><<<dim3((items + 255) / 256 + reorder_blocks(qa.also, 256)), dim3(256), 0, st>>>(qa, first, items);
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
