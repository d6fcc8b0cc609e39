// Device side of MX4: 32 neighbours share a power of two and hold an E2M1 value each.
//
//   a = max |x_i|,  e = max(floor(log2 a) - 2, -127),  code_i = E2M1(x_i 2^-e), nearest, ties to even, saturating at 6;
// the scale is the byte e + 127.  floor(log2 a) is the exponent field of a, so the byte is max(field - 2, 0), and the largest value
// of a block lies in [4, 8) units.  A block with a value that is not finite gets byte 255, which the matrix cores read as NaN, and codes 0.
// The conversions are the hardware's; they take the scale as a float of which only the exponent field counts, so that byte << 23 serves for all
// bytes, 2^-127 among them.
#pragma once
#include <hip/hip_runtime.h>

#include "omc_layer.h"

namespace omc {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kMx4NaN = 255;

// Magnitudes are compared as integers: above all finite ones come infinity and the NaNs.
struct F32 {
    typedef float type;
    static constexpr uint32_t kBytes = 4, kFinite = 0x7f7fffffu, kField = 23;
};
struct BF16 {
    typedef uint16_t type;
    static constexpr uint32_t kBytes = 2, kFinite = 0x7f7fu, kField = 7;
};
__device__ __forceinline__ float load_f32(const float *p) { return *p; }
__device__ __forceinline__ float load_f32(const uint16_t *p) { return __builtin_bit_cast(float, static_cast<uint32_t>(*p) << 16); }
__device__ __forceinline__ float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_bf16_pair(float a, float b) {   // nearest, ties to even
    const bf16x2 t = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, t);
}
__device__ __forceinline__ uint16_t to_bf16(float a) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(a)); }

// Eight neighbours of a row, as they lie in memory.  Rows begin at any element; the hardware takes 16 bytes from any address.
template <typename T>
struct Eight {
    uint32_t w[2 * T::kBytes];
    // fetch and then settle: a row's values from col on, and zeros past its end.  There the row's last eight are fetched and moved down, so that all lanes load alike, whole vectors, and
    // nothing waits between the loads of several pieces.  SHORT: rows may have fewer than eight.
    template <bool SHORT>
    __device__ __forceinline__ void fetch(const typename T::type *row, uint32_t col, uint32_t cols) {
        if (SHORT && cols < 8) {
            clear();
#pragma unroll 1                               // (unrolled, its loads would be merged with the others', and these be cut into elements)
            for (uint32_t i = 0; i < cols; ++i) {   // from above
#pragma unroll
                for (uint32_t k = 0; k + 1 < 2 * T::kBytes; ++k) w[k] = T::kBytes == 4 ? w[k + 1] : w[k + 1] << 16 | w[k] >> 16;
                if constexpr (T::kBytes == 4) w[7] = __float_as_uint(row[i]);
                else w[3] = static_cast<uint32_t>(row[i]) << 16 | w[3] >> 16;
            }
        } else {
            __builtin_memcpy(w, row + min(col, cols - 8), 8 * T::kBytes);
        }
    }
    static __device__ __forceinline__ uint32_t missing(uint32_t col, uint32_t cols) { return col + 8 <= cols ? 0u : min(8u, col + 8 - cols); }
    __device__ __forceinline__ void settle(uint32_t missing) {
        if (missing == 0) return;
        constexpr uint32_t kWords = 2 * T::kBytes;
        if constexpr (T::kBytes == 2) {
            const uint32_t by = missing & 1u ? 16u : 0u;
#pragma unroll
            for (uint32_t i = 0; i < kWords; ++i) w[i] = __builtin_amdgcn_alignbit(i + 1 < kWords ? w[i + 1] : 0u, w[i], by);
        }
#pragma unroll
        for (uint32_t by = 1; by <= kWords; by *= 2) {
            const bool move = missing & (by * 4 / T::kBytes);
#pragma unroll
            for (uint32_t i = 0; i < kWords; ++i) w[i] = move ? (i + by < kWords ? w[i + by] : 0u) : w[i];
        }
    }
    template <bool SHORT = true>
    __device__ __forceinline__ void load(const typename T::type *row, uint32_t col, uint32_t cols) {
        fetch<SHORT>(row, col, cols);
        settle(missing(col, cols));
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (uint32_t i = 0; i < 2 * T::kBytes; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float value(int i) const {
        if constexpr (T::kBytes == 4) return __builtin_bit_cast(float, w[i]);
        else return i & 1 ? bf16_high(w[i / 2]) : bf16_low(w[i / 2]);
    }
    // largest magnitude's bits
    __device__ __forceinline__ uint32_t top() const {
        if constexpr (T::kBytes == 4) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
            return m;
        } else {
            u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
            for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
            return max(static_cast<uint32_t>(m[0]), static_cast<uint32_t>(m[1]));
        }
    }
    __device__ __forceinline__ uint32_t codes(float scale) const {
        uint32_t c = 0;
        if constexpr (T::kBytes == 4) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value(0), value(1), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value(2), value(3), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value(4), value(5), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, value(6), value(7), scale, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
        }
        return c;
    }
};

// Scale byte of a block whose largest magnitude has these bits.
template <typename T>
__device__ __forceinline__ uint32_t mx4_scale(uint32_t top) {
    const uint32_t field = top >> T::kField;
    return top > T::kFinite ? kMx4NaN : field > 2 ? field - 2 : 0u;
}
__device__ __forceinline__ float mx4_unit(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// A lane's block of an operand, 32 codes.
__device__ __forceinline__ i32x8 mx4_operand(i32x4 x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

// acc += a b^T over 128 values: lane l holds of either operand row l % 16, block l / 16, its scale in byte BYTE_A or BYTE_B of a register.  The result's value v of
// lane l is row 4 (l / 16) + v of a, row l % 16 of b.
constexpr int kE2M1 = 4;                       // the operands' type, as the instructions name it
template <int BYTE_A, int BYTE_B>
__device__ __forceinline__ f32x4 mx4_multiply(i32x4 a, uint32_t scale_a, i32x4 b, uint32_t scale_b, f32x4 acc) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(a), mx4_operand(b), acc, kE2M1, kE2M1, BYTE_A, static_cast<int>(scale_a), BYTE_B,
                                                            static_cast<int>(scale_b));
}
// The same over 64 values and 32 x 32 results: row l % 32, block l / 32; value v is row 8 (v / 4) + 4 (l / 32) + v % 4 of a, row l % 32 of b.
template <int BYTE>
__device__ __forceinline__ f32x16 mx4_multiply_32(i32x4 a, uint32_t scale_a, i32x4 b, uint32_t scale_b, f32x16 acc) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(a), mx4_operand(b), acc, kE2M1, kE2M1, BYTE, static_cast<int>(scale_a), BYTE,
                                                           static_cast<int>(scale_b));
}

// COUNT neighbours of a result's row, in fp32 or bf16: `left` of them lie inside.
template <typename T, int COUNT>
__device__ __forceinline__ void store_run(typename T::type *to, const float (&v)[COUNT], uint32_t left) {
    if (left >= COUNT) {
        if constexpr (T::kBytes == 4) {
            __builtin_memcpy(to, v, 4 * COUNT);
        } else {
            uint32_t w[COUNT / 2];
#pragma unroll
            for (int i = 0; i < COUNT / 2; ++i) w[i] = to_bf16_pair(v[2 * i], v[2 * i + 1]);
            __builtin_memcpy(to, w, 2 * COUNT);
        }
    } else {
#pragma unroll
        for (uint32_t i = 0; i < COUNT; ++i)
            if (i < left) {
                if constexpr (T::kBytes == 4) to[i] = v[i];
                else to[i] = to_bf16(v[i]);
            }
    }
}

}  // namespace omc
