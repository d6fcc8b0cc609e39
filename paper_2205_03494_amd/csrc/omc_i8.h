// Device side of I8: a row of values shares a scale and holds a whole number each.
//
//   a = max |x_i|,  s = a * (1 / 127), both rounded to fp32,  code_i = the whole number nearest to x_i / s, ties to even.
// (The product and not the quotient a / 127, which is a last place away for one fp32 row in twenty and for 6 of bf16's 128 significands.  That place decides a value halfway between two codes by its row's scale, as a / 2 is in
// bf16, so the format has to name one of them.)
// The quotient is never formed exactly: r = rint(x * (1 / s)) is off by at most one, and d = x - r s, which fp32 holds exactly (r = 0: x itself; r = 1: both are within a factor of two; otherwise x > s, and d is a
// multiple of s' last place below s / 2 and a little), says whether the neighbour is nearer.  That is asked where x * (1 / s) comes within 2^-12 of halfway between two whole numbers (it is off by 2^-15 at most).  Scales below 2^-100 are handled times 2^100, which is exact.
#pragma once
#include "omc_mx4.h"

namespace omc {

struct Rounding {
    float scale, up, s, inverse;
    __device__ __forceinline__ void of(float top, bool is_nan) { with(is_nan ? __builtin_nanf("") : top * (1.0f / 127.0f)); }
    __device__ __forceinline__ void with(float its_scale) {
        scale = its_scale;
        up = scale < 0x1p-100f ? 0x1p100f : 1.0f;
        const bool some = scale > 0.0f;                              // (a NaN is not)
        s = some ? scale * up : 1.0f;
        inverse = some ? 1.0f / s : 0.0f;                            // 0: all codes are 0
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
    // The same where x / s is not about halfway between two whole numbers, which `far` says (the largest distance so far): adding 1.5 * 2^23 rounds, ties to even.
    __device__ __forceinline__ float near(float x, float &far) const {
        constexpr float kWhole = 12582912.0f;
        const float f = x * inverse, r = (f + kWhole) - kWhole;
        far = fmaxf(far, fabsf(f - r));
        return r;
    }
    static constexpr float kFar = 0.499755859375f;                   // 1/2 - 2^-12
    __device__ __forceinline__ bool special() const { return up != 1.0f || inverse == 0.0f; }
    // Of eight values, where lanes seldom need code().
    __device__ __forceinline__ void eight(const float (&x)[8], float (&r)[8]) const {
        float far = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = near(x[i], far);
        if (far > kFar || special()) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = code(x[i]);
        }
    }
    __device__ __forceinline__ float value(float r) const { return r * scale; }
};
__device__ __forceinline__ uint32_t four_bytes(const float *r) {   // of whole numbers
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(r[i] + 12582912.0f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
}
template <typename T>
__device__ __forceinline__ float from_top(uint32_t top) {
    return __uint_as_float(T::kBytes == 4 ? top : top << 16);
}

}  // namespace omc
