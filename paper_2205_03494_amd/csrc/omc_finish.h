// Device side of what a product's sums become: scales, bias, the gate with its slopes, and rounding.
#pragma once
#include "omc_mx4.h"
#include "omc_product.h"

namespace omc {

// act(g) and act'(g):
//   sigmoid  s = 1 / (1 + exp(-g)),       s (1 - s)
//   swish    g s,                         s (1 + g (1 - s))
//   gelu     g P, P = erfc(-g / sqrt 2) / 2,   P + g exp(-g^2 / 2) / sqrt(2 pi)
struct Gate {
    float value, slope;
};
__device__ __forceinline__ Gate gate_of(int kind, float g) {
    if (kind == OMC_GATE_GELU) {
        const float p = 0.5f * erfcf(-0.70710678118654752f * g);
        return {g * p, p + g * (0.39894228040143268f * expf(-0.5f * g * g))};
    }
    const float e = expf(-g), s = 1.0f / (1.0f + e);
    const float rest = e < __builtin_inff() ? e * s : 1.0f;          // 1 - s without its cancellation
    return kind == OMC_GATE_SIGMOID ? Gate{s, s * rest} : Gate{g * s, s * (1.0f + g * rest)};
}

__device__ __forceinline__ float sum_value(float sum, float, float) { return sum; }
__device__ __forceinline__ float sum_value(int sum, float row_scale, float scale) { return static_cast<float>(sum) * row_scale * scale; }

// A lane's four neighbours of a row of C, n .. n + 3, from their sums.  `left`: how many of them lie inside (4 or more: all).
struct Four {
    float v[4];
};
template <typename V>
__device__ __forceinline__ Four finish_plain(const Finish &f, const V &sum, float row_scale, uint32_t n, uint32_t left) {
    Four r;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t at = n + (e < left ? e : 0);
        r.v[e] = sum_value(sum[e], row_scale, f.scale ? f.scale[at] : 1.0f);
        if (f.bias) r.v[e] += f.bias[at];
    }
    return r;
}
template <typename V>
__device__ __forceinline__ Four finish_gated(const Finish &f, const V &first, const V &second, float row_scale, uint32_t n, uint32_t left, Four &slope_g, Four &slope_u) {
    Four r;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t at = n + (e < left ? e : 0);
        float g = sum_value(first[e], row_scale, f.scale ? f.scale[at] : 1.0f), u = sum_value(second[e], row_scale, f.scale2 ? f.scale2[at] : 1.0f);
        if (f.bias) g += f.bias[at];
        if (f.bias2) u += f.bias2[at];
        const Gate gate = gate_of(f.gate, g);
        r.v[e] = gate.value * u;
        slope_g.v[e] = u * gate.slope;
        slope_u.v[e] = gate.value;
    }
    return r;
}

// Row m of C; null for one that is nowhere.
template <typename T>
__device__ __forceinline__ typename T::type *row_of(const Finish &f, uint32_t m) {
    if (m < f.rows) return static_cast<typename T::type *>(f.c) + m * f.ldc;
    return f.c2 && m >= f.second && m - f.second < f.rows ? static_cast<typename T::type *>(f.c2) + (m - f.second) * f.ldc : nullptr;
}

}  // namespace omc
