// Device side of what a product's sums become: scales, bias, the gate with its slopes, and rounding.
#pragma once
#include "omc_mx4.h"
#include "omc_product.h"

namespace omc {

// act(g), and act'(g) from what that left:
//   sigmoid  s = 1 / (1 + exp(-g)),          s (1 - s)
//   swish    g s,                            s (1 + g (1 - s))
//   gelu     g P, P = erfc(-g / sqrt 2) / 2, P + g exp(-g^2 / 2) / sqrt(2 pi)
// With the hardware's exp2 and reciprocal, an error of 2^-23 each: while a wave finishes results it multiplies nothing (8192 x 4096 x 1024 in 8 bits, swish: 155 us with the library's expf and divisions and every column's scale
// and bias fetched for every value, 102 so and with these in LDS, 84 with a kind's arithmetic in a branch of its own; 70 - 73 now that one wave multiplies while another finishes).  The exponent's rounding counts |x| 2^-24 of exp(x), which is worth 0.3 * 2^-24 of s and 0.4 * 2^-24 of P at most.
// P's tail, exp(-g^2 / 2) q(t) with t = 1 / (1 + 0.295 |g|) and q of degree 8, was fitted here to erfc by least squares, reweighted until the errors were even, 4.4e-7 of itself.  In fp32, measured: P is within 2.2e-7 in all; the tail
// within 7e-7 of itself up to |g| = 3, and farther out by what the exponent's two roundings are worth, g^2 2^-24: 1.8e-6 at 5, 5e-6 at 10, 8.4e-6 at 13.  s for g < 0 likewise, by |g| 2^-24: 3.4e-7 up to 5, 9e-7 at 12, 3.9e-6 at 80.
struct Gate {
    float value, part, rest;
};
template <int KIND>
__device__ __forceinline__ Gate gate_of(float g) {
    constexpr float kLog2e = 1.44269504088896340736f;
    if constexpr (KIND == OMC_GATE_GELU) {
        const float e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * g * g), t = __builtin_amdgcn_rcpf(fmaf(0.295f, fabsf(g), 1.0f));
        float q = 0.0363113738f;
        q = fmaf(q, t, -0.168342339f);
        q = fmaf(q, t, 0.240175284f);
        q = fmaf(q, t, -0.0823553353f);
        q = fmaf(q, t, 0.142894139f);
        q = fmaf(q, t, 0.0943672353f);
        q = fmaf(q, t, 0.119349668f);
        q = fmaf(q, t, 0.117599973f);
        const float tail = q * t * e, p = g < 0.0f ? tail : 1.0f - tail;
        return {g * p, p, e};
    } else {
        const float e = __builtin_amdgcn_exp2f(-kLog2e * g), s = __builtin_amdgcn_rcpf(1.0f + e);
        return {KIND == OMC_GATE_SIGMOID ? s : g * s, s, e};
    }
}
template <int KIND>
__device__ __forceinline__ float slope_of(float g, const Gate &gate) {
    if constexpr (KIND == OMC_GATE_GELU) {
        return fmaf(g * 0.39894228040143268f, gate.rest, gate.part);
    } else {
        const float rest = gate.rest > 0x1p100f ? 1.0f : gate.rest * gate.part;   // 1 - s without its cancellation
        return KIND == OMC_GATE_SIGMOID ? gate.part * rest : fmaf(gate.value, rest, gate.part);
    }
}

// A lane's four neighbours of a row of C, from their sums, scales and biases (those of absent ones are 0).
struct Four {
    float v[4];
};
struct Columns {                               // of four columns, of either matrix
    f32x4 scale, scale2, bias, bias2;
};
__device__ __forceinline__ float sum_value(float sum, float, float, float bias) { return sum + bias; }
__device__ __forceinline__ float sum_value(int sum, float row_scale, float scale, float bias) { return fmaf(static_cast<float>(sum) * row_scale, scale, bias); }
template <typename V>
__device__ __forceinline__ Four finish_plain(const V &sum, float row_scale, const Columns &c) {
    Four r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r.v[e] = sum_value(sum[e], row_scale, c.scale[e], c.bias[e]);
    return r;
}
// KEEP: with the slopes of the result
template <int KIND, bool KEEP, typename V>
__device__ __forceinline__ Four finish_gated(const V &first, const V &second, float row_scale, const Columns &c, Four &slope_g, Four &slope_u) {
    Four r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float g = sum_value(first[e], row_scale, c.scale[e], c.bias[e]), u = sum_value(second[e], row_scale, c.scale2[e], c.bias2[e]);
        const Gate gate = gate_of<KIND>(g);
        r.v[e] = gate.value * u;
        if constexpr (KEEP) {
            slope_g.v[e] = u * slope_of<KIND>(g, gate);
            slope_u.v[e] = gate.value;
        }
    }
    return r;
}
template <int V>
struct IntTag {
    static constexpr int value = V;
};
// f(IntTag<kind>)
template <typename F>
__device__ __forceinline__ void for_gate(int kind, F &&f) {
    if (kind == OMC_GATE_SWISH) f(IntTag<OMC_GATE_SWISH>{});
    else if (kind == OMC_GATE_SIGMOID) f(IntTag<OMC_GATE_SIGMOID>{});
    else f(IntTag<OMC_GATE_GELU>{});
}
// A gated result's run of a row, and its slopes' if f keeps them, from row m and column n on.
template <typename T, typename V>
__device__ __forceinline__ void store_gated(const Finish &f, const V &first, const V &second, float row_scale, const Columns &c, typename T::type *to, uint32_t m, uint32_t n, uint32_t left) {
    for_gate(f.gate, [&](auto kind) {
        Four sg, su;
        store_run<T, 4>(to, finish_gated<decltype(kind)::value, true>(first, second, row_scale, c, sg, su).v, left);
        if (f.slope_g) {
            store_run<BF16, 4>(f.slope_g + m * f.ld_slope + n, sg.v, left);
            store_run<BF16, 4>(f.slope_u + m * f.ld_slope + n, su.v, left);
        }
    });
}

// Columns n .. n + 3 from memory; those past the end are the last one's.
template <bool I8, bool GATED>
__device__ __forceinline__ Columns columns_from(const Finish &f, uint32_t n, uint32_t N) {
    Columns c;
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    auto from = [&](const float *p) {
        f32x4 v = zero;
        if (n + 4 <= N) {
            __builtin_memcpy(&v, p + n, 16);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) v[e] = p[min(n + e, N - 1)];
        }
        return v;
    };
    c.scale = I8 ? from(f.scale) : zero;
    c.scale2 = I8 && GATED ? from(f.scale2) : zero;
    c.bias = f.bias ? from(f.bias) : zero;
    c.bias2 = GATED && f.bias2 ? from(f.bias2) : zero;
    return c;
}

// Row m of C; null for one that is nowhere.
template <typename T>
__device__ __forceinline__ typename T::type *row_of(const Finish &f, uint32_t m) {
    if (m < f.rows) return static_cast<typename T::type *>(f.c) + m * f.ldc;
    return f.c2 && m >= f.second && m - f.second < f.rows ? static_cast<typename T::type *>(f.c2) + (m - f.second) * f.ldc : nullptr;
}

}  // namespace omc
