// Entry points of the layer's operators: argument checks, the layout of workspaces, and which kernels a call takes.  No device code here.
#include <cmath>

#include "omc_layer.h"

namespace omc {

constexpr uint32_t kMostDim = 1u << 24;        // a tile's rows within 32-bit offsets
constexpr uint64_t kMostElems = 1ull << 37;    // a launch's work-items within 32 bits

static bool dims_ok(uint32_t a, uint32_t b) { return a >= 1 && b >= 1 && a <= kMostDim && b <= kMostDim && static_cast<uint64_t>(a) * b <= kMostElems; }
static bool type_ok(omc_type t) { return t == OMC_F32 || t == OMC_BF16; }
static bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool element_aligned(const void *p, omc_type t) { return aligned(p, t == OMC_BF16 ? 2 : 4); }
static bool mx4_aligned(const void *codes, const void *scales) { return aligned(codes, 16) && aligned(scales, 4); }
static omc_status from_hip(int rc) { return rc == 0 ? OMC_OK : OMC_ERR_DEVICE; }

// Parts of a workspace, one after the other, 256 bytes apart at least.
struct Parts {
    uint8_t *base;
    uint64_t used = 0;
    uint8_t *take(uint64_t bytes) {
        uint8_t *p = base + used;
        used += (bytes + 255) / 256 * 256;
        return p;
    }
};
static const uint8_t *bytes(const void *p) { return static_cast<const uint8_t *>(p); }

// A product's way: few rows of the first operand, or tiles, whose scales are reordered first.
static uint64_t parts_bytes(uint32_t M, uint32_t N, uint32_t K) { return mx4_few(M, N, K) ? 0 : mx4_gemm_workspace(M, N, K); }
static int launch_product(const Mx4GemmArgs &ga, bool bf16, void *stream) {
    return mx4_few(ga.M, ga.N, ga.K) ? launch_mx4_few(ga, nullptr, bf16, stream) : launch_mx4_gemm(ga, false, bf16, stream);
}

struct GemmLayout {
    uint8_t *a_image, *b_image;
    float *parts;
    uint64_t bytes;
};
static GemmLayout gemm_layout(uint8_t *ws, uint32_t M, uint32_t N, uint32_t K) {
    GemmLayout l{};
    if (mx4_few(M, N, K)) return l;
    Parts p{ws};
    l.a_image = p.take(mx4_image_bytes(M, K));
    l.b_image = p.take(mx4_image_bytes(N, K));
    l.parts = reinterpret_cast<float *>(p.take(parts_bytes(M, N, K)));
    l.bytes = p.used;
    return l;
}

struct LinearLayout {
    uint8_t *codes, *scales, *w_image;
    float *parts;
    uint64_t bytes;
};
static LinearLayout linear_layout(uint8_t *ws, uint32_t M, uint32_t N, uint32_t K) {
    LinearLayout l{};
    const bool few = mx4_few(M, N, K);
    if (few && mx4_few_rounds(M, K)) return l;
    Parts p{ws};
    l.codes = p.take(mx4_code_bytes(M, K));
    l.scales = p.take(few ? mx4_scale_bytes(M, K) : mx4_image_bytes(M, K));
    if (!few) l.w_image = p.take(mx4_image_bytes(N, K));
    l.parts = reinterpret_cast<float *>(p.take(parts_bytes(M, N, K)));
    l.bytes = p.used;
    return l;
}

// Either product may go in tiles or, if its first operand has few rows (dX's M, dW's K), the other way; the larger image has room for the scales in either order.
struct BackwardLayout {
    uint8_t *dy, *dy_scales, *dy_t, *dy_t_scales, *x_t, *x_t_scales, *w_image;
    float *sums, *parts;
    uint64_t bytes;
};
static BackwardLayout backward_layout(uint8_t *ws, uint32_t M, uint32_t N, uint32_t K) {
    BackwardLayout l{};
    Parts p{ws};
    l.dy = p.take(mx4_code_bytes(M, N));
    l.dy_scales = p.take(mx4_image_bytes(M, N));
    l.dy_t = p.take(mx4_code_bytes(N, M));
    l.dy_t_scales = p.take(mx4_image_bytes(N, M));
    l.x_t = p.take(mx4_code_bytes(K, M));
    l.x_t_scales = p.take(mx4_image_bytes(K, M));
    l.w_image = p.take(mx4_image_bytes(K, N));
    l.sums = reinterpret_cast<float *>(p.take(4ull * ((M + 255) / 256 * 4) * N));
    const uint64_t dx = parts_bytes(M, K, N), dw = parts_bytes(K, N, M);
    l.parts = reinterpret_cast<float *>(p.take(dx > dw ? dx : dw));
    l.bytes = p.used;
    return l;
}

}  // namespace omc

using namespace omc;

extern "C" {

size_t omc_mx4_code_bytes(uint32_t rows, uint32_t cols) { return dims_ok(rows, cols) ? mx4_code_bytes(rows, cols) : 0; }
size_t omc_mx4_scale_bytes(uint32_t rows, uint32_t cols) { return dims_ok(rows, cols) ? mx4_scale_bytes(rows, cols) : 0; }

omc_status omc_mx4_quantize(const void *x, omc_type type, uint32_t rows, uint32_t cols, uint64_t ldx, void *codes, void *scales, void *codes_t,
                            void *scales_t, void *values, uint64_t ldv, void *stream) {
    if (!x || !codes != !scales || !codes_t != !scales_t || (!codes && !codes_t && !values)) return OMC_ERR_NULL;
    if (!type_ok(type)) return OMC_ERR_FORMAT;
    if (!dims_ok(rows, cols) || ldx < cols || (values && ldv < cols)) return OMC_ERR_SIZE;
    if (!element_aligned(x, type) || !element_aligned(values, type) || !mx4_aligned(codes, scales) || !mx4_aligned(codes_t, scales_t)) return OMC_ERR_ALIGN;
    const QuantArgs qa{x, ldx, rows, cols, static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales), static_cast<uint8_t *>(codes_t),
                       static_cast<uint8_t *>(scales_t), values, ldv, nullptr, false, {}};
    return from_hip(launch_mx4_quantize(qa, type == OMC_BF16, stream));
}

size_t omc_mx4_gemm_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) {
    return dims_ok(M, N) && dims_ok(M, K) && dims_ok(N, K) ? gemm_layout(nullptr, M, N, K).bytes : 0;
}

omc_status omc_mx4_gemm(const void *a_codes, const void *a_scales, const void *b_codes, const void *b_scales, const float *bias, void *C,
                        omc_type c_type, uint64_t ldc, uint32_t M, uint32_t N, uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!a_codes || !a_scales || !b_codes || !b_scales || !C) return OMC_ERR_NULL;
    if (!type_ok(c_type)) return OMC_ERR_FORMAT;
    if (!dims_ok(M, N) || !dims_ok(M, K) || !dims_ok(N, K) || ldc < N) return OMC_ERR_SIZE;
    if (!mx4_aligned(a_codes, a_scales) || !mx4_aligned(b_codes, b_scales) || !aligned(bias, 4) || !element_aligned(C, c_type)) return OMC_ERR_ALIGN;
    const GemmLayout l = gemm_layout(static_cast<uint8_t *>(ws), M, N, K);
    if (l.bytes > 0 && (!ws || ws_bytes < l.bytes)) return OMC_ERR_WORKSPACE;
    if (l.bytes > 0 && !aligned(ws, 16)) return OMC_ERR_ALIGN;
    Mx4GemmArgs ga{{bytes(a_codes), bytes(a_scales)}, {bytes(b_codes), bytes(b_scales)}, bias, C, ldc, M, N, K, l.parts};
    int rc = 0;
    if (!mx4_few(M, N, K)) {
        rc = launch_mx4_reorder({ga.a.scales, l.a_image, M, K}, {ga.b.scales, l.b_image, N, K}, stream);
        ga.a.scales = l.a_image;
        ga.b.scales = l.b_image;
    }
    return from_hip(rc != 0 ? rc : launch_product(ga, c_type == OMC_BF16, stream));
}

size_t omc_mx4_linear_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) {
    return dims_ok(M, N) && dims_ok(M, K) && dims_ok(N, K) ? linear_layout(nullptr, M, N, K).bytes : 0;
}

omc_status omc_mx4_linear(const void *X, omc_type x_type, uint64_t ldx, const void *w_codes, const void *w_scales, const float *bias, void *Y,
                          omc_type y_type, uint64_t ldy, uint32_t M, uint32_t N, uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!X || !w_codes || !w_scales || !Y) return OMC_ERR_NULL;
    if (!type_ok(x_type) || !type_ok(y_type)) return OMC_ERR_FORMAT;
    if (!dims_ok(M, N) || !dims_ok(M, K) || !dims_ok(N, K) || ldx < K || ldy < N) return OMC_ERR_SIZE;
    if (!element_aligned(X, x_type) || !element_aligned(Y, y_type) || !mx4_aligned(w_codes, w_scales) || !aligned(bias, 4)) return OMC_ERR_ALIGN;
    const LinearLayout l = linear_layout(static_cast<uint8_t *>(ws), M, N, K);
    if (l.bytes > 0 && (!ws || ws_bytes < l.bytes)) return OMC_ERR_WORKSPACE;
    if (l.bytes > 0 && !aligned(ws, 16)) return OMC_ERR_ALIGN;
    const bool x_bf16 = x_type == OMC_BF16, y_bf16 = y_type == OMC_BF16, few = mx4_few(M, N, K);
    const Mx4 w{bytes(w_codes), few ? bytes(w_scales) : l.w_image};
    const Mx4GemmArgs ga{{l.codes, l.scales}, w, bias, Y, ldy, M, N, K, l.parts};
    if (!l.codes) {
        const Mx4Rows rows{X, ldx, x_bf16};
        return from_hip(launch_mx4_few(ga, &rows, y_bf16, stream));
    }
    const QuantArgs qa{X, ldx, M, K, l.codes, l.scales, nullptr, nullptr, nullptr, 0, nullptr, !few, {bytes(w_scales), l.w_image, N, K}};
    const int rc = launch_mx4_quantize(qa, x_bf16, stream);
    return from_hip(rc != 0 ? rc : launch_product(ga, y_bf16, stream));
}

size_t omc_mx4_linear_backward_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) {
    return dims_ok(M, N) && dims_ok(M, K) && dims_ok(N, K) ? backward_layout(nullptr, M, N, K).bytes : 0;
}

omc_status omc_mx4_linear_backward(const void *dY, uint64_t lddy, const void *X, uint64_t ldx, omc_type type, const void *w_codes,
                                   const void *w_scales, void *dX, omc_type dx_type, uint64_t lddx, float *dW, float *dbias, uint32_t M,
                                   uint32_t N, uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!dY || (!dX && !dW && !dbias) || (dX && (!w_codes || !w_scales)) || (dW && !X)) return OMC_ERR_NULL;
    if (!type_ok(type) || (dX && !type_ok(dx_type))) return OMC_ERR_FORMAT;
    if (!dims_ok(M, N) || !dims_ok(M, K) || !dims_ok(N, K) || lddy < N || (dW && ldx < K) || (dX && lddx < K)) return OMC_ERR_SIZE;
    if (!element_aligned(dY, type) || !aligned(dW, 4) || !aligned(dbias, 4) || (dW && !element_aligned(X, type)) ||
        (dX && (!element_aligned(dX, dx_type) || !mx4_aligned(w_codes, w_scales))))
        return OMC_ERR_ALIGN;
    const BackwardLayout l = backward_layout(static_cast<uint8_t *>(ws), M, N, K);
    if (!ws || ws_bytes < l.bytes) return OMC_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return OMC_ERR_ALIGN;
    const bool bf16 = type == OMC_BF16;

    // all roundings in one launch; dY's in one pass, unless its two products want their scales in different orders
    const bool whole = mx4_backward_whole(M, N, K), dx_tiles = whole || !mx4_few(M, K, N), dw_tiles = whole || !mx4_few(K, N, M);
    const int together = whole && dX && dW ? mx4_pair_tile(M, N, K, dbias != nullptr) : -1;
    const Mx4Reorder weights = dX && dx_tiles ? Mx4Reorder{bytes(w_scales), l.w_image, K, N} : Mx4Reorder{};
    QuantArgs jobs[kMostJobs];
    uint32_t count = 1;
    jobs[0] = QuantArgs{dY, lddy, M, N, nullptr, nullptr, nullptr, nullptr, nullptr, 0, dbias ? l.sums : nullptr, dx_tiles, {}};
    if (dX) {
        jobs[0].codes = l.dy;
        jobs[0].scales = l.dy_scales;
    }
    if (dW) {
        QuantArgs &along_columns = !dX || dx_tiles == dw_tiles ? jobs[0] : jobs[count++];
        if (&along_columns != jobs) along_columns = QuantArgs{dY, lddy, M, N, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr, dw_tiles, {}};
        along_columns.codes_t = l.dy_t;
        along_columns.scales_t = l.dy_t_scales;
        along_columns.images = dw_tiles;
        jobs[count++] = QuantArgs{X, ldx, M, K, nullptr, nullptr, l.x_t, l.x_t_scales, nullptr, 0, nullptr, dw_tiles, {}};
    }
    int rc;
    if (!dW && !dbias) {
        jobs[0].also = weights;
        rc = launch_mx4_quantize(jobs[0], bf16, stream);
    } else {
        rc = launch_mx4_tiles(jobs, count, weights, bf16, stream);
    }
    if (rc != 0) return from_hip(rc);
    const uint32_t sum_rows = (M + 255) / 256;
    const bool fours = mx4_tile_height(jobs, count) == 64;
    const Mx4GemmArgs for_dx{{l.dy, l.dy_scales}, {bytes(w_codes), dx_tiles ? l.w_image : bytes(w_scales)}, nullptr, dX, lddx, M, K, N, l.parts};
    const Mx4GemmArgs for_dw{{l.x_t, l.x_t_scales}, {l.dy_t, l.dy_t_scales}, nullptr, dW, N, K, N, M, l.parts};
    if (together >= 0) return from_hip(launch_mx4_pair(together, for_dx, dx_type == OMC_BF16, for_dw, l.sums, sum_rows, fours, dbias, stream));
    if (dbias) rc = launch_column_sums(l.sums, sum_rows, fours, N, N, dbias, nullptr, stream);
    if (rc == 0 && dX) rc = whole ? launch_mx4_gemm(for_dx, true, dx_type == OMC_BF16, stream) : launch_product(for_dx, dx_type == OMC_BF16, stream);
    if (rc == 0 && dW) rc = whole ? launch_mx4_gemm(for_dw, true, false, stream) : launch_product(for_dw, false, stream);
    return from_hip(rc);
}

omc_status omc_layer_norm(const void *x, omc_type x_type, uint64_t ldx, const float *gamma, const float *beta, float eps, void *y,
                          omc_type y_type, uint64_t ldy, float *mean, float *rstd, uint32_t rows, uint32_t cols, void *stream) {
    if (!x || !y) return OMC_ERR_NULL;
    if (!type_ok(x_type) || !type_ok(y_type)) return OMC_ERR_FORMAT;
    if (!dims_ok(rows, cols) || ldx < cols || ldy < cols) return OMC_ERR_SIZE;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return OMC_ERR_OPT;
    if (!element_aligned(x, x_type) || !element_aligned(y, y_type) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return OMC_ERR_ALIGN;
    const NormArgs na{x, ldx, gamma, beta, eps, y, ldy, mean, rstd, rows, cols};
    return from_hip(launch_layer_norm(na, x_type == OMC_BF16, y_type == OMC_BF16, stream));
}

size_t omc_layer_norm_backward_workspace_bytes(uint32_t rows, uint32_t cols) { return dims_ok(rows, cols) ? layer_norm_backward_workspace(rows, cols) : 0; }

omc_status omc_layer_norm_backward(const void *dy, omc_type dy_type, uint64_t lddy, const void *x, omc_type x_type, uint64_t ldx,
                                   const float *gamma, const float *mean, const float *rstd, void *dx, uint64_t lddx, float *dgamma,
                                   float *dbeta, uint32_t rows, uint32_t cols, void *ws, size_t ws_bytes, void *stream) {
    if (!dy || !x || !mean || !rstd || (!dx && !dgamma && !dbeta)) return OMC_ERR_NULL;
    if (!type_ok(x_type) || !type_ok(dy_type)) return OMC_ERR_FORMAT;
    if (!dims_ok(rows, cols) || lddy < cols || ldx < cols || (dx && lddx < cols)) return OMC_ERR_SIZE;
    if (!element_aligned(dy, dy_type) || !element_aligned(x, x_type) || !element_aligned(dx, x_type) || !aligned(gamma, 4) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
        return OMC_ERR_ALIGN;
    if (!ws || ws_bytes < layer_norm_backward_workspace(rows, cols)) return OMC_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return OMC_ERR_ALIGN;
    const NormGradArgs na{dy, lddy, x, ldx, gamma, mean, rstd, dx, lddx, dgamma, dbeta, rows, cols, static_cast<float *>(ws)};
    return from_hip(launch_layer_norm_backward(na, x_type == OMC_BF16, dy_type == OMC_BF16, stream));
}

}  // extern "C"
