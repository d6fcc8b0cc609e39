// Entry points of the products on 8-bit integers and of the gated linear layer: argument checks, the layout of workspaces, and which kernels a call takes.  No device code here.
#include "omc_product.h"

namespace omc {

constexpr uint32_t kMostDim = 1u << 24;        // rows of a matrix
constexpr uint64_t kMostElems = 1ull << 37;    // a launch's work-items within 32 bits
constexpr uint32_t kMostI8 = 131071;           // values of a contraction whose sum of products of two codes fits 32 bits
constexpr uint32_t kMostGated = 1u << 22;      // a tile's rows within 32-bit offsets

static bool dims_ok(uint32_t a, uint32_t b) { return a >= 1 && b >= 1 && a <= kMostDim && b <= kMostDim && static_cast<uint64_t>(a) * b <= kMostElems; }
static bool i8_dims_ok(uint32_t M, uint32_t N, uint32_t K) { return dims_ok(M, N) && dims_ok(M, K) && dims_ok(N, K) && K <= kMostI8; }
static bool gated_dims_ok(uint32_t M, uint32_t N, uint32_t K) {
    return M <= kMostGated && N <= kMostGated && K <= kMostGated && dims_ok(M, N) && dims_ok(M, K) && dims_ok(N, K);
}
static bool type_ok(omc_type t) { return t == OMC_F32 || t == OMC_BF16; }
static bool gate_ok(omc_gate g) { return g == OMC_GATE_SIGMOID || g == OMC_GATE_SWISH || g == OMC_GATE_GELU; }
static bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool element_aligned(const void *p, omc_type t) { return aligned(p, t == OMC_BF16 ? 2 : 4); }
static omc_status from_hip(int rc) { return rc == 0 ? OMC_OK : OMC_ERR_DEVICE; }
static uint32_t to_64(uint32_t n) { return (n + 63) / 64 * 64; }
static ElementType element(omc_type t) { return t == OMC_BF16 ? kE16 : kE32; }

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
static omc_status check_workspace(const void *ws, size_t have, uint64_t need) {
    if (need == 0) return OMC_OK;
    if (!ws || have < need) return OMC_ERR_WORKSPACE;
    return aligned(ws, 16) ? OMC_OK : OMC_ERR_ALIGN;
}

static Finish finish(void *c, uint64_t ldc, uint32_t M) {
    Finish f{};
    f.c = c;
    f.ldc = ldc;
    f.rows = f.second = M;
    return f;
}

// ---- 8-bit integers
struct I8Operands {
    const void *w, *w2;
    const float *w_scale, *w2_scale, *bias, *bias2;
    int gate;
};
static uint64_t i8_parts(ProductKind kind, uint32_t M, uint32_t N, uint32_t K) {
    return product_few(kind, M, N, K, false) ? 0 : product_workspace(kind, M, N, static_cast<uint32_t>(i8_pitch(K) / 128));
}
static Finish i8_finish(const float *scales, const I8Operands &o, void *C, uint64_t ldc, uint32_t M) {
    Finish f = finish(C, ldc, M);
    f.row_scale = scales;
    f.scale = o.w_scale;
    f.scale2 = o.w2_scale;
    f.bias = o.bias;
    f.bias2 = o.bias2;
    f.gate = o.gate;
    return f;
}
static int i8_product(const void *codes, const float *scales, const I8Operands &o, bool gated, void *C, bool c_bf16, uint64_t ldc, uint32_t M, uint32_t N, uint32_t K, void *parts, void *stream) {
    const uint64_t pitch = i8_pitch(K);
    const Finish f = i8_finish(scales, o, C, ldc, M);
    if (product_few(gated ? kI8Gated : kI8Plain, M, N, K, false)) return launch_product_few(kE8, kE8, gated, FewArgs{codes, pitch, o.w, o.w2, pitch, M, N, static_cast<uint32_t>(pitch), 0, f}, c_bf16, stream);
    const uint32_t stages = static_cast<uint32_t>(pitch / 128);
    return launch_product_tiles(gated ? kI8Gated : kI8Plain, TiledArgs{codes, o.w, o.w2, pitch, pitch, M, N, stages, stages, N, f, parts}, false, c_bf16, stream);
}
struct I8Layout {
    uint8_t *codes;
    float *scales;
    void *parts;
    uint64_t bytes;
};
static I8Layout i8_layout(uint8_t *ws, bool gated, uint32_t M, uint32_t N, uint32_t K) {
    I8Layout l{};
    if (product_few_rounds(M, K) && product_few(gated ? kI8Gated : kI8Plain, M, N, K, true)) return l;   // codes stay in LDS
    Parts p{ws};
    l.codes = p.take(M * i8_pitch(K));
    l.scales = reinterpret_cast<float *>(p.take(4ull * M));
    l.parts = p.take(i8_parts(gated ? kI8Gated : kI8Plain, M, N, K));
    l.bytes = p.used;
    return l;
}
static omc_status i8_layer(const void *X, omc_type x_type, uint64_t ldx, const I8Operands &o, bool gated, void *Y, omc_type y_type, uint64_t ldy, uint32_t M, uint32_t N, uint32_t K, void *ws,
                           size_t ws_bytes, void *stream) {
    if (!type_ok(x_type) || !type_ok(y_type)) return OMC_ERR_FORMAT;
    if (!i8_dims_ok(M, N, K) || ldx < K || ldy < N) return OMC_ERR_SIZE;
    if (!element_aligned(X, x_type) || !element_aligned(Y, y_type) || !aligned(o.w, 16) || !aligned(o.w2, 16) || !aligned(o.w_scale, 4) || !aligned(o.w2_scale, 4) || !aligned(o.bias, 4) ||
        !aligned(o.bias2, 4))
        return OMC_ERR_ALIGN;
    const I8Layout l = i8_layout(static_cast<uint8_t *>(ws), gated, M, N, K);
    if (const omc_status s = check_workspace(ws, ws_bytes, l.bytes)) return s;
    if (l.bytes == 0) {
        const uint64_t pitch = i8_pitch(K);
        const FewArgs fa{X, ldx, o.w, o.w2, pitch, M, N, static_cast<uint32_t>(pitch), K, i8_finish(nullptr, o, Y, ldy, M)};
        return from_hip(launch_product_few(element(x_type), kE8, gated, fa, y_type == OMC_BF16, stream));
    }
    const int rc = launch_i8_rows(I8Args{X, ldx, M, K, l.codes, l.scales, nullptr, 0}, x_type == OMC_BF16, stream);
    return from_hip(rc != 0 ? rc : i8_product(l.codes, l.scales, o, gated, Y, y_type == OMC_BF16, ldy, M, N, K, l.parts, stream));
}

// ---- the gated layer.  An operand that lies as the tiles take it is used in place, others are copied first.
struct Matrix {
    const void *x;
    uint64_t ld;                               // in elements
    omc_type type;
};
constexpr uint64_t kMostPitch = 1u << 24;      // bytes
static bool whole_rows(const Matrix &m) { return m.type == OMC_BF16 && aligned(m.x, 16) && m.ld % 8 == 0 && 2 * m.ld < kMostPitch; }

struct GatedLayout {
    uint16_t *x, *wg, *wu;
    void *parts;
    uint64_t bytes;
};
static GatedLayout gated_layout(uint8_t *ws, uint32_t M, uint32_t N, uint32_t K) {
    GatedLayout l{};
    if (product_few(kBF16Gated, M, N, K, false)) return l;
    Parts p{ws};
    const uint64_t pitch = to_64(K);
    l.x = reinterpret_cast<uint16_t *>(p.take(2 * M * pitch));
    l.wg = reinterpret_cast<uint16_t *>(p.take(2 * N * pitch));
    l.wu = reinterpret_cast<uint16_t *>(p.take(2 * N * pitch));
    l.parts = p.take(product_workspace(kBF16Gated, M, N, to_64(K) / 64));
    l.bytes = p.used;
    return l;
}
// Asked of the sizes alone, so that a gradient's bits do not depend on what is asked for beside it: tiles add up the contraction in the same order, whichever they are, but for where it is cut.
static int backward_pair(uint32_t M, uint32_t N, uint32_t K) { return product_pair_tile(M, K, to_64(N) / 64 * 2, 2 * to_64(N), K, to_64(M) / 64); }
static uint32_t sum_rows(uint32_t M, uint32_t N) { return (M + slope_rows(M, N) - 1) / slope_rows(M, N); }
struct GatedBackwardLayout {
    uint16_t *dgu, *x, *wg, *wu;
    float *sums;
    void *parts;
    uint64_t sum_bytes, bytes;                 // of the columns' sums alone (they come first, whatever K is), of all
};
static GatedBackwardLayout gated_backward_layout(uint8_t *ws, uint32_t M, uint32_t N, uint32_t K) {
    GatedBackwardLayout l{};
    Parts p{ws};
    const uint64_t m = to_64(M), n = to_64(N), k = to_64(K);
    l.sums = reinterpret_cast<float *>(p.take(8ull * sum_rows(M, N) * N));
    l.sum_bytes = p.used;
    l.dgu = reinterpret_cast<uint16_t *>(p.take(4 * m * n));
    l.x = reinterpret_cast<uint16_t *>(p.take(2 * m * k));
    l.wg = reinterpret_cast<uint16_t *>(p.take(2 * n * k));
    l.wu = reinterpret_cast<uint16_t *>(p.take(2 * n * k));
    const bool whole = backward_pair(M, N, K) >= 0;
    const uint64_t dx = whole ? 0 : product_workspace(kBF16AcrossB, M, K, to_64(N) / 64 * 2), dw = whole ? 0 : product_workspace(kBF16AcrossBoth, 2 * to_64(N), K, to_64(M) / 64);
    l.parts = p.take(dx > dw ? dx : dw);
    l.bytes = p.used;
    return l;
}

}  // namespace omc

using namespace omc;

extern "C" {

size_t omc_i8_code_bytes(uint32_t rows, uint32_t cols) { return dims_ok(rows, cols) ? rows * i8_pitch(cols) : 0; }

omc_status omc_i8_quantize(const void *x, omc_type type, uint32_t rows, uint32_t cols, uint64_t ldx, int by_columns, void *codes, float *scales, void *values, uint64_t ldv, void *stream) {
    if (!x || !codes || !scales) return OMC_ERR_NULL;
    if (!type_ok(type)) return OMC_ERR_FORMAT;
    if (!dims_ok(rows, cols) || ldx < cols || (values && ldv < cols)) return OMC_ERR_SIZE;
    if (!element_aligned(x, type) || !element_aligned(values, type) || !aligned(codes, 16) || !aligned(scales, 4)) return OMC_ERR_ALIGN;
    const I8Args ia{x, ldx, rows, cols, static_cast<uint8_t *>(codes), scales, values, ldv};
    return from_hip(by_columns ? launch_i8_columns(ia, type == OMC_BF16, stream) : launch_i8_rows(ia, type == OMC_BF16, stream));
}

size_t omc_i8_gemm_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) { return i8_dims_ok(M, N, K) ? i8_parts(kI8Plain, M, N, K) : 0; }

omc_status omc_i8_gemm(const void *a_codes, const float *a_scales, const void *b_codes, const float *b_scales, const float *bias, void *C, omc_type c_type, uint64_t ldc, uint32_t M, uint32_t N,
                       uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!a_codes || !a_scales || !b_codes || !b_scales || !C) return OMC_ERR_NULL;
    if (!type_ok(c_type)) return OMC_ERR_FORMAT;
    if (!i8_dims_ok(M, N, K) || ldc < N) return OMC_ERR_SIZE;
    if (!aligned(a_codes, 16) || !aligned(b_codes, 16) || !aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(bias, 4) || !element_aligned(C, c_type)) return OMC_ERR_ALIGN;
    if (const omc_status s = check_workspace(ws, ws_bytes, i8_parts(kI8Plain, M, N, K))) return s;
    const I8Operands o{b_codes, nullptr, b_scales, nullptr, bias, nullptr, 0};
    return from_hip(i8_product(a_codes, a_scales, o, false, C, c_type == OMC_BF16, ldc, M, N, K, ws, stream));
}

size_t omc_i8_linear_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) { return i8_dims_ok(M, N, K) ? i8_layout(nullptr, false, M, N, K).bytes : 0; }

omc_status omc_i8_linear(const void *X, omc_type x_type, uint64_t ldx, const void *w_codes, const float *w_scales, const float *bias, void *Y, omc_type y_type, uint64_t ldy, uint32_t M, uint32_t N,
                         uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!X || !w_codes || !w_scales || !Y) return OMC_ERR_NULL;
    return i8_layer(X, x_type, ldx, I8Operands{w_codes, nullptr, w_scales, nullptr, bias, nullptr, 0}, false, Y, y_type, ldy, M, N, K, ws, ws_bytes, stream);
}

size_t omc_i8_gated_linear_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) { return i8_dims_ok(M, N, K) ? i8_layout(nullptr, true, M, N, K).bytes : 0; }

omc_status omc_i8_gated_linear(const void *X, omc_type x_type, uint64_t ldx, const void *wg_codes, const float *wg_scales, const void *wu_codes, const float *wu_scales, const float *bg, const float *bu,
                               omc_gate gate, void *H, omc_type h_type, uint64_t ldh, uint32_t M, uint32_t N, uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!X || !wg_codes || !wg_scales || !wu_codes || !wu_scales || !H) return OMC_ERR_NULL;
    if (!gate_ok(gate)) return OMC_ERR_OPT;
    return i8_layer(X, x_type, ldx, I8Operands{wg_codes, wu_codes, wg_scales, wu_scales, bg, bu, static_cast<int>(gate)}, true, H, h_type, ldh, M, N, K, ws, ws_bytes, stream);
}

size_t omc_gated_linear_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) { return gated_dims_ok(M, N, K) ? gated_layout(nullptr, M, N, K).bytes : 0; }

omc_status omc_gated_linear(const void *X, omc_type x_type, uint64_t ldx, const void *Wg, const void *Wu, omc_type w_type, uint64_t ldw, const float *bg, const float *bu, omc_gate gate, void *H,
                            omc_type h_type, uint64_t ldh, void *slope_g, void *slope_u, uint64_t ld_slope, uint32_t M, uint32_t N, uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!X || !Wg || !Wu || !H || !slope_g != !slope_u) return OMC_ERR_NULL;
    if (!type_ok(x_type) || !type_ok(w_type) || !type_ok(h_type)) return OMC_ERR_FORMAT;
    if (!gate_ok(gate)) return OMC_ERR_OPT;
    if (!gated_dims_ok(M, N, K) || ldx < K || ldw < K || ldh < N || (slope_g && ld_slope < N)) return OMC_ERR_SIZE;
    if (!element_aligned(X, x_type) || !element_aligned(Wg, w_type) || !element_aligned(Wu, w_type) || !element_aligned(H, h_type) || !aligned(bg, 4) || !aligned(bu, 4) || !aligned(slope_g, 2) ||
        !aligned(slope_u, 2))
        return OMC_ERR_ALIGN;
    const GatedLayout l = gated_layout(static_cast<uint8_t *>(ws), M, N, K);
    if (const omc_status s = check_workspace(ws, ws_bytes, l.bytes)) return s;
    Finish f = finish(H, ldh, M);
    f.bias = bg;
    f.bias2 = bu;
    f.gate = static_cast<int>(gate);
    f.slope_g = static_cast<uint16_t *>(slope_g);
    f.slope_u = static_cast<uint16_t *>(slope_u);
    f.ld_slope = ld_slope;
    if (product_few(kBF16Gated, M, N, K, false)) return from_hip(launch_product_few(element(x_type), element(w_type), true, FewArgs{X, ldx, Wg, Wu, ldw, M, N, K, 0, f}, h_type == OMC_BF16, stream));
    const uint32_t pitch = to_64(K);
    PackArgs packs[kMostPacks];
    uint32_t count = 0;
    const Matrix x{X, ldx, x_type}, wg{Wg, ldw, w_type}, wu{Wu, ldw, w_type};
    TiledArgs ta{X, Wg, Wu, 2 * ldx, 2 * ldw, M, N, pitch / 64, pitch / 64, N, f, l.parts};
    if (K % 64 != 0 || !whole_rows(x)) {
        packs[count++] = PackArgs{X, ldx, x_type == OMC_BF16, M, K, l.x, M, pitch};
        ta.a = l.x;
        ta.a_pitch = 2 * pitch;
    }
    if (K % 64 != 0 || !whole_rows(wg) || !whole_rows(wu)) {
        packs[count++] = PackArgs{Wg, ldw, w_type == OMC_BF16, N, K, l.wg, N, pitch};
        packs[count++] = PackArgs{Wu, ldw, w_type == OMC_BF16, N, K, l.wu, N, pitch};
        ta.b = l.wg;
        ta.b2 = l.wu;
        ta.b_pitch = 2 * pitch;
    }
    const int rc = count > 0 ? launch_pack(packs, count, stream) : 0;
    return from_hip(rc != 0 ? rc : launch_product_tiles(kBF16Gated, ta, false, h_type == OMC_BF16, stream));
}

size_t omc_gated_linear_backward_workspace_bytes(uint32_t M, uint32_t N, uint32_t K) { return gated_dims_ok(M, N, K) ? gated_backward_layout(nullptr, M, N, K).bytes : 0; }

omc_status omc_gated_linear_backward(const void *dH, omc_type dh_type, uint64_t lddh, const void *slope_g, const void *slope_u, uint64_t ld_slope, const void *X, omc_type x_type, uint64_t ldx,
                                     const void *Wg, const void *Wu, omc_type w_type, uint64_t ldw, void *dX, omc_type dx_type, uint64_t lddx, float *dWg, float *dWu, float *dbg, float *dbu,
                                     uint32_t M, uint32_t N, uint32_t K, void *ws, size_t ws_bytes, void *stream) {
    if (!dH || !slope_g || !slope_u || !dWg != !dWu || (!dX && !dWg && !dbg && !dbu) || (dX && (!Wg || !Wu)) || (dWg && !X)) return OMC_ERR_NULL;
    if (!type_ok(dh_type) || (dWg && !type_ok(x_type)) || (dX && (!type_ok(w_type) || !type_ok(dx_type)))) return OMC_ERR_FORMAT;
    if (!gated_dims_ok(M, N, K) || lddh < N || ld_slope < N || (dWg && ldx < K) || (dX && (ldw < K || lddx < K))) return OMC_ERR_SIZE;
    if (!element_aligned(dH, dh_type) || !aligned(slope_g, 2) || !aligned(slope_u, 2) || !aligned(dWg, 4) || !aligned(dWu, 4) || !aligned(dbg, 4) || !aligned(dbu, 4) ||
        (dWg && !element_aligned(X, x_type)) || (dX && (!element_aligned(Wg, w_type) || !element_aligned(Wu, w_type) || !element_aligned(dX, dx_type))))
        return OMC_ERR_ALIGN;
    const GatedBackwardLayout l = gated_backward_layout(static_cast<uint8_t *>(ws), M, N, K);
    if (const omc_status s = check_workspace(ws, ws_bytes, dX || dWg ? l.bytes : l.sum_bytes)) return s;
    const bool sums = dbg || dbu;
    const uint32_t rows = to_64(M), half = to_64(N), k = to_64(K);
    PackArgs packs[kMostPacks];
    uint32_t count = 0;
    TiledArgs for_dx{l.dgu, Wg, Wu, 4ull * half, 2 * ldw, M, K, half / 64 * 2, half / 64, K, finish(dX, lddx, M), l.parts};
    TiledArgs for_dw{l.dgu, X, nullptr, 4ull * half, 2 * ldx, 2 * half, K, rows / 64, rows / 64, K, finish(dWg, K, N), l.parts};
    for_dw.f.c2 = dWu;
    for_dw.f.second = half;
    if (dX && (K % 8 != 0 || N % 64 != 0 || !whole_rows(Matrix{Wg, ldw, w_type}) || !whole_rows(Matrix{Wu, ldw, w_type}))) {
        packs[count++] = PackArgs{Wg, ldw, w_type == OMC_BF16, N, K, l.wg, half, k};
        packs[count++] = PackArgs{Wu, ldw, w_type == OMC_BF16, N, K, l.wu, half, k};
        for_dx.b = l.wg;
        for_dx.b2 = l.wu;
        for_dx.b_pitch = 2ull * k;
        for_dx.b_cols = k;
    }
    if (dWg && (K % 8 != 0 || M % 64 != 0 || !whole_rows(Matrix{X, ldx, x_type}))) {
        packs[count++] = PackArgs{X, ldx, x_type == OMC_BF16, M, K, l.x, rows, k};
        for_dw.b = l.x;
        for_dw.b_pitch = 2ull * k;
        for_dw.b_cols = k;
    }
    const SlopeArgs sa{dH, lddh, dh_type == OMC_BF16, static_cast<const uint16_t *>(slope_g), static_cast<const uint16_t *>(slope_u), ld_slope, M, N, rows, half, dX || dWg ? l.dgu : nullptr,
                       sums ? l.sums : nullptr};
    int rc = launch_slopes(sa, packs, count, stream);
    const int pair = backward_pair(M, N, K);
    if (rc == 0 && pair >= 0 && dX && dWg) return from_hip(launch_product_pair(pair, for_dx, dx_type == OMC_BF16, for_dw, l.sums, sum_rows(M, N), N, dbg, dbu, stream));
    if (rc == 0 && sums) rc = launch_column_sums(l.sums, sum_rows(M, N), false, N, 2 * N, dbg, dbu, stream);
    if (rc == 0 && dX) rc = launch_product_tiles(kBF16AcrossB, for_dx, pair >= 0, dx_type == OMC_BF16, stream);
    if (rc == 0 && dWg) rc = launch_product_tiles(kBF16AcrossBoth, for_dw, pair >= 0, false, stream);
    return from_hip(rc);
}

}  // extern "C"
