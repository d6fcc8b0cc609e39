// Launchers of the products on 8-bit integers and on bf16, of the gated linear layer, and of what prepares their operands.  Arguments already validated; return hipError_t as int.
#pragma once
#include "omc_layer.h"

namespace omc {

// What a product's sums become.  rows_scale and scale (, scale2) turn sums of 8-bit integers into values; bias (, bias2) is added; of a gated product, whose second sums belong to b2, the result is
// act(first) * second, and slope_g, slope_u (bf16, or both null) get its derivatives with respect to either.
struct Finish {
    const float *row_scale, *scale, *scale2, *bias, *bias2;
    int gate;                            // omc_gate
    void *c, *c2;                        // rows from `second` on go to c2, row 0 of which is row `second`; rows `rows` .. `second` are nowhere
    uint64_t ldc;
    uint32_t rows, second;
    uint16_t *slope_g, *slope_u;
    uint64_t ld_slope;
};

// C[M x N] = A B^T in tiles.  An operand lies in rows along the contraction, of whole stages of 128 bytes (64 values of bf16, 128 of 8 bits), or (bf16 only) across it: a row for every k, whole 64s of
// them, and whole 8s of columns.  16-byte aligned rows, `pitch` bytes apart.  Across, B may lie in two parts: from stage `turn` on it is b2.
enum ProductKind { kI8Plain, kI8Gated, kBF16Gated, kBF16AcrossB, kBF16AcrossBoth };
struct TiledArgs {
    const void *a, *b, *b2;
    uint64_t a_pitch, b_pitch;
    uint32_t M, N, stages, turn, b_cols;   // b_cols: of B across, whole 8s, N at least
    Finish f;
    void *parts;                         // of a split contraction
};
size_t product_workspace(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages);   // bytes of parts
double product_tiles_cost(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages);  // an estimate, us
int launch_product_tiles(ProductKind kind, const TiledArgs &pa, bool whole, bool c_bf16, void *stream);   // whole: the contraction is not cut
// Of a gated layer's backward products, M x N as kBF16AcrossB and M2 x N2 as kBF16AcrossBoth (its result in fp32): the tile in which both go together, uncut, in one launch; -1: each goes its own way.
int product_pair_tile(uint32_t M, uint32_t N, uint32_t stages, uint32_t M2, uint32_t N2, uint32_t stages2);
// In the same launch columns' sums, of `count` rows of partial sums, 2 * cols floats each, to out0 and out1 (as launch_column_sums; both may be null: none).
int launch_product_pair(int tile, const TiledArgs &dx, bool dx_bf16, const TiledArgs &dw, const float *sums, uint32_t count, uint32_t cols, float *out0, float *out1, void *stream);

// The same for few rows of A (product_few).  x_type and w_type: 8-bit codes in padded rows (then K is whole 128s), or fp32 or bf16 as they lie, which are rounded to bf16 on the way; pitches in bytes.
// rounds: A comes in fp32 or bf16 and becomes 8-bit codes on the way (product_few_rounds).
enum ElementType { kE8, kE16, kE32 };
struct FewArgs {
    const void *x;
    uint64_t ldx;                        // in elements
    const void *w, *w2;
    uint64_t ldw;
    uint32_t M, N, K;
    uint32_t columns;                    // values of a row of A, where it becomes codes
    Finish f;
};
bool product_few(ProductKind kind, uint32_t M, uint32_t N, uint32_t K, bool rounds);   // rounds: A would become codes on the way
bool product_few_rounds(uint32_t M, uint32_t K);
int launch_product_few(ElementType x, ElementType w, bool gated, const FewArgs &fa, bool c_bf16, void *stream);

// 8-bit codes and scales of a matrix' rows, or of its columns (codes are then its transpose's rows); values may be null.
constexpr uint64_t i8_pitch(uint32_t cols) { return (static_cast<uint64_t>(cols) + 127) / 128 * 128; }
struct I8Args {
    const void *x;
    uint64_t ldx;
    uint32_t rows, cols;
    uint8_t *codes;
    float *scales;
    void *values;
    uint64_t ldv;
};
int launch_i8_rows(const I8Args &ia, bool bf16, void *stream);
int launch_i8_columns(const I8Args &ia, bool bf16, void *stream);

// Copies in bf16 with rows of `pitch` values, zeros behind a row's end and behind the last row up to to_rows; several in one launch.
struct PackArgs {
    const void *x;
    uint64_t ldx;
    bool bf16;
    uint32_t rows, cols;
    uint16_t *to;
    uint32_t to_rows, pitch;
};
constexpr uint32_t kMostPacks = 3;
int launch_pack(const PackArgs *packs, uint32_t count, void *stream);

// dg and du: dh times its slopes in fp32, rounded to bf16, side by side in rows of 2 * half values (zeros behind N and up to to_rows; may be null), and partial sums of their columns, a row of 2 N floats for every
// slope_rows rows (may be null).  By the same launch copies, as above.
uint32_t slope_rows(uint32_t M, uint32_t N);
struct SlopeArgs {
    const void *dh;
    uint64_t lddh;
    bool bf16;
    const uint16_t *slope_g, *slope_u;
    uint64_t ld_slope;
    uint32_t M, N, to_rows, half;
    uint16_t *to;
    float *sums;
};
int launch_slopes(const SlopeArgs &sa, const PackArgs *packs, uint32_t count, void *stream);

}  // namespace omc
