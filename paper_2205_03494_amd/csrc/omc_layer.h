// Launchers of the layer's operators: 4-bit microscaled products and the layer norm.  Arguments already validated; return hipError_t as int.
#pragma once
#include <cstddef>
#include <cstdint>

#include "omc.h"

namespace omc {

// A matrix in MX4: rows of `blocks` blocks of 32 values (whole multiples of 4 blocks), 16 bytes of codes and a scale byte each.
struct Mx4 {
    const uint8_t *codes, *scales;
};
constexpr uint32_t mx4_padded(uint32_t cols) { return (cols + 127) / 128 * 128; }   // (cols <= 2^32 - 128)
constexpr uint64_t mx4_code_bytes(uint64_t rows, uint32_t cols) { return rows * (mx4_padded(cols) / 2); }
constexpr uint64_t mx4_scale_bytes(uint64_t rows, uint32_t cols) { return rows * (mx4_padded(cols) / 32); }

// The scales as the tiles of launch_mx4_gemm read them: for every 256 values of a row, one after the other, 8 bytes of every row (rows padded to 256, which need not be
// written), those of its blocks 0, 1, 4, 5, 2, 3, 6, 7, and 0 for the second 128 values if the row has none.
constexpr uint32_t mx4_image_byte(uint32_t block) { return 4 * (block / 2 % 2) + 2 * (block / 4) + block % 2; }
constexpr uint64_t mx4_image_pitch(uint32_t rows) { return (static_cast<uint64_t>(rows) + 255) / 256 * 2048; }
constexpr uint64_t mx4_image_bytes(uint32_t rows, uint32_t cols) { return (static_cast<uint64_t>(cols) + 255) / 256 * mx4_image_pitch(rows); }

// Scales in the order of omc.h, to be brought into that of the tiles.
struct Mx4Reorder {
    const uint8_t *scales;
    uint8_t *image;                // null: nothing to do
    uint32_t rows, cols;
};

struct QuantArgs {
    const void *x;
    uint64_t ldx;
    uint32_t rows, cols;
    uint8_t *codes, *scales;       // blocks along a row; may be null
    uint8_t *codes_t, *scales_t;   // blocks along a column; may be null
    void *values;                  // may be null
    uint64_t ldv;
    float *colsum;                 // partial sums of the columns, a row of them for every tile of rows, of whole 256s (mx4_tile_height); may be null
    bool images;                   // scales and scales_t in the tiles' order
    Mx4Reorder also;               // another matrix' scales, by the same launch (along rows only; see launch_mx4_tiles)
};
// Several matrices in one launch, in any directions but without values, and another one's scales.
constexpr uint32_t kMostJobs = 3;
uint32_t mx4_tile_height(const QuantArgs *args, uint32_t count);   // rows of a tile of such a launch, 64 or 256
int launch_mx4_tiles(const QuantArgs *args, uint32_t count, const Mx4Reorder &also, bool bf16, void *stream);
int launch_mx4_reorder(const Mx4Reorder &a, const Mx4Reorder &b, void *stream);
int launch_mx4_quantize(const QuantArgs &qa, bool bf16, void *stream);   // no sums

struct Mx4GemmArgs {
    Mx4 a, b;
    const float *bias;
    void *c;
    uint64_t ldc;
    uint32_t M, N, K;
    float *parts;                  // partial results of a split contraction
};
// c = a b^T + bias, c in bf16 or fp32; the operands' scales in the tiles' order.  whole: the contraction is not cut.
size_t mx4_gemm_workspace(uint32_t M, uint32_t N, uint32_t K);   // bytes of parts
int launch_mx4_gemm(const Mx4GemmArgs &ga, bool whole, bool bf16, void *stream);
// Of a layer's backward pass, dX[M x K] over N and dW[K x N] over M: are both products uncut and in tiles; the tile in which such should go together, -1: each in a launch of its own.
bool mx4_backward_whole(uint32_t M, uint32_t N, uint32_t K);
int mx4_pair_tile(uint32_t M, uint32_t N, uint32_t K, bool sums);
// Two products, the second one's result in fp32, in one launch, and in it dbias, whose columns are the second one's, from partial sums as for launch_column_sums (dbias may be null).
int launch_mx4_pair(int tile, const Mx4GemmArgs &ga, bool bf16, const Mx4GemmArgs &gb, const float *parts, uint32_t count, bool fours, float *dbias, void *stream);
// The same for few rows of a (mx4_few, 32 at most), with scales in the order of omc.h.  Where mx4_few_rounds, these may come as they are (`rows`), and are rounded on the way.
struct Mx4Rows {
    const void *x;
    uint64_t ldx;
    bool bf16;
};
bool mx4_few(uint32_t M, uint32_t N, uint32_t K);
bool mx4_few_rounds(uint32_t M, uint32_t K);
int launch_mx4_few(const Mx4GemmArgs &ga, const Mx4Rows *rows, bool bf16, void *stream);

// Of `count` rows of partial sums, `width` floats each: the columns' sums, the first `cols` of them to out0, the others to out1 (either may be null).  fours: each is four rows that lie one after the other,
// which are added first; 256 of them at most.  The order of all is fixed by count.
int launch_column_sums(const float *parts, uint32_t count, bool fours, uint32_t cols, uint32_t width, float *out0, float *out1, void *stream);

struct NormArgs {
    const void *x;
    uint64_t ldx;
    const float *gamma, *beta;
    float eps;
    void *y;
    uint64_t ldy;
    float *mean, *rstd;
    uint32_t rows, cols;
};
int launch_layer_norm(const NormArgs &na, bool x_bf16, bool y_bf16, void *stream);

struct NormGradArgs {
    const void *dy;
    uint64_t lddy;
    const void *x;
    uint64_t ldx;
    const float *gamma, *mean, *rstd;
    void *dx;
    uint64_t lddx;
    float *dgamma, *dbeta;
    uint32_t rows, cols;
    float *parts;
};
size_t layer_norm_backward_workspace(uint32_t rows, uint32_t cols);
int launch_layer_norm_backward(const NormGradArgs &na, bool x_bf16, bool dy_bf16, void *stream);

}  // namespace omc
