// The gated linear layer's backward products on bf16 in tiles (see omc_tiles.h): dX = [dg | du] [Wg; Wu], the weights across the contraction, and dW = [dg | du]^T X, both operands across it.
#include "omc_tiles.h"

namespace omc {

int launch_across_b(const TiledArgs &pa, bool whole, bool c_bf16, hipStream_t st) {
    return c_bf16 ? launch_tiles<false, false, false, true, BF16>(pa, whole, st) : launch_tiles<false, false, false, true, F32>(pa, whole, st);
}
int launch_across_both(const TiledArgs &pa, bool whole, bool c_bf16, hipStream_t st) {
    return c_bf16 ? launch_tiles<false, false, true, true, BF16>(pa, whole, st) : launch_tiles<false, false, true, true, F32>(pa, whole, st);
}

// Both in one launch, in tiles of one size, and the biases' gradients.  8192 x 4096 x 1024: 256 tiles of 256 x 256 in one launch, a backward pass
// of 270 us with the slopes before them; in two launches, whose 128 such tiles leave half of the chip idle, in tiles of 256 x 128 at best, 302.
template <typename T>
static int launch_pair_typed(int tile, const TiledArgs &dx, const TiledArgs &dw, const ColumnSums &sums, hipStream_t st) {
    PairGrid pg{grid_of(dx, tile, false, 1), grid_of(dw, tile, false, 1), 0, sums};
    pg.groups = (pg.first.tiles_m * pg.first.tiles_n + 7) / 8 * 8 + pg.second.tiles_m * pg.second.tiles_n;
    for_tile(tile, [&](auto wm, auto wn, auto tm, auto tn, auto s, auto occ, auto) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, TM = decltype(tm)::value, TN = decltype(tn)::value, S = decltype(s)::value;
        tiles_pair_kernel<Tiles<false, false, false, true, WM, WN, TM, TN, S, false, T>, Tiles<false, false, true, true, WM, WN, TM, TN, S, false, F32>, decltype(occ)::value>
            <<<dim3(pg.groups + (sums.width + 31) / 32), dim3(64 * WM * WN), 0, st>>>(pg);
    });
    return static_cast<int>(hipGetLastError());
}
int launch_product_pair(int tile, const TiledArgs &dx, bool dx_bf16, const TiledArgs &dw, const float *sums, uint32_t count, uint32_t cols, float *out0, float *out1, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const ColumnSums cs{sums, count, cols, out0 || out1 ? 2 * cols : 0, out0, out1};
    return dx_bf16 ? launch_pair_typed<BF16>(tile, dx, dw, cs, st) : launch_pair_typed<F32>(tile, dx, dw, cs, st);
}

}  // namespace omc
