// The gated linear layer's backward products on bf16 in tiles (see omc_tiles.h): dX = [dg | du] [Wg; Wu], the weights across the contraction, and dW = [dg | du]^T X, both operands across it.
#include "omc_tiles.h"

namespace omc {

int launch_across_b(const TiledArgs &pa, bool c_bf16, hipStream_t st) {
    return c_bf16 ? launch_tiles<false, false, false, true, BF16>(pa, st) : launch_tiles<false, false, false, true, F32>(pa, st);
}
int launch_across_both(const TiledArgs &pa, bool c_bf16, hipStream_t st) {
    return c_bf16 ? launch_tiles<false, false, true, true, BF16>(pa, st) : launch_tiles<false, false, true, true, F32>(pa, st);
}

}  // namespace omc
