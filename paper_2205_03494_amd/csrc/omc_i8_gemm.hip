// Products on 8-bit integers in tiles, plain and gated (see omc_tiles.h).
#include "omc_tiles.h"

namespace omc {

int launch_i8_plain(const TiledArgs &pa, bool c_bf16, hipStream_t st) {
    return c_bf16 ? launch_tiles<true, false, false, false, BF16>(pa, false, st) : launch_tiles<true, false, false, false, F32>(pa, false, st);
}
int launch_i8_gated(const TiledArgs &pa, bool c_bf16, hipStream_t st) {
    return c_bf16 ? launch_tiles<true, true, false, false, BF16>(pa, false, st) : launch_tiles<true, true, false, false, F32>(pa, false, st);
}

}  // namespace omc
