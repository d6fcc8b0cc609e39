// The gated linear layer's forward product on bf16 in tiles (see omc_tiles.h), and which tile a product takes.
#include "omc_tiles.h"

namespace omc {

TileChoice choose_tile(uint32_t M, uint32_t cols, uint32_t stages) {
    (void)stages;
    for (int i = 0; i < 3; ++i)
        if (static_cast<uint64_t>((M + kTileRows[i] - 1) / kTileRows[i]) * ((cols + kTileCols[i] - 1) / kTileCols[i]) >= 200) return {i, 1};
    return {3, 1};
}

int launch_i8_plain(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_i8_gated(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_across_b(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_across_both(const TiledArgs &pa, bool c_bf16, hipStream_t st);

static uint32_t columns_of(ProductKind kind, uint32_t N) { return kind == kI8Gated || kind == kBF16Gated ? 2 * N : N; }
size_t product_workspace(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages) {
    const TileChoice c = choose_tile(M, columns_of(kind, N), stages);
    return c.splits > 1 ? 4ull * c.splits * M * columns_of(kind, N) : 0;
}

int launch_product_tiles(ProductKind kind, const TiledArgs &pa, bool c_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (kind) {
        case kI8Plain: return launch_i8_plain(pa, c_bf16, st);
        case kI8Gated: return launch_i8_gated(pa, c_bf16, st);
        case kBF16Gated: return c_bf16 ? launch_tiles<false, true, false, false, BF16>(pa, st) : launch_tiles<false, true, false, false, F32>(pa, st);
        case kBF16AcrossB: return launch_across_b(pa, c_bf16, st);
        default: return launch_across_both(pa, c_bf16, st);
    }
}

}  // namespace omc
