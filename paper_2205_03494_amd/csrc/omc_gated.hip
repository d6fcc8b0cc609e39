// The gated linear layer's forward product on bf16 in tiles (see omc_tiles.h), and which tile a product takes.
#include "omc_tiles.h"

namespace omc {

struct TileCost {
    double base, alone, busy, uneven, store;
};
static constexpr TileCost kCosts[5][4] = {
    {{6.0, 1.1, 1.1, 0.6, 4.0}, {5.0, 0.6, 0.6, 0.6, 2.0}, {4.0, 0.3, 0.35, 0.6, 1.0}, {3.0, 0.12, 0.12, 0.6, 0.4}},
    {{6.0, 1.1, 1.1, 0.6, 8.0}, {5.0, 0.6, 0.6, 0.6, 4.0}, {4.0, 0.3, 0.35, 0.6, 2.0}, {3.0, 0.12, 0.12, 0.6, 0.6}},
    {{6.0, 1.3, 1.4, 0.6, 8.0}, {5.0, 0.7, 0.75, 0.6, 4.0}, {4.0, 0.35, 0.42, 0.6, 2.0}, {3.0, 0.14, 0.14, 0.6, 0.6}},
    {{6.0, 1.3, 1.4, 0.6, 4.0}, {5.0, 0.7, 0.75, 0.6, 2.0}, {4.0, 0.35, 0.42, 0.6, 1.0}, {3.0, 0.14, 0.14, 0.6, 0.4}},
    {{6.0, 1.3, 1.4, 0.6, 4.0}, {5.0, 0.7, 0.75, 0.6, 2.0}, {4.0, 0.35, 0.42, 0.6, 1.0}, {3.0, 0.14, 0.14, 0.6, 0.4}},
};
static constexpr uint32_t kResident[] = {1, 1, 2, 2};

static bool gated_kind(ProductKind kind) { return kind == kI8Gated || kind == kBF16Gated; }
static uint64_t tiles_of(ProductKind kind, int tile, uint32_t M, uint32_t N) {
    const uint32_t bm = kTileRows[tile], bn = kTileCols[tile] / (gated_kind(kind) ? 2 : 1);
    return static_cast<uint64_t>((M + bm - 1) / bm) * ((N + bn - 1) / bn);
}
static double cost(const TileCost &t, uint32_t resident, double items, double stages) {   // stages: of an item
    const double units = static_cast<double>((static_cast<uint64_t>(items) + 255) / 256), rounds = static_cast<double>((static_cast<uint64_t>(items) + 256 * resident - 1) / (256 * resident)), per_unit = items / 256.0;
    const double alone = t.alone * stages * rounds, busy = t.busy * stages * (per_unit + t.uneven * (units - per_unit));
    return t.base + (alone > busy ? alone : busy) + t.store * (per_unit > 1.0 ? per_unit : 1.0);
}
TileChoice choose_tile(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages, bool whole) {
    TileChoice best{-1, 1, 0.0};
    for (int i = 0; i < 4; ++i) {
        const uint64_t tiles = tiles_of(kind, i, M, N);
        if (tiles > 0x7fffffffu) continue;
        for (uint32_t splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && (whole || tiles * splits > 256 * kResident[i] || 2 * splits > stages)) break;
            double c = cost(kCosts[kind][i], kResident[i], static_cast<double>(tiles * splits), static_cast<double>((stages + splits - 1) / splits));
            if (splits > 1) c += 3.2 + 2e-6 * splits * M * N * (gated_kind(kind) ? 2 : 1);
            if (best.tile < 0 || c < best.cost) best = TileChoice{i, splits, c};
        }
    }
    const uint32_t each = (stages + best.splits - 1) / best.splits;
    best.splits = (stages + each - 1) / each;
    return best;
}
int product_pair_tile(uint32_t M, uint32_t N, uint32_t stages, uint32_t M2, uint32_t N2, uint32_t stages2) {
    int tile = -1;
    double least = choose_tile(kBF16AcrossB, M, N, stages, false).cost + choose_tile(kBF16AcrossBoth, M2, N2, stages2, false).cost;
    for (int i = 0; i < 4; ++i) {
        const double a = static_cast<double>(tiles_of(kBF16AcrossB, i, M, N)), b = static_cast<double>(tiles_of(kBF16AcrossBoth, i, M2, N2));
        if (a + b > 0x7ffffff0u) continue;
        const double c = cost(kCosts[kBF16AcrossBoth][i], kResident[i], a + b, (a * stages + b * stages2) / (a + b));
        if (c < least) {
            least = c;
            tile = i;
        }
    }
    return tile;
}

int launch_i8_plain(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_i8_gated(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_across_b(const TiledArgs &pa, bool whole, bool c_bf16, hipStream_t st);
int launch_across_both(const TiledArgs &pa, bool whole, bool c_bf16, hipStream_t st);

size_t product_workspace(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages) {
    const TileChoice c = choose_tile(kind, M, N, stages, false);
    return c.splits > 1 ? 4ull * c.splits * M * N * (gated_kind(kind) ? 2 : 1) : 0;
}

int launch_product_tiles(ProductKind kind, const TiledArgs &pa, bool whole, bool c_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (kind) {
        case kI8Plain: return launch_i8_plain(pa, c_bf16, st);
        case kI8Gated: return launch_i8_gated(pa, c_bf16, st);
        case kBF16Gated: return c_bf16 ? launch_tiles<false, true, false, false, BF16>(pa, false, st) : launch_tiles<false, true, false, false, F32>(pa, false, st);
        case kBF16AcrossB: return launch_across_b(pa, whole, c_bf16, st);
        default: return launch_across_both(pa, whole, c_bf16, st);
    }
}

}  // namespace omc
