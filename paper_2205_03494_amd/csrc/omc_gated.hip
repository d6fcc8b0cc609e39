// The gated linear layer's forward product on bf16 in tiles (see omc_tiles.h), and which tile a product takes.
#include "omc_tiles.h"

namespace omc {

// By an estimate of the time in us: `base` is a launch; `alone` a stage of workgroups that nothing else slows down, `resident` of them on a compute unit; `busy` what a stage costs per workgroup of a unit where all units have some
// (of the last workgroups' unevenness over the units `uneven` counts); `store` the end of 256 tiles.  A row for every kind of product, the last one for both backward products in one launch, which takes no less than its longest
// contraction.  Fitted to 2100 sizes of 33 .. 16384 x 64 .. 8192 x 64 .. 8192 in bf16, 60 % of them with whole cache lines: 4 - 16 % (standard deviation).  On these the chosen way takes 0.5 - 1.4 % longer than the best one (both
// backward products together or apart: 2.6 %), at worst 13 - 50 %, of a few us.
// 8192 x 4096 x 1024, gated: 256 x 256 150 us, 256 x 128 152, 128 x 128 157, 64 x 64 238; in 8 bits, plain: 42, 46, 43, 60; 8192 x 1024 x 4096: 48, 34, 35, 38.
// 128 x 128 has two stages and two workgroups on a unit; with four stages, eight waves and the unit for itself 8192 x 4096 x 1024, gated, took 168 us.
// A cut costs a second launch and the parts' way through memory.
struct TileCost {
    double base, alone, busy, uneven, store;
};
static constexpr int kPair = 5;
static constexpr TileCost kCosts[6][4] = {
    {{2.031, 1.341, 0.3, 0.5, 10.24}, {2.936, 0.497, 1.121, 0.441, 3.521}, {4.058, 0.246, 0.593, 0.637, 1.522}, {3.617, 0.239, 0.188, 1.105, 0.686}},
    {{2.781, 1.406, 0.1, 0.5, 8.55}, {4.195, 0.495, 0.856, 0.675, 3.131}, {4.303, 0.508, 0.429, 1.007, 1.445}, {3.653, 0.261, 0.181, 1.204, 0.68}},
    {{0.0, 1.286, 0.3, 0.5, 14.292}, {3.132, 0.454, 0.855, 0.691, 6.042}, {2.881, 0.562, 0.428, 1.104, 3.168}, {3.507, 0.272, 0.183, 1.279, 1.214}},
    {{2.467, 1.219, 0.1, 0.5, 8.363}, {3.369, 0.405, 0.793, 0.774, 2.976}, {2.535, 0.572, 0.393, 1.177, 1.887}, {3.34, 0.264, 0.188, 1.099, 0.497}},
    {{8.689, 1.217, 1.015, 0.5, 17.326}, {7.594, 0.075, 0.749, 0.883, 8.209}, {3.302, 0.619, 0.387, 1.442, 4.197}, {3.518, 0.278, 0.194, 1.256, 0.832}},
    {{0.0, 1.145, 0.357, 0.5, 24.809}, {5.328, 0.66, 0.783, 0.986, 8.287}, {0.246, 0.623, 0.399, 1.662, 4.664}, {2.813, 0.276, 0.195, 1.667, 1.257}},
};
static constexpr uint32_t kResident[] = {1, 1, 2, 2};

static bool gated_kind(ProductKind kind) { return kind == kI8Gated || kind == kBF16Gated; }
static uint64_t tiles_of(ProductKind kind, int tile, uint32_t M, uint32_t N) {
    const uint32_t bm = kTileRows[tile], bn = kTileCols[tile] / (gated_kind(kind) ? 2 : 1);
    return static_cast<uint64_t>((M + bm - 1) / bm) * ((N + bn - 1) / bn);
}
static double cost(const TileCost &t, uint32_t resident, uint64_t items, double stages, double longest) {   // stages: of an item, on average
    const double units = static_cast<double>((items + 255) / 256), rounds = static_cast<double>((items + 256 * resident - 1) / (256 * resident)), per_unit = static_cast<double>(items) / 256.0;
    const double in_turn = stages * rounds, alone = t.alone * (in_turn > longest ? in_turn : longest), busy = t.busy * stages * (per_unit + t.uneven * (units - per_unit));
    return t.base + (alone > busy ? alone : busy) + t.store * (per_unit > 1.0 ? per_unit : 1.0);
}
TileChoice choose_tile(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages, bool whole) {
    TileChoice best{-1, 1, 0.0};
    for (int i = 0; i < 4; ++i) {
        const uint64_t tiles = tiles_of(kind, i, M, N);
        if (tiles > 0x7fffffffu) continue;
        for (uint32_t splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && (whole || tiles * splits > 256 * kResident[i] || 2 * splits > stages)) break;
            const double each = static_cast<double>((stages + splits - 1) / splits);
            double c = cost(kCosts[kind][i], kResident[i], tiles * splits, each, each);
            if (splits > 1) c += 2.5 + 1.6e-6 * splits * M * N * (gated_kind(kind) ? 2 : 1);   // (8 bytes of a part at 5 TB/s)
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
        const uint64_t a = tiles_of(kBF16AcrossB, i, M, N), b = tiles_of(kBF16AcrossBoth, i, M2, N2);
        if (a + b > 1u << 22) continue;        // (a workgroup for every tile, and a launch's work-items within 32 bits)
        const double c = cost(kCosts[kPair][i], kResident[i], a + b, static_cast<double>(a * stages + b * stages2) / static_cast<double>(a + b), stages > stages2 ? stages : stages2);
        if (c < least) {
            least = c;
            tile = i;
        }
    }
    return tile;
}

double product_tiles_cost(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages) { return choose_tile(kind, M, N, stages, false).cost; }

// Host only, not part of the interface: the tile's index, and 16 times the parts, that a product takes; the tile in which both backward products of a gated layer go together, or -1.
extern "C" int omc_internal_product_tile(int kind, uint32_t M, uint32_t N, uint32_t stages) {
    const TileChoice c = choose_tile(static_cast<ProductKind>(kind), M, N, stages, false);
    return c.tile + 16 * static_cast<int>(c.splits);
}
extern "C" int omc_internal_product_pair_tile(uint32_t M, uint32_t N, uint32_t K) {
    const uint32_t half = (N + 63) / 64;
    return product_pair_tile(M, K, 2 * half, 128 * half, K, (M + 63) / 64);
}

int launch_i8_plain(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_i8_gated(const TiledArgs &pa, bool c_bf16, hipStream_t st);
int launch_across_b(const TiledArgs &pa, bool whole, bool c_bf16, hipStream_t st);
int launch_across_both(const TiledArgs &pa, bool whole, bool c_bf16, hipStream_t st);

size_t product_workspace(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages) {
    const TileChoice c = choose_tile(kind, M, N, stages, false);
    return c.splits > 1 ? 4ull * c.splits * M * parts_columns(N) * (gated_kind(kind) ? 2 : 1) : 0;
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
