// The gated linear layer's forward product on bf16 in tiles (see omc_tiles.h), and which tile a product takes.
#include "omc_tiles.h"

namespace omc {

// By an estimate of the time in us: `base` is a launch; `alone` a stage of workgroups that nothing else slows down, `resident` of them on a compute unit; `busy` what a stage costs per workgroup of a unit where all units have some
// (of the last workgroups' unevenness over the units `uneven` counts); `store` the end of 256 tiles.  A row for every kind of product, the last one for both backward products in one launch, which takes no less than its longest
// contraction.  Fitted to 1500 sizes of 33 .. 16384 x 64 .. 8192 x 64 .. 8192 in bf16, 60 % of them with whole cache lines: 4 - 18 % (standard deviation).  On these the chosen way takes 0.8 - 1.7 % longer than the best one (both
// backward products together or apart: 3 %), at worst 20 - 40 %.
// In 256 x 256, 256 x 128, 128 x 128, 64 x 64: 8192 x 4096 x 1024 gated with slopes 143 us, 170, 166, 300; without 110, 127, 127, 218; plain in 8 bits 40, 46, 46, 73; 8192 x 1024 x 4096 in 8 bits 48, 36, 37, 54.
// 128 x 128 has two stages and two workgroups on a unit; with four stages, eight waves and the unit for itself 8192 x 4096 x 1024, gated, took 7 % longer.  64 x 64 is bound by its fragments' reads: a ring of eight stages, or
// whole stages of fragments read ahead, do not help it.
// A cut costs a second launch and the parts' way through memory.
struct TileCost {
    double base, alone, busy, uneven, store;
};
static constexpr int kPair = 5;
static constexpr TileCost kCosts[6][4] = {
    {{3.466, 0.337, 1.563, 0.488, 7.359}, {2.402, 0.457, 1.072, 0.428, 4.107}, {3.841, 0.328, 0.542, 0.732, 1.766}, {3.612, 0.244, 0.176, 1.296, 0.717}},
    {{4.011, 1.148, 1.016, 0.5, 6.658}, {3.992, 0.478, 0.808, 0.675, 3.359}, {4.219, 0.512, 0.396, 1.099, 1.552}, {3.664, 0.267, 0.171, 1.308, 0.703}},
    {{0.0, 1.13, 0.1, 0.5, 13.894}, {2.922, 0.058, 0.81, 0.679, 6.142}, {3.016, 0.578, 0.401, 1.109, 3.066}, {3.502, 0.292, 0.17, 1.385, 1.221}},
    {{3.21, 1.116, 1.0, 0.5, 6.889}, {3.37, 0.0, 0.782, 0.783, 2.987}, {2.343, 0.591, 0.349, 1.276, 2.005}, {3.259, 0.279, 0.174, 1.207, 0.559}},
    {{13.282, 1.166, 0.295, 0.5, 14.331}, {8.797, 0.568, 0.767, 0.878, 7.586}, {3.843, 0.633, 0.355, 1.452, 4.038}, {3.567, 0.271, 0.182, 1.415, 0.82}},
    {{0.0, 1.042, 1.365, 0.679, 18.915}, {7.069, 0.678, 0.801, 0.908, 6.896}, {0.0, 0.637, 0.362, 1.654, 4.634}, {2.755, 0.29, 0.186, 1.903, 1.317}},
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
