// omc_mx4_gemm: C[M x N] = A[M x K] B[N x K]^T + bias, both operands in MX4, on the scaled matrix instructions (32 x 32 results over 64 values).
//
// Codes and scales go from global memory straight into a ring of S LDS stages of 256 values of K: a row's stage is 128 bytes of codes, eight pieces of 16 bytes that are a block each, and 8 scale
// bytes.  (Rows of 64 bytes, stages of 128 values, would make a deeper ring, but the load path moves a cache line in two clocks, whole or half: 54 bytes a clock and compute unit with rows of
// 128 bytes, 27 with rows of 64.)  In step s of a stage's four, lane l multiplies block 2 (l / 32) + s % 2 + 4 (s / 2) of its row.  Which blocks meet in a step is
// free as long as both operands agree, and the scales are reordered before (mx4_image_pitch), so that a lane's four are a dword and a load of them is as dense as one of the codes:
// read from rows of K / 32 bytes, 8 bytes a row, they take as many cache lines as the codes (16384 x 8192 x 8192: 600 us with such loads, 490 without any scales).  Of an odd number of 128s the last
// stage's second half is its first one again, with scales of 2^-127 on both sides: what it adds is below 2^-240.
//
// Pieces are XOR-swizzled on their way in, so that the 16 that one read takes at a time lie on different ones of the 64 banks.  The B operand comes first in the instruction, and its
// tiles' row i is column 16 (i / 4 % 2) + 4 (i / 8) + i % 4: a lane then holds 16 neighbours of a row of C.
//
// 16384 x 8192 x 8192: 480 - 500 us, 4.5 PFLOP/s, the matrix cores busy 59 % of the time at a clock that the power limit sets: the instructions alone take 325 us, reading their fragments adds 65, the
// loads 60.  8192 x 4096 x 1024: 27 - 30 us; stores alone 13, products 10, loads 7, which all but add up.
//
// The fragments of a step are read while the step before is multiplied; a stage's last step is multiplied behind the barrier of the next one, under that one's first reads and loads.  A
// workgroup goes on to its next tile without a break: the loads run ahead of the products by S - 1 stages, whosever they are, and nothing waits for a tile's stores.  These overlap little all the same
// where tiles have few stages: all waves of a unit convert and store at the same time, and its matrix cores idle meanwhile.
#include <type_traits>

#include "omc_mma.h"
#include "omc_column_sums.h"
#include "omc_mx4.h"
#include "omc_pieces.h"

namespace omc {

// Keeps a product between the reads and loads that it is written between: without it the compiler gathers the products behind all of them.
__device__ __forceinline__ void stays_here(f32x16 &x) { asm volatile("" : "+v"(x)); }

constexpr uint32_t kCorner = 2560;             // LDS of a wave for its results on their way out

struct Mx4TileArgs {
    Mx4GemmArgs g;
    uint32_t tiles_m, tiles_n, splits, stages_per_split;
    bool streams;                              // C is more than the caches hold, in whole cache lines
};

// Two products whose tiles one launch deals out, the second one's, whose result is fp32, after the first one's; in workgroups behind theirs, which are `groups`, sums of columns.
struct Mx4PairArgs {
    Mx4TileArgs first, second;
    uint32_t groups;
    bool fours;
    ColumnSums sums;
};

// WM x WN waves of TM x TN matrix tiles, and LOADERS that load for all (0: every wave loads its share), OCC waves per SIMD.  SPLIT: the contraction is cut into parts, whose results go to g.parts in fp32.
// PAIR: two products.
template <int WM, int WN, int TM, int TN, int LOADERS, int S, int OCC, typename T, bool SPLIT, bool PAIR>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * (WM * WN + LOADERS), 64 * (WM * WN + LOADERS)))) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
void mx4_gemm_kernel(typename std::conditional<PAIR, Mx4PairArgs, Mx4TileArgs>::type ta) {
    constexpr int NW = WM * WN, kLoaders = LOADERS > 0 ? LOADERS : NW, BM = 32 * TM * WM, BN = 32 * TN * WN;
    constexpr int kALoads = BM / 8 / kLoaders, kBLoads = BN / 8 / kLoaders, kLoads = kALoads + kBLoads + 1;
    constexpr uint32_t kB = BM * 128, kS = kB + BN * 128, kStage = kS + (BM + BN) * 8, kScaleLoads = (BM + BN + 127) / 128, kCorners = S * kStage;
    constexpr int kStores = TM * TN * (T::kBytes == 2 && !SPLIT ? 2 : 4);
    static_assert(!PAIR || LOADERS > 0, "a wave that loads counts one type's stores");
    static_assert(BM % (8 * kLoaders) == 0 && BN % (8 * kLoaders) == 0 && kScaleLoads <= kLoaders && 256 % BM == 0 && 256 % BN == 0, "whole loads");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kCorners + NW * kCorner];
    auto product = [&](uint32_t which) {       // (field by field: the arguments stay where they are)
        if constexpr (PAIR) {
            const Mx4TileArgs &x = ta.first, &y = ta.second;
            auto of = [which](auto a, auto b) { return which == 0 ? a : b; };
            return Mx4TileArgs{{{of(x.g.a.codes, y.g.a.codes), of(x.g.a.scales, y.g.a.scales)}, {of(x.g.b.codes, y.g.b.codes), of(x.g.b.scales, y.g.b.scales)}, of(x.g.bias, y.g.bias),
                                of(x.g.c, y.g.c), of(x.g.ldc, y.g.ldc), of(x.g.M, y.g.M), of(x.g.N, y.g.N), of(x.g.K, y.g.K), nullptr},
                               of(x.tiles_m, y.tiles_m), of(x.tiles_n, y.tiles_n), 1, of(x.stages_per_split, y.stages_per_split), of(x.streams, y.streams)};
        } else {
            return ta;
        }
    };
    const uint32_t lds0 = lds_offset(lds);
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const uint32_t tiles_first = product(0).tiles_m * product(0).tiles_n;
    uint32_t groups = gridDim.x, items = SPLIT ? tiles_first * product(0).splits : tiles_first;
    if constexpr (PAIR) {
        groups = ta.groups;
        items += ta.second.tiles_m * ta.second.tiles_n;
        if (blockIdx.x >= groups) {
            float(*part)[32] = reinterpret_cast<float(*)[32]>(lds);
            // (with eight chains of fours the tiles' waves spill; fours are 255 at most)
            auto take = [&](auto chains, auto fours) { column_sums<NW + LOADERS, decltype(chains)::value, decltype(fours)::value>(ta.sums, blockIdx.x - groups, part); };
            if (ta.fours) ta.sums.count <= 64 ? take(UintTag<1>{}, BoolTag<true>{}) : take(UintTag<4>{}, BoolTag<true>{});
            else ta.sums.count <= 64 ? take(UintTag<1>{}, BoolTag<false>{}) : take(UintTag<8>{}, BoolTag<false>{});
            return;
        }
    }

    // Product, tile and part of a work item.  Workgroups go to the 8 dies in turn (the grid is a multiple of 8, or there is no second item).
    struct Place {
        uint32_t which, m0, n0, part, first, stages;
    };
    auto locate = [&](uint32_t item) {
        Place p;                               // (divisions go through vector registers)
        p.which = PAIR && item >= tiles_first ? 1 : 0;
        const Mx4TileArgs t = product(p.which);
        const uint32_t tiles = t.tiles_m * t.tiles_n, all_stages = ((t.g.K + 127) / 128 + 1) / 2;
        p.part = SPLIT ? __builtin_amdgcn_readfirstlane(item / tiles) : 0u;
        tile_of(item - (PAIR ? p.which * tiles_first : p.part * tiles), BM == 256 ? 4 : 8, t.tiles_m, t.tiles_n, p.m0, p.n0);
        p.m0 = __builtin_amdgcn_readfirstlane(p.m0) * BM;
        p.n0 = __builtin_amdgcn_readfirstlane(p.n0) * BN;
        p.first = SPLIT ? p.part * t.stages_per_split : 0u;
        p.stages = SPLIT ? min(t.stages_per_split, all_stages - p.first) : all_stages;
        return p;
    };

    // ---- global -> LDS: load i of a loader is the rows 8 (loader + kLoaders i) .. + 8 of an operand, lane l's piece l % 8 of row l / 8 (before the swizzle).  Rows past the end: the last one
    // again.
    const uint32_t loader = LOADERS > 0 ? wave - NW : wave;   // (LOADERS > 0: of the waves that load)
    const uint8_t *a_from, *b_from, *s_from;
    uint32_t off[kALoads + kBLoads];
    auto load_row = [&](uint32_t i) { return 8 * (loader + kLoaders * i) + (lane >> 3); };
    auto a_piece = [&](uint32_t i) { return 16 * ((lane & 7u) ^ (load_row(i) >> 1 & 7u)); };
    auto b_piece = [&](uint32_t i) { return 16 * ((lane & 7u) ^ ((load_row(i) >> 1 & 3u) + 4 * (load_row(i) >> 4 & 1u))); };
    const uint32_t s_unit = loader % kScaleLoads, s_row = 2 * (64 * s_unit + lane);                 // two rows' scales a lane (some waves bring the same)
    const uint64_t s_lanes = __ballot(s_row < BM + BN);
    uint32_t ask_item = blockIdx.x, ask_stage, ask_end, half_at;
    uint64_t s_pitch;
    uint64_t lanes = ~0ull;                    // that load: none once everything has been asked for
    auto upper_is_lower = [&]() {              // before half a stage
#pragma unroll
        for (uint32_t i = 0; i < kALoads + kBLoads; ++i) off[i] -= (i < kALoads ? a_piece(i) : b_piece(i - kALoads)) & 64u;
    };
    auto ask_for = [&](uint32_t item) {
        const Place p = locate(item);
        const Mx4GemmArgs g = product(p.which).g;
        const uint32_t k128 = (g.K + 127) / 128, row_bytes = k128 * 64;
        half_at = (k128 & 1u) != 0 ? k128 / 2 : ~0u;
        s_pitch = mx4_image_pitch(s_row < BM ? g.M : g.N);
        a_from = g.a.codes + static_cast<uint64_t>(p.m0) * row_bytes + p.first * 128;
        b_from = g.b.codes + static_cast<uint64_t>(p.n0) * row_bytes + p.first * 128;
        s_from = (s_row < BM ? g.a.scales + 8ull * (p.m0 + s_row) : g.b.scales + 8ull * (p.n0 + s_row - BM)) + p.first * s_pitch;
        const uint32_t last_m = g.M - 1 - p.m0, last_n = g.N - 1 - p.n0;
#pragma unroll
        for (uint32_t i = 0; i < kALoads; ++i) off[i] = min(load_row(i), last_m) * row_bytes + a_piece(i);
#pragma unroll
        for (uint32_t i = 0; i < kBLoads; ++i) off[kALoads + i] = min(load_row(i), last_n) * row_bytes + b_piece(i);
        ask_stage = p.first;
        ask_end = p.first + p.stages;
        if (ask_stage == half_at) upper_is_lower();
    };
    const uint32_t codes_to = lds0 + 1024 * loader, scales_to = lds0 + kS + 1024 * s_unit;
    struct From {
        const uint8_t *a, *b;
    };
    auto from_now = [&]() { return From{in_scalars(a_from), in_scalars(b_from)}; };
    auto load_one = [&](const From &from, uint32_t at, auto index) {
        constexpr uint32_t I = decltype(index)::value;
        if constexpr (I < kALoads) load_pieces<1024 * kLoaders * I>(from.a, off[I], codes_to + at, lanes);
        else if constexpr (I < kALoads + kBLoads) load_pieces<kB + 1024 * kLoaders * (I - kALoads)>(from.b, off[I], codes_to + at, lanes);
        else load_pieces<0>(s_from, scales_to + at, lanes & s_lanes);
    };
    auto load_stage = [&](uint32_t at) {
        const From from = from_now();
        for_constants<kLoads>([&](auto i) { load_one(from, at, i); });
    };
    auto next_stage = [&]() {
        if (lanes == 0) return;
        if (++ask_stage == ask_end) {
            ask_item += groups;
            if (ask_item < items) ask_for(ask_item);
            else lanes = 0;
        } else {
            a_from += 128;
            b_from += 128;
            s_from += s_pitch;
            if (ask_stage == half_at) upper_is_lower();
        }
    };

    uint32_t far = (S - 1) * kStage;           // the stage that is asked for
    if (LOADERS > 0 && wave >= NW) {                 // as many barriers as the other waves, which have one for every stage and one before the first
        ask_for(ask_item);
#pragma unroll
        for (uint32_t i = 0; i < S - 1; ++i) {
            load_stage(i * kStage);
            next_stage();
        }
        uint32_t stages = 0;
        for (uint32_t item = blockIdx.x; item < items; item += groups) stages += locate(item).stages;
        for (uint32_t j = 0; j <= stages; ++j) {
            if (lanes != 0) wait_loads_and_sync<(S - 2) * kLoads>();
            else wait_loads_and_sync<0>();
            load_stage(far);
            next_stage();
            far = far == (S - 1) * kStage ? 0 : far + kStage;
        }
        return;
    }

    // ---- LDS -> fragments
    const uint32_t r = lane & 31u, h = lane >> 5;
    const uint32_t a_row = 32 * TM * wm + r, b_col = 32 * TN * wn + 16 * ((r >> 2) & 1u) + 4 * (r >> 3) + (r & 3u);
    const uint32_t a_swz = (r >> 1) & 7u, b_swz = ((b_col >> 1) & 3u) + 4 * ((b_col >> 4) & 1u);
    f32x16 acc[TM][TN];
    i32x4 a[2][TM], b[2][TN];
    uint32_t sa[2][TM], sb[2][TN];             // of this stage, of the next
    uint32_t a_at[4], b_at[4];
#pragma unroll
    for (uint32_t s = 0; s < 4; ++s) {
        const uint32_t piece = 2 * h + s % 2 + 4 * (s / 2);
        a_at[s] = a_row * 128 + ((piece ^ a_swz) << 4);
        b_at[s] = kB + b_col * 128 + ((piece ^ b_swz) << 4);
    }
    const uint32_t sa_at = kS + a_row * 8 + 4 * h, sb_at = kS + (BM + b_col) * 8 + 4 * h;
    // read `index` of a step's: B's fragments first
    auto read_one = [&](uint32_t at, auto step, auto index) {
        constexpr uint32_t s = decltype(step)::value, I = decltype(index)::value;
        if constexpr (I < TN) b[s & 1][I] = *reinterpret_cast<const i32x4 *>(lds + at + b_at[s] + 4096 * I);
        else a[s & 1][I - TN] = *reinterpret_cast<const i32x4 *>(lds + at + a_at[s] + 4096 * (I - TN));
    };
    auto read_scale = [&](uint32_t at, auto index, auto set) {
        constexpr uint32_t I = decltype(index)::value, s = decltype(set)::value;
        if constexpr (I < TN) sb[s][I] = *reinterpret_cast<const uint32_t *>(lds + at + sb_at + 256 * I);
        else sa[s][I - TN] = *reinterpret_cast<const uint32_t *>(lds + at + sa_at + 256 * (I - TN));
    };
    constexpr int kReads = TM + TN, kProducts = TM * TN;
    uint32_t cur = 0;                          // the stage that is read
    // The products of step s, and beside them the reads of the next step; after a stage's last one of the next stage, with its scales, and the loads of the stage that is asked for.
    auto multiply = [&](auto step) {
        constexpr uint32_t s = decltype(step)::value, N = (s + 1) % 4;
        constexpr int kR = s == 3 ? 2 * kReads : kReads, kL = s == 3 && LOADERS == 0 ? kLoads : 0;
        const From from = kL > 0 ? from_now() : From{};
        for_constants<kProducts>([&](auto product) {
            constexpr int P = decltype(product)::value, i = P / TN, j = P % TN;
            constexpr int R0 = P * kR / kProducts, R1 = (P + 1) * kR / kProducts, L0 = P * kL / kProducts, L1 = (P + 1) * kL / kProducts;
            for_constants<R1 - R0>([&](auto x) {
                constexpr int I = R0 + decltype(x)::value;
                if constexpr (I < kReads) read_one(cur, UintTag<N>{}, UintTag<I>{});
                else read_scale(cur, UintTag<I - kReads>{}, UintTag<1>{});
            });
            for_constants<L1 - L0>([&](auto x) { load_one(from, far, UintTag<L0 + decltype(x)::value>{}); });
            acc[i][j] = mx4_multiply_32<s>(b[s & 1][j], sb[0][j], a[s & 1][i], sa[0][i], acc[i][j]);
            stays_here(acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // Waits for the next stage: it is there when at most the loads of the S - 2 after it, and the stores behind loads of its own age, are on their way.  (At the end it is nothing that is
    // waited for, read and asked for.  Loads without lanes are not relied on to count.)
    uint32_t behind = 0;                       // so many stages yet that were asked for before the last stores
    auto wait_for_next = [&]() {
        constexpr int kLater = (S - 2) * kLoads;
        if (LOADERS > 0) sync_lds();
        else if (lanes == 0) wait_loads_and_sync<0>();
        else if (behind > 0) wait_loads_and_sync<(kLater + kStores < 63 ? kLater + kStores : 63)>();
        else wait_loads_and_sync<kLater>();
        behind -= behind > 0 ? 1 : 0;
        cur = cur == (S - 1) * kStage ? 0 : cur + kStage;
        if (LOADERS == 0) far = far == (S - 1) * kStage ? 0 : far + kStage;
    };

    if constexpr (LOADERS > 0) {
        sync_lds();
    } else {
        ask_for(ask_item);
#pragma unroll
        for (uint32_t i = 0; i < S - 1; ++i) {
            load_stage(i * kStage);
            next_stage();
        }
        if (lanes != 0) wait_loads_and_sync<(S - 2) * kLoads>();
        else wait_loads_and_sync<0>();
        load_stage(far);
        next_stage();
    }
    for_constants<kReads>([&](auto i) {
        read_one(0, UintTag<0>{}, i);
        read_scale(0, i, UintTag<0>{});
    });
    for (uint32_t item = blockIdx.x; item < items; item += groups) {
        const Place p = locate(item);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
        for (uint32_t left = p.stages; left > 0; --left) {
            multiply(UintTag<0>{});
            multiply(UintTag<1>{});
            multiply(UintTag<2>{});
            wait_for_next();
            multiply(UintTag<3>{});
            if (LOADERS == 0) next_stage();
#pragma unroll
            for (int i = 0; i < TM; ++i) sa[0][i] = sa[1][i];
#pragma unroll
            for (int i = 0; i < TN; ++i) sb[0][i] = sb[1][i];
        }

        // ---- through the wave's own corner of LDS, so that 128 bytes of a row are stored together (64 of a bf16 result where a wave has one tile across): halves of cache lines from two tiles in turn
        // made 12 - 18 % more traffic to memory, and 8192 x 4096 x 1024 took 28.4 us, 27 with whole ones
        const Mx4TileArgs of = product(p.which);
        const Mx4GemmArgs &g = of.g;
        const bool stored = p.m0 + BM <= g.M && p.n0 + BN <= g.N;   // a whole tile
        auto store = [&](auto type) {
            typedef decltype(type) Out;
            constexpr uint32_t kTogether = Out::kBytes == 2 && TN % 2 == 0 ? 2 : 1;   // tiles side by side: 64 columns in bf16 are a cache line
            constexpr uint32_t kRun = 16 / Out::kBytes, kLanes = 32 * kTogether / kRun, kRows = 64 / kLanes, kPitch = 32 * kTogether * Out::kBytes + 16;
            constexpr uint32_t kPass = kPitch > 80 ? 16 : 32;
            static_assert(kPass * kPitch <= kCorner, "fits");
            uint8_t *corner = lds + kCorners + wave * kCorner;
            typename Out::type *c;
            uint64_t ldc;
            if constexpr (SPLIT) {
                c = g.parts + static_cast<uint64_t>(p.part) * g.M * g.N;
                ldc = g.N;
            } else {
                c = static_cast<typename Out::type *>(g.c);
                ldc = g.ldc;
            }
            const uint32_t s_row = lane / kLanes, s_col = kRun * (lane % kLanes);
            const bool streams = !SPLIT && of.streams;
#pragma unroll
            for (uint32_t j0 = 0; j0 < TN; j0 += kTogether) {
                const uint32_t n = p.n0 + 32 * (TN * wn + j0) + s_col;
                float bias[kTogether][16];    // of the lane's 16 columns, by scalar loads, which wait for none of the loads on their way
                const bool whole_bias = !SPLIT && g.bias && stored;
#pragma unroll
                for (uint32_t jj = 0; jj < kTogether; ++jj) {
                    const uint32_t n_tile = p.n0 + 32 * (TN * wn + j0 + jj);
                    if (whole_bias) {
                        const __attribute__((address_space(4))) float *from = reinterpret_cast<const __attribute__((address_space(4))) float *>(reinterpret_cast<uintptr_t>(g.bias + n_tile));
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) bias[jj][e] = h == 0 ? from[e] : from[16 + e];
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < 16; ++e) bias[jj][e] = 0.0f;
                        if (!SPLIT && g.bias) {
#pragma unroll
                            for (uint32_t e = 0; e < 16; ++e) bias[jj][e] = g.bias[min(n_tile + 16 * h + e, g.N - 1)];
                        }
                    }
                }
#pragma unroll
                for (uint32_t i = 0; i < TM; ++i)
#pragma unroll
                    for (uint32_t pass = 0; pass < 32 / kPass; ++pass) {
                        if (kPass == 32 || r / kPass == pass) {
#pragma unroll
                            for (uint32_t jj = 0; jj < kTogether; ++jj) {
                                float v[16];
#pragma unroll
                                for (uint32_t e = 0; e < 16; ++e) v[e] = acc[i][j0 + jj][e] + bias[jj][e];
                                uint8_t *to = corner + (r % kPass) * kPitch + (32 * jj + 16 * h) * Out::kBytes;
                                if constexpr (Out::kBytes == 4) {
#pragma unroll
                                    for (uint32_t e = 0; e < 4; ++e) *reinterpret_cast<f32x4 *>(to + 16 * e) = f32x4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
                                } else {
#pragma unroll
                                    for (uint32_t e = 0; e < 2; ++e)
                                        *reinterpret_cast<u32x4 *>(to + 16 * e) = u32x4{to_bf16_pair(v[8 * e], v[8 * e + 1]), to_bf16_pair(v[8 * e + 2], v[8 * e + 3]),
                                                                                        to_bf16_pair(v[8 * e + 4], v[8 * e + 5]), to_bf16_pair(v[8 * e + 6], v[8 * e + 7])};
                                }
                            }
                        }
                        lanes_exchange();
#pragma unroll
                        for (uint32_t k = 0; k < kPass / kRows; ++k) {
                            const u32x4 w = *reinterpret_cast<const u32x4 *>(corner + (kRows * k + s_row) * kPitch + 16 * (lane % kLanes));
                            const uint32_t m = p.m0 + 32 * (TM * wm + i) + kPass * pass + kRows * k + s_row;
                            typename Out::type *to = c + m * ldc + n;
                            if (streams && stored) {
                                __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(to));
                            } else if (stored || (m < g.M && n + kRun <= g.N)) {
                                __builtin_memcpy(to, &w, 16);
                            } else if (m < g.M) {
#pragma unroll
                                for (uint32_t e = 0; e < kRun; ++e)
                                    if (n + e < g.N) {
                                        if constexpr (Out::kBytes == 4) to[e] = __uint_as_float(w[e]);
                                        else to[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                                    }
                            }
                        }
                        lanes_exchange();
                    }
            }
        };
        if constexpr (SPLIT) store(F32{});
        else if constexpr (PAIR && T::kBytes == 2) p.which == 0 ? store(T{}) : store(F32{});
        else store(T{});
        behind = stored ? S - 1 : 0;
    }
}

// The parts of a split contraction, added in order.  512 x 512 x 65536 in four parts: 5.0 us after a product of 25.
template <typename T>
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4GemmArgs g, uint32_t splits) {
    const uint32_t n = 4 * (blockIdx.x * 64 + (threadIdx.x & 63u)), m = blockIdx.y * 4 + (threadIdx.x >> 6);
    if (m >= g.M || n >= g.N) return;
    const uint32_t left = g.N - n;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t s = 0; s < splits; ++s) {
        const float *p = g.parts + (static_cast<uint64_t>(s) * g.M + m) * g.N + n;
        float w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (left >= 4) {
            __builtin_memcpy(w, p, 16);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (e < left) w[e] = p[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    if (g.bias) {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) v[e] += g.bias[min(n + e, g.N - 1)];
    }
    store_run<T, 4>(static_cast<typename T::type *>(g.c) + m * g.ldc + n, v, left);
}

// Which tile a product takes, and into how many parts its contraction is cut, by an estimate of the time in us: `base` is a launch; `alone` a stage of workgroups that nothing else slows down,
// `resident` of them on a compute unit; `busy` what a stage costs per workgroup of a unit where all units have some (of the last workgroups' unevenness over the units `uneven` counts); `store` the
// stores of 256 tiles, `store_lines` where a row of C is whole cache lines.  Fitted to 408 sizes (301 for the largest tile) of 33 .. 16384 x 64 .. 8192 x 64 .. 8192, half of them with whole lines,
// bf16 results: 6 - 9 % (standard deviation).  (The result's type is not asked for: fp32 results, dW's among them, are chosen for by the same figures.)  On these the chosen tile takes 0.7 % longer than the best one, at worst 17 % (13450 x 3516 x 1101), but for some of a few us.
// 16384 x 8192 x 8192: 256 x 256 480 - 500 us, 128 x 128 628, 64 x 64 940; 8192 x 4096 x 1024: 27 - 30, 28 - 33, 42; 4096 x 1024 x 8192: 49, 22, 32; 1003 x 971 x 243: 10.4, 5.1, 4.1.
// The largest tile's eight waves load for themselves; beside the others are four that only load (64 x 8192 x 8192 in tiles of 64 x 64: 12.8 us without them, 10 with).  128 x 128 has three stages
// and the unit for itself: a stage more on its way counts for more than a second workgroup with two stages where each unit has one tile (4096 x 1024 x 8192: 26 us), and for less in a
// row of tiles with few stages each (8192 x 4096 x 1024: 29 us).
// Cutting the contraction costs a second launch, 3.2 us, and the parts' way through memory; it is worth that for few tiles of a very long one.
struct Mx4Tile {
    uint32_t bm, bn, resident;
    bool cut;
    double base, alone, busy, uneven, store, store_lines;
};
static constexpr Mx4Tile kMx4Tiles[] = {
    {256, 256, 1, false, -0.109, 1.199, 2.024, 0.591, 10.182, 8.107}, {128, 128, 1, true, 2.632, 0.085, 0.597, 0.566, 1.92, 1.404}, {64, 64, 2, true, 2.979, 0.012, 0.229, 0.848, 0.519, 0.46},
};
static double cost(const Mx4Tile &t, uint32_t splits, uint32_t M, uint32_t N, uint32_t K) {
    const uint32_t stages = (K + 255) / 256;
    const uint64_t items = static_cast<uint64_t>((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn) * splits, units = (items + 255) / 256, rounds = (items + 256 * t.resident - 1) / (256 * t.resident);
    const double per_unit = static_cast<double>(items) / 256.0, steps = (stages + splits - 1) / splits;
    const double alone = t.alone * steps * static_cast<double>(rounds), busy = t.busy * steps * (per_unit + t.uneven * (static_cast<double>(units) - per_unit));
    const double whole = t.base + (alone > busy ? alone : busy) + (N % 64 == 0 ? t.store_lines : t.store) * (per_unit > 1.0 ? per_unit : 1.0);
    return splits > 1 ? whole + 3.2 + 2e-6 * splits * M * N : whole;   // (8 bytes of a part at 4 TB/s)
}
struct Mx4Choice {
    int tile;
    uint32_t splits;
    double cost;
};
static Mx4Choice choose(uint32_t M, uint32_t N, uint32_t K, bool whole) {   // whole: not cut
    const uint32_t stages = (K + 255) / 256;
    Mx4Choice best{-1, 1, 0.0};
    for (int i = 0; i < 3; ++i) {
        const Mx4Tile &t = kMx4Tiles[i];
        const uint64_t tiles = static_cast<uint64_t>((M + t.bm - 1) / t.bm) * ((N + t.bn - 1) / t.bn);
        for (uint32_t splits = 1; splits <= 16; splits *= 2) {
            if (splits > 1 && (whole || !t.cut || tiles * splits > 256 || splits > stages)) break;
            const double c = cost(t, splits, M, N, K);
            if (best.tile < 0 || c < best.cost) best = Mx4Choice{i, splits, c};
        }
    }
    const uint32_t each = (stages + best.splits - 1) / best.splits;
    best.splits = (stages + each - 1) / each;
    return best;
}
// Host only, not part of the interface: the tile's index, and 16 times the parts, that a product takes.
extern "C" int omc_internal_mx4_tile(uint32_t M, uint32_t N, uint32_t K) {
    const Mx4Choice c = choose(M, N, K, false);
    return c.tile + 16 * static_cast<int>(c.splits);
}

size_t mx4_gemm_workspace(uint32_t M, uint32_t N, uint32_t K) {
    const Mx4Choice c = choose(M, N, K, false);
    return c.splits > 1 ? 4ull * c.splits * M * N : 0;
}

template <int WM, int WN, int TM, int TN, int LOADERS, int S, int OCC, bool CUT, typename T>
static void launch_tile(const Mx4TileArgs &ta, hipStream_t st) {
    constexpr uint32_t kLds = 32 * (TM * WM + TN * WN) * S * 136 + WM * WN * kCorner, kByLds = 163840 / kLds, kByWaves = 4 * OCC / (WM * WN + LOADERS);
    const uint32_t items = ta.tiles_m * ta.tiles_n * ta.splits, most = 256 * (kByLds < kByWaves ? kByLds : kByWaves);
    const dim3 grid(items < most ? items : most), block(64 * (WM * WN + LOADERS));
    if constexpr (CUT) {
        if (ta.splits > 1) {
            mx4_gemm_kernel<WM, WN, TM, TN, LOADERS, S, OCC, T, true, false><<<grid, block, 0, st>>>(ta);
            return;
        }
    }
    mx4_gemm_kernel<WM, WN, TM, TN, LOADERS, S, OCC, T, false, false><<<grid, block, 0, st>>>(ta);
}

// Stores past the caches (8 x 4 MB of L2): 8192 x 4096 in bf16, K of 1024, in tiles of 128 x 128: 31.3 -> 29.8 us; 16384 x 8192 x 8192 in these: 667 -> 630 us.  Of parts of cache lines it costs more
// than it gives (2948 x 3118 x 932: 13.8 us, 16 - 23 with it), and 0.3 us where C stays in the caches.
template <typename T>
static bool past_caches(const Mx4GemmArgs &g) {
    const uint64_t pitch = g.ldc * T::kBytes;
    return g.M * pitch >= 32u << 20 && (pitch | reinterpret_cast<uintptr_t>(g.c)) % 128 == 0;
}

template <typename T>
static int launch(const Mx4GemmArgs &ga, bool whole, hipStream_t st) {
    const Mx4Choice c = choose(ga.M, ga.N, ga.K, whole);
    const Mx4Tile &t = kMx4Tiles[c.tile];
    const uint32_t stages = (ga.K + 255) / 256;
    const bool streams = past_caches<T>(ga);
    const Mx4TileArgs ta{ga, (ga.M + t.bm - 1) / t.bm, (ga.N + t.bn - 1) / t.bn, c.splits, (stages + c.splits - 1) / c.splits, streams};
    switch (c.tile) {
        case 0: launch_tile<4, 2, 2, 4, 0, 2, 2, false, T>(ta, st); break;
        case 1: launch_tile<2, 4, 2, 1, 4, 3, 3, true, T>(ta, st); break;
        default: launch_tile<2, 2, 1, 1, 4, 4, 4, true, T>(ta, st); break;
    }
    if (c.splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return static_cast<int>(e);
        mx4_join_kernel<T><<<dim3((ga.N + 255) / 256, (ga.M + 3) / 4), dim3(256), 0, st>>>(ga, c.splits);
    }
    return static_cast<int>(hipGetLastError());
}

// Tile in which two products of M x N over K and M2 x N2 over K2 take the least time together, uncut, and that time.
static int best_pair(uint32_t M, uint32_t N, uint32_t K, uint32_t M2, uint32_t N2, uint32_t K2, double &time) {
    int tile = -1;
    for (int i = 1; i < 3; ++i) {
        const double c = cost(kMx4Tiles[i], 1, M, N, K) + cost(kMx4Tiles[i], 1, M2, N2, K2) - kMx4Tiles[i].base;
        if (tile < 0 || c <= time) {
            time = c;
            tile = i;
        }
    }
    return tile;
}
// Both products of a backward pass are uncut and in tiles, so that they can go together, where by the estimate that takes no more than each its own way, with a launch of its own and one for dbias' sums.
// Asked of the sizes alone: tiles add up the contraction in the same order, whichever they are, so that a gradient's bits do not depend on what is asked for beside it.  Backward of a linear layer with its bias,
// 64 x 64 x 64: 13.4 us in four launches, 8.9 in two; 1003 x 971 x 243 in fp32: 16.9 and 11.1; 4057 x 832 x 562 in bf16: 24.4 and 19.2;
// 8192 x 1024 x 4096: 78.7 and 75.3; 4096 x 2048 x 2048: 46.2 and 41.3.
// A product of few rows would go another way by itself (mx4_few), which the estimate does not know.  Where its contraction is short both ways take the same within 1 or 2 us, and together pays; where
// it is long it loses by itself more than both gain: all three gradients apart and together, and the product's alone in its own way and in tiles, 1 x 64 x 64 12.6 and 10.2,
// dX 5.4 and 6.3 us; 32 x 1024 x 4096 17.9 and 16.2, 6.7 and 7.4; 16 x 4096 x 4096 29.0 and 25.7, 8.1 and 11.0; 1 x 8192 x 2048 30.5 and 29.5, 8.1 and 14.3; 8 x 8192 x 8192 68.9 and 71.3; dW of 1000 x 1000 x 32 15.2
// and 11.9, 8.5 and 9.6; 8192 x 300 x 20 20.5 and 19.6, 12.5 and 17.0; 16000 x 300 x 32 27.8 and 28.4, 18.9 and 26.0.  Apart, dW of few rows has a rounding of dY to itself: 8192 x 4096 x 32 50.4 and 37.7, 28.6 and 31.4.
constexpr double kSumsLaunch = 2.5;
constexpr uint32_t kLongAlone = 4096;
constexpr uint64_t kRoundedTwice = 1u << 23;
bool mx4_backward_whole(uint32_t M, uint32_t N, uint32_t K) {
    if (mx4_few(M, K, N) && N > kLongAlone) return false;
    if (mx4_few(K, N, M) && M > kLongAlone && static_cast<uint64_t>(M) * N <= kRoundedTwice) return false;
    double together;
    best_pair(M, K, N, K, N, M, together);
    return together <= choose(M, K, N, false).cost + choose(K, N, M, false).cost + kSumsLaunch;
}
// (Of few rows, uncut tiles in a launch of their own take longer than the estimate says: 16 x 4096 x 4096 without dbias 30.3 us, 25.5 together.)
int mx4_pair_tile(uint32_t M, uint32_t N, uint32_t K, bool sums) {
    double together;
    const int tile = best_pair(M, K, N, K, N, M, together);
    return mx4_few(M, K, N) || mx4_few(K, N, M) || together <= choose(M, K, N, true).cost + choose(K, N, M, true).cost + (sums ? kSumsLaunch : 0.0) ? tile : -1;
}
// Host only, not part of the interface: the tile in which both products of a backward pass with its bias go together; -1: each in a launch of its own.
extern "C" int omc_internal_mx4_pair_tile(uint32_t M, uint32_t N, uint32_t K) { return mx4_backward_whole(M, N, K) ? mx4_pair_tile(M, N, K, true) : -1; }

template <typename T>
static int launch_pair(int tile, const Mx4GemmArgs &ga, const Mx4GemmArgs &gb, const ColumnSums &sums, bool fours, hipStream_t st) {
    const uint32_t b = kMx4Tiles[tile].bm, most = 256 * kMx4Tiles[tile].resident;
    auto tiles = [b](const Mx4GemmArgs &g, bool streams) { return Mx4TileArgs{g, (g.M + b - 1) / b, (g.N + b - 1) / b, 1, (g.K + 255) / 256, streams}; };
    Mx4PairArgs pa{tiles(ga, past_caches<T>(ga)), tiles(gb, past_caches<F32>(gb)), 0, fours, sums};
    const uint32_t items = pa.first.tiles_m * pa.first.tiles_n + pa.second.tiles_m * pa.second.tiles_n;
    pa.groups = items < most ? items : most;
    const dim3 grid(pa.groups + (sums.width + 31) / 32);
    if (tile == 1) mx4_gemm_kernel<2, 4, 2, 1, 4, 3, 3, T, false, true><<<grid, dim3(768), 0, st>>>(pa);
    else mx4_gemm_kernel<2, 2, 1, 1, 4, 4, 4, T, false, true><<<grid, dim3(512), 0, st>>>(pa);
    return static_cast<int>(hipGetLastError());
}
int launch_mx4_pair(int tile, const Mx4GemmArgs &ga, bool bf16, const Mx4GemmArgs &gb, const float *parts, uint32_t count, bool fours, float *dbias, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const ColumnSums sums{parts, count, dbias ? gb.N : 0, dbias ? gb.N : 0, dbias, nullptr};
    return bf16 ? launch_pair<BF16>(tile, ga, gb, sums, fours, st) : launch_pair<F32>(tile, ga, gb, sums, fours, st);
}

int launch_mx4_gemm(const Mx4GemmArgs &ga, bool whole, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch<BF16>(ga, whole, st) : launch<F32>(ga, whole, st);
}

}  // namespace omc
