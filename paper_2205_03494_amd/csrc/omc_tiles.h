// C[M x N] = A B^T in tiles, on 8-bit integers or bf16: the kernel's body, instantiated by omc_i8_gemm.hip, omc_gated.hip and omc_gated_grad.hip.
//
// Both types' matrix instructions take 16 bytes of a row in a lane (16 x 16 results over 64 values of 8 bits or 32 of bf16), so that one kernel serves both.  Operands go from global memory straight into a
// ring of S LDS stages of 128 bytes of K (8 bits) or 64 k (bf16).
//   Along K: a row's stage is 128 bytes, eight pieces of 16, XOR-swizzled by half the row on their way in: the sixteen rows of a read lie on different banks.
//   Across K (a row of the operand for every k, bf16): the stage's 64 rows as they are, fragments by the transposing read (of 16 lanes that point at four rows x 16 columns, lane c receives column
//   c's four rows).  The 64-byte groups of a row are exchanged by the lowest bits of the row and the 16-byte pieces in them by its bit 3.
// A stage has two steps.  B's rows are the instruction's first operand: a lane then holds four neighbours of a row of C.  A gated product's tile holds rows of both its matrices, every
// wave the same columns of the two, and the gate needs no other wave's sums.
//
// The order of reads and products is written down: a column of tiles at a time, A's fragments of the next step beside the first products, B's each as soon as its predecessor has been multiplied for the last time; a
// stage's second step is multiplied behind the barrier of the next stage, under that one's first reads and the loads of the one that is asked for.  A workgroup's tiles follow each other without a gap: the loads
// of the next tile are under way while the last stages of this one are multiplied.
// What bounds it: large products the power limit (16384 x 8192 x 8192 in 8 bits 780 - 830 us, 2.65 - 2.8 POP/s, the library's 957 - 978; gated 8192 x 4096 x 4096 in bf16 412 us, 1.33 PFLOP/s); a gated one with a short contraction the
// way of its results, 200 MB with slopes, which the products hide in part: 8192 x 4096 x 1024 124 - 145 us, 40 of which its results take by themselves at 5 TB/s, and its products 95.
#pragma once
#include "omc_column_sums.h"
#include "omc_finish.h"
#include "omc_pieces.h"

namespace omc {

template <bool I8>
struct SumOf {
    typedef f32x4 type;
    typedef float scalar;
};
template <>
struct SumOf<true> {
    typedef i32x4 type;
    typedef int scalar;
};
__device__ __forceinline__ f32x4 multiply_16(i32x4 a, i32x4 b, f32x4 acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ i32x4 multiply_16(i32x4 a, i32x4 b, i32x4 acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc, 0, 0, 0); }

struct TileGrid {
    TiledArgs g;
    uint32_t tiles_m, tiles_n, splits, stages_per_split;
};

// Parts of a cut contraction lie in rows of whole fours of columns, so that a lane's four are there for all lanes.
constexpr uint64_t parts_columns(uint32_t N) { return (static_cast<uint64_t>(N) + 3) / 4 * 4; }

// Two tiles side by side in bf16, so that a lane has eight neighbours: of tile 0 (even) or 1 (odd lane / 16), columns 8 (lane / 32) ..
__device__ __forceinline__ u32x4 side_by_side_bf16(const float (&x)[4], const float (&y)[4]) {
    const auto lo = __builtin_amdgcn_permlane16_swap(to_bf16_pair(x[0], x[1]), to_bf16_pair(y[0], y[1]), false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(to_bf16_pair(x[2], x[3]), to_bf16_pair(y[2], y[3]), false, false);
    return u32x4{static_cast<uint32_t>(lo[0]), static_cast<uint32_t>(hi[0]), static_cast<uint32_t>(lo[1]), static_cast<uint32_t>(hi[1])};
}

// WM x WN waves of TM x TN matrix tiles, S stages.  GATED: the tile's columns are TN / 2 tiles of a wave of either matrix.  SPLIT: the contraction is cut, sums go to parts as they are.
template <bool I8_, bool GATED_, bool ACROSS_A_, bool ACROSS_B_, int WM_, int WN_, int TM_, int TN_, int S_, bool SPLIT_, typename T_>
struct Tiles {
    static constexpr bool I8 = I8_, GATED = GATED_, ACROSS_A = ACROSS_A_, ACROSS_B = ACROSS_B_, SPLIT = SPLIT_;
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, S = S_;
    typedef T_ T;
    static constexpr int NW = WM * WN, BM = 16 * TM * WM, BN = 16 * TN * WN, kColsOut = GATED ? BN / 2 : BN, TH = GATED ? TN / 2 : TN;
    static constexpr uint32_t kB = BM * 128, kStage = kB + BN * 128;
    // scales and biases of a tile's columns and scales of its rows, in LDS, for every tile that is under way (a tile may have one stage): a slot is kLines lines of kColsOut floats and BM floats
    static constexpr uint32_t kLines = SPLIT || ACROSS_B ? 0 : (I8 ? 2 : 1) * (GATED ? 2 : 1), kSlot = 4 * (kLines * kColsOut + (I8 && !SPLIT ? BM : 0)), kSlots = S + 2, kParams = S * kStage;
    static constexpr uint32_t kLds = kParams + kSlots * kSlot;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0 && (!GATED || TN % 2 == 0) && !(I8 && (ACROSS_A || ACROSS_B)) && !(GATED && ACROSS_B), "whole loads");
};

// The tiles that workgroup `block` of `groups` takes.
template <typename C>
__device__ __forceinline__ void tiles_body(const TileGrid &tg, const uint32_t block, const uint32_t groups, uint8_t *lds) {
    constexpr bool I8 = C::I8, GATED = C::GATED, ACROSS_A = C::ACROSS_A, ACROSS_B = C::ACROSS_B, SPLIT = C::SPLIT;
    constexpr int WN = C::WN, TM = C::TM, TN = C::TN, S = C::S, NW = C::NW, BM = C::BM, BN = C::BN, kColsOut = C::kColsOut, TH = C::TH;
    constexpr uint32_t kB = C::kB, kStage = C::kStage, kLines = C::kLines, kSlot = C::kSlot, kSlots = C::kSlots, kParams = C::kParams;
    typedef typename C::T T;
    constexpr int kALoads = BM / 8 / NW, kBLoads = BN / 8 / NW, kLoads = kALoads + kBLoads;
    constexpr int kParamLoads = (kSlot / 4 + 64 * NW - 1) / (64 * NW);
    constexpr int kStores = TM * (T::kBytes == 2 && TH % 2 == 0 ? TH / 2 : TH);
    typedef typename SumOf<I8>::type Sum;
    const TiledArgs &g = tg.g;
    const uint32_t lds0 = lds_offset(lds);
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const uint32_t tiles = tg.tiles_m * tg.tiles_n, items = SPLIT ? tiles * tg.splits : tiles;

    struct Place {
        uint32_t m0, n0, part, first, stages;
    };
    auto locate = [&](uint32_t item) {
        Place p;
        p.part = SPLIT ? __builtin_amdgcn_readfirstlane(item / tiles) : 0u;
        tile_of(item - p.part * tiles, BM == 256 ? (GATED ? 2 : 4) : 8, tg.tiles_m, tg.tiles_n, p.m0, p.n0);
        p.m0 = __builtin_amdgcn_readfirstlane(p.m0) * BM;
        p.n0 = __builtin_amdgcn_readfirstlane(p.n0) * kColsOut;
        p.first = SPLIT ? p.part * tg.stages_per_split : 0u;
        p.stages = SPLIT ? min(tg.stages_per_split, g.stages - p.first) : g.stages;
        return p;
    };

    // ---- global -> LDS, 1 KB a load.  Rows, or columns' pieces, past the end: the last ones again.
    auto across_row = [&](auto width, uint32_t i) { return (wave + NW * i) * (512 / decltype(width)::value) + lane / (decltype(width)::value / 8); };
    auto across_piece = [&](auto width, uint32_t i) {
        constexpr uint32_t W = decltype(width)::value;
        const uint32_t row = across_row(width, i), slot = lane % (W / 8), swz = W >= 128 ? row & 3u : (row >> 1) & 1u;
        return (((slot >> 2) ^ swz) << 2) | ((slot & 3u) ^ ((row >> 2) & 2u));
    };
    auto load_row = [&](uint32_t i) { return 8 * (wave + NW * i) + (lane >> 3); };
    auto load_piece = [&](uint32_t i) { return 16 * ((lane & 7u) ^ (load_row(i) >> 1 & 7u)); };
    const uint8_t *a_from, *b_from, *b2_from = nullptr;
    uint32_t off[kLoads];
    uint32_t ask_item = block, ask_stage, ask_end, ask_slot = 0, slot = 0;
    uint64_t lanes = ~0ull;                    // none once everything has been asked for
    const uint64_t a_step = ACROSS_A ? 64 * g.a_pitch : 128, b_step = ACROSS_B ? 64 * g.b_pitch : 128;
    auto ask_for = [&](uint32_t item) {
        const Place p = locate(item);
        if constexpr (ACROSS_A) {
            a_from = static_cast<const uint8_t *>(g.a) + p.first * a_step;
            for_constants<kALoads>([&](auto i) { off[i.value] = across_row(UintTag<BM>{}, i.value) * static_cast<uint32_t>(g.a_pitch) + 2 * min(p.m0 + 8 * across_piece(UintTag<BM>{}, i.value), g.M - 8); });
        } else {
            a_from = static_cast<const uint8_t *>(g.a) + p.m0 * g.a_pitch + p.first * 128;
            for_constants<kALoads>([&](auto i) { off[i.value] = min(load_row(i.value), g.M - 1 - p.m0) * static_cast<uint32_t>(g.a_pitch) + load_piece(i.value); });
        }
        if constexpr (ACROSS_B) {
            b_from = p.first < g.turn ? static_cast<const uint8_t *>(g.b) + p.first * b_step : static_cast<const uint8_t *>(g.b2) + (p.first - g.turn) * b_step;
            for_constants<kBLoads>([&](auto i) { off[kALoads + i.value] = across_row(UintTag<BN>{}, i.value) * static_cast<uint32_t>(g.b_pitch) + 2 * min(p.n0 + 8 * across_piece(UintTag<BN>{}, i.value), g.b_cols - 8); });
        } else {
            const uint64_t at = p.n0 * g.b_pitch + p.first * 128;
            b_from = static_cast<const uint8_t *>(g.b) + at;
            if constexpr (GATED) b2_from = static_cast<const uint8_t *>(g.b2) + at;
            for_constants<kBLoads>([&](auto i) {
                const uint32_t row = load_row(i.value), col = GATED ? 16 * (TH * (row / (16 * TN)) + row / 16 % TH) + row % 16 : row;
                off[kALoads + i.value] = min(col, g.N - 1 - p.n0) * static_cast<uint32_t>(g.b_pitch) + load_piece(i.value);
            });
        }
        ask_stage = p.first;
        ask_end = p.first + p.stages;
        // (more loads on their way than the waits count make these stricter)
        for_constants<kParamLoads>([&](auto i) {
            const uint32_t x = 64 * (wave + NW * i.value) + lane, line = x / kColsOut, rows_from = kLines * kColsOut;
            const float *array = line % 4 == 0 ? (I8 ? g.f.scale : g.f.bias) : line % 4 == 1 ? (I8 ? g.f.bias : g.f.bias2) : line % 4 == 2 ? g.f.scale2 : g.f.bias2;
            const float *own = array + min(p.n0 + x % kColsOut, g.N - 1);
            if (I8 && x >= rows_from) {
                array = g.f.row_scale;
                own = array + min(p.m0 + x - rows_from, g.M - 1);
            }
            const uint64_t mine = __ballot(x < kSlot / 4 && array);
            load_dwords(own, __builtin_amdgcn_readfirstlane(lds0 + kParams + ask_slot * kSlot + 256 * (wave + NW * i.value)), mine);
        });
        ask_slot = ask_slot + 1 == kSlots ? 0 : ask_slot + 1;
    };
    const uint32_t to = lds0 + 1024 * wave;
    struct From {
        const uint8_t *a, *b, *b2;
    };
    auto from_now = [&]() { return From{in_scalars(a_from), in_scalars(b_from), GATED ? in_scalars(b2_from) : nullptr}; };
    auto load_one = [&](const From &from, uint32_t at, auto index) {
        constexpr uint32_t I = decltype(index)::value;
        if constexpr (I < kALoads) {
            load_pieces<1024 * NW * I>(from.a, off[I], to + at, lanes);
        } else {
            constexpr uint32_t J = I - kALoads;
            const bool second = GATED && 8 * (wave + NW * J) / 16 % TN >= TH;
            load_pieces<kB + 1024 * NW * J>(second ? from.b2 : from.b, off[I], to + at, lanes);
        }
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
            a_from += a_step;
            b_from += b_step;
            if constexpr (GATED) b2_from += 128;
            if (ACROSS_B && ask_stage == g.turn) b_from = static_cast<const uint8_t *>(g.b2);
        }
    };

    // ---- LDS -> fragments
    const uint32_t r = lane & 15u, q = lane >> 4;
    auto along_place = [&](uint32_t row, uint32_t step) { return row * 128 + (((q + 4 * step) ^ ((r >> 1) & 7u)) << 4); };   // (row % 16 is r)
    const uint32_t t_row = 8 * q + (r >> 2);
    auto across_place = [&](auto width, uint32_t tile) {
        constexpr uint32_t W = decltype(width)::value;
        const uint32_t piece = 2 * (tile & 1u) + ((lane >> 1) & 1u), swz = W >= 128 ? t_row & 3u : (t_row >> 1) & 1u;
        return t_row * (2 * W) + (((tile >> 1) ^ swz) * 4 + (piece ^ ((t_row >> 2) & 2u))) * 16 + 8 * (lane & 1u);
    };
    uint32_t a_at[ACROSS_A ? TM : 2], b_at[ACROSS_B ? TN : 2];
#pragma unroll
    for (uint32_t i = 0; i < (ACROSS_A ? TM : 2); ++i) a_at[i] = ACROSS_A ? across_place(UintTag<BM>{}, TM * wm + i) : along_place(16 * TM * wm + r, i);
#pragma unroll
    for (uint32_t i = 0; i < (ACROSS_B ? TN : 2); ++i) b_at[i] = kB + (ACROSS_B ? across_place(UintTag<BN>{}, TN * wn + i) : along_place(16 * TN * wn + r, i));
    uint32_t cur = 0, far = (S - 1) * kStage;
    auto transposed = [&](uint32_t at, uint32_t four_rows) {
        uint8_t *p = lds + at;
        const i32x2 lo = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((OMC_LDS s16x4 *)(p)));
        const i32x2 hi = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((OMC_LDS s16x4 *)(p + four_rows)));
        return i32x4{lo[0], lo[1], hi[0], hi[1]};
    };
    Sum acc[TM][TN];
    i32x4 a[2][TM], b[TN];
    auto read_a = [&](auto step, auto index) {
        constexpr uint32_t s = decltype(step)::value, I = decltype(index)::value;
        if constexpr (ACROSS_A) a[s][I] = transposed(cur + a_at[I] + 32 * 2 * BM * s, 4 * 2 * BM);
        else a[s][I] = *reinterpret_cast<const i32x4 *>(lds + cur + a_at[s] + 2048 * I);
    };
    auto read_b = [&](auto step, auto index) {
        constexpr uint32_t s = decltype(step)::value, I = decltype(index)::value;
        if constexpr (ACROSS_B) b[I] = transposed(cur + b_at[I] + 32 * 2 * BN * s, 4 * 2 * BN);
        else b[I] = *reinterpret_cast<const i32x4 *>(lds + cur + b_at[s] + 2048 * I);
    };
    // The products of step s and the reads of the next one; beside the second step's the loads of the stage that is asked for.  Of the waves of a SIMD the one that is further in its products goes first (priority 1 from the second
    // column on): they part, and one finishes results, or waits, while the other multiplies.  8192 x 4096 x 1024: gated 137 -> 112 us, with slopes 164 -> 153 (and 145 by tile rows in twos instead of fours), in 8 bits
    // 99 -> 86, plain in 8 bits 41 -> 37; 16384 x 8192 x 8192 825 -> 804.  One priority for whole steps, or for half of the waves, changes nothing.
    auto multiply = [&](auto step) {
        constexpr uint32_t s = decltype(step)::value, NEXT = 1 - s;
        constexpr int kL = s == 1 ? kLoads : 0;
        const From from = kL > 0 ? from_now() : From{};
        for_constants<TN>([&](auto column) {
            constexpr int J = decltype(column)::value, R0 = J * TM / TN, R1 = (J + 1) * TM / TN, L0 = J * kL / TN, L1 = (J + 1) * kL / TN;
            for_constants<R1 - R0>([&](auto i) { read_a(UintTag<NEXT>{}, UintTag<R0 + decltype(i)::value>{}); });
            for_constants<L1 - L0>([&](auto i) { load_one(from, far, UintTag<L0 + decltype(i)::value>{}); });
#pragma unroll
            for (int i = 0; i < TM; ++i) acc[i][J] = multiply_16(b[J], a[s][i], acc[i][J]);
            __builtin_amdgcn_s_setprio(J == TN - 1 ? 0 : 1);
            read_b(UintTag<NEXT>{}, column);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // Waits for the next stage: it is there when at most the loads of the S - 2 after it, and the stores behind loads of its own age, are on their way.  (At the end it is nothing that is waited for, read and asked for.
    // Loads without lanes are not relied on to count.)
    uint32_t behind = 0;                       // so many stages yet that were asked for before the last stores
    auto wait_for_next = [&]() {
        constexpr int kLater = (S - 2) * kLoads;
        if (lanes == 0) wait_loads_and_sync<0>();
        else if (behind > 0) wait_loads_and_sync<(kLater + kStores < 63 ? kLater + kStores : 63)>();
        else wait_loads_and_sync<kLater>();
        behind -= behind > 0 ? 1 : 0;
        cur = cur == (S - 1) * kStage ? 0 : cur + kStage;
        far = far == (S - 1) * kStage ? 0 : far + kStage;
    };

    if constexpr (kLines > 0) {                // absent biases are zeros
        for (uint32_t x = threadIdx.x; x < kSlots * kSlot / 4; x += 64 * NW) *reinterpret_cast<float *>(lds + kParams + 4 * x) = 0.0f;
        sync_lds();
    }
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
    // (read again behind the largest tile's results, which need the registers)
    constexpr bool kReadAgain = !SPLIT && TM * TN == 32;
    auto first_reads = [&]() {
        for_constants<TM>([&](auto i) { read_a(UintTag<0>{}, i); });
        for_constants<TN>([&](auto i) { read_b(UintTag<0>{}, i); });
    };
    first_reads();
    for (uint32_t item = block; item < items; item += groups) {
        const Place p = locate(item);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = Sum{0, 0, 0, 0};
        for (uint32_t left = p.stages; left > 0; --left) {
            multiply(UintTag<0>{});
            wait_for_next();
            multiply(UintTag<1>{});
            next_stage();
        }

        // ---- results: tile (i, j)'s lane holds row r, columns 4 q .. of it
        const uint32_t m_wave = p.m0 + 16 * TM * wm + r, n_wave = p.n0 + 16 * TH * wn;
        if constexpr (SPLIT) {
            const uint64_t half = parts_columns(g.N), width = GATED ? 2 * half : half;
            typedef typename SumOf<I8>::scalar Scalar;
#pragma unroll
            for (uint32_t i = 0; i < TM; ++i) {
                const uint32_t m = m_wave + 16 * i;
#pragma unroll
                for (uint32_t j = 0; j < TN; ++j) {
                    const uint32_t n = n_wave + 16 * (j % TH) + 4 * q;
                    if (m < g.M && n < g.N) *reinterpret_cast<Sum *>(static_cast<Scalar *>(g.parts) + (static_cast<uint64_t>(p.part) * g.M + m) * width + (j / TH) * half + n) = acc[i][j];
                }
            }
        } else {
            const Finish &f = g.f;
            const uint8_t *params = lds + kParams + slot * kSlot;
            slot = slot + 1 == kSlots ? 0 : slot + 1;
            const bool upper = p.m0 + BM <= f.rows, lower = f.c2 && p.m0 >= f.second && p.m0 - f.second + BM <= f.rows;
            const bool stored = (upper || lower) && p.n0 + kColsOut <= g.N;   // a whole tile
            typename T::type *const c_tile = upper ? static_cast<typename T::type *>(f.c) + p.m0 * f.ldc : static_cast<typename T::type *>(f.c2) + (p.m0 - f.second) * f.ldc;   // (of a whole tile)
            auto line = [&](uint32_t index, uint32_t j) { return *reinterpret_cast<const f32x4 *>(params + 4 * (index * kColsOut + 16 * (TH * wn + j) + 4 * q)); };
            auto columns = [&](uint32_t j) {
                const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
                if constexpr (kLines == 0) return Columns{zero, zero, zero, zero};
                else if constexpr (I8 && GATED) return Columns{line(0, j), line(2, j), line(1, j), line(3, j)};
                else if constexpr (I8) return Columns{line(0, j), zero, line(1, j), zero};
                else return Columns{zero, zero, line(0, j), line(1, j)};
            };
            constexpr uint32_t kTogether = TH % 2 == 0 ? 2 : 1;
            // A gated product's large results in bf16 go past the caches: 8192 x 4096 x 1024 with slopes 156 -> 145 us, without 116 -> 113.  Plain ones do not: 8192 x 4096 x 1024 in 8 bits 37 us, 45 so.
            const bool streams = GATED && static_cast<uint64_t>(g.M) * g.N >= 16u << 20 && (f.ldc | f.ld_slope) % 64 == 0 &&
                                 ((reinterpret_cast<uintptr_t>(f.c) | reinterpret_cast<uintptr_t>(f.slope_g) | reinterpret_cast<uintptr_t>(f.slope_u)) & 15u) == 0;
            auto rows = [&](auto kind, auto keep, auto whole) {
                constexpr bool KEEP = decltype(keep)::value, WHOLE = decltype(whole)::value;
                const uint32_t two_from = n_wave + 16 * (q & 1u) + 8 * (q >> 1), four_from = n_wave + 4 * q;
                auto store_eight = [&](uint16_t *to_row, const u32x4 &w, uint32_t j) {
                    uint16_t *const at = to_row + 16 * j;
                    if constexpr (WHOLE) {
                        if (streams) __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(at));
                        else __builtin_memcpy(at, &w, 16);
                    } else {
                        const uint32_t n = two_from + 16 * j;
                        if (!to_row || n >= g.N) return;
                        if (n + 8 <= g.N) {
                            __builtin_memcpy(at, &w, 16);
                        } else {
#pragma unroll
                            for (uint32_t e = 0; e < 8; ++e)
                                if (n + e < g.N) at[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                        }
                    }
                };
                auto store_four = [&](auto type, auto *to_row, const float (&x)[4], uint32_t j) {
                    const uint32_t n = n_wave + 16 * j + 4 * q;
                    if (WHOLE || (to_row && n < g.N)) store_run<decltype(type), 4>(to_row + 16 * j, x, WHOLE ? 4 : g.N - n);
                };
                constexpr bool kTwo = T::kBytes == 2 && kTogether >= 2;
#pragma unroll
                for (uint32_t i = 0; i < TM; ++i) {
                    const uint32_t m = m_wave + 16 * i;
                    const float row_scale = I8 ? *reinterpret_cast<const float *>(params + 4 * (kLines * kColsOut + 16 * (TM * wm + i) + r)) : 1.0f;
                    typename T::type *row = WHOLE ? c_tile + (m - p.m0) * f.ldc : m < g.M ? row_of<T>(f, m) : nullptr;
                    if (WHOLE || row) row += kTwo ? two_from : four_from;
                    uint16_t *row_g = nullptr, *row_u = nullptr;
                    if (KEEP && (WHOLE || m < g.M)) {
                        row_g = f.slope_g + m * f.ld_slope + (kTogether >= 2 ? two_from : four_from);
                        row_u = f.slope_u + m * f.ld_slope + (kTogether >= 2 ? two_from : four_from);
                    }
#pragma unroll
                    for (uint32_t j = 0; j < TH; j += kTogether) {
                        Four x[kTogether], sg[kTogether], su[kTogether];
#pragma unroll
                        for (uint32_t k = 0; k < kTogether; ++k) {
                            const Columns c = columns(j + k);
                            if constexpr (GATED) x[k] = finish_gated<decltype(kind)::value, KEEP>(acc[i][j + k], acc[i][j + k + TH], row_scale, c, sg[k], su[k]);
                            else x[k] = finish_plain(acc[i][j + k], row_scale, c);
                        }
                        // (all lanes take part in the exchange)
                        auto store_pairs = [&](uint16_t *to_row, const Four(&v)[kTogether]) {
#pragma unroll
                            for (uint32_t k = 0; k < kTogether; k += 2) store_eight(to_row, side_by_side_bf16(v[k].v, v[(k + 1) % kTogether].v), j + k);
                        };
                        if constexpr (kTwo) {
                            store_pairs(row, x);
                        } else {
#pragma unroll
                            for (uint32_t k = 0; k < kTogether; ++k) store_four(T{}, row, x[k].v, j + k);
                        }
                        if constexpr (KEEP && kTogether >= 2) {
                            store_pairs(row_g, sg);
                            store_pairs(row_u, su);
                        } else if constexpr (KEEP) {
                            store_four(BF16{}, row_g, sg[0].v, j);
                            store_four(BF16{}, row_u, su[0].v, j);
                        }
                    }
                }
            };
            auto all = [&](auto kind, auto keep) { stored ? rows(kind, keep, BoolTag<true>{}) : rows(kind, keep, BoolTag<false>{}); };
            if constexpr (!GATED) all(IntTag<0>{}, BoolTag<false>{});
            else for_gate(f.gate, [&](auto kind) { !I8 && f.slope_g ? all(kind, BoolTag<true>{}) : all(kind, BoolTag<false>{}); });
            behind = stored ? S - 1 : 0;
            if constexpr (kReadAgain) first_reads();
        }
    }
}

template <typename C, int OCC>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * C::NW, 64 * C::NW))) __attribute__((amdgpu_waves_per_eu(OCC, OCC))) void tiles_kernel(TileGrid tg) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[C::kLds];
    tiles_body<C>(tg, blockIdx.x, gridDim.x, lds);
}

// Two products in one launch, a workgroup for every tile; the second one's begin at a multiple of 8, so that both keep their order over the dies.
struct PairGrid {
    TileGrid first, second;
    uint32_t groups;                           // of both; behind them come the columns' sums
    ColumnSums sums;
};
template <typename C, typename D, int OCC>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * C::NW, 64 * C::NW))) __attribute__((amdgpu_waves_per_eu(OCC, OCC))) void tiles_pair_kernel(PairGrid pg) {
    static_assert(C::NW == D::NW, "one workgroup size");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[C::kLds > D::kLds ? C::kLds : D::kLds];
    const uint32_t first = pg.first.tiles_m * pg.first.tiles_n, second = (first + 7) / 8 * 8;
    if (blockIdx.x >= pg.groups) {
        float(*part)[32] = reinterpret_cast<float(*)[32]>(lds);
        pg.sums.count <= 64 ? column_sums<C::NW, 1, false>(pg.sums, blockIdx.x - pg.groups, part) : column_sums<C::NW, 8, false>(pg.sums, blockIdx.x - pg.groups, part);
    } else if (blockIdx.x >= second) {
        tiles_body<D>(pg.second, blockIdx.x - second, pg.second.tiles_m * pg.second.tiles_n, lds);
    } else if (blockIdx.x < first) {
        tiles_body<C>(pg.first, blockIdx.x, first, lds);
    }
}

// The parts of a split contraction, added in order, and what becomes of the sums.
template <bool I8, bool GATED, typename T>
__global__ __launch_bounds__(64) void join_kernel(TiledArgs g, uint32_t splits) {
    typedef typename SumOf<I8>::type Sum;
    typedef typename SumOf<I8>::scalar Scalar;
    const uint32_t at = blockIdx.x * 64 + threadIdx.x, quads = (g.N + 3) / 4, m = at / quads, n = 4 * (at - m * quads);   // (M N < 2^28: tiles are few where they are cut)
    if (m >= g.M || n >= g.N) return;
    const uint32_t left = g.N - n;
    const uint64_t half = parts_columns(g.N), width = GATED ? 2 * half : half;
    auto sum_from = [&](uint64_t column) {
        constexpr uint32_t kTogether = 8;      // loads on their way: other dies wrote what they bring
        Sum t = {0, 0, 0, 0};
        for (uint32_t first = 0; first < splits; first += kTogether) {
            Sum w[kTogether];
#pragma unroll
            for (uint32_t s = 0; s < kTogether; ++s)
                w[s] = *reinterpret_cast<const Sum *>(static_cast<const Scalar *>(g.parts) + (static_cast<uint64_t>(min(first + s, splits - 1)) * g.M + m) * width + column);
#pragma unroll
            for (uint32_t s = 0; s < kTogether; ++s)
                if (first + s < splits) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) t[e] += w[s][e];
                }
        }
        return t;
    };
    const float row_scale = I8 ? g.f.row_scale[m] : 1.0f;
    const Columns columns = columns_from<I8, GATED>(g.f, n, g.N);
    typename T::type *row = row_of<T>(g.f, m);
    if constexpr (GATED) {
        store_gated<T>(g.f, sum_from(n), sum_from(half + n), row_scale, columns, row + n, m, n, left);
    } else if (row) {
        store_run<T, 4>(row + n, finish_plain(sum_from(n), row_scale, columns).v, left);
    }
}

// Which tile a product takes, and into how many parts its contraction is cut (omc_gated.hip).
struct TileChoice {
    int tile;
    uint32_t splits;
    double cost;
};
constexpr uint32_t kTileRows[] = {256, 256, 128, 64}, kTileCols[] = {256, 128, 128, 64};
TileChoice choose_tile(ProductKind kind, uint32_t M, uint32_t N, uint32_t stages, bool whole);   // whole: not cut

static inline TileGrid grid_of(const TiledArgs &pa, int tile, bool gated, uint32_t splits) {
    const uint32_t bm = kTileRows[tile], bn = kTileCols[tile] / (gated ? 2 : 1);
    return TileGrid{pa, (pa.M + bm - 1) / bm, (pa.N + bn - 1) / bn, splits, (pa.stages + splits - 1) / splits};
}
// f(waves in rows, in columns, matrix tiles of a wave in rows, in columns, stages, waves per SIMD, workgroups of a compute unit)
template <typename F>
static void for_tile(int tile, F &&f) {
    switch (tile) {
        case 0: f(IntTag<4>{}, IntTag<2>{}, IntTag<4>{}, IntTag<8>{}, IntTag<2>{}, IntTag<2>{}, IntTag<1>{}); break;
        case 1: f(IntTag<4>{}, IntTag<2>{}, IntTag<4>{}, IntTag<4>{}, IntTag<3>{}, IntTag<2>{}, IntTag<1>{}); break;
        case 2: f(IntTag<2>{}, IntTag<2>{}, IntTag<4>{}, IntTag<4>{}, IntTag<2>{}, IntTag<2>{}, IntTag<2>{}); break;
        default: f(IntTag<2>{}, IntTag<2>{}, IntTag<2>{}, IntTag<2>{}, IntTag<4>{}, IntTag<2>{}, IntTag<2>{}); break;
    }
}
template <bool I8, bool GATED, bool ACROSS_A, bool ACROSS_B, typename T>
static int launch_tiles(const TiledArgs &pa, bool whole, hipStream_t st) {
    const TileChoice c = choose_tile(ACROSS_A ? kBF16AcrossBoth : ACROSS_B ? kBF16AcrossB : I8 ? (GATED ? kI8Gated : kI8Plain) : kBF16Gated, pa.M, pa.N, pa.stages, whole);
    const TileGrid tg = grid_of(pa, c.tile, GATED, c.splits);
    for_tile(c.tile, [&](auto wm, auto wn, auto tm, auto tn, auto s, auto occ, auto resident) {
        constexpr int WM = decltype(wm)::value, WN = decltype(wn)::value, TM = decltype(tm)::value, TN = decltype(tn)::value, S = decltype(s)::value, OCC = decltype(occ)::value;
        const uint32_t items = tg.tiles_m * tg.tiles_n * tg.splits, most = 256 * decltype(resident)::value;
        const dim3 grid(items < most ? items : most), block(64 * WM * WN);
        if (tg.splits > 1) tiles_kernel<Tiles<I8, GATED, ACROSS_A, ACROSS_B, WM, WN, TM, TN, S, true, T>, OCC><<<grid, block, 0, st>>>(tg);
        else tiles_kernel<Tiles<I8, GATED, ACROSS_A, ACROSS_B, WM, WN, TM, TN, S, false, T>, OCC><<<grid, block, 0, st>>>(tg);
    });
    if (c.splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return static_cast<int>(e);
        join_kernel<I8, GATED, T><<<dim3((pa.M * ((pa.N + 3) / 4) + 63) / 64), dim3(64), 0, st>>>(pa, c.splits);
    }
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
