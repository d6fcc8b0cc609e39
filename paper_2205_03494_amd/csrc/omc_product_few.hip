// Products of few rows of A (frames of streams): 8-bit integers and bf16, plain and gated.
//
// Bound by memory, or by a launch: every weight is read once.  A workgroup takes 16 rows of the weights (of each matrix where gated) and all rows of A; its waves share out K, and their sums are joined in order
// through LDS.  A wave's weights go from memory straight into the matrix instruction's operand registers, two units on their way while two are multiplied.
// A lane's pieces are 16 bytes of its own row, so that a load fetches halves of 16 cache lines and the next one their other halves: that, more than memory, bounds a long contraction (1 x 8192 x 8192 in 8 bits 15 us, 4.4 TB/s; a large copy 5.1).
// 1 x 4096 x 1024 in 8 bits 4.7 us, 29 x 8200 x 971 from codes 6.2, gated 16 x 4096 x 1024 in 8 bits 7.7: a launch, two round trips and the join; the last rounds its 16 rows in every workgroup, 2 us.
#include "omc_finish.h"
#include "omc_i8.h"
#include "omc_mma.h"

namespace omc {

template <int BYTES>
struct TypeOf {
    typedef BF16 type;
};
template <>
struct TypeOf<4> {
    typedef F32 type;
};

// A lane's 16 bytes of an operand for one matrix instruction, as they lie in memory.  WHOLE: a row is whole pieces.
template <ElementType E, bool WHOLE>
struct Piece {
    typedef typename TypeOf<E == kE32 ? 4 : 2>::type Type;
    Eight<Type> v;
    __device__ __forceinline__ void load(const uint8_t *row, uint32_t k, uint32_t K) {
        const typename Type::type *from = reinterpret_cast<const typename Type::type *>(row);
        if constexpr (WHOLE) {
            __builtin_memcpy(v.w, from + (k < K ? k : 0), sizeof(v.w));
        } else {
            v.clear();
            if (k < K) v.load(from, k, K);
        }
    }
    __device__ __forceinline__ i32x4 operand() const {
        i32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = static_cast<int>(E == kE32 ? to_bf16_pair(v.value(2 * i), v.value(2 * i + 1)) : v.w[i]);
        return w;
    }
};
template <>
struct Piece<kE8, true> {
    i32x4 w;
    __device__ __forceinline__ void load(const uint8_t *row, uint32_t k, uint32_t) { w = *reinterpret_cast<const i32x4 *>(row + k); }
    __device__ __forceinline__ i32x4 operand() const { return w; }
};
__device__ __forceinline__ f32x4 multiply_few(i32x4 a, i32x4 b, f32x4 acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ i32x4 multiply_few(i32x4 a, i32x4 b, i32x4 acc) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc, 0, 0, 0); }
template <bool I8>
struct FewSum {
    typedef f32x4 type;
};
template <>
struct FewSum<true> {
    typedef i32x4 type;
};

// MT row tiles of A.  kPieces: of eight values, of a lane at most, where A becomes codes.
constexpr uint32_t kPieces = 4, kRoundedValues = 16384;
template <ElementType X, ElementType W, bool GATED, int PARTS, int MT, bool WHOLE, typename T>
__global__ __launch_bounds__(512) void few_kernel(FewArgs fa) {
    constexpr bool I8 = W == kE8, ROUNDS = I8 && X != kE8;
    constexpr uint32_t kStep = I8 ? 64 : 32, kUnit = 2 * kStep, kPer = I8 ? 16 : 8, kBytes = W == kE8 ? 1 : W == kE16 ? 2 : 4, kXBytes = X == kE8 ? 1 : X == kE16 ? 2 : 4;
    static_assert(!GATED || PARTS == 2, "both matrices");
    constexpr int U = MT == 2 && X == kE32 && W == kE32 ? 1 : 2;   // units that are asked for together (two of fp32 would spill)
    typedef typename FewSum<I8>::type Sum;
    extern __shared__ __attribute__((aligned(16))) uint8_t few_lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t r = lane & 15u, q = lane >> 4, n0 = blockIdx.x * (GATED ? 16 : 16 * PARTS);
    const uint32_t units = (fa.K + kUnit - 1) / kUnit;
    const uint32_t begin = static_cast<uint32_t>(static_cast<uint64_t>(wave) * units / waves), end = static_cast<uint32_t>(static_cast<uint64_t>(wave + 1) * units / waves);
    const uint8_t *w_row[PARTS], *x_row[MT];
#pragma unroll
    for (uint32_t i = 0; i < PARTS; ++i) w_row[i] = static_cast<const uint8_t *>(GATED && i == 1 ? fa.w2 : fa.w) + min(n0 + (GATED ? 0 : 16 * i) + r, fa.N - 1) * (fa.ldw * kBytes);
#pragma unroll
    for (uint32_t i = 0; i < MT; ++i) x_row[i] = static_cast<const uint8_t *>(fa.x) + min(16 * i + r, fa.M - 1) * (fa.ldx * kXBytes);
    struct Group {
        Piece<W, WHOLE> w[U][2][PARTS];
        Piece<I8 ? kE8 : X, WHOLE> x[U][2][ROUNDS ? 1 : MT];
    } even, odd;
    auto load_group = [&](Group &g, uint32_t unit) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (unit + u >= end) break;
#pragma unroll
            for (uint32_t s = 0; s < 2; ++s) {
                const uint32_t k = (unit + u) * kUnit + s * kStep + q * kPer;
#pragma unroll
                for (int i = 0; i < PARTS; ++i) g.w[u][s][i].load(w_row[i], k, fa.K);
                if constexpr (!ROUNDS) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) g.x[u][s][i].load(x_row[i], k, fa.K);
                }
            }
        }
    };
    Sum acc[PARTS][MT];
#pragma unroll
    for (int i = 0; i < PARTS; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = Sum{0, 0, 0, 0};
    load_group(even, begin);

    // ROUNDS: A's codes, rows apart by 16 bytes more than they are long, and scales in LDS, while the weights are on their way.  fa.K is whole 128s.
    const uint32_t pitch = fa.K + 16;
    uint8_t *row_codes = few_lds + 64;
    float scale_of_row = 1.0f;
    if constexpr (ROUNDS) {
        typedef typename TypeOf<X == kE32 ? 4 : 2>::type XT;
        uint32_t *tops = reinterpret_cast<uint32_t *>(few_lds);
        const uint32_t pieces = fa.K / 8, all = fa.M * pieces;                 // of eight values; whole sixteens of a row
        Eight<XT> v[kPieces];
        if (threadIdx.x < 16) tops[threadIdx.x] = 0;
        uint32_t row[kPieces], col[kPieces];
#pragma unroll
        for (uint32_t k = 0; k < kPieces; ++k) {
            const uint32_t at = k * blockDim.x + threadIdx.x;
            row[k] = at / pieces;
            col[k] = 8 * (at - row[k] * pieces);
            v[k].clear();
            if (at < all && col[k] < fa.columns) v[k].load(static_cast<const typename XT::type *>(fa.x) + row[k] * fa.ldx, col[k], fa.columns);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < kPieces; ++k) {
            uint32_t top = v[k].top();
            auto with = [&](int other) { top = max(top, static_cast<uint32_t>(other)); };
            with(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0xb1, 0xf, 0xf, true));    // lanes 1 0 3 2
            with(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x4e, 0xf, 0xf, true));    // lanes 2 3 0 1
            with(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x141, 0xf, 0xf, true));   // of eight, backwards
            with(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x140, 0xf, 0xf, true));   // of sixteen, backwards
            if (r == 0 && row[k] < fa.M) atomicMax(&tops[row[k]], top);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < kPieces; ++k) {
            if (row[k] >= fa.M) continue;
            Rounding to;
            to.of(from_top<XT>(tops[row[k]]), tops[row[k]] > XT::kFinite);
            float x8[8], c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x8[i] = v[k].value(i);
            to.eight(x8, c);
            *reinterpret_cast<uint64_t *>(row_codes + row[k] * pitch + col[k]) = four_bytes(c) | static_cast<uint64_t>(four_bytes(c + 4)) << 32;
        }
        const uint32_t own = tops[min(r, fa.M - 1)];
        Rounding to;
        to.of(from_top<XT>(own), own > XT::kFinite);
        scale_of_row = to.scale;
        __syncthreads();
    }
    auto multiply_group = [&](const Group &g, uint32_t unit) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) {
            if (unit + u >= end) break;
            const bool past = WHOLE && !I8 && (unit + u + 1) * kUnit > fa.K;   // a unit with lanes past the rows' end
#pragma unroll
            for (uint32_t s = 0; s < 2; ++s) {
                const uint32_t k = (unit + u) * kUnit + s * kStep + q * kPer;
                const i32x4 zero = {0, 0, 0, 0};
                i32x4 x[MT];
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    if constexpr (ROUNDS) x[j] = *reinterpret_cast<const i32x4 *>(row_codes + min(r, fa.M - 1) * pitch + k);
                    else x[j] = g.x[u][s][j].operand();
                    if (past && k >= fa.K) x[j] = zero;
                }
#pragma unroll
                for (int i = 0; i < PARTS; ++i) {
                    i32x4 w = g.w[u][s][i].operand();
                    if (past && k >= fa.K) w = zero;
#pragma unroll
                    for (int j = 0; j < MT; ++j) acc[i][j] = multiply_few(w, x[j], acc[i][j]);
                }
            }
        }
    };
    for (uint32_t unit = begin; unit < end; unit += 2 * U) {
        load_group(odd, unit + U);
        multiply_group(even, unit);
        load_group(even, unit + 2 * U);
        multiply_group(odd, unit + U);
    }

    if constexpr (ROUNDS) __syncthreads();     // nobody reads A any more
    Sum *sums = reinterpret_cast<Sum *>(few_lds);
#pragma unroll
    for (int i = 0; i < PARTS; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) sums[((wave * MT + j) * PARTS + i) * 64 + lane] = acc[i][j];
    __syncthreads();
    constexpr uint32_t kOut = GATED ? 1 : PARTS;              // tiles of results
    for (uint32_t t = threadIdx.x; t < 64 * MT * kOut; t += blockDim.x) {   // (blockDim.x is a multiple of 64: r and q stay)
        const uint32_t j = t / 64 % MT, part = t / (64 * MT), m = 16 * j + r, n = n0 + 16 * part + 4 * q;
        if (m >= fa.M || n >= fa.N) continue;
        auto total = [&](uint32_t i) {
            Sum s = sums[(j * PARTS + i) * 64 + lane];
            for (uint32_t w = 1; w < waves; ++w) s += sums[((w * MT + j) * PARTS + i) * 64 + lane];
            return s;
        };
        const float row_scale = ROUNDS ? scale_of_row : I8 ? fa.f.row_scale[m] : 1.0f;
        typename T::type *to = static_cast<typename T::type *>(fa.f.c) + m * fa.f.ldc + n;
        const uint32_t left = fa.N - n;
        const Columns columns = columns_from<I8, GATED>(fa.f, n, fa.N);
        if constexpr (GATED) store_gated<T>(fa.f, total(0), total(1), row_scale, columns, to, m, n, left);
        else store_run<T, 4>(to, finish_plain(total(part), row_scale, columns).v, left);
    }
}

// Up to 32 rows, where by estimates (us) that takes less than tiles, which cut a long contraction over the chip: a workgroup's eight waves take `rounds` units one after the other, at the rate at which a compute unit's loads bring
// halves of 16 rows' cache lines; all workgroups together are bound by memory.  Fitted to 490 sizes of 1 .. 32 x 16 .. 16384 x 64 .. 32768 of each kind, 10 - 12 % (standard deviation); the chosen way takes 0.5 - 1.8 % longer
// than the better one on average.  1 x 4096 x 1024 in 8 bits 5.5 us with its rounding, in tiles 9.3; 1 x 512 x 32768 36 and 26; gated in bf16 1 x 4096 x 1024 6.4 and 8.6, 16 x 8192 x 8192 50 and 45.
bool product_few(ProductKind kind, uint32_t M, uint32_t N, uint32_t K, bool rounds) {
    if (M > 32) return false;
    const bool i8 = kind != kBF16Gated, gated = kind != kI8Plain;
    const uint32_t unit = i8 ? 128 : 64, stages = (K + unit - 1) / unit, waves = stages < 8 ? stages : 8, parts = gated ? 2 : 1;
    const double per_unit = static_cast<double>((N + 15) / 16) / 256.0, uneven = 1.0 + (per_unit > 1.0 ? 0.1 * (per_unit - 1.0) : 0.0);
    const double turns = static_cast<double>((stages + waves - 1) / waves) * (0.43 * parts + (M <= 16 ? 0.13 : 0.26) + 0.3 / 16 * M) * uneven;
    const double memory = static_cast<double>(N) * K * parts * (i8 ? 1 : 2) / 4.4e6;
    const double few = 3.2 + (turns > memory ? turns : memory) - (rounds ? 2.0 : 0.0);   // a launch less
    return few <= product_tiles_cost(kind, M, N, stages);
}
// A becomes codes in every workgroup where that is worth less than a launch, of which the host's part counts too.  With it, and with one before, from a graph: 1 x 4096 x 1024 5.5 us and 7.5, 8 x 4096 x 1024 6.8 and 8.2,
// 16 x 4096 x 1024 8.3 and 8.5, 16 x 512 x 512 7.6 and 6.8; gated 16 x 4096 x 1024, call after call from Python, 9.6 and 13.
bool product_few_rounds(uint32_t M, uint32_t K) { return M <= 16 && M * i8_pitch(K) <= kRoundedValues; }

// With more than 16 rows of A a plain product's workgroup takes 32 columns where that leaves one for every compute unit, so that A is read half as often: 29 x 8192 x 8192 in 8 bits 29.8 -> 26.8 us with the rounding, 29 x 16384 x 4096
// 28 -> 24.5; 16 rows 24.2 either way, one 15.4 -> 17.4.
constexpr uint32_t kWideN = 32 * 256;
template <ElementType X, ElementType W, bool GATED, int PARTS, int MT, typename T>
static int launch_parts(const FewArgs &fa, hipStream_t st) {
    const uint32_t unit = W == kE8 ? 128 : 64, units = (fa.K + unit - 1) / unit, waves = units < 8 ? units : 8, joined = waves * MT * PARTS * 1024, columns = GATED ? 16 : 16 * PARTS;
    const uint32_t rounded = W == kE8 && X != kE8 ? 64 + fa.M * (fa.K + 16) : 0;
    const dim3 grid((fa.N + columns - 1) / columns), block(64 * waves);
    const uint32_t lds = rounded > joined ? rounded : joined;
    if constexpr (W == kE8) few_kernel<X, W, GATED, PARTS, MT, true, T><<<grid, block, lds, st>>>(fa);
    else if (fa.K % 8 == 0) few_kernel<X, W, GATED, PARTS, MT, true, T><<<grid, block, lds, st>>>(fa);
    else few_kernel<X, W, GATED, PARTS, MT, false, T><<<grid, block, lds, st>>>(fa);
    return static_cast<int>(hipGetLastError());
}
template <ElementType X, ElementType W, bool GATED, int MT, typename T>
static int launch_rows(const FewArgs &fa, hipStream_t st) {
    if constexpr (GATED) return launch_parts<X, W, GATED, 2, MT, T>(fa, st);
    else if constexpr (MT == 1) return launch_parts<X, W, GATED, 1, MT, T>(fa, st);
    else return fa.N >= kWideN ? launch_parts<X, W, GATED, 2, MT, T>(fa, st) : launch_parts<X, W, GATED, 1, MT, T>(fa, st);
}
template <ElementType X, ElementType W, bool GATED>
static int launch_typed(const FewArgs &fa, bool c_bf16, hipStream_t st) {
    if constexpr (W == kE8 && X != kE8) return c_bf16 ? launch_rows<X, W, GATED, 1, BF16>(fa, st) : launch_rows<X, W, GATED, 1, F32>(fa, st);
    else if (c_bf16) return fa.M <= 16 ? launch_rows<X, W, GATED, 1, BF16>(fa, st) : launch_rows<X, W, GATED, 2, BF16>(fa, st);
    else return fa.M <= 16 ? launch_rows<X, W, GATED, 1, F32>(fa, st) : launch_rows<X, W, GATED, 2, F32>(fa, st);
}
template <bool GATED>
static int launch_i8(ElementType x, const FewArgs &fa, bool c_bf16, hipStream_t st) {
    if (x == kE8) return launch_typed<kE8, kE8, GATED>(fa, c_bf16, st);
    return x == kE16 ? launch_typed<kE16, kE8, GATED>(fa, c_bf16, st) : launch_typed<kE32, kE8, GATED>(fa, c_bf16, st);
}
int launch_product_few(ElementType x, ElementType w, bool gated, const FewArgs &fa, bool c_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (w == kE8) return gated ? launch_i8<true>(x, fa, c_bf16, st) : launch_i8<false>(x, fa, c_bf16, st);
    if (w == kE16) return x == kE16 ? launch_typed<kE16, kE16, true>(fa, c_bf16, st) : launch_typed<kE32, kE16, true>(fa, c_bf16, st);
    return x == kE16 ? launch_typed<kE16, kE32, true>(fa, c_bf16, st) : launch_typed<kE32, kE32, true>(fa, c_bf16, st);
}

}  // namespace omc
