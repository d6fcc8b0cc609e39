// Products of few rows of A (frames of streams): 8-bit integers and bf16, plain and gated.
//
// Bound by memory, or by a launch: every weight is read once.  A workgroup takes 16 rows of the weights (of each matrix where gated) and all rows of A; its waves share out K, and their sums are joined in order
// through LDS.  A wave's weights go from memory straight into the matrix instruction's operand registers, two units on their way while two are multiplied.
#include "omc_finish.h"
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

// A lane's 16 bytes of an operand for one matrix instruction, as they lie in memory.
template <ElementType E>
struct Piece {
    Eight<typename TypeOf<E == kE32 ? 4 : 2>::type> v;
    __device__ __forceinline__ void load(const void *row, uint32_t k, uint32_t K) { v.load(static_cast<const typename TypeOf<E == kE32 ? 4 : 2>::type::type *>(row), k, K); }
    __device__ __forceinline__ void clear() { v.clear(); }
    __device__ __forceinline__ i32x4 operand() const {
        i32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = static_cast<int>(E == kE32 ? to_bf16_pair(v.value(2 * i), v.value(2 * i + 1)) : v.w[i]);
        return w;
    }
};
template <>
struct Piece<kE8> {
    i32x4 w;
    __device__ __forceinline__ void load(const void *row, uint32_t k, uint32_t) { w = *reinterpret_cast<const i32x4 *>(static_cast<const uint8_t *>(row) + k); }
    __device__ __forceinline__ void clear() { w = i32x4{0, 0, 0, 0}; }
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

// MT row tiles of A.
template <ElementType X, ElementType W, bool GATED, int MT, typename T>
__global__ __launch_bounds__(512) void few_kernel(FewArgs fa) {
    constexpr bool I8 = W == kE8;
    static_assert(I8 == (X == kE8), "operands of one kind");
    constexpr uint32_t kStep = I8 ? 64 : 32, kUnit = 2 * kStep, kPer = I8 ? 16 : 8, kBytes = W == kE8 ? 1 : W == kE16 ? 2 : 4, kXBytes = X == kE8 ? 1 : X == kE16 ? 2 : 4;
    constexpr int MATRICES = GATED ? 2 : 1, U = 2;
    typedef typename FewSum<I8>::type Sum;
    extern __shared__ __attribute__((aligned(16))) uint8_t few_lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t r = lane & 15u, q = lane >> 4, n0 = blockIdx.x * 16;
    const uint32_t units = (fa.K + kUnit - 1) / kUnit;
    const uint32_t begin = static_cast<uint32_t>(static_cast<uint64_t>(wave) * units / waves), end = static_cast<uint32_t>(static_cast<uint64_t>(wave + 1) * units / waves);
    const uint8_t *w_row[MATRICES], *x_row[MT];
#pragma unroll
    for (int i = 0; i < MATRICES; ++i) w_row[i] = static_cast<const uint8_t *>(i == 0 ? fa.w : fa.w2) + min(n0 + r, fa.N - 1) * (fa.ldw * kBytes);
#pragma unroll
    for (uint32_t i = 0; i < MT; ++i) x_row[i] = static_cast<const uint8_t *>(fa.x) + min(16 * i + r, fa.M - 1) * (fa.ldx * kXBytes);
    struct Group {
        Piece<W> w[U][2][MATRICES];
        Piece<X> x[U][2][MT];
    } now, next;
    auto load_group = [&](Group &g, uint32_t unit) {
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t s = 0; s < 2; ++s) {
                const uint32_t k = (unit + u) * kUnit + s * kStep + q * kPer;
                const bool there = unit + u < end && k < fa.K;
#pragma unroll
                for (int i = 0; i < MATRICES; ++i) {
                    g.w[u][s][i].clear();
                    if (there) g.w[u][s][i].load(w_row[i], k, fa.K);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    g.x[u][s][i].clear();
                    if (there) g.x[u][s][i].load(x_row[i], k, fa.K);
                }
            }
    };
    Sum acc[MATRICES][MT];
#pragma unroll
    for (int i = 0; i < MATRICES; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = Sum{0, 0, 0, 0};
    load_group(now, begin);
    for (uint32_t unit = begin; unit < end; unit += U) {
        load_group(next, unit + U);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < MATRICES; ++i)
#pragma unroll
                    for (int j = 0; j < MT; ++j) acc[i][j] = multiply_few(now.w[u][s][i].operand(), now.x[u][s][j].operand(), acc[i][j]);
        now = next;
    }

    Sum *sums = reinterpret_cast<Sum *>(few_lds);
#pragma unroll
    for (int i = 0; i < MATRICES; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) sums[((wave * MT + j) * MATRICES + i) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 64 * MT; t += blockDim.x) {   // (blockDim.x is a multiple of 64: r and q stay)
        const uint32_t j = t / 64, m = 16 * j + r, n = n0 + 4 * q;
        if (m >= fa.M || n >= fa.N) continue;
        Sum total[MATRICES];
#pragma unroll
        for (int i = 0; i < MATRICES; ++i) {
            total[i] = sums[(j * MATRICES + i) * 64 + lane];
            for (uint32_t w = 1; w < waves; ++w) total[i] += sums[((w * MT + j) * MATRICES + i) * 64 + lane];
        }
        const float row_scale = I8 ? fa.f.row_scale[m] : 1.0f;
        typename T::type *to = static_cast<typename T::type *>(fa.f.c) + m * fa.f.ldc + n;
        const uint32_t left = fa.N - n;
        const Columns columns = columns_from<I8, GATED>(fa.f, n, fa.N);
        if constexpr (GATED) {
            store_gated<T>(fa.f, total[0], total[MATRICES - 1], row_scale, columns, to, m, n, left);
        } else {
            store_run<T, 4>(to, finish_plain(total[0], row_scale, columns).v, left);
        }
    }
}

bool product_few(uint32_t M, uint32_t N, uint32_t K) {
    (void)N;
    (void)K;
    return M <= 32;
}
bool product_few_rounds(uint32_t M, uint32_t K) {
    (void)M;
    (void)K;
    return false;
}

template <ElementType X, ElementType W, bool GATED, int MT, typename T>
static int launch_rows(const FewArgs &fa, hipStream_t st) {
    const uint32_t unit = W == kE8 ? 128 : 64, units = (fa.K + unit - 1) / unit, waves = units < 8 ? units : 8;
    few_kernel<X, W, GATED, MT, T><<<dim3((fa.N + 15) / 16), dim3(64 * waves), waves * MT * (GATED ? 2048 : 1024), st>>>(fa);
    return static_cast<int>(hipGetLastError());
}
template <ElementType X, ElementType W, bool GATED>
static int launch_typed(const FewArgs &fa, bool c_bf16, hipStream_t st) {
    if (c_bf16) return fa.M <= 16 ? launch_rows<X, W, GATED, 1, BF16>(fa, st) : launch_rows<X, W, GATED, 2, BF16>(fa, st);
    return fa.M <= 16 ? launch_rows<X, W, GATED, 1, F32>(fa, st) : launch_rows<X, W, GATED, 2, F32>(fa, st);
}
int launch_product_few(ElementType x, ElementType w, bool gated, const FewArgs &fa, bool c_bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (w == kE8) return gated ? launch_typed<kE8, kE8, true>(fa, c_bf16, st) : launch_typed<kE8, kE8, false>(fa, c_bf16, st);
    if (w == kE16) return x == kE16 ? launch_typed<kE16, kE16, true>(fa, c_bf16, st) : launch_typed<kE32, kE16, true>(fa, c_bf16, st);
    return x == kE16 ? launch_typed<kE16, kE32, true>(fa, c_bf16, st) : launch_typed<kE32, kE32, true>(fa, c_bf16, st);
}

}  // namespace omc
