// omc_mx4_gemm and omc_mx4_linear for few rows of A (M <= 64: frames of streams, a batch's end).
//
// Bound by memory, or by a launch: every weight is read once, N K 17/32 bytes.  A workgroup takes 16 rows of B and all rows of A; its waves share out K
// in units of 256 values, one unit after the other to one wave after the other, and their sums are joined in order through LDS.  B's codes go from memory straight into the registers
// of the matrix instruction's operand: lane l takes blocks 2 (l / 16) and 2 (l / 16) + 1 of a unit of row l % 16, whose scales are two neighbouring bytes.
// FUSED: A comes as it is and is rounded by every workgroup for itself into LDS, which saves a launch and costs M K roundings in each.
#include "omc_mma.h"
#include "omc_mx4.h"

namespace omc {

// MT row tiles of A; T the result's type, X A's where FUSED.
template <int MT, typename T, bool FUSED, typename X>
__global__ __launch_bounds__(1024) void mx4_few_kernel(Mx4GemmArgs g, Mx4Rows rows) {
    extern __shared__ __attribute__((aligned(16))) uint8_t few_lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t r = lane & 15u, q = lane >> 4, n0 = blockIdx.x * 16;
    const uint32_t blocks = mx4_padded(g.K) / 32, units = (blocks + 7) / 8;
    const uint8_t *a_codes = g.a.codes, *a_scales = g.a.scales;
    if constexpr (FUSED) {
        const uint32_t eights = blocks * 4, items = g.M * eights;
        uint8_t *scales = few_lds + static_cast<uint64_t>(g.M) * blocks * 16;
        for (uint32_t base = 0; base < items; base += blockDim.x) {   // (blocks stay together: both counts are multiples of 4)
            const uint32_t item = base + threadIdx.x, row = item / eights, col = 8 * (item % eights);
            Eight<X> v;
            v.clear();
            if (item < items && col < g.K) v.load(static_cast<const typename X::type *>(rows.x) + row * rows.ldx + col, g.K - col);
            uint32_t top = v.top();
            top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0xb1, 0xf, 0xf, true)));
            top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x4e, 0xf, 0xf, true)));
            const uint32_t byte = mx4_scale<X>(top);
            const uint32_t codes = byte == kMx4NaN ? 0u : v.codes(mx4_unit(byte));
            if (item < items) {
                reinterpret_cast<uint32_t *>(few_lds)[item] = codes;
                if (item % 4 == 0) scales[item / 4] = static_cast<uint8_t>(byte);
            }
        }
        __syncthreads();
        a_codes = few_lds;
        a_scales = scales;
    }
    const uint64_t b_row = min(n0 + r, g.N - 1);
    const uint8_t *b_codes = g.b.codes + b_row * (blocks * 16), *b_scales = g.b.scales + b_row * blocks;
    uint32_t a_row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) a_row[i] = min(16 * i + r, g.M - 1) * blocks;   // (M <= 64: in blocks)
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    constexpr int kAhead = MT == 1 ? 4 : 2;    // units whose B is asked for together
    for (uint32_t u0 = wave; u0 < units; u0 += kAhead * waves) {
        i32x4 b[kAhead][2];
        uint32_t sb[kAhead], at[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t block = 8 * (u0 + k * waves) + 2 * q;
            at[k] = min(block, blocks - 2);    // past the end (half a unit, or no unit at all): other codes' place, and zeros
            b[k][0] = *reinterpret_cast<const i32x4 *>(b_codes + 16ull * at[k]);
            b[k][1] = *reinterpret_cast<const i32x4 *>(b_codes + 16ull * at[k] + 16);
            sb[k] = *reinterpret_cast<const uint16_t *>(b_scales + at[k]);
            if (block != at[k]) b[k][0] = b[k][1] = i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const uint8_t *a = a_codes + 16ull * (a_row[i] + at[k]);
                const uint32_t sa = *reinterpret_cast<const uint16_t *>(a_scales + a_row[i] + at[k]);
                acc[i] = mx4_multiply<0, 0>(b[k][0], sb[k], *reinterpret_cast<const i32x4 *>(a), sa, acc[i]);
                acc[i] = mx4_multiply<1, 1>(b[k][1], sb[k], *reinterpret_cast<const i32x4 *>(a + 16), sa, acc[i]);
            }
    }

    __syncthreads();                           // A's codes are done with
    f32x4 *sums = reinterpret_cast<f32x4 *>(few_lds);
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[(wave * MT + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 64 * MT; t += blockDim.x) {   // (blockDim.x is a multiple of 64: lane and r, q stay)
        f32x4 s = sums[t];
        for (uint32_t w = 1; w < waves; ++w) s += sums[w * (64 * MT) + t];
        const uint32_t m = 16 * (t / 64) + r, n = n0 + 4 * q;
        if (m < g.M && n < g.N) {
            float v[4];
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) v[e] = g.bias ? s[e] + g.bias[min(n + e, g.N - 1)] : s[e];
            store_run<T, 4>(static_cast<typename T::type *>(g.c) + m * g.ldc + n, v, g.N - n);
        }
    }
}

// LDS that a rounded A may take.
constexpr uint64_t kFusedBytes = 16384;
static uint64_t rounded_bytes(uint32_t M, uint32_t K) { return static_cast<uint64_t>(M) * (mx4_padded(K) / 32) * 17; }
bool mx4_few_rounds(uint32_t M, uint32_t, uint32_t K) { return M <= kMx4FewRows && rounded_bytes(M, K) <= kFusedBytes; }

template <int MT, typename T>
static int launch_rows(const Mx4GemmArgs &ga, const Mx4Rows *rows, hipStream_t st) {
    const uint32_t units = (ga.K + 255) / 256;
    uint32_t waves = 1;
    while (waves < 8 && 2 * waves <= units) waves *= 2;
    const size_t joined = waves * MT * 1024, lds = rows && rounded_bytes(ga.M, ga.K) > joined ? rounded_bytes(ga.M, ga.K) : joined;
    const dim3 grid((ga.N + 15) / 16), block(64 * waves);
    if (!rows) mx4_few_kernel<MT, T, false, T><<<grid, block, lds, st>>>(ga, Mx4Rows{});
    else if (rows->bf16) mx4_few_kernel<MT, T, true, BF16><<<grid, block, lds, st>>>(ga, *rows);
    else mx4_few_kernel<MT, T, true, F32><<<grid, block, lds, st>>>(ga, *rows);
    return static_cast<int>(hipGetLastError());
}

template <typename T>
static int launch_typed(const Mx4GemmArgs &ga, const Mx4Rows *rows, hipStream_t st) {
    if (ga.M <= 16) return launch_rows<1, T>(ga, rows, st);
    if (ga.M <= 32) return launch_rows<2, T>(ga, rows, st);
    return launch_rows<4, T>(ga, rows, st);
}

int launch_mx4_few(const Mx4GemmArgs &ga, const Mx4Rows *rows, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch_typed<BF16>(ga, rows, st) : launch_typed<F32>(ga, rows, st);
}

}  // namespace omc
