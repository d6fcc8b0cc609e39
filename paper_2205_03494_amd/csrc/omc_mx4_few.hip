// omc_mx4_gemm and omc_mx4_linear for few rows of A (frames of streams, a batch's end).
//
// Bound by memory, or by a launch: every weight is read once, N K 17/32 bytes.  A workgroup takes 16 rows of B and all rows of A; its waves share out K, each a run of
// units of 256 values, and their sums are joined in order through LDS.  A wave brings its units into an LDS ring of its own, whole cache lines of B's and A's rows (a load straight into the matrix
// instruction's operands takes half a line of a row at a time, which costs the load path as much as a whole one), and waits for nobody.  Lane l multiplies blocks 2 (l / 16) and
// 2 (l / 16) + 1 of a unit of row l % 16, whose scales are two neighbouring bytes.
// FUSED: A comes as it is and is rounded by every workgroup for itself into LDS, while B is on its way, which saves a launch and costs M K roundings in each.
// 1 x 8192 x 8192: 8.6 us, 4.1 TB/s of weights; 1 x 4096 x 1024: 3.4 us; 29 x 8200 x 8192: 12.1 us and 2.5 for the rounding before.  There, with more than 16 rows, the ring has two stages:
// a wave has one unit on its way while it multiplies another, eight round trips in a row.  What is loaded, B once and A for every 16 columns, 109 MB, would take a third of that time at the rate of the tiles' loads.
#include "omc_mma.h"
#include "omc_mx4.h"

namespace omc {

// Direct loads into LDS as in load_to_lds, 4 bytes a lane.
__device__ __forceinline__ void load_dwords_to_lds(const uint8_t *base, uint32_t off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(dst), "v"(off), "s"(base) : "memory", "m0");
}
// This wave's accesses to LDS are done, and all but LATER of its loads.
template <int LATER>
__device__ __forceinline__ void wait_own() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory");
}

// MT row tiles of A, S stages in a wave's ring; T the result's type, X A's where FUSED.
template <int MT, int S, bool FUSED, typename T, typename X>
__global__ __launch_bounds__(512) void mx4_few_kernel(Mx4GemmArgs g, Mx4Rows rows) {
    constexpr uint32_t kOperands = FUSED ? 1 : 1 + MT, kScales = 2048 * kOperands, kScaleLoads = (kOperands + 1) / 2, kStage = kScales + 256 * kScaleLoads;   // B, then A's tiles; 8 bytes of scales a row
    constexpr int kLoads = 2 * kOperands + kScaleLoads;
    extern __shared__ __attribute__((aligned(16))) uint8_t few_lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t r = lane & 15u, q = lane >> 4, n0 = blockIdx.x * 16;
    const uint32_t k128 = mx4_padded(g.K) / 128, blocks = 4 * k128, units = (k128 + 1) / 2, row_bytes = 64 * k128;
    const uint32_t begin = __builtin_amdgcn_readfirstlane(wave * units / waves), end = __builtin_amdgcn_readfirstlane((wave + 1) * units / waves);

    // ---- global -> LDS: a load is 8 rows of an operand, lane l's piece l % 8 of row l / 8, XOR-swizzled by half the row
    uint8_t *ring = few_lds + wave * (S * kStage);
    const uint32_t ring0 = lds_offset(few_lds) + wave * (S * kStage), last_n = g.N - 1 - n0;
    uint32_t off[2 * kOperands], piece[2];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) piece[i] = (lane & 7u) ^ ((4 * i + (lane >> 4)) & 7u);
#pragma unroll
    for (uint32_t i = 0; i < 2 * kOperands; ++i) {
        const uint32_t row = 8 * (i % 2) + (lane >> 3);
        off[i] = (i < 2 ? min(row, last_n) : min(16 * (i / 2 - 1) + row, g.M - 1)) * row_bytes + 16 * piece[i % 2];
    }
    const uint8_t *b_from = g.b.codes + static_cast<uint64_t>(n0) * row_bytes + 128 * begin, *a_from = g.a.codes + 128 * begin;
    // scales, two dwords a row: B's rows and in the upper lanes A's first tile, then A's second tile
    const uint32_t s_row = lane >> 1, s_dword = 4 * (lane & 1u);
    const uint8_t *b_scales = g.b.scales + static_cast<uint64_t>(n0) * blocks + 8 * begin, *a_scales = FUSED ? b_scales : g.a.scales + 8 * begin;
    const uint8_t *first_scales = (FUSED || lane < 32 ? b_scales + min(s_row % 16, last_n) * blocks : a_scales + min(s_row - 16, g.M - 1) * blocks) + s_dword;   // (the lane's own)
    const uint32_t second_scales = min(16 + s_row, g.M - 1) * blocks + s_dword;
    auto load_unit = [&](uint32_t unit, uint32_t at) {
        const bool half = 2 * unit + 1 == k128;               // its second half is not there: the first one twice
#pragma unroll
        for (uint32_t i = 0; i < 2 * kOperands; ++i)
            load_to_lds(i < 2 ? b_from : a_from, off[i] - (half ? 16 * (piece[i % 2] & 4u) : 0u), ring0 + at + 1024 * i);
        const uint8_t *own = first_scales - (half ? s_dword : 0u);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(ring0 + at + kScales), "v"(own) : "memory", "m0");
        if constexpr (kScaleLoads > 1) load_dwords_to_lds(a_scales, second_scales - (half ? s_dword : 0u), ring0 + at + kScales + 256);
        b_from += 128;
        a_from += 128;
        first_scales += 8;
        a_scales += 8;
    };
#pragma unroll
    for (uint32_t i = 0; i < S - 1; ++i)
        if (begin + i < end) load_unit(begin + i, i * kStage);

    const uint8_t *a_codes = nullptr, *a_bytes = nullptr;     // FUSED: A's rows in LDS
    if constexpr (FUSED) {
        uint8_t *codes_lds = few_lds + waves * (S * kStage), *scales_lds = codes_lds + g.M * blocks * 16;
        const uint32_t eights = blocks * 4, items = g.M * eights;
        constexpr uint32_t kTogether = 4;                     // loads on their way at a time
        for (uint32_t base = 0; base < items; base += kTogether * blockDim.x) {   // (blocks stay together: both counts are multiples of 4)
            Eight<X> v[kTogether];
#pragma unroll
            for (uint32_t k = 0; k < kTogether; ++k) {
                const uint32_t item = base + k * blockDim.x + threadIdx.x, row = item / eights, col = 8 * (item % eights);
                v[k].clear();
                if (item < items && col < g.K) v[k].load(static_cast<const typename X::type *>(rows.x) + row * rows.ldx, col, g.K);
            }
#pragma unroll
            for (uint32_t k = 0; k < kTogether; ++k) {
                const uint32_t item = base + k * blockDim.x + threadIdx.x;
                uint32_t top = v[k].top();
                top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0xb1, 0xf, 0xf, true)));
                top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x4e, 0xf, 0xf, true)));
                const uint32_t byte = mx4_scale<X>(top);
                const uint32_t codes = byte == kMx4NaN ? 0u : v[k].codes(mx4_unit(byte));
                if (item < items) {
                    reinterpret_cast<uint32_t *>(codes_lds)[item] = codes;
                    if (item % 4 == 0) scales_lds[item / 4] = static_cast<uint8_t>(byte);
                }
            }
        }
        sync_lds();
        a_codes = codes_lds;
        a_bytes = scales_lds;
    }

    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t at[2];                            // a row's two pieces
#pragma unroll
    for (uint32_t s = 0; s < 2; ++s) at[s] = r * 128 + (((2 * q + s) ^ ((r >> 1) & 7u)) << 4);
    uint32_t cur = 0, far = (S - 1) * kStage;
    for (uint32_t unit = begin; unit < end; ++unit) {
        if (unit + S - 2 < end) wait_own<(S - 2) * kLoads>();
        else wait_own<0>();
        if (unit + S - 1 < end) load_unit(unit + S - 1, far);
        const bool absent = 2 * unit + 1 == k128 && q >= 2;   // blocks past the end: zeros
        i32x4 b[2];
        const uint32_t sb = *reinterpret_cast<const uint16_t *>(ring + cur + kScales + 8 * r + 2 * q);
#pragma unroll
        for (uint32_t s = 0; s < 2; ++s) {
            b[s] = *reinterpret_cast<const i32x4 *>(ring + cur + at[s]);
            if (absent) b[s] = i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (uint32_t i = 0; i < MT; ++i) {
            i32x4 a[2];
            uint32_t sa;
            if constexpr (FUSED) {
                const uint32_t block = min(16 * i + r, g.M - 1) * blocks + min(8 * unit + 2 * q, blocks - 2);
                sa = *reinterpret_cast<const uint16_t *>(a_bytes + block);
                a[0] = *reinterpret_cast<const i32x4 *>(a_codes + 16 * block);
                a[1] = *reinterpret_cast<const i32x4 *>(a_codes + 16 * block + 16);
            } else {
                sa = *reinterpret_cast<const uint16_t *>(ring + cur + kScales + 128 * (1 + i) + 8 * r + 2 * q);
                a[0] = *reinterpret_cast<const i32x4 *>(ring + cur + 2048 * (1 + i) + at[0]);
                a[1] = *reinterpret_cast<const i32x4 *>(ring + cur + 2048 * (1 + i) + at[1]);
            }
            acc[i] = mx4_multiply<0, 0>(b[0], sb, a[0], sa, acc[i]);
            acc[i] = mx4_multiply<1, 1>(b[1], sb, a[1], sa, acc[i]);
        }
        cur = cur == (S - 1) * kStage ? 0 : cur + kStage;
        far = far == (S - 1) * kStage ? 0 : far + kStage;
    }

    sync_lds();                                // nobody reads a ring or A any more
    f32x4 *sums = reinterpret_cast<f32x4 *>(few_lds);
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[(wave * MT + i) * 64 + lane] = acc[i];
    sync_lds();
    for (uint32_t t = threadIdx.x; t < 64 * MT; t += blockDim.x) {   // (blockDim.x is a multiple of 64: r and q stay)
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

// A is rounded by every workgroup where that is worth less than a launch: up to 16 rows and 8 KB of codes and scales (1 x 4096 x 1024: 3.4 us, 4.5 with a launch before; 16 x 4096 x 1024, 8.7 KB:
// 5.1 and 4.8; 29 x 4096 x 1024: 7.6 and 5.1).
constexpr uint32_t kFusedRows = 16;
constexpr uint64_t kFusedBytes = 8192;
static uint64_t rounded_bytes(uint32_t M, uint32_t K) { return static_cast<uint64_t>(M) * (mx4_padded(K) / 32) * 17; }
bool mx4_few_rounds(uint32_t M, uint32_t K) { return M <= kFusedRows && rounded_bytes(M, K) <= kFusedBytes; }

// Up to 32 rows, unless the contraction is long and B narrow: it is cut into four waves' shares here, whose units of 256 take 0.24 us each one after the other (0.44 with more than 16 rows, since the ring
// has two stages then), while tiles cut it over the whole chip.  Linear layers in bf16, us, here and in tiles, 16 rows: 16 x 32768 13.1 and 14.5, 16 x 49152 19.8 and 15.7, 33 x 1048576 518 and 93, 2048 x 20480
// 18.3 and 17.7, 2048 x 49152 34.0 and 26.5; wider ones are bound by the weights' way through memory, 4096 x 49152 39.5 and 40.8, 8192 x 49152 70 and 69 (one row 50).  32 rows: 512 x 16384 12.8 and 14.8, 16 x 24576
// 16.2 and 14.2, 512 x 32768 22.9 and 16.8, 33 x 1048576 749 and 93, 4096 x 24576 27.5 and 25.2, 8192 x 16384 31.3 and 30.3, 8192 x 28672 53.6 and 43.5.
constexpr uint32_t kLongOf16 = 40960, kLongOf32 = 20480, kWide = 2048;
bool mx4_few(uint32_t M, uint32_t N, uint32_t K) {
    if (M <= 16) return K <= kLongOf16 || N > kWide;
    return M <= 32 && K <= kLongOf32;
}

template <int MT, int S, bool FUSED, typename T, typename X>
static int launch_rows(const Mx4GemmArgs &ga, const Mx4Rows &rows, hipStream_t st) {
    constexpr uint32_t kOperands = FUSED ? 1 : 1 + MT, kStage = 2048 * kOperands + 256 * ((kOperands + 1) / 2);
    const uint32_t units = (ga.K + 255) / 256, waves = units < 4 ? units : 4;
    const size_t ring = waves * S * kStage + (FUSED ? rounded_bytes(ga.M, ga.K) : 0), joined = waves * MT * 1024;
    mx4_few_kernel<MT, S, FUSED, T, X><<<dim3((ga.N + 15) / 16), dim3(64 * waves), ring > joined ? ring : joined, st>>>(ga, rows);
    return static_cast<int>(hipGetLastError());
}

template <typename T>
static int launch_typed(const Mx4GemmArgs &ga, const Mx4Rows *rows, hipStream_t st) {
    if (!rows) return ga.M <= 16 ? launch_rows<1, 3, false, T, T>(ga, Mx4Rows{}, st) : launch_rows<2, 2, false, T, T>(ga, Mx4Rows{}, st);
    return rows->bf16 ? launch_rows<1, 4, true, T, BF16>(ga, *rows, st) : launch_rows<1, 4, true, T, F32>(ga, *rows, st);
}

int launch_mx4_few(const Mx4GemmArgs &ga, const Mx4Rows *rows, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch_typed<BF16>(ga, rows, st) : launch_typed<F32>(ga, rows, st);
}

}  // namespace omc
