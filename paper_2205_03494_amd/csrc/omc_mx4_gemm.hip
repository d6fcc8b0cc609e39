// omc_mx4_gemm: C[M x N] = A[M x K] B[N x K]^T + bias, both operands in MX4, on the scaled matrix instructions (16 x 16 results over 128 values).
//
// Codes and scales go from global memory straight into a ring of S LDS stages of 256 values of K: a row's stage is 128 bytes of codes, eight pieces of 16 bytes that are
// a block each, and 8 scale bytes.  In step s of a stage's two, lane l multiplies block 2 (l / 16) + s of its row: the order of K is free as long as both operands agree, and this
// one puts the scales of a lane's two steps next to each other.  The last stage may be half one (an odd number of 128s): its lanes bring the
// first half twice instead of reading past the row, and one step multiplies the blocks l / 16.
//
// Pieces are XOR-swizzled on their way in, so that the 16 that one read takes at a time lie on different banks.  The B operand comes first in the instruction, and row i of B's tile t in a
// group of four is column 16 (i / 4) + 4 t + i % 4 of the group's 64: a lane then holds 16 neighbours of a row of C, and four lanes 64.
#include "omc_mma.h"
#include "omc_mx4.h"

namespace omc {

// One wave copies 64 dwords from global memory into 256 bytes of LDS at `dst`, lane l's to dst + 4 l.  (See load_to_lds.)
__device__ __forceinline__ void load_dwords_to_lds(const uint8_t *base, uint32_t off, uint32_t dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(dst), "v"(off), "s"(base) : "memory", "m0");
}

struct Mx4TileArgs {
    Mx4GemmArgs g;
    uint32_t tiles_m, tiles_n;
    uint32_t stages_per_split;
};

// WM x WN waves of TM x (4 TG) matrix tiles.  SPLIT: the contraction is cut into gridDim.y parts, whose results go to g.parts in fp32.
template <int WM, int WN, int TM, int TG, int S, int OCC, typename T, bool SPLIT>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * WM * WN, 64 * WM * WN))) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
void mx4_gemm_kernel(Mx4TileArgs ta) {
    constexpr int NW = WM * WN, BM = 16 * TM * WM, BN = 64 * TG * WN, TN = 4 * TG;
    constexpr int kALoads = BM / 8 / NW, kBLoads = BN / 8 / NW, kScaleUnits = (BM + BN) / 32, kSLoads = (kScaleUnits + NW - 1) / NW;
    constexpr int kLoads = kALoads + kBLoads + kSLoads;
    constexpr uint32_t kA = 0, kB = BM * 128, kSA = kB + BN * 128, kStage = kSA + (BM + BN) * 8;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole loads");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[S * kStage];
    const Mx4GemmArgs &g = ta.g;
    const uint32_t lds0 = lds_offset(lds);
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    uint32_t m0, n0;
    tile_of_block(BM == 256 ? 4 : 8, ta.tiles_m, ta.tiles_n, m0, n0);
    m0 *= BM;
    n0 *= BN;
    const uint32_t k128 = (g.K + 127) / 128, all_stages = (k128 + 1) / 2;
    const uint32_t first = SPLIT ? blockIdx.y * ta.stages_per_split : 0u;
    const uint32_t stages = SPLIT ? min(ta.stages_per_split, all_stages - first) : all_stages;
    const bool half_end = (k128 & 1u) != 0 && first + stages == all_stages;
    const uint32_t row_bytes = k128 * 64, row_scales = k128 * 4;

    // ---- global -> LDS
    const uint8_t *a_from = g.a.codes + static_cast<uint64_t>(m0) * row_bytes + first * 128;
    const uint8_t *b_from = g.b.codes + static_cast<uint64_t>(n0) * row_bytes + first * 128;
    const uint8_t *sa_from = g.a.scales + static_cast<uint64_t>(m0) * row_scales + first * 8;
    const uint8_t *sb_from = g.b.scales + static_cast<uint64_t>(n0) * row_scales + first * 8;
    const uint32_t last_m = g.M - 1 - m0, last_n = g.N - 1 - n0;   // rows past the end: the last one again
    uint32_t a_off[kALoads], b_off[kBLoads], s_off[kSLoads];
    uint32_t upper = 0;                        // bit i: this lane's piece of load i lies in the second half of a stage
#pragma unroll
    for (uint32_t i = 0; i < kALoads; ++i) {
        const uint32_t row = 8 * (wave + NW * i) + (lane >> 3), piece = (lane & 7u) ^ ((row >> 1) & 7u);
        a_off[i] = min(row, last_m) * row_bytes + piece * 16;
        upper |= (piece >> 2) << i;
    }
#pragma unroll
    for (uint32_t i = 0; i < kBLoads; ++i) {
        const uint32_t row = 8 * (wave + NW * i) + (lane >> 3), piece = (lane & 7u) ^ (((row >> 1) & 1u) + 2 * ((row >> 4) & 3u));
        b_off[i] = min(row, last_n) * row_bytes + piece * 16;
        upper |= (piece >> 2) << (kALoads + i);
    }
#pragma unroll
    for (uint32_t i = 0; i < kSLoads; ++i) {
        const uint32_t unit = min(wave + NW * i, static_cast<uint32_t>(kScaleUnits - 1)), row = 32 * unit + (lane >> 1);
        s_off[i] = (row < BM ? min(row, last_m) : min(row - BM, last_n)) * row_scales + 4 * (lane & 1u);
    }
    auto load_stage = [&](uint32_t at, bool half) {
#pragma unroll
        for (uint32_t i = 0; i < kALoads; ++i)
            load_to_lds(a_from, half ? a_off[i] - 64 * ((upper >> i) & 1u) : a_off[i], lds0 + at + kA + 1024 * (wave + NW * i));
#pragma unroll
        for (uint32_t i = 0; i < kBLoads; ++i)
            load_to_lds(b_from, half ? b_off[i] - 64 * ((upper >> (kALoads + i)) & 1u) : b_off[i], lds0 + at + kB + 1024 * (wave + NW * i));
#pragma unroll
        for (uint32_t i = 0; i < kSLoads; ++i) {
            const uint32_t unit = min(wave + NW * i, static_cast<uint32_t>(kScaleUnits - 1));
            load_dwords_to_lds(unit < BM / 32 ? sa_from : sb_from, half ? s_off[i] - 4 * (lane & 1u) : s_off[i], lds0 + at + kSA + 256 * unit);
        }
        a_from += 128;
        b_from += 128;
        sa_from += 8;
        sb_from += 8;
    };

    // ---- LDS -> fragments
    const uint32_t r = lane & 15u, q = lane >> 4;
    const uint32_t a_row = 16 * TM * wm + r, b_row = 64 * TG * wn + 16 * (r >> 2) + (r & 3u);
    const uint32_t a_swz = (r >> 1) & 7u, b_swz = ((r >> 1) & 1u) + 2 * (r >> 2);
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto code = [&](uint32_t at) { return *reinterpret_cast<const i32x4 *>(lds + at); };
    auto multiply_stage = [&](uint32_t at) {
        uint32_t sa[TM], sb[TN];
#pragma unroll
        for (uint32_t i = 0; i < TM; ++i) sa[i] = *reinterpret_cast<const uint16_t *>(lds + at + kSA + (a_row + 16 * i) * 8 + 2 * q);
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) sb[j] = *reinterpret_cast<const uint16_t *>(lds + at + kSA + (BM + b_row + 64 * (j / 4) + 4 * (j % 4)) * 8 + 2 * q);
        for_constants<2>([&](auto step) {
            constexpr int s = decltype(step)::value;
            const uint32_t a_at = at + kA + a_row * 128 + (((2 * q + s) ^ a_swz) << 4), b_at = at + kB + b_row * 128 + (((2 * q + s) ^ b_swz) << 4);
            i32x4 b[TN];
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j) b[j] = code(b_at + 8192 * (j / 4) + 512 * (j % 4));
#pragma unroll
            for (uint32_t i = 0; i < TM; ++i) {
                const i32x4 a = code(a_at + 2048 * i);
#pragma unroll
                for (uint32_t j = 0; j < TN; ++j) acc[i][j] = mx4_multiply<s, s>(b[j], sb[j], a, sa[i], acc[i][j]);
            }
        });
    };
    auto multiply_half = [&](uint32_t at) {
        const uint32_t a_at = at + kA + a_row * 128 + ((q ^ a_swz) << 4), b_at = at + kB + b_row * 128 + ((q ^ b_swz) << 4);
        i32x4 b[TN];
        uint32_t sb[TN];
#pragma unroll
        for (uint32_t j = 0; j < TN; ++j) {
            b[j] = code(b_at + 8192 * (j / 4) + 512 * (j % 4));
            sb[j] = lds[at + kSA + (BM + b_row + 64 * (j / 4) + 4 * (j % 4)) * 8 + q];
        }
#pragma unroll
        for (uint32_t i = 0; i < TM; ++i) {
            const i32x4 a = code(a_at + 2048 * i);
            const uint32_t sa = lds[at + kSA + (a_row + 16 * i) * 8 + q];
#pragma unroll
            for (uint32_t j = 0; j < TN; ++j) acc[i][j] = mx4_multiply<0, 0>(b[j], sb[j], a, sa, acc[i][j]);
        }
    };

    uint32_t cur = 0, far = (S - 1) * kStage;
#pragma unroll
    for (uint32_t i = 0; i < S - 1; ++i)
        if (i < stages) load_stage(i * kStage, half_end && i + 1 == stages);
    for (uint32_t j = 0; j < stages; ++j) {
        wait_stage<S, kLoads>(j, stages);
        if (j + S - 1 < stages) load_stage(far, half_end && j + S == stages);
        if (half_end && j + 1 == stages) multiply_half(cur);
        else multiply_stage(cur);
        cur = cur == (S - 1) * kStage ? 0 : cur + kStage;
        far = far == (S - 1) * kStage ? 0 : far + kStage;
    }

    // ---- a lane's runs of 16 neighbours
    float *parts = SPLIT ? g.parts + static_cast<uint64_t>(blockIdx.y) * g.M * g.N : nullptr;
#pragma unroll
    for (uint32_t gr = 0; gr < TG; ++gr) {
        const uint32_t n = n0 + 64 * (TG * wn + gr) + 16 * q;
        if (n >= g.N) continue;
        const uint32_t left = g.N - n;
        float bias[16];
#pragma unroll
        for (uint32_t e = 0; e < 16; ++e) bias[e] = !SPLIT && g.bias ? g.bias[min(n + e, g.N - 1)] : 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < TM; ++i) {
            const uint32_t m = m0 + a_row + 16 * i;
            if (m >= g.M) continue;
            float v[16];
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) v[e] = acc[i][4 * gr + e / 4][e % 4] + bias[e];
            if (SPLIT) store_run<F32, 16>(parts + static_cast<uint64_t>(m) * g.N + n, v, left);
            else store_run<T, 16>(static_cast<typename T::type *>(g.c) + m * g.ldc + n, v, left);
        }
    }
}

// The parts of a split contraction, added in order.
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

struct Mx4Choice {
    int tile;
    uint32_t bm, bn, splits;
};
static Mx4Choice choose(uint32_t M, uint32_t N, uint32_t K) {
    const uint32_t stages = (K + 255) / 256;
    const uint32_t sizes[3][2] = {{256, 256}, {128, 128}, {64, 64}};
    Mx4Choice c{2, 64, 64, 1};
    for (int i = 0; i < 3; ++i) {
        c = Mx4Choice{i, sizes[i][0], sizes[i][1], 1};
        if (static_cast<uint64_t>((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn) >= 256) return c;
    }
    const uint32_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
    uint32_t splits = 256 / tiles;
    if (splits > stages / 4) splits = stages / 4;
    if (splits > 8) splits = 8;
    c.splits = splits < 1 ? 1 : splits;
    return c;
}

size_t mx4_gemm_workspace(uint32_t M, uint32_t N, uint32_t K) {
    const Mx4Choice c = choose(M, N, K);
    return c.splits > 1 ? 4ull * c.splits * M * N : 0;
}

template <int WM, int WN, int TM, int TG, int S, int OCC, typename T>
static void launch_tile(const Mx4TileArgs &ta, uint32_t splits, hipStream_t st) {
    const dim3 grid(ta.tiles_m * ta.tiles_n, splits), block(64 * WM * WN);
    if (splits > 1) mx4_gemm_kernel<WM, WN, TM, TG, S, OCC, T, true><<<grid, block, 0, st>>>(ta);
    else mx4_gemm_kernel<WM, WN, TM, TG, S, OCC, T, false><<<grid, block, 0, st>>>(ta);
}

template <typename T>
static int launch(const Mx4GemmArgs &ga, hipStream_t st) {
    const Mx4Choice c = choose(ga.M, ga.N, ga.K);
    const uint32_t stages = (ga.K + 255) / 256, each = (stages + c.splits - 1) / c.splits, splits = (stages + each - 1) / each;
    const Mx4TileArgs ta{ga, (ga.M + c.bm - 1) / c.bm, (ga.N + c.bn - 1) / c.bn, each};
    switch (c.tile) {
        case 0: launch_tile<2, 4, 8, 1, 2, 2, T>(ta, splits, st); break;
        case 1: launch_tile<2, 2, 4, 1, 2, 2, T>(ta, splits, st); break;
        default: launch_tile<4, 1, 1, 1, 2, 4, T>(ta, splits, st); break;
    }
    if (splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return static_cast<int>(e);
        mx4_join_kernel<T><<<dim3((ga.N + 255) / 256, (ga.M + 3) / 4), dim3(256), 0, st>>>(ga, splits);
    }
    return static_cast<int>(hipGetLastError());
}

int launch_mx4_gemm(const Mx4GemmArgs &ga, bool bf16, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bf16 ? launch<BF16>(ga, st) : launch<F32>(ga, st);
}

}  // namespace omc
