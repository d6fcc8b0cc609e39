// What the gated linear layer's products take: operands in bf16 with padded rows, and dg and du with partial sums of their columns.  Bound by memory.
// 8192 x 4096 in bf16: 58 - 61 us, 5.6 TB/s of 335 MB, a large copy's rate.
#include "omc_mx4.h"
#include "omc_product.h"

namespace omc {

struct Packs {
    PackArgs p[kMostPacks];
    uint32_t groups[kMostPacks];               // workgroups of each
};

template <typename T>
__device__ __forceinline__ u32x4 eight_bf16(const Eight<T> &v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T::kBytes == 2) w[i] = v.w[i];
        else w[i] = to_bf16_pair(v.value(2 * i), v.value(2 * i + 1));
    }
    return w;
}
// A lane takes eight values; workgroups more than one, where a launch has too few.
template <typename T>
__device__ __forceinline__ void pack_pieces(const PackArgs &p, uint32_t group, uint32_t groups) {
    const uint32_t pieces = p.pitch / 8;
    const uint64_t step = groups * 256ull;
    uint64_t at = group * 256ull;
    for (;;) {
        const uint32_t row0 = static_cast<uint32_t>(at / pieces), rest = static_cast<uint32_t>(at - static_cast<uint64_t>(row0) * pieces) + threadIdx.x;
        if (row0 >= p.to_rows) return;
        const uint32_t down = rest / pieces, row = row0 + down, col = 8 * (rest - down * pieces);
        if (row < p.to_rows) {
            Eight<T> v;
            v.clear();
            if (row < p.rows && col < p.cols) v.load(static_cast<const typename T::type *>(p.x) + row * p.ldx, col, p.cols);
            *reinterpret_cast<u32x4 *>(p.to + row * static_cast<uint64_t>(p.pitch) + col) = eight_bf16(v);
        }
        at += step;
    }
}
__device__ __forceinline__ void pack(const Packs &packs, uint32_t group) {
    const uint32_t second = packs.groups[0], third = second + packs.groups[1], i = group < second ? 0u : group < third ? 1u : 2u;
    const PackArgs &p = packs.p[i];            // (by number: the arguments stay where they are)
    group -= i == 0 ? 0u : i == 1 ? second : third;
    p.bf16 ? pack_pieces<BF16>(p, group, packs.groups[i]) : pack_pieces<F32>(p, group, packs.groups[i]);
}
constexpr uint64_t kMostGroups = 1u << 21;     // of a copy; a launch's work-items within 32 bits
static Packs packs_of(const PackArgs *packs, uint32_t count, uint32_t &groups) {
    Packs all{};
    groups = 0;
    for (uint32_t i = 0; i < count; ++i) {
        all.p[i] = packs[i];
        const uint64_t n = static_cast<uint64_t>(packs[i].to_rows) * (packs[i].pitch / 8);
        const uint64_t wanted = (n + 255) / 256;
        all.groups[i] = static_cast<uint32_t>(wanted < kMostGroups ? wanted : kMostGroups);
        groups += all.groups[i];
    }
    return all;
}
__global__ __launch_bounds__(256) void pack_kernel(Packs packs) { pack(packs, blockIdx.x); }
int launch_pack(const PackArgs *packs, uint32_t count, void *stream) {
    uint32_t groups;
    const Packs all = packs_of(packs, count, groups);
    pack_kernel<<<dim3(groups), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(all);
    return static_cast<int>(hipGetLastError());
}

// A workgroup takes 4 * EACH rows x 512 columns, a wave every fourth row, a lane eight columns.  The workgroups behind theirs copy operands.  Of few rows a wave asks for all four together; of many for one at a time, which leaves
// registers for more waves (8192 x 4096, bf16, sums alone: four at a time 47 us, two 44, one 41).
struct SlopeGrid {
    SlopeArgs s;
    uint32_t across, groups;
    Packs packs;
};
// (SHORT: rows of fewer than eight values.)
template <typename T, int EACH, bool SHORT>
__global__ __launch_bounds__(256) void slopes_kernel(SlopeGrid sg) {
    __shared__ float sums[4][2][512];
    if (blockIdx.x >= sg.groups) {
        pack(sg.packs, blockIdx.x - sg.groups);
        return;
    }
    const SlopeArgs &sa = sg.s;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, down = blockIdx.x / sg.across, col0 = (blockIdx.x - down * sg.across) * 512, col = col0 + 8 * lane, row0 = down * (4 * EACH);
    constexpr uint32_t kTogether = EACH == 4 ? 4 : 1;
    float s[2][8] = {};
#pragma unroll 1
    for (uint32_t first = 0; first < EACH; first += kTogether) {
        Eight<T> dh[kTogether];
        Eight<BF16> slope[kTogether][2];
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k) {
            const uint32_t row = row0 + 4 * (first + k) + wave;
            dh[k].clear();
            slope[k][0].clear();
            slope[k][1].clear();
            if (row < sa.M && col < sa.N) {
                dh[k].template fetch<SHORT>(static_cast<const typename T::type *>(sa.dh) + row * sa.lddh, col, sa.N);
                slope[k][0].template fetch<SHORT>(sa.slope_g + row * sa.ld_slope, col, sa.N);
                slope[k][1].template fetch<SHORT>(sa.slope_u + row * sa.ld_slope, col, sa.N);
            }
        }
        const uint32_t missing = Eight<T>::missing(col, sa.N);   // of a row's last piece; nothing waits between the loads
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k) {
            dh[k].settle(missing);
            slope[k][0].settle(missing);
            slope[k][1].settle(missing);
        }
#pragma unroll
        for (uint32_t k = 0; k < kTogether; ++k) {
            const uint32_t row = row0 + 4 * (first + k) + wave;
            u32x4 w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[e] = dh[k].value(e) * slope[k][h].value(e);
                    s[h][e] += d[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) w[h][e] = to_bf16_pair(d[2 * e], d[2 * e + 1]);
            }
            if (sa.to && row < sa.to_rows && col < sa.half) {
                uint16_t *to = sa.to + row * (2ull * sa.half) + col;
                *reinterpret_cast<u32x4 *>(to) = w[0];
                *reinterpret_cast<u32x4 *>(to + sa.half) = w[1];
            }
        }
    }
    if (!sa.sums || row0 >= sa.M) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave][h][8 * lane + e] = s[h][e];
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 1024; t += 256) {
        const uint32_t h = t / 512, c = t % 512, n = col0 + c;
        if (n < sa.N) sa.sums[(static_cast<uint64_t>(down) * 2 + h) * sa.N + n] = ((sums[0][h][c] + sums[1][h][c]) + sums[2][h][c]) + sums[3][h][c];
    }
}
// 16 rows a workgroup where 64 would leave compute units without one: 1003 x 971 in fp32, with copies of X and the weights in the same launch, 23 us with 64 rows and 6.7 with 16.
uint32_t slope_rows(uint32_t M, uint32_t N) { return static_cast<uint64_t>((M + 63) / 64) * ((N + 511) / 512) >= 512 ? 64 : 16; }

template <typename T>
static void launch_typed(const SlopeGrid &sg, uint32_t rows, uint32_t groups, hipStream_t st) {
    if (sg.s.N < 8) rows == 64 ? slopes_kernel<T, 16, true><<<dim3(groups), dim3(256), 0, st>>>(sg) : slopes_kernel<T, 4, true><<<dim3(groups), dim3(256), 0, st>>>(sg);
    else if (rows == 64) slopes_kernel<T, 16, false><<<dim3(groups), dim3(256), 0, st>>>(sg);
    else slopes_kernel<T, 4, false><<<dim3(groups), dim3(256), 0, st>>>(sg);
}
int launch_slopes(const SlopeArgs &sa, const PackArgs *packs, uint32_t count, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t rows = slope_rows(sa.M, sa.N), across = (sa.half + 511) / 512, groups = (sa.to_rows + rows - 1) / rows * across;
    uint32_t more;
    const Packs all = packs_of(packs, count, more);
    const SlopeGrid sg{sa, across, groups, all};
    if (sa.bf16) launch_typed<BF16>(sg, rows, groups + more, st);
    else launch_typed<F32>(sg, rows, groups + more, st);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
