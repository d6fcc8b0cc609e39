// Device code of the sums over rows of partial sums (dgamma, dbeta, dbias).
#pragma once
#include "omc_mx4.h"

namespace omc {

// The first `cols` of the `width` columns' sums over `count` rows go to out0, the others to out1; either may be null.
struct ColumnSums {
    const float *parts;
    uint32_t count, cols, width;
    float *out0, *out1;
};

// A workgroup takes 32 columns and the rows in 16 shares, as many as it has waves at a time: sixteen lanes of a share take two columns each, so that the groups of sixteen lanes read a cache line of 64
// rows between them, and CHAINS such reads are on their way together.  The chains, the groups of a share and the shares are joined in order.  The order is the same for all numbers of waves, and for all of chains
// from count / 64 on, or from 8 on: chains without a row add zeros.  FOURS: a row is four that lie one after the other, added first, in order.  Bound by the way to memory and back, since other XCDs' caches hold what it reads: 4 us for 16 rows or 512, of 1024 columns,
// against 2.4 us for next to none.
template <int WAVES, int CHAINS, bool FOURS>
__device__ __forceinline__ void column_sums(const ColumnSums &cs, uint32_t block, float (*part)[32]) {
    constexpr uint32_t kShares = 16, kEach = FOURS ? 4 : 1;
    const float *parts = cs.parts;
    const uint32_t count = cs.count, cols = cs.cols, width = cs.width;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = block * 32 + 2 * (lane & 15u);
    const float *p = parts + min(col, width - 1);
    const uint32_t pair = col + 1 < width ? 1 : 0;
    for (uint32_t share = wave; share < kShares; share += WAVES) {
        const uint32_t mine = 4 * share + (lane >> 4);
        float s[CHAINS][2] = {};
        for (uint32_t first = 0; first + 4 * share < count; first += 4 * kShares * CHAINS) {
            float v[CHAINS][kEach][2];
#pragma unroll
            for (uint32_t c = 0; c < CHAINS; ++c)
#pragma unroll
                for (uint32_t k = 0; k < kEach; ++k) {
                    const float *from = p + (static_cast<uint64_t>(min(first + 4 * kShares * c + mine, count - 1)) * kEach + k) * width;
                    v[c][k][0] = from[0];
                    v[c][k][1] = from[pair];
                }
#pragma unroll
            for (uint32_t c = 0; c < CHAINS; ++c)
#pragma unroll
                for (uint32_t k = 1; k < kEach; ++k) {
                    v[c][0][0] += v[c][k][0];
                    v[c][0][1] += v[c][k][1];
                }
#pragma unroll
            for (uint32_t c = 0; c < CHAINS; ++c) {
                const bool there = first + 4 * kShares * c + mine < count;
                s[c][0] += there ? v[c][0][0] : 0.0f;
                s[c][1] += there ? v[c][0][1] : 0.0f;
            }
        }
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e) {
            float sum = s[0][e];
#pragma unroll
            for (uint32_t c = 1; c < CHAINS; ++c) sum += s[c][e];
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (lane < 16) part[share][2 * lane + e] = sum;
        }
    }
    __syncthreads();
    const uint32_t mine_col = block * 32 + lane;
    if (threadIdx.x >= 32 || mine_col >= width) return;
    float sum = part[0][lane];
#pragma unroll
    for (uint32_t w = 1; w < kShares; ++w) sum += part[w][lane];
    if (mine_col < cols) {
        if (cs.out0) cs.out0[mine_col] = sum;
    } else if (cs.out1) {
        cs.out1[mine_col - cols] = sum;
    }
}

}  // namespace omc
