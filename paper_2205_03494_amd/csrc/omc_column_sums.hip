// The last step of every sum over rows (dgamma, dbeta, dbias): the partial sums that the workgroups left, added up in a fixed order.
#include "omc_mx4.h"

namespace omc {

// A workgroup takes 32 columns: sixteen lanes two each, so that the groups of sixteen lanes read a cache line of 64 rows at a time, and CHAINS such reads are on their way together.  The
// chains, the groups of a wave and the waves are joined in order.  Bound by the way to memory and back, since other XCDs' caches hold what it reads: 4 us for 16 rows or 512, of 1024 columns,
// against 2.4 us for next to none.
template <int CHAINS>
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *parts, uint32_t count, uint32_t cols, uint32_t width, float *out0, float *out1) {
    __shared__ float part[16][32];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, mine = threadIdx.x >> 4, col = blockIdx.x * 32 + 2 * (lane & 15u);
    const float *p = parts + min(col, width - 1);
    const uint32_t pair = col + 1 < width ? 1 : 0;
    float s[CHAINS][2] = {};
    for (uint32_t first = 0; first < count; first += 64 * CHAINS) {
        float v[CHAINS][2];
#pragma unroll
        for (uint32_t c = 0; c < CHAINS; ++c) {
            const float *from = p + static_cast<uint64_t>(min(first + 64 * c + mine, count - 1)) * width;
            v[c][0] = from[0];
            v[c][1] = from[pair];
        }
#pragma unroll
        for (uint32_t c = 0; c < CHAINS; ++c) {
            const bool there = first + 64 * c + mine < count;
            s[c][0] += there ? v[c][0] : 0.0f;
            s[c][1] += there ? v[c][1] : 0.0f;
        }
    }
#pragma unroll
    for (uint32_t e = 0; e < 2; ++e) {
        float sum = s[0][e];
#pragma unroll
        for (uint32_t c = 1; c < CHAINS; ++c) sum += s[c][e];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) part[wave][2 * lane + e] = sum;
    }
    __syncthreads();
    const uint32_t mine_col = blockIdx.x * 32 + lane;
    if (threadIdx.x >= 32 || mine_col >= width) return;
    float sum = part[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += part[w][lane];
    if (mine_col < cols) {
        if (out0) out0[mine_col] = sum;
    } else if (out1) {
        out1[mine_col - cols] = sum;
    }
}

int launch_column_sums(const float *parts, uint32_t count, uint32_t cols, uint32_t width, float *out0, float *out1, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((width + 31) / 32), block(1024);
    if (count <= 64) column_sums_kernel<1><<<grid, block, 0, st>>>(parts, count, cols, width, out0, out1);
    else if (count <= 128) column_sums_kernel<2><<<grid, block, 0, st>>>(parts, count, cols, width, out0, out1);
    else if (count <= 256) column_sums_kernel<4><<<grid, block, 0, st>>>(parts, count, cols, width, out0, out1);
    else column_sums_kernel<8><<<grid, block, 0, st>>>(parts, count, cols, width, out0, out1);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
