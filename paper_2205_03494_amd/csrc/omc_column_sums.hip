// The last step of every sum over rows (dgamma, dbeta, dbias): the partial sums that the workgroups left, added up in a fixed order.
#include "omc_mx4.h"

namespace omc {

// A workgroup takes 64 columns; its sixteen waves share out the rows, each in four chains, and are joined in order.
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *parts, uint32_t count, uint32_t cols, uint32_t width, float *out0, float *out1) {
    __shared__ float part[16][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < width) {
        const float *p = parts + col;
        uint32_t i = wave;
        for (; i + 48 < count; i += 64) {
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c) s[c] += p[static_cast<uint64_t>(i + 16 * c) * width];
        }
        for (uint32_t c = 0; i < count; i += 16, ++c) s[c] += p[static_cast<uint64_t>(i) * width];
    }
    part[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wave > 0 || col >= width) return;
    float sum = part[0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += part[w][lane];
    if (col < cols) {
        if (out0) out0[col] = sum;
    } else if (out1) {
        out1[col - cols] = sum;
    }
}

int launch_column_sums(const float *parts, uint32_t count, uint32_t cols, uint32_t width, float *out0, float *out1, void *stream) {
    column_sums_kernel<<<dim3((width + 63) / 64), dim3(1024), 0, static_cast<hipStream_t>(stream)>>>(parts, count, cols, width, out0, out1);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
