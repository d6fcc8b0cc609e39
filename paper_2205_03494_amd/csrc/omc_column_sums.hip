// The last step of every sum over rows (dgamma, dbeta, dbias): the partial sums that the workgroups left, added up in a fixed order.
#include "omc_column_sums.h"

namespace omc {

template <int CHAINS>
__global__ __launch_bounds__(1024) void column_sums_kernel(ColumnSums cs) {
    __shared__ float part[16][32];
    column_sums<16, CHAINS>(cs, blockIdx.x, part);
}

int launch_column_sums(const float *parts, uint32_t count, uint32_t cols, uint32_t width, float *out0, float *out1, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const ColumnSums cs{parts, count, cols, width, out0, out1};
    const dim3 grid((width + 31) / 32), block(1024);
    if (count <= 64) column_sums_kernel<1><<<grid, block, 0, st>>>(cs);
    else if (count <= 128) column_sums_kernel<2><<<grid, block, 0, st>>>(cs);
    else if (count <= 256) column_sums_kernel<4><<<grid, block, 0, st>>>(cs);
    else column_sums_kernel<8><<<grid, block, 0, st>>>(cs);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
