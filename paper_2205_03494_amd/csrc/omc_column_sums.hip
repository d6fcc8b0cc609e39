// The last step of every sum over rows (dgamma, dbeta, dbias): the partial sums that the workgroups left, added up in a fixed order.
#include "omc_column_sums.h"

namespace omc {

template <int CHAINS, bool FOURS>
__global__ __launch_bounds__(1024) void column_sums_kernel(ColumnSums cs) {
    __shared__ float part[16][32];
    column_sums<16, CHAINS, FOURS>(cs, blockIdx.x, part);
}

template <bool FOURS>
static void launch(const ColumnSums &cs, hipStream_t st) {
    const dim3 grid((cs.width + 31) / 32), block(1024);
    if (cs.count <= 64) column_sums_kernel<1, FOURS><<<grid, block, 0, st>>>(cs);
    else if (cs.count <= 128) column_sums_kernel<2, FOURS><<<grid, block, 0, st>>>(cs);
    else if (FOURS || cs.count <= 256) column_sums_kernel<4, FOURS><<<grid, block, 0, st>>>(cs);
    else column_sums_kernel<8, false><<<grid, block, 0, st>>>(cs);
}
int launch_column_sums(const float *parts, uint32_t count, bool fours, uint32_t cols, uint32_t width, float *out0, float *out1, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const ColumnSums cs{parts, count, cols, width, out0, out1};
    if (fours) launch<true>(cs, st);
    else launch<false>(cs, st);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
