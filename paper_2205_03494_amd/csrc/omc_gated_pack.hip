// What the gated linear layer's products take: operands in bf16 with padded rows, and dg and du.
#include "omc_mx4.h"
#include "omc_product.h"

namespace omc {

struct Packs {
    PackArgs p[kMostPacks];
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
__global__ __launch_bounds__(256) void pack_kernel(Packs packs) {
    const PackArgs &p = packs.p[blockIdx.y];
    const uint32_t pieces = p.pitch / 8;
    const uint64_t count = static_cast<uint64_t>(p.to_rows) * pieces;
    for (uint64_t at = blockIdx.x * 256ull + threadIdx.x; at < count; at += gridDim.x * 256ull) {
        const uint32_t row = static_cast<uint32_t>(at / pieces), col = 8 * static_cast<uint32_t>(at % pieces);
        u32x4 w = {0, 0, 0, 0};
        if (row < p.rows && col < p.cols) {
            if (p.bf16) {
                Eight<BF16> v;
                v.load(static_cast<const uint16_t *>(p.x) + row * p.ldx, col, p.cols);
                w = eight_bf16(v);
            } else {
                Eight<F32> v;
                v.load(static_cast<const float *>(p.x) + row * p.ldx, col, p.cols);
                w = eight_bf16(v);
            }
        }
        *reinterpret_cast<u32x4 *>(p.to + row * static_cast<uint64_t>(p.pitch) + col) = w;
    }
}
int launch_pack(const PackArgs *packs, uint32_t count, void *stream) {
    Packs all{};
    uint64_t most = 0;
    for (uint32_t i = 0; i < count; ++i) {
        all.p[i] = packs[i];
        const uint64_t n = static_cast<uint64_t>(packs[i].to_rows) * (packs[i].pitch / 8);
        most = n > most ? n : most;
    }
    const uint64_t groups = (most + 255) / 256;
    pack_kernel<<<dim3(static_cast<uint32_t>(groups < 8192 ? groups : 8192), count), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(all);
    return static_cast<int>(hipGetLastError());
}

// A workgroup takes kSlopeRows rows x 512 columns, a wave every fourth row, a lane eight columns.
template <typename T>
__global__ __launch_bounds__(256) void slopes_kernel(SlopeArgs sa) {
    __shared__ float sums[4][2][512];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = blockIdx.x * 512 + 8 * lane, row0 = blockIdx.y * kSlopeRows;
    float s[2][8] = {};
#pragma unroll 4
    for (uint32_t i = 0; i < kSlopeRows / 4; ++i) {
        const uint32_t row = row0 + 4 * i + wave;
        if (row >= sa.to_rows) break;
        u32x4 w[2] = {};
        if (row < sa.M && col < sa.N) {
            Eight<T> dh;
            Eight<BF16> slope[2];
            dh.load(static_cast<const typename T::type *>(sa.dh) + row * sa.lddh, col, sa.N);
            slope[0].load(sa.slope_g + row * sa.ld_slope, col, sa.N);
            slope[1].load(sa.slope_u + row * sa.ld_slope, col, sa.N);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[e] = dh.value(e) * slope[h].value(e);
                    s[h][e] += d[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) w[h][e] = to_bf16_pair(d[2 * e], d[2 * e + 1]);
            }
        }
        if (sa.to && col < sa.half) {
            uint16_t *to = sa.to + row * (2ull * sa.half) + col;
            *reinterpret_cast<u32x4 *>(to) = w[0];
            *reinterpret_cast<u32x4 *>(to + sa.half) = w[1];
        }
    }
    if (!sa.sums || row0 >= sa.M) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave][h][8 * lane + e] = s[h][e];
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < 1024; t += 256) {
        const uint32_t h = t / 512, c = t % 512, n = blockIdx.x * 512 + c;
        if (n < sa.N) sa.sums[(static_cast<uint64_t>(blockIdx.y) * 2 + h) * sa.N + n] = ((sums[0][h][c] + sums[1][h][c]) + sums[2][h][c]) + sums[3][h][c];
    }
}
int launch_slopes(const SlopeArgs &sa, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((sa.half + 511) / 512, (sa.to_rows + kSlopeRows - 1) / kSlopeRows), block(256);
    if (sa.bf16) slopes_kernel<BF16><<<grid, block, 0, st>>>(sa);
    else slopes_kernel<F32><<<grid, block, 0, st>>>(sa);
    return static_cast<int>(hipGetLastError());
}

}  // namespace omc
