// Matrix products in 8 bits, on the CUDA cores: tiles of 32 rows by 128 features, 32 elements of k at a time in shared memory.
#include <cuda_fp8.h>

#include "speca_matmul8_common.cuh"

namespace speca {
namespace {

constexpr int kTileM = 32, kTileN = 128, kTileK = 32;

__device__ __forceinline__ float from_e4m3(uint8_t code) {
    __nv_fp8_e4m3 v;
    v.__x = code;
    return static_cast<float>(v);
}
__device__ __forceinline__ float value8(const uint8_t* codes, int64_t stride, const uint8_t* scales, int64_t scale_stride, int row, int rows, int c, int k) {
    if (row >= rows || c >= k) return 0.f;
    const uint32_t byte = scales[c / (4 * kBlock8) * scale_stride + 4 * static_cast<int64_t>(row) + c / kBlock8 % 4];
    return from_e4m3(codes[row * stride + c]) * scale_of(byte);
}

template <int DT>
__global__ void __launch_bounds__(256) matmul8_kernel(const __grid_constant__ Matmul8Params p) {
    __shared__ float a[kTileM][kTileK + 1], w[kTileN][kTileK + 1];
    const int m0 = blockIdx.x * kTileM, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int n0 = blockIdx.y * kTileN; n0 < p.n; n0 += gridDim.y * kTileN) {
        float sum[4][4] = {};
        for (int k0 = 0; k0 < p.k; k0 += kTileK) {
            __syncthreads();
            for (int i = threadIdx.x; i < kTileM * kTileK; i += 256)
                a[i / kTileK][i % kTileK] = value8(p.a, p.a_stride, p.a_scales, p.a_scale_stride, m0 + i / kTileK, p.m, k0 + i % kTileK, p.k);
            for (int i = threadIdx.x; i < kTileN * kTileK; i += 256)
                w[i / kTileK][i % kTileK] = value8(p.w, p.w_stride, p.w_scales, p.w_scale_stride, n0 + i / kTileK, p.n, k0 + i % kTileK, p.k);
            __syncthreads();
            for (int k = 0; k < kTileK; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[i][j] = fmaf(a[warp * 4 + i][k], w[lane * 4 + j][k], sum[i][j]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = m0 + warp * 4 + i;
            if (row >= p.m) continue;
            const int seq = p.row_seq[row];
            if (p.dev_mask != nullptr && p.dev_mask[seq] == 0) continue;
            finish_block<DT>(p, row, seq, n0, lane, sum[i]);
        }
    }
}

}  // namespace

cudaError_t launch_matmul8(const Matmul8Params& p, int dtype, int, cudaStream_t stream) {
    if (p.m == 0) return cudaSuccess;
    const dim3 grid((p.m + kTileM - 1) / kTileM, min(65535, (p.n + kTileN - 1) / kTileN));
    if (dtype == SPECA_BF16)
        matmul8_kernel<SPECA_BF16><<<grid, 256, 0, stream>>>(p);
    else
        matmul8_kernel<SPECA_F32><<<grid, 256, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace speca
