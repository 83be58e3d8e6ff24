// Joins the partial results of rows whose keys were shared out over several units.
//
// Share s of a row left sums O_s, their divisor d_s, their weights' sum l_s and the maximum m_s they refer to; the row is
// sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) d_s with m the largest m_s, its log-sum that of the l_s, added up in the order of the
// shares. One warp per row: the statistics of 32 shares at once by the lanes, then the sums with the lanes across the head.
#include "speca_attention_common.cuh"

namespace speca {
namespace {

constexpr int kJoinWarps = 8;
constexpr int kAhead = 8;  // shares whose sums are on their way at once

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <typename T>
__global__ void __launch_bounds__(kJoinWarps * 32) join_kernel(const __grid_constant__ AttnParams p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");  // launched ahead of the end of the units
    const JoinBlock jb = p.joins[blockIdx.x];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int row = blockIdx.y * kJoinWarps + warp;
    if (row >= jb.rows || (p.dev_mask != nullptr && p.dev_mask[jb.seq] == 0)) return;
    const int64_t pitch = part_row_floats(p.head_dim), stride = jb.rows * pitch;
    const float* base = reinterpret_cast<const float*>(p.parts + jb.part) + row * pitch;
    float m = -CUDART_INF_F;
    for (int s = lane; s < jb.n_splits; s += 32) {
        const float2 stat = *reinterpret_cast<const float2*>(base + s * stride + pitch - 4);
        if (stat.y != 0.f) m = fmaxf(m, stat.x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float l = 0.f, d = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const bool holds = lane * 4 < p.head_dim;
    for (int s0 = 0; s0 < jb.n_splits; s0 += 32) {
        float w = 0.f, wl = 0.f, wd = 0.f;  // a share that saw nothing left its sums unwritten: weight zero, not read
        if (s0 + lane < jb.n_splits) {
            const float4 stat = *reinterpret_cast<const float4*>(base + (s0 + lane) * stride + pitch - 4);
            if (stat.y != 0.f) {
                w = exp2f(stat.x - m);
                wl = w * stat.y;
                wd = w * stat.z;
            }
        }
        const int n = min(32, jb.n_splits - s0);
        for (int s = 0; s < n; s += kAhead) {
            float4 v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float ws = __shfl_sync(0xffffffffu, w, (s + k) % 32);
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (s + k < n && holds && ws != 0.f) v[k] = *reinterpret_cast<const float4*>(base + (s0 + s + k) * stride + lane * 4);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (s + k >= n) break;
                const float ws = __shfl_sync(0xffffffffu, w, s + k);
                l += __shfl_sync(0xffffffffu, wl, s + k);
                d += __shfl_sync(0xffffffffu, wd, s + k);
                acc.x = fmaf(ws, v[k].x, acc.x);
                acc.y = fmaf(ws, v[k].y, acc.y);
                acc.z = fmaf(ws, v[k].z, acc.z);
                acc.w = fmaf(ws, v[k].w, acc.w);
            }
        }
    }
    const int pr = jb.row0 + row, tok = jb.q_start + pr / p.group, head = jb.kv_head * p.group + pr % p.group;
    const float inv = l == 0.f ? 0.f : 1.f / d;
    T* o = reinterpret_cast<T*>(p.o) + tok * p.o_row + head * p.o_head + lane * 4;
    const float out[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (lane * 4 + e < p.head_dim) put(o + e, out[e]);
    if (p.lse != nullptr && lane == 0)
        p.lse[static_cast<int64_t>(head) * p.total_q + tok] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
}

}  // namespace

cudaError_t launch_attention_join(const AttnParams& p, int dtype, cudaStream_t stream) {
    if (p.n_joins == 0) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.n_joins, (p.join_rows + kJoinWarps - 1) / kJoinWarps);
    cfg.blockDim = dim3(kJoinWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, dtype == SPECA_BF16 ? join_kernel<__nv_bfloat16> : join_kernel<float>, p);
}

}  // namespace speca
