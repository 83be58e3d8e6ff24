// Device code that the attention kernels share: units, visibility, the join of shared rows.
#pragma once
#include <cuda_bf16.h>
#include <math_constants.h>

#include "speca_layer_internal.h"

namespace speca {
namespace {

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ AttnUnit load_unit(const AttnUnit* units, int i) {
    AttnUnit u;
    const int4* src = reinterpret_cast<const int4*>(units + i);
    int4* dst = reinterpret_cast<int4*>(&u);
#pragma unroll
    for (int k = 0; k < 3; ++k) dst[k] = __ldg(src + k);
    return u;
}

// Keys of the unit's sequence that hold data.
__device__ __forceinline__ int kv_length(const AttnParams& p, const AttnUnit& u) {
    return p.dev_kv_len == nullptr ? u.kv_cap : max(0, min(u.kv_cap, p.dev_kv_len[u.seq]));
}
// Keys that query `i` of the sequence sees: those in front of this index.
__device__ __forceinline__ int visible_keys(const AttnParams& p, const AttnUnit& u, int kv_len, int i) {
    return p.causal ? max(0, min(kv_len, i + 1 + kv_len - u.q_len)) : kv_len;
}

constexpr float kLn2 = 0.6931471805599453f;

// Joins the partial results of a row block whose last share has just been written: weights exp2(m_s - m)
// in the order of the shares, whoever came last. One warp per row, lanes across the head.
template <typename T>
__device__ void join_rows(const AttnParams& p, const AttnUnit& u, int row0, int rows, int64_t part, int64_t split_stride, int warp,
                          int n_warps) {
    const int lane = threadIdx.x % 32;
    const int64_t pitch = part_row_floats(p.head_dim);
    for (int r = warp; r < rows; r += n_warps) {
        const float* base = reinterpret_cast<const float*>(p.parts + part) + r * pitch;
        float m = -CUDART_INF_F;
        for (int s = 0; s < u.n_splits; ++s) m = fmaxf(m, __ldcg(base + s * split_stride + pitch - 4));
        float l = 0.f, acc[SPECA_MAX_HEAD_DIM / 32] = {};
        for (int s = 0; s < u.n_splits; ++s) {
            const float* q = base + s * split_stride;
            const float ls = __ldcg(q + pitch - 3);
            if (ls == 0.f) continue;  // this share saw nothing and left its sums unwritten
            const float w = exp2f(__ldcg(q + pitch - 4) - m);
            l = fmaf(w, ls, l);
#pragma unroll
            for (int i = 0; i < SPECA_MAX_HEAD_DIM / 32; ++i)
                if (lane + i * 32 < p.head_dim) acc[i] = fmaf(w, __ldcg(q + lane + i * 32), acc[i]);
        }
        const int pr = row0 + r, tok = u.q_start + pr / p.group, head = u.kv_head * p.group + pr % p.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* o = reinterpret_cast<T*>(p.o) + tok * p.o_row + head * p.o_head;
#pragma unroll
        for (int i = 0; i < SPECA_MAX_HEAD_DIM / 32; ++i)
            if (lane + i * 32 < p.head_dim) put(o + lane + i * 32, acc[i] * inv);
        if (p.lse != nullptr && lane == 0)
            p.lse[static_cast<int64_t>(head) * p.total_q + tok] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
    }
}

}  // namespace
}  // namespace speca
