// Attention of the verification layer in fp32, on the CUDA cores.

#include "speca_attention_common.cuh"

namespace speca {
namespace {

// ------------------------------------------------------------------------------------------------
// fp32 arithmetic on the CUDA cores
// ------------------------------------------------------------------------------------------------
// 32 packed rows against tiles of 64 keys: 128 threads, each with 4 rows x 4 keys of the scores and 4 rows x 8
// columns of the output in registers; running maximum and sum per row, so scores never leave the chip. Bound by latency:
// two samples of 64 rows x 6 heads of 64 take 11.6 us (one tile per block: four rounds of loads, then one pass), 2000 rows
// x 6 heads of 128 run at 14 TFLOP/s, and 4 single rows x 24 heads of 128 against 8192 keys take 656 us (1.2 TB/s: a block
// computes 32 rows of which one is there).
constexpr int kSimtThreads = 128;
constexpr int kSimtPitch = SPECA_MAX_HEAD_DIM + 4;  // floats; rows 4 banks apart: 16-byte reads of 8 rows do not collide

struct SimtSmem {
    float q[kSimtRows][kSimtPitch];
    float k[kSimtKeys][kSimtPitch];
    float v[kSimtKeys][kSimtPitch];
    float p[kSimtRows][kSimtKeys + 4];
};

// Eight rows of up to 128 elements (row 4 i of `row`, i < 8) by one warp, zeros behind their end (up to a multiple of 4) or
// where there is none. All loads are issued before the first store waits for one: row by row, a tile's 32 rows
// per warp took 12 us of latency.
template <typename Row>
__device__ __forceinline__ void fill_rows(float (*dst)[kSimtPitch], const Row& row, int hd, int lane, bool vectors) {
    if (vectors) {
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float* src = row(i * 4);
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (src != nullptr && lane * 4 < hd) v[i] = __ldg(reinterpret_cast<const float4*>(src + lane * 4));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane * 4 < hd) *reinterpret_cast<float4*>(&dst[i * 4][lane * 4]) = v[i];
        return;
    }
#pragma unroll 1
    for (int c = lane; c < (hd + 3) / 4 * 4; c += 32) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float* src = row(i * 4);
            v[i] = 0.f;
            if (src != nullptr && c < hd) v[i] = __ldg(src + c);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) dst[i * 4][c] = v[i];
    }
}

__global__ void __launch_bounds__(kSimtThreads) attention_f32_kernel(const __grid_constant__ AttnParams p) {
    extern __shared__ __align__(16) char smem_raw[];
    SimtSmem& sm = *reinterpret_cast<SimtSmem*>(smem_raw);
    const AttnUnit u = load_unit(p.units, blockIdx.x);
    if (p.dev_mask != nullptr && p.dev_mask[u.seq] == 0) return;
    const int kv_len = kv_length(p, u);
    const int rows = min(kSimtRows, u.q_len * p.group - u.row0);
    const int tiles = (kv_len + kSimtKeys - 1) / kSimtKeys, share = (tiles + u.n_splits - 1) / u.n_splits;
    const int seen = visible_keys(p, u, kv_len, (u.row0 + rows - 1) / p.group);  // by the block's last row
    const int t0 = u.split * share, t1 = min(min(tiles, t0 + share), (seen + kSimtKeys - 1) / kSimtKeys);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int hd = p.head_dim, hd4 = (hd + 3) / 4;

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const float* pq = reinterpret_cast<const float*>(p.q);
    const float* pk = reinterpret_cast<const float*>(p.k) + u.kv_start * p.k_row + u.kv_head * p.k_head;
    const float* pv = reinterpret_cast<const float*>(p.v) + u.kv_start * p.v_row + u.kv_head * p.v_head;
    static_assert(kSimtRows == 32 && kSimtKeys == 64, "8 rows of Q and 16 of K and V per warp");
    auto query = [&](int r) -> const float* {
        const int pr = u.row0 + warp + r;
        if (warp + r >= rows) return nullptr;
        return pq + (u.q_start + pr / p.group) * p.q_row + (u.kv_head * p.group + pr % p.group) * p.q_head;
    };
    fill_rows(sm.q + warp, query, hd, lane, p.vectors);
    int limit[4];
    float m[4], l[4], acc[4][8];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = ty * 4 + r;
        limit[r] = row < rows ? visible_keys(p, u, kv_len, (u.row0 + row) / p.group) : 0;
        m[r] = -CUDART_INF_F;
        l[r] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[r][c] = 0.f;
    }
    for (int t = t0; t < t1; ++t) {
        const int key0 = t * kSimtKeys;
        __syncthreads();  // the previous tile has been read
        // keys behind kv_len are not read: a weight of zero times whatever they hold may be NaN
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            const int r0 = half * 32 + warp;
            auto key = [&](int r) { return key0 + r0 + r < kv_len ? pk + (key0 + r0 + r) * p.k_row : nullptr; };
            auto value = [&](int r) { return key0 + r0 + r < kv_len ? pv + (key0 + r0 + r) * p.v_row : nullptr; };
            fill_rows(sm.k + r0, key, hd, lane, p.vectors);
            fill_rows(sm.v + r0, value, hd, lane, p.vectors);
        }
        __syncthreads();
        float s[4][4] = {};
#pragma unroll 2  // a tile's code runs once or a few times: written out in full, fetching it took longer than running it
        for (int c = 0; c < hd4; ++c) {
            float4 qa[4], kb[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) qa[r] = *reinterpret_cast<const float4*>(&sm.q[ty * 4 + r][c * 4]);
#pragma unroll
            for (int j = 0; j < 4; ++j) kb[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][c * 4]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[r][j] = fmaf(qa[r].w, kb[j].w, fmaf(qa[r].z, kb[j].z, fmaf(qa[r].y, kb[j].y, fmaf(qa[r].x, kb[j].x, s[r][j]))));
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float top = -CUDART_INF_F;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[r][j] = key0 + tx + 16 * j < limit[r] ? s[r][j] * p.scale_log2 : -CUDART_INF_F;
                top = fmaxf(top, s[r][j]);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            top = fmaxf(top, m[r]);
            const float ref = top == -CUDART_INF_F ? 0.f : top;  // a row that has seen nothing yet
            const float f = exp2f(m[r] - ref);
            m[r] = top;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e = exp2f(s[r][j] - ref);
                sum += e;
                sm.p[ty * 4 + r][tx + 16 * j] = e;
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l[r] = fmaf(l[r], f, sum);
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[r][c] *= f;
        }
        __syncwarp();  // rows of p belong to one half warp
#pragma unroll 1
        for (int k = 0; k < kSimtKeys; k += 4) {
            float4 pr[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) pr[r] = *reinterpret_cast<const float4*>(&sm.p[ty * 4 + r][k]);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (tx * 4 + h * 64 >= hd) continue;
                    const float4 v = *reinterpret_cast<const float4*>(&sm.v[k + kk][tx * 4 + h * 64]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float w = kk == 0 ? pr[r].x : kk == 1 ? pr[r].y : kk == 2 ? pr[r].z : pr[r].w;
                        acc[r][h * 4 + 0] = fmaf(w, v.x, acc[r][h * 4 + 0]);
                        acc[r][h * 4 + 1] = fmaf(w, v.y, acc[r][h * 4 + 1]);
                        acc[r][h * 4 + 2] = fmaf(w, v.z, acc[r][h * 4 + 2]);
                        acc[r][h * 4 + 3] = fmaf(w, v.w, acc[r][h * 4 + 3]);
                    }
                }
            }
        }
        __syncwarp();
    }
    const int64_t pitch = part_row_floats(hd), split_stride = static_cast<int64_t>(rows) * pitch;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = ty * 4 + r, pr = u.row0 + row;
        if (row >= rows) continue;
        if (u.n_splits > 1) {
            float* part = reinterpret_cast<float*>(p.parts + u.part) + u.split * split_stride + row * pitch;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int col = tx * 4 + (c / 4) * 64 + c % 4;
                if (col < hd) part[col] = acc[r][c];
            }
            if (tx == 0) {
                part[pitch - 4] = m[r];
                part[pitch - 3] = part[pitch - 2] = l[r];
            }
            continue;
        }
        const int tok = u.q_start + pr / p.group, head = u.kv_head * p.group + pr % p.group;
        const float inv = 1.f / l[r];
        float* o = reinterpret_cast<float*>(p.o) + tok * p.o_row + head * p.o_head;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int col = tx * 4 + (c / 4) * 64 + c % 4;
            // a row that sees nothing: zero, also where a weight of zero met a value that is not finite
            if (col < hd) o[col] = l[r] == 0.f ? 0.f : acc[r][c] * inv;
        }
        if (p.lse != nullptr && tx == 0)
            p.lse[static_cast<int64_t>(head) * p.total_q + tok] = l[r] == 0.f ? -CUDART_INF_F : (m[r] + log2f(l[r])) * kLn2;
    }
}

}  // namespace

cudaError_t launch_attention_f32(const AttnParams& p, cudaStream_t stream) {
    if (p.n_units == 0) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(attention_f32_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SimtSmem));
    if (e != cudaSuccess) return e;
    attention_f32_kernel<<<p.n_units, kSimtThreads, sizeof(SimtSmem), stream>>>(p);
    return cudaGetLastError();
}

}  // namespace speca
