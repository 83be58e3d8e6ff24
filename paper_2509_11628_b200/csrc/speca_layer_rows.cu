// The row-wise operators of the verification layer: adaptive layer norm and rotary positions.
#include <cuda_bf16.h>

#include "speca_layer_internal.h"

namespace speca {
namespace {

template <int DT>
struct Type;
template <>
struct Type<SPECA_F32> {
    using T = float;
    static constexpr int kBytes = 4;
};
template <>
struct Type<SPECA_BF16> {
    using T = __nv_bfloat16;
    static constexpr int kBytes = 2;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
    return x;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) {
    return __float2bfloat16_rn(x);
}

// E consecutive elements as one access of up to 16 bytes (the address is a multiple of it).
template <typename T, int E>
struct alignas(sizeof(T) * E <= 16 ? sizeof(T) * E : 16) Pack {
    T e[E];
};
template <typename T, int E>
__device__ __forceinline__ Pack<T, E> load(const char* base, int64_t i) {
    return *reinterpret_cast<const Pack<T, E>*>(reinterpret_cast<const T*>(base) + i);
}
template <typename T, int E>
__device__ __forceinline__ void store(char* base, int64_t i, const Pack<T, E>& v) {
    *reinterpret_cast<Pack<T, E>*>(reinterpret_cast<T*>(base) + i) = v;
}

// Sum over the G lanes (a power of two) of a group inside a warp.
template <int G>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// ------------------------------------------------------------------------------------------------
// adaptive layer norm
// ------------------------------------------------------------------------------------------------
// x' = x + gate * branch, y = (x' - mean) * rstd * (1 + scale) + shift. One pass over memory: the G
// threads of a row keep it in registers (NV accesses of E elements each), so the variance is the
// mean of squared deviations from the finished mean and nothing is read twice.

// Sum over the row's threads: inside the warp, then through shared memory if the row has several warps (`red`: one
// float per warp, of this sum alone, so that one barrier is enough).
template <int G>
__device__ __forceinline__ float sum_row(float x, float* red) {
    if constexpr (G <= 32) return sum_lanes<G>(x);
    x = sum_lanes<32>(x);
    const int warp = threadIdx.x / 32, first = warp / (G / 32) * (G / 32);
    if (threadIdx.x % 32 == 0) red[warp] = x;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < G / 32; ++i) s += red[first + i];
    return s;
}

template <int DT, int E, int NV, int G, int NT>
__global__ void __launch_bounds__(NT) modulate_kernel(const __grid_constant__ ModulateParams p) {
    using T = typename Type<DT>::T;
    __shared__ float red[2][NT / 32];
    const int row = blockIdx.x * (NT / G) + threadIdx.x / G;
    const int t = threadIdx.x % G;
    bool live = row < p.rows;
    int seq = 0;
    if (live) {
        seq = p.row_seq[row];
        live = p.dev_mask == nullptr || p.dev_mask[seq] != 0;
    }
    float x[NV][E];
    float sum = 0.f;
    if (live) {
        const char* px = p.x + row * p.x_stride * static_cast<int64_t>(sizeof(T));
        Pack<T, E> in[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * G) * E;
            if (c < p.dim) in[i] = load<T, E>(px, c);
        }
        if (p.branch != nullptr) {
            const char* pb = p.branch + row * p.branch_stride * static_cast<int64_t>(sizeof(T));
            const char* pg = p.gate == nullptr ? nullptr : p.gate + seq * p.mod_stride * static_cast<int64_t>(sizeof(T));
            char* po = p.x_out == nullptr ? nullptr : p.x_out + row * p.x_out_stride * static_cast<int64_t>(sizeof(T));
            Pack<T, E> br[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * G) * E;
                if (c < p.dim) br[i] = load<T, E>(pb, c);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * G) * E;
                if (c >= p.dim) continue;
                if (pg != nullptr) {
                    const Pack<T, E> g = load<T, E>(pg, c);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[i][e] = fmaf(to_float(g.e[e]), to_float(br[i].e[e]), to_float(in[i].e[e]));
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[i][e] = to_float(in[i].e[e]) + to_float(br[i].e[e]);
                }
                if (po != nullptr) {
                    Pack<T, E> out;
#pragma unroll
                    for (int e = 0; e < E; ++e) out.e[e] = from_float<T>(x[i][e]);
                    store<T, E>(po, c, out);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * G) * E;
                if (c >= p.dim) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) x[i][e] = to_float(in[i].e[e]);
                if (p.x_out != nullptr) store<T, E>(p.x_out + row * p.x_out_stride * static_cast<int64_t>(sizeof(T)), c, in[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((t + i * G) * E >= p.dim) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) sum += x[i][e];
        }
    }
    // every thread takes part in the sums: a row's threads may share a warp or a barrier with a dead row's
    const float mean = sum_row<G>(sum, red[0]) / p.dim;
    float sq = 0.f;
    if (live) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((t + i * G) * E >= p.dim) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[i][e] -= mean;
                sq = fmaf(x[i][e], x[i][e], sq);
            }
        }
    }
    const float rstd = 1.f / sqrtf(sum_row<G>(sq, red[1]) / p.dim + p.eps);
    if (!live) return;
    const char* ps = p.scale == nullptr ? nullptr : p.scale + seq * p.mod_stride * static_cast<int64_t>(sizeof(T));
    const char* pt = p.shift == nullptr ? nullptr : p.shift + seq * p.mod_stride * static_cast<int64_t>(sizeof(T));
    char* py = p.y + row * p.y_stride * static_cast<int64_t>(sizeof(T));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * G) * E;
        if (c >= p.dim) continue;
        Pack<T, E> s, b, out;
        if (ps != nullptr) s = load<T, E>(ps, c);
        if (pt != nullptr) b = load<T, E>(pt, c);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float a = x[i][e] * rstd;
            out.e[e] = from_float<T>(fmaf(a, ps != nullptr ? 1.f + to_float(s.e[e]) : 1.f, pt != nullptr ? to_float(b.e[e]) : 0.f));
        }
        store<T, E>(py, c, out);
    }
}

// Rows too long for the registers of one block: three passes, the second and third out of L2.
template <int DT>
__global__ void __launch_bounds__(1024) modulate_long_kernel(const __grid_constant__ ModulateParams p) {
    using T = typename Type<DT>::T;
    __shared__ float red[2][32];
    const int row = blockIdx.x;
    const int seq = p.row_seq[row];
    if (p.dev_mask != nullptr && p.dev_mask[seq] == 0) return;
    const T* px = reinterpret_cast<const T*>(p.x) + row * p.x_stride;
    const T* pb = p.branch == nullptr ? nullptr : reinterpret_cast<const T*>(p.branch) + row * p.branch_stride;
    const T* pg = p.gate == nullptr ? nullptr : reinterpret_cast<const T*>(p.gate) + seq * p.mod_stride;
    const T* ps = p.scale == nullptr ? nullptr : reinterpret_cast<const T*>(p.scale) + seq * p.mod_stride;
    const T* pt = p.shift == nullptr ? nullptr : reinterpret_cast<const T*>(p.shift) + seq * p.mod_stride;
    auto value = [&](int c) {
        const float v = to_float(px[c]);
        return pb == nullptr ? v : fmaf(pg == nullptr ? 1.f : to_float(pg[c]), to_float(pb[c]), v);
    };
    float sum = 0.f;
    for (int c = threadIdx.x; c < p.dim; c += 1024) sum += value(c);
    const float mean = sum_row<1024>(sum, red[0]) / p.dim;
    float sq = 0.f;
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float d = value(c) - mean;
        sq = fmaf(d, d, sq);
    }
    const float rstd = 1.f / sqrtf(sum_row<1024>(sq, red[1]) / p.dim + p.eps);
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float v = value(c);
        if (p.x_out != nullptr) (reinterpret_cast<T*>(p.x_out) + row * p.x_out_stride)[c] = from_float<T>(v);
        (reinterpret_cast<T*>(p.y) + row * p.y_stride)[c] =
            from_float<T>(fmaf((v - mean) * rstd, ps == nullptr ? 1.f : 1.f + to_float(ps[c]), pt == nullptr ? 0.f : to_float(pt[c])));
    }
}

template <int DT, int E, int NV, int G, int NT>
void run_modulate(const ModulateParams& p, cudaStream_t stream) {
    const int per = NT / G;
    modulate_kernel<DT, E, NV, G, NT><<<(p.rows + per - 1) / per, NT, 0, stream>>>(p);
}

// A row's threads hold NV accesses of E elements each. Few threads with two or three accesses beat one access per thread
// (loads in flight) and many accesses per thread (registers): on rows of 3072 bf16 elements 128 threads x 3 ran at
// 5.8 TB/s over 20926 rows, 128 x 4 at 5.0, 384 x 1 at 4.0, 32 x 12 at 3.6. Rows that do not divide into 16 bytes go element by
// element, above 2048 of them in three passes: 4608 rows with the residual take 35 us at 1151 bf16 elements (21 at 1152), 129 at
// 4097 bf16 and 126 at 3071 fp32 (44 at 3072).
template <int DT, int E>
void dispatch_modulate(const ModulateParams& p, cudaStream_t stream) {
    const int n = (p.dim + E - 1) / E;  // accesses per row
    if (n <= 32 * 2) return run_modulate<DT, E, 2, 32, 128>(p, stream);
    if (n <= 64 * 2) return run_modulate<DT, E, 2, 64, 128>(p, stream);
    if (n <= 128 * 2) return run_modulate<DT, E, 2, 128, 128>(p, stream);
    if (n <= 128 * 3) return run_modulate<DT, E, 3, 128, 128>(p, stream);
    if (n <= 128 * 5) return run_modulate<DT, E, 5, 128, 128>(p, stream);
    if (n <= 256 * 4) return run_modulate<DT, E, 4, 256, 256>(p, stream);
    if (n <= 512 * 4) return run_modulate<DT, E, 4, 512, 512>(p, stream);
    modulate_long_kernel<DT><<<p.rows, 1024, 0, stream>>>(p);
}

// ------------------------------------------------------------------------------------------------
// rotary positions
// ------------------------------------------------------------------------------------------------
// L lanes share one head of one row; each holds 4 pairs (with vectors: consecutive pairs, one or two
// accesses; else pairs lane, lane + L, ...). Several lane groups share a row: each takes its part of the heads of q
// and k. The block first forms the rotations of its rows in shared memory: an angle serves every head of a row.
// Bound by memory in the end (read once, written once), by instructions on the way there: 20926 rows x 48 heads of 128 bf16 with the
// norm take 106 us = 4.8 TB/s; with angles formed by every lane group, weights read per head and applied apart
// from the rotation it was 295 us. 3 heads in flight per lane and 4 blocks per SM beat 2, 4 and 6 heads (119, 120, 128 us)
// and 3 or 5 blocks.
constexpr int kRopeThreads = 256;
constexpr int kRopePairs = 4;   // pairs per lane
constexpr int kRopeAhead = 3;   // heads whose loads are in flight per lane
constexpr int kRopeBlocks = 4;  // per SM
constexpr float kKept = 2.f;    // no cosine: the pair is copied, so that an infinity in it stays where it is

// The 8 elements that a lane holds of a head, as pairs (a, b).
template <int DT, bool VEC, bool HALVES, int L>
struct HeadPart {
    using T = typename Type<DT>::T;
    int first, n_pairs, half;  // first pair, pairs of the head, distance of a pair's elements (HALVES)
    bool split;                // VEC, HALVES: the lane's pairs lie in the rotated part
    __device__ __forceinline__ HeadPart(int lane, int n, int h)
        : first(VEC ? lane * kRopePairs : lane), n_pairs(n), half(h), split(HALVES && lane * kRopePairs < h) {}
    __device__ __forceinline__ int pair(int i) const { return VEC ? first + i : first + i * L; }
    __device__ __forceinline__ bool holds(int i) const { return VEC ? first < n_pairs : pair(i) < n_pairs; }
    // HALVES, behind the rotated part: the remaining elements two by two
    __device__ __forceinline__ int e0(int i) const { return HALVES && pair(i) < half ? pair(i) : 2 * pair(i); }
    __device__ __forceinline__ int e1(int i) const { return HALVES && pair(i) < half ? pair(i) + half : 2 * pair(i) + 1; }
    // VEC, HALVES: a = 4 elements, b = their partners, or the 4 elements behind them where nothing turns
    __device__ __forceinline__ int second() const { return split ? first + half : 2 * first + kRopePairs; }
    __device__ __forceinline__ int start() const { return split ? first : 2 * first; }

    __device__ __forceinline__ void read(const char* src, int64_t at, T (&a)[kRopePairs], T (&b)[kRopePairs]) const {
        if constexpr (VEC && !HALVES) {
            if (first >= n_pairs) return;
            const Pack<T, 2 * kRopePairs> v = load<T, 2 * kRopePairs>(src, at + 2 * first);
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) a[i] = v.e[2 * i], b[i] = v.e[2 * i + 1];
        } else if constexpr (VEC) {
            if (first >= n_pairs) return;
            const Pack<T, kRopePairs> u = load<T, kRopePairs>(src, at + start()), v = load<T, kRopePairs>(src, at + second());
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) a[i] = u.e[i], b[i] = v.e[i];
        } else {
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) {
                if (!holds(i)) continue;
                a[i] = reinterpret_cast<const T*>(src)[at + e0(i)];
                b[i] = reinterpret_cast<const T*>(src)[at + e1(i)];
            }
        }
    }
    __device__ __forceinline__ void write(char* dst, int64_t at, const float (&a)[kRopePairs], const float (&b)[kRopePairs]) const {
        if constexpr (VEC && !HALVES) {
            if (first >= n_pairs) return;
            Pack<T, 2 * kRopePairs> v;
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) v.e[2 * i] = from_float<T>(a[i]), v.e[2 * i + 1] = from_float<T>(b[i]);
            store<T, 2 * kRopePairs>(dst, at + 2 * first, v);
        } else if constexpr (VEC) {
            if (first >= n_pairs) return;
            Pack<T, kRopePairs> u, v;
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) u.e[i] = from_float<T>(a[i]), v.e[i] = from_float<T>(b[i]);
            store<T, kRopePairs>(dst, at + start(), u);
            store<T, kRopePairs>(dst, at + second(), v);
        } else {
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) {
                if (!holds(i)) continue;
                reinterpret_cast<T*>(dst)[at + e0(i)] = from_float<T>(a[i]);
                reinterpret_cast<T*>(dst)[at + e1(i)] = from_float<T>(b[i]);
            }
        }
    }
};

// All heads of q or of k of one row, by the row's lane groups. A head x turns into r R(w x), r the reciprocal root mean
// square, w the weight: the rotation is linear, so w goes into its coefficients once and r is applied behind it.
template <int DT, bool VEC, bool HALVES, bool KEPT, bool NORM, int L>
__device__ __forceinline__ void turn_heads(const HeadPart<DT, VEC, HALVES, L>& part, const char* src, int64_t head_in, char* dst,
                                           int64_t head_out, int n_heads, int head0, int step, const char* w,
                                           const float2 (&cs)[kRopePairs], bool live, float inv_dim, float eps) {
    using T = typename Type<DT>::T;
    float ca[kRopePairs], sb[kRopePairs], sa[kRopePairs], cb[kRopePairs];  // (a, b) -> (ca a - sb b, sa a + cb b)
    {
        T wa[kRopePairs], wb[kRopePairs];
        if (NORM && w != nullptr) part.read(w, 0, wa, wb);
#pragma unroll
        for (int i = 0; i < kRopePairs; ++i) {
            const bool weighted = NORM && w != nullptr && part.holds(i);
            const float fa = weighted ? to_float(wa[i]) : 1.f, fb = weighted ? to_float(wb[i]) : 1.f;
            const bool kept = KEPT && cs[i].x == kKept;
            ca[i] = (kept ? 1.f : cs[i].x) * fa;
            cb[i] = (kept ? 1.f : cs[i].x) * fb;
            sa[i] = cs[i].y * fa;
            sb[i] = cs[i].y * fb;
        }
    }
    // the groups of a warp run the same number of rounds: sums over the head are shuffles of the whole warp
    for (int first = 0; first < n_heads; first += step * kRopeAhead) {
        T in[kRopeAhead][2][kRopePairs];
#pragma unroll
        for (int j = 0; j < kRopeAhead; ++j) {
            const int h = first + j * step + head0;
            if (live && h < n_heads) part.read(src, h * head_in, in[j][0], in[j][1]);
        }
#pragma unroll
        for (int j = 0; j < kRopeAhead; ++j) {
            if (first + j * step >= n_heads) break;  // the same for every group
            const int h = first + j * step + head0;
            const bool use = live && h < n_heads;
            float a[kRopePairs], b[kRopePairs], r = 1.f;
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) {
                const bool has = use && part.holds(i);
                a[i] = has ? to_float(in[j][0][i]) : 0.f;
                b[i] = has ? to_float(in[j][1][i]) : 0.f;
            }
            if (NORM && w != nullptr) {
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < kRopePairs; ++i) sq = fmaf(a[i], a[i], fmaf(b[i], b[i], sq));
                r = rsqrtf(fmaf(sum_lanes<L>(sq), inv_dim, eps));
            }
            if (!use) continue;
            float ra[kRopePairs], rb[kRopePairs];
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) {
                const bool kept = KEPT && cs[i].x == kKept;
                ra[i] = kept ? ca[i] * a[i] : fmaf(ca[i], a[i], -sb[i] * b[i]);
                rb[i] = kept ? cb[i] * b[i] : fmaf(sa[i], a[i], cb[i] * b[i]);
                if (NORM) ra[i] *= r, rb[i] *= r;
            }
            part.write(dst, h * head_out, ra, rb);
        }
    }
}

template <int DT, bool VEC, bool HALVES, bool KEPT, bool NORM, int L>
__global__ void __launch_bounds__(kRopeThreads, kRopeBlocks) rope_kernel(const __grid_constant__ RopeParams p, int groups_per_row) {
    constexpr int kGroups = kRopeThreads / L;
    constexpr int64_t kBytes = Type<DT>::kBytes;
    __shared__ float2 turn[kGroups * kRopePairs * L];  // [row of the block][pair]: cosine, sine
    const int group = threadIdx.x / L;
    const int rows_per_block = kGroups / groups_per_row, row0 = blockIdx.x * rows_per_block;
    const int own = group / groups_per_row, row = row0 + own, head0 = group % groups_per_row;
    const int n_pairs = p.head_dim / 2;
    const bool live = row < p.rows && (p.dev_mask == nullptr || p.dev_mask[p.row_seq[row]] != 0);
    const HeadPart<DT, VEC, HALVES, L> part(threadIdx.x % L, n_pairs, p.half);
    for (int i = threadIdx.x; i < rows_per_block * n_pairs; i += kRopeThreads) {
        const int r = i / n_pairs, pair = i % n_pairs;
        const RopePair f = p.pairs[pair];
        float2 t = make_float2(kKept, 0.f);
        if (f.axis >= 0 && row0 + r < p.rows) {
            // the angle in turns, reduced in fp64 to half a turn either way
            const double turns = f.turns * static_cast<double>(p.positions[static_cast<int64_t>(row0 + r) * p.n_axes + f.axis]);
            sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &t.y, &t.x);
        }
        turn[i] = t;
    }
    __syncthreads();
    float2 cs[kRopePairs];
#pragma unroll
    for (int i = 0; i < kRopePairs; ++i) cs[i] = part.holds(i) ? turn[own * n_pairs + part.pair(i)] : make_float2(kKept, 0.f);
    const float inv_dim = 1.f / p.head_dim;
    turn_heads<DT, VEC, HALVES, KEPT, NORM, L>(part, p.q + row * p.q_row * kBytes, p.q_head, p.q_out + row * p.qo_row * kBytes, p.qo_head,
                                               p.n_heads, head0, groups_per_row, p.q_weight, cs, live, inv_dim, p.eps);
    if (p.k != nullptr)
        turn_heads<DT, VEC, HALVES, KEPT, NORM, L>(part, p.k + row * p.k_row * kBytes, p.k_head, p.k_out + row * p.ko_row * kBytes,
                                                   p.ko_head, p.n_kv_heads, head0, groups_per_row, p.k_weight, cs, live, inv_dim, p.eps);
}

template <int DT, bool VEC, bool HALVES, bool KEPT, int L>
void run_rope(const RopeParams& p, cudaStream_t stream) {
    const int groups = kRopeThreads / L;
    // Lane groups per row: as many rows per block as give every thread an angle to form, or (few rows: SMs idle)
    // enough groups that each keeps no more than kRopeAhead heads in flight.
    int gpr = groups;
    while (gpr > 1 && groups / gpr * (p.head_dim / 2) < kRopeThreads) gpr /= 2;
    while (gpr < groups && gpr * kRopeAhead < p.n_heads && static_cast<int64_t>(p.rows) * gpr < groups * 592ll) gpr *= 2;
    const int per = groups / gpr, grid = (p.rows + per - 1) / per;
    if (p.q_weight != nullptr || p.k_weight != nullptr)
        rope_kernel<DT, VEC, HALVES, KEPT, true, L><<<grid, kRopeThreads, 0, stream>>>(p, gpr);
    else
        rope_kernel<DT, VEC, HALVES, KEPT, false, L><<<grid, kRopeThreads, 0, stream>>>(p, gpr);
}

template <int DT, bool VEC, bool HALVES, bool KEPT>
void dispatch_rope(const RopeParams& p, cudaStream_t stream) {
    const int lanes = (p.head_dim / 2 + kRopePairs - 1) / kRopePairs;
    if (lanes <= 4) return run_rope<DT, VEC, HALVES, KEPT, 4>(p, stream);
    if (lanes <= 8) return run_rope<DT, VEC, HALVES, KEPT, 8>(p, stream);
    return run_rope<DT, VEC, HALVES, KEPT, 16>(p, stream);
}
template <int DT, bool VEC>
void dispatch_rope(const RopeParams& p, cudaStream_t stream) {
    const bool kept = p.rotated < p.head_dim;
    if (p.half > 0)
        kept ? dispatch_rope<DT, VEC, true, true>(p, stream) : dispatch_rope<DT, VEC, true, false>(p, stream);
    else
        kept ? dispatch_rope<DT, VEC, false, true>(p, stream) : dispatch_rope<DT, VEC, false, false>(p, stream);
}

}  // namespace

cudaError_t launch_modulate(const ModulateParams& p, int dtype, int vec, cudaStream_t stream) {
    if (p.rows == 0) return cudaSuccess;
    if (dtype == SPECA_BF16) {
        vec > 1 ? dispatch_modulate<SPECA_BF16, 8>(p, stream) : dispatch_modulate<SPECA_BF16, 1>(p, stream);
    } else {
        vec > 1 ? dispatch_modulate<SPECA_F32, 4>(p, stream) : dispatch_modulate<SPECA_F32, 1>(p, stream);
    }
    return cudaGetLastError();
}

cudaError_t launch_rope(const RopeParams& p, int dtype, bool vectors, cudaStream_t stream) {
    if (p.rows == 0) return cudaSuccess;
    if (dtype == SPECA_BF16)
        vectors ? dispatch_rope<SPECA_BF16, true>(p, stream) : dispatch_rope<SPECA_BF16, false>(p, stream);
    else
        vectors ? dispatch_rope<SPECA_F32, true>(p, stream) : dispatch_rope<SPECA_F32, false>(p, stream);
    return cudaGetLastError();
}

}  // namespace speca
