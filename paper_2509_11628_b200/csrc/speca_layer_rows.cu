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
constexpr int kModThreads = 128;

// Sum over the row's threads: inside the warp, then through shared memory if the row has several warps.
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
    __syncthreads();
    return s;
}

template <int DT, int E, int NV, int G, int NT>
__global__ void __launch_bounds__(NT) modulate_kernel(const __grid_constant__ ModulateParams p) {
    using T = typename Type<DT>::T;
    __shared__ float red[NT / 32];
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
    const float mean = sum_row<G>(sum, red) / p.dim;
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
    const float rstd = 1.f / sqrtf(sum_row<G>(sq, red) / p.dim + p.eps);
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
    __shared__ float red[32];
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
    const float mean = sum_row<1024>(sum, red) / p.dim;
    float sq = 0.f;
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float d = value(c) - mean;
        sq = fmaf(d, d, sq);
    }
    const float rstd = 1.f / sqrtf(sum_row<1024>(sq, red) / p.dim + p.eps);
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

// Elements a row's threads can hold: NV accesses of E elements by G threads.
template <int DT, int E>
void dispatch_modulate(const ModulateParams& p, cudaStream_t stream) {
    const int n = (p.dim + E - 1) / E;  // accesses per row
    if (n <= 32 * 2) return run_modulate<DT, E, 2, 32, kModThreads>(p, stream);
    if (n <= 32 * 6) return run_modulate<DT, E, 6, 32, kModThreads>(p, stream);
    if (n <= 128 * 4) return run_modulate<DT, E, 4, 128, 128>(p, stream);
    if (n <= 512 * 4) return run_modulate<DT, E, 4, 512, 512>(p, stream);
    if (n <= 512 * 8) return run_modulate<DT, E, 8, 512, 512>(p, stream);
    modulate_long_kernel<DT><<<p.rows, 1024, 0, stream>>>(p);
}

// ------------------------------------------------------------------------------------------------
// rotary positions
// ------------------------------------------------------------------------------------------------
// L lanes share one head of one row; each holds 4 pairs (with vectors: consecutive pairs, one or two
// accesses; else pairs lane, lane + L, ...). The angle of a pair is the same for every head of a row, so
// a lane keeps its row, computes 4 angles once and turns its share of all heads of q and k with them.
constexpr int kRopeThreads = 256;
constexpr int kRopePairs = 4;   // pairs per lane
constexpr int kRopeAhead = 4;   // heads whose loads are in flight per lane

template <int DT, bool VEC, bool HALVES, int L>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p, int groups_per_row) {
    using T = typename Type<DT>::T;
    constexpr int kGroups = kRopeThreads / L;
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int rows_per_block = kGroups / groups_per_row;
    const int row = blockIdx.x * rows_per_block + group / groups_per_row;
    const int head0 = group % groups_per_row;
    const int n_pairs = p.head_dim / 2, n_all = p.n_heads + (p.k == nullptr ? 0 : p.n_kv_heads);
    const bool live = row < p.rows && (p.dev_mask == nullptr || p.dev_mask[p.row_seq[row]] != 0);

    // pair i of this lane and the elements it consists of
    int pair[kRopePairs], e0[kRopePairs], e1[kRopePairs];
#pragma unroll
    for (int i = 0; i < kRopePairs; ++i) {
        pair[i] = VEC ? lane * kRopePairs + i : lane + i * L;
        // HALVES: pairs behind the rotated part hold its remaining elements two by two
        const bool split = HALVES && pair[i] < p.half;
        e0[i] = split ? pair[i] : 2 * pair[i];
        e1[i] = split ? pair[i] + p.half : 2 * pair[i] + 1;
    }
    float c[kRopePairs], s[kRopePairs];
    bool kept[kRopePairs];  // copied, so that an infinity in it stays where it is
#pragma unroll
    for (int i = 0; i < kRopePairs; ++i) kept[i] = true;
    if (live) {
#pragma unroll
        for (int i = 0; i < kRopePairs; ++i) {
            c[i] = 1.f;
            s[i] = 0.f;
            if (pair[i] >= n_pairs) continue;
            const RopePair f = p.pairs[pair[i]];
            if (f.axis < 0) continue;
            kept[i] = false;
            const double turns = f.turns * static_cast<double>(p.positions[static_cast<int64_t>(row) * p.n_axes + f.axis]);
            sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s[i], &c[i]);
        }
    }
    // the groups of a warp run the same number of rounds: sums over the head are shuffles of the whole warp
    const int rounds = (n_all + groups_per_row * kRopeAhead - 1) / (groups_per_row * kRopeAhead);
    for (int round = 0; round < rounds; ++round) {
        float a[kRopeAhead][kRopePairs], b[kRopeAhead][kRopePairs];
#pragma unroll
        for (int j = 0; j < kRopeAhead; ++j) {
            const int h = head0 + (round * kRopeAhead + j) * groups_per_row;
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) a[j][i] = b[j][i] = 0.f;
            if (!live || h >= n_all) continue;
            const char* src = h < p.n_heads ? p.q : p.k;
            const int64_t at = h < p.n_heads ? row * p.q_row + h * p.q_head : row * p.k_row + (h - p.n_heads) * p.k_head;
            if constexpr (VEC && !HALVES) {
                if (pair[0] < n_pairs) {
                    const Pack<T, 2 * kRopePairs> v = load<T, 2 * kRopePairs>(src, at + 2 * pair[0]);
#pragma unroll
                    for (int i = 0; i < kRopePairs; ++i) {
                        a[j][i] = to_float(v.e[2 * i]);
                        b[j][i] = to_float(v.e[2 * i + 1]);
                    }
                }
            } else if constexpr (VEC) {
                if (pair[0] < n_pairs) {
                    // rotated: 4 elements and their 4 partners; kept: 8 consecutive ones
                    const bool split = pair[0] < p.half;
                    const Pack<T, kRopePairs> u = load<T, kRopePairs>(src, at + e0[0]);
                    const Pack<T, kRopePairs> v = load<T, kRopePairs>(src, at + (split ? e1[0] : e0[0] + kRopePairs));
#pragma unroll
                    for (int i = 0; i < kRopePairs; ++i) {
                        a[j][i] = to_float(u.e[i]);
                        b[j][i] = to_float(v.e[i]);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRopePairs; ++i) {
                    if (pair[i] >= n_pairs) continue;
                    a[j][i] = to_float(reinterpret_cast<const T*>(src)[at + e0[i]]);
                    b[j][i] = to_float(reinterpret_cast<const T*>(src)[at + e1[i]]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kRopeAhead; ++j) {
            const int h = head0 + (round * kRopeAhead + j) * groups_per_row;
            const bool is_q = h < p.n_heads;
            const char* w = is_q ? p.q_weight : p.k_weight;
            if (p.q_weight != nullptr || p.k_weight != nullptr) {
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < kRopePairs; ++i) sq = fmaf(a[j][i], a[j][i], fmaf(b[j][i], b[j][i], sq));
                sq = sum_lanes<L>(sq);
                if (w != nullptr) {
                    const float r = 1.f / sqrtf(sq / p.head_dim + p.eps);
                    // in registers a kept pair of HALVES holds elements 4 apart (see the load)
#pragma unroll
                    for (int i = 0; i < kRopePairs; ++i) {
                        if (pair[i] >= n_pairs) continue;
                        const bool apart = VEC && HALVES && pair[i] >= p.half;
                        a[j][i] *= r * to_float(reinterpret_cast<const T*>(w)[apart ? e0[0] + i : e0[i]]);
                        b[j][i] *= r * to_float(reinterpret_cast<const T*>(w)[apart ? e0[0] + kRopePairs + i : e1[i]]);
                    }
                }
            }
            if (!live || h >= n_all) continue;
            char* dst = is_q ? p.q_out : p.k_out;
            const int64_t at = is_q ? row * p.qo_row + h * p.qo_head : row * p.ko_row + (h - p.n_heads) * p.ko_head;
            float ra[kRopePairs], rb[kRopePairs];
#pragma unroll
            for (int i = 0; i < kRopePairs; ++i) {
                ra[i] = kept[i] ? a[j][i] : fmaf(a[j][i], c[i], -b[j][i] * s[i]);
                rb[i] = kept[i] ? b[j][i] : fmaf(a[j][i], s[i], b[j][i] * c[i]);
            }
            if constexpr (VEC && !HALVES) {
                if (pair[0] < n_pairs) {
                    Pack<T, 2 * kRopePairs> v;
#pragma unroll
                    for (int i = 0; i < kRopePairs; ++i) {
                        v.e[2 * i] = from_float<T>(ra[i]);
                        v.e[2 * i + 1] = from_float<T>(rb[i]);
                    }
                    store<T, 2 * kRopePairs>(dst, at + 2 * pair[0], v);
                }
            } else if constexpr (VEC) {
                if (pair[0] < n_pairs) {
                    const bool split = pair[0] < p.half;
                    Pack<T, kRopePairs> u, v;
#pragma unroll
                    for (int i = 0; i < kRopePairs; ++i) {
                        u.e[i] = from_float<T>(ra[i]);
                        v.e[i] = from_float<T>(rb[i]);
                    }
                    store<T, kRopePairs>(dst, at + e0[0], u);
                    store<T, kRopePairs>(dst, at + (split ? e1[0] : e0[0] + kRopePairs), v);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRopePairs; ++i) {
                    if (pair[i] >= n_pairs) continue;
                    reinterpret_cast<T*>(dst)[at + e0[i]] = from_float<T>(ra[i]);
                    reinterpret_cast<T*>(dst)[at + e1[i]] = from_float<T>(rb[i]);
                }
            }
        }
    }
}

template <int DT, bool VEC, bool HALVES, int L>
void run_rope(const RopeParams& p, cudaStream_t stream) {
    const int groups = kRopeThreads / L;
    const int heads = p.n_heads + (p.k == nullptr ? 0 : p.n_kv_heads);
    // lane groups per row: enough that each keeps about kRopeAhead heads in flight
    int gpr = 1;
    while (gpr < groups && gpr * kRopeAhead < heads) gpr *= 2;
    const int per = groups / gpr;
    rope_kernel<DT, VEC, HALVES, L><<<(p.rows + per - 1) / per, kRopeThreads, 0, stream>>>(p, gpr);
}

template <int DT, bool VEC, bool HALVES>
void dispatch_rope(const RopeParams& p, cudaStream_t stream) {
    const int lanes = (p.head_dim / 2 + kRopePairs - 1) / kRopePairs;
    if (lanes <= 4) return run_rope<DT, VEC, HALVES, 4>(p, stream);
    if (lanes <= 8) return run_rope<DT, VEC, HALVES, 8>(p, stream);
    return run_rope<DT, VEC, HALVES, 16>(p, stream);
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
    const bool halves = p.half > 0;
    if (dtype == SPECA_BF16) {
        if (vectors)
            halves ? dispatch_rope<SPECA_BF16, true, true>(p, stream) : dispatch_rope<SPECA_BF16, true, false>(p, stream);
        else
            halves ? dispatch_rope<SPECA_BF16, false, true>(p, stream) : dispatch_rope<SPECA_BF16, false, false>(p, stream);
    } else {
        if (vectors)
            halves ? dispatch_rope<SPECA_F32, true, true>(p, stream) : dispatch_rope<SPECA_F32, true, false>(p, stream);
        else
            halves ? dispatch_rope<SPECA_F32, false, true>(p, stream) : dispatch_rope<SPECA_F32, false, false>(p, stream);
    }
    return cudaGetLastError();
}

}  // namespace speca
