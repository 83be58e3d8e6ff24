// Rows into 8 bits, after an RMS or layer norm with the residual's addition, or as they are.
//
//   z = x + gate * branch;  u = (z - mean) * rsqrt(mean((z - mean)^2) + eps), mean = 0 for the RMS norm
//   y = u * weight * (1 + scale) + shift;  per 128 elements of y: the scale byte, the codes
// One pass over memory: the G threads of a row keep it in registers (NV accesses of 8 elements each), 16 lanes share a block of 128,
// so its largest magnitude takes four shuffles. y is rounded once, to its code. Bound by memory.
#include "speca_eight_common.cuh"
#include "speca_rows_common.cuh"

namespace speca {
namespace {

// Eight elements of a block of 128 that lane l of 16 holds: consecutive ones, as accesses of 16 bytes, or every 16th from l on, one
// access each, where rows do not start on 16 bytes or hold no multiple of 8.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const char* base, int first, int l, int dim, T (&out)[8]) {
    if constexpr (VEC) {
        constexpr int E = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < 8; i += E) {
            const Pack<T, E> v = load<T, E>(base, first + 8 * l + i);
#pragma unroll
            for (int e = 0; e < E; ++e) out[i + e] = v.e[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (first + l + 16 * e < dim) out[e] = reinterpret_cast<const T*>(base)[first + l + 16 * e];
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(char* base, int first, int l, int dim, const float (&v)[8]) {
    if constexpr (VEC) {
        constexpr int E = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < 8; i += E) {
            Pack<T, E> out;
#pragma unroll
            for (int e = 0; e < E; ++e) out.e[e] = from_float<T>(v[i + e]);
            store<T, E>(base, first + 8 * l + i, out);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (first + l + 16 * e < dim) reinterpret_cast<T*>(base)[first + l + 16 * e] = from_float<T>(v[e]);
    }
}

// One block of 128 of row `row`, 8 values in each of 16 lanes (zeros behind the end), to codes and scale. The whole warp calls.
template <bool VEC>
__device__ __forceinline__ void put8(const Out8& o, int row, int first, int l, int dim, bool write, float (&v)[8]) {
    const uint32_t byte = scale_byte(block_top<8, 8>(v));
    const float inv = inverse_of(byte);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= inv;
    if (!write || first >= dim) return;
    const uint32_t lo = pack_e4m3(v[0], v[1], v[2], v[3]), hi = pack_e4m3(v[4], v[5], v[6], v[7]);
    uint8_t* codes = o.codes + row * o.code_stride + first;
    if constexpr (VEC) {
        if (first + 8 * l < dim) *reinterpret_cast<uint2*>(codes + 8 * l) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (first + l + 16 * e < dim) codes[l + 16 * e] = static_cast<uint8_t>((e < 4 ? lo : hi) >> 8 * (e % 4));
    }
    if (l == 0) o.scales[first / (4 * kBlock8) * o.scale_stride + 4 * static_cast<int64_t>(row) + first / kBlock8 % 4] = static_cast<uint8_t>(byte);
}

template <int DT, bool VEC, int NV, int G, int NT>
__global__ void __launch_bounds__(NT) norm8_kernel(const __grid_constant__ Norm8Params p) {
    using T = typename Type<DT>::T;
    __shared__ float red[2][NT / 32];
    const int row = blockIdx.x * (NT / G) + threadIdx.x / G;
    const int t = threadIdx.x % G, l = t % 16;
    // where the 8 elements of access i begin, and which of them there are
    auto first = [&](int i) { return (t / 16 + i * (G / 16)) * kBlock8; };
    auto there = [&](int i, int e) { return first(i) + (VEC ? 8 * l : l + 16 * e) < p.dim; };
    bool live = row < p.rows;
    int seq = 0;
    if (live && p.row_seq != nullptr) {
        seq = p.row_seq[row];
        live = p.dev_mask == nullptr || p.dev_mask[seq] != 0;
    }
    float z[NV][8];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[i][e] = 0.f;
    auto at = [&](const char* base, int64_t index, int64_t stride) { return base + index * stride * static_cast<int64_t>(sizeof(T)); };
    if (live) {
        const char* px = at(p.x, row, p.x_stride);
        T in[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (there(i, 0)) load8<T, VEC>(px, first(i), l, p.dim, in[i]);
        if (p.branch != nullptr) {
            const char* pb = at(p.branch, row, p.branch_stride);
            T br[NV][8];
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (there(i, 0)) load8<T, VEC>(pb, first(i), l, p.dim, br[i]);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!there(i, 0)) continue;
                T g[8];
                if (p.gate != nullptr) load8<T, VEC>(at(p.gate, seq, p.mod_stride), first(i), l, p.dim, g);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (there(i, e)) z[i][e] = fmaf(p.gate != nullptr ? to_float(g[e]) : 1.f, to_float(br[i][e]), to_float(in[i][e]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (there(i, e)) z[i][e] = to_float(in[i][e]);
        }
        if (p.x_out != nullptr) {
            char* po = p.x_out + row * p.x_out_stride * static_cast<int64_t>(sizeof(T));
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (there(i, 0)) store8<T, VEC>(po, first(i), l, p.dim, z[i]);
        }
    }
    if (p.norm) {
        // every thread takes part in the sums: a row's threads may share a barrier with a dead row's
        if (p.centre) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += z[i][e];
            const float mean = sum_row<G>(sum, red[0]) / p.dim;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (there(i, e)) z[i][e] -= mean;
        }
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(z[i][e], z[i][e], sq);
        const float rstd = 1.f / sqrtf(sum_row<G>(sq, red[1]) / p.dim + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            T w[8], s[8], b[8];
            const bool some = live && there(i, 0);
            if (some && p.weight != nullptr) load8<T, VEC>(p.weight, first(i), l, p.dim, w);
            if (some && p.scale != nullptr) load8<T, VEC>(at(p.scale, seq, p.mod_stride), first(i), l, p.dim, s);
            if (some && p.shift != nullptr) load8<T, VEC>(at(p.shift, seq, p.mod_stride), first(i), l, p.dim, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!live || !there(i, e)) continue;
                float y = z[i][e] * rstd;
                if (p.weight != nullptr) y *= to_float(w[e]);
                z[i][e] = fmaf(y, p.scale != nullptr ? 1.f + to_float(s[e]) : 1.f, p.shift != nullptr ? to_float(b[e]) : 0.f);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) put8<VEC>(p.out, row, first(i), l, p.dim, live, z[i]);
}

// Rows too long for the registers of one block: passes over memory, the later ones out of L2. A thread meets the same elements in each.
template <int DT>
__global__ void __launch_bounds__(1024) norm8_long_kernel(const __grid_constant__ Norm8Params p) {
    using T = typename Type<DT>::T;
    __shared__ float red[2][32];
    const int row = blockIdx.x;
    const int seq = p.row_seq == nullptr ? 0 : p.row_seq[row];
    if (p.row_seq != nullptr && p.dev_mask != nullptr && p.dev_mask[seq] == 0) return;
    auto row_of = [&](const char* base, int64_t i, int64_t stride) { return base == nullptr ? nullptr : reinterpret_cast<const T*>(base) + i * stride; };
    const T *px = row_of(p.x, row, p.x_stride), *pb = row_of(p.branch, row, p.branch_stride), *pw = row_of(p.weight, 0, 0);
    const T *pg = row_of(p.gate, seq, p.mod_stride), *ps = row_of(p.scale, seq, p.mod_stride), *pt = row_of(p.shift, seq, p.mod_stride);
    T* po = p.x_out == nullptr ? nullptr : reinterpret_cast<T*>(p.x_out) + row * p.x_out_stride;
    const int l = threadIdx.x % 16, start = threadIdx.x / 16 * kBlock8;
    auto value = [&](int c) {
        const float v = to_float(px[c]);
        return pb == nullptr ? v : fmaf(pg == nullptr ? 1.f : to_float(pg[c]), to_float(pb[c]), v);
    };
    float mean = 0.f, rstd = 1.f;
    if (p.norm) {
        if (p.centre) {
            float sum = 0.f;
            for (int f = start; f < p.dim; f += 64 * kBlock8)
                for (int c = f + l; c < min(f + kBlock8, p.dim); c += 16) sum += value(c);
            mean = sum_row<1024>(sum, red[0]) / p.dim;
        }
        float sq = 0.f;
        for (int f = start; f < p.dim; f += 64 * kBlock8)
            for (int c = f + l; c < min(f + kBlock8, p.dim); c += 16) {
                const float d = value(c) - mean;
                sq = fmaf(d, d, sq);
            }
        rstd = 1.f / sqrtf(sum_row<1024>(sq, red[1]) / p.dim + p.eps);
    }
    const int last = threadIdx.x / 32 * 2 * kBlock8;  // both blocks of a warp go through the loop together
    for (int f = start, g = last; g < p.dim; f += 64 * kBlock8, g += 64 * kBlock8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = f + l + 16 * e;
            v[e] = 0.f;
            if (c >= p.dim) continue;
            v[e] = value(c);
            if (po != nullptr) po[c] = from_float<T>(v[e]);
            if (!p.norm) continue;
            float y = (v[e] - mean) * rstd;
            if (pw != nullptr) y *= to_float(pw[c]);
            v[e] = fmaf(y, ps == nullptr ? 1.f : 1.f + to_float(ps[c]), pt == nullptr ? 0.f : to_float(pt[c]));
        }
        put8<false>(p.out, row, f, l, p.dim, true, v);
    }
}

template <int DT, bool VEC, int NV, int G, int NT>
void run_norm8(const Norm8Params& p, cudaStream_t stream) {
    const int per = NT / G;
    norm8_kernel<DT, VEC, NV, G, NT><<<(p.rows + per - 1) / per, NT, 0, stream>>>(p);
}

template <int DT, bool VEC>
void dispatch_norm8(const Norm8Params& p, cudaStream_t stream) {
    const int n = (p.dim + kBlock8 - 1) / kBlock8 * 16;  // accesses per row: 16 lanes a block
    if (n <= 32 * 2) return run_norm8<DT, VEC, 2, 32, 128>(p, stream);
    if (n <= 64 * 2) return run_norm8<DT, VEC, 2, 64, 128>(p, stream);
    if (n <= 128 * 2) return run_norm8<DT, VEC, 2, 128, 128>(p, stream);
    if (n <= 128 * 3) return run_norm8<DT, VEC, 3, 128, 128>(p, stream);
    if (n <= 128 * 5) return run_norm8<DT, VEC, 5, 128, 128>(p, stream);
    if (n <= 256 * 4) return run_norm8<DT, VEC, 4, 256, 256>(p, stream);
    if (n <= 512 * 4) return run_norm8<DT, VEC, 4, 512, 512>(p, stream);
    norm8_long_kernel<DT><<<p.rows, 1024, 0, stream>>>(p);
}

}  // namespace

cudaError_t launch_norm8(const Norm8Params& p, int dtype, bool vectors, cudaStream_t stream) {
    if (p.rows == 0) return cudaSuccess;
    if (dtype == SPECA_BF16)
        vectors ? dispatch_norm8<SPECA_BF16, true>(p, stream) : dispatch_norm8<SPECA_BF16, false>(p, stream);
    else
        vectors ? dispatch_norm8<SPECA_F32, true>(p, stream) : dispatch_norm8<SPECA_F32, false>(p, stream);
    return cudaGetLastError();
}

}  // namespace speca
