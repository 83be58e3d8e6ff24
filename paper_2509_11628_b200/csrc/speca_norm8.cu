// Rows into 8 bits, after an RMS or layer norm with the residual's addition, or as they are.
//
//   z = x + gate * branch;  u = (z - mean) * rsqrt(mean((z - mean)^2) + eps), mean = 0 for the RMS norm
//   y = u * weight * (1 + scale) + shift;  per 128 elements of y: the scale byte, the codes
// One pass over memory: the G threads of a row keep it in registers (NV accesses of 16 elements each). Eight lanes share a block of 128,
// so its largest magnitude takes three shuffles. y is rounded once, to its code. Bound by memory in the end, by instructions and by the blocks that
// registers leave room for on the way there: 20926 rows x 4096 bf16 with branch, gate and weight 113 us (5.3 TB/s), as they are 49 us (5.2 TB/s); with 8 elements a
// lane (four shuffles, one scale and one set of addresses for half as much) 210 and 84. Tried and not kept, 20926 x 4096: weight, scale and shift loaded in
// front of the sums 155 us (registers), asked into L1 there 117, bounds on the registers 114 to 146, the row map read before the wait 118.
#include "speca_early.cuh"
#include "speca_eight_common.cuh"
#include "speca_rows_common.cuh"

namespace speca {
namespace {

constexpr int kPer = 16, kLanes = kBlock8 / kPer;  // elements of an access, lanes of a block

// Sixteen elements of a block of 128 that lane l of 8 holds: consecutive ones, as accesses of 16 bytes; or every 8th from l on, one access
// each, where rows do not start on 16 bytes or hold no multiple of 16. `at`: the block's first element of the row.
template <typename T, bool VEC>
__device__ __forceinline__ void load16(const T* row, int at, int l, int dim, float (&out)[kPer]) {
    if constexpr (VEC) {
        constexpr int E = 16 / sizeof(T);
        Pack<T, E> v[kPer / E];
#pragma unroll
        for (int i = 0; i < kPer / E; ++i) v[i] = *reinterpret_cast<const Pack<T, E>*>(row + at + kPer * l + i * E);
#pragma unroll
        for (int i = 0; i < kPer; ++i) out[i] = to_float(v[i / E].e[i % E]);
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e) out[e] = at + l + kLanes * e < dim ? to_float(row[at + l + kLanes * e]) : 0.f;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store16(T* row, int at, int l, int dim, const float (&v)[kPer]) {
    if constexpr (VEC) {
        constexpr int E = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < kPer; i += E) {
            Pack<T, E> out;
#pragma unroll
            for (int e = 0; e < E; ++e) out.e[e] = from_float<T>(v[i + e]);
            *reinterpret_cast<Pack<T, E>*>(row + at + kPer * l + i) = out;
        }
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (at + l + kLanes * e < dim) row[at + l + kLanes * e] = from_float<T>(v[e]);
    }
}

// One block of 128 of row `row`, 16 values in each of 8 lanes (zeros behind the end), to codes and scale. The whole warp calls.
template <bool VEC>
__device__ __forceinline__ void put16(const Out8& o, int64_t row, int at, int l, int dim, bool write, float (&v)[kPer]) {
    const uint32_t byte = scale_byte(block_top<kPer, kLanes / 2>(v));
    const float inv = inverse_of(byte);
    uint32_t w[kPer / 4];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) w[i] = pack_e4m3(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
    if (!write || at >= dim) return;
    uint8_t* codes = o.codes + row * o.code_stride + at;
    if constexpr (VEC) {
        if (at + kPer * l < dim) *reinterpret_cast<uint4*>(codes + kPer * l) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (at + l + kLanes * e < dim) codes[l + kLanes * e] = static_cast<uint8_t>(w[e / 4] >> 8 * (e % 4));
    }
    if (l == 0) o.scales[at / (4 * kBlock8) * o.scale_stride + 4 * row + at / kBlock8 % 4] = static_cast<uint8_t>(byte);
}

// Rows as they are: nothing ties a row's blocks of 128 together, so 8 lanes take one after another of all rows' blocks, kBlocks of them at once.
constexpr int kQuantThreads = 256, kBlocks = 2;
template <int DT, bool VEC>
__global__ void __launch_bounds__(kQuantThreads) quantize8_kernel(const __grid_constant__ Norm8Params p, const int64_t total, const int per_row) {
    using T = typename Type<DT>::T;
    constexpr int kGroups = kQuantThreads / kLanes;
    wait_for_stream();
    const int l = threadIdx.x % kLanes;
    const int64_t index = static_cast<int64_t>(blockIdx.x) * (kGroups * kBlocks) + threadIdx.x / kLanes;
    int64_t row = total <= 0xffffffff ? static_cast<uint32_t>(index) / static_cast<uint32_t>(per_row) : index / per_row;
    int64_t block = index - row * per_row;
    float v[kBlocks][kPer];
    int64_t rows[kBlocks];
    int at[kBlocks];
    bool live[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
        rows[i] = row;
        at[i] = static_cast<int>(block) * kBlock8;
        live[i] = row < p.rows && (p.dev_mask == nullptr || p.dev_mask[p.row_seq[row]] != 0);
        for (block += kGroups; block >= per_row; block -= per_row) ++row;
#pragma unroll
        for (int e = 0; e < kPer; ++e) v[i][e] = 0.f;
        if (live[i] && (!VEC || at[i] + kPer * l < p.dim))
            load16<T, VEC>(reinterpret_cast<const T*>(p.x) + rows[i] * p.x_stride, at[i], l, p.dim, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) put16<VEC>(p.out, rows[i], at[i], l, p.dim, live[i], v[i]);
}

template <int DT, bool VEC, int NV, int G, int NT>
__global__ void __launch_bounds__(NT) norm8_kernel(const __grid_constant__ Norm8Params p) {
    using T = typename Type<DT>::T;
    __shared__ float red[2][NT / 32];
    const int row = blockIdx.x * (NT / G) + threadIdx.x / G;
    const int t = threadIdx.x % G, l = t % kLanes;
    auto at = [&](int i) { return (t / kLanes + i * (G / kLanes)) * kBlock8; };                // block of access i
    auto some = [&](int i) { return VEC ? at(i) + kPer * l < p.dim : at(i) < p.dim; };         // whether any of it exists
    auto there = [&](int i, int e) { return VEC ? some(i) : at(i) + l + kLanes * e < p.dim; };
    auto row_of = [&](const char* base, int64_t i, int64_t stride) { return reinterpret_cast<const T*>(base) + i * stride; };
    wait_for_stream();
    bool live = row < p.rows;
    int seq = 0;
    if (live) {
        seq = p.row_seq[row];
        live = p.dev_mask == nullptr || p.dev_mask[seq] != 0;
    }
    float z[NV][kPer];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < kPer; ++e) z[i][e] = 0.f;
    if (live) {
        const T* px = row_of(p.x, row, p.x_stride);
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (some(i)) load16<T, VEC>(px, at(i), l, p.dim, z[i]);
        if (p.branch != nullptr) {
            const T* pb = row_of(p.branch, row, p.branch_stride);
            const T* pg = row_of(p.gate, seq, p.mod_stride);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!some(i)) continue;
                float b[kPer];
                load16<T, VEC>(pb, at(i), l, p.dim, b);
                if (p.gate != nullptr) {
                    float g[kPer];
                    load16<T, VEC>(pg, at(i), l, p.dim, g);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) z[i][e] = fmaf(g[e], b[e], z[i][e]);
                } else {
#pragma unroll
                    for (int e = 0; e < kPer; ++e) z[i][e] += b[e];
                }
            }
        }
        if (p.x_out != nullptr) {
            T* po = reinterpret_cast<T*>(p.x_out) + row * p.x_out_stride;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (some(i)) store16<T, VEC>(po, at(i), l, p.dim, z[i]);
        }
    }
    // every thread takes part in the sums: a row's threads may share a barrier with a dead row's
    if (p.centre) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) sum += z[i][e];
        const float mean = sum_row<G>(sum, red[0]) / p.dim;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (there(i, e)) z[i][e] -= mean;
    }
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < kPer; ++e) sq = fmaf(z[i][e], z[i][e], sq);
    const float rstd = 1.f / sqrtf(sum_row<G>(sq, red[1]) / p.dim + p.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (live && some(i)) {
            float f[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e) z[i][e] *= rstd;
            if (p.weight != nullptr) {
                load16<T, VEC>(row_of(p.weight, 0, 0), at(i), l, p.dim, f);
#pragma unroll
                for (int e = 0; e < kPer; ++e) z[i][e] *= f[e];
            }
            if (p.scale != nullptr) {
                load16<T, VEC>(row_of(p.scale, seq, p.mod_stride), at(i), l, p.dim, f);
#pragma unroll
                for (int e = 0; e < kPer; ++e) z[i][e] = fmaf(z[i][e], f[e], z[i][e]);
            }
            if (p.shift != nullptr) {
                load16<T, VEC>(row_of(p.shift, seq, p.mod_stride), at(i), l, p.dim, f);
#pragma unroll
                for (int e = 0; e < kPer; ++e) z[i][e] += f[e];
            }
        }
        put16<VEC>(p.out, row, at(i), l, p.dim, live, z[i]);
    }
}

// Sum of what the row's 1024 threads hold in 64 bits.
__device__ __forceinline__ double sum_long(double x, double* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = x;
    __syncthreads();
    x = red[threadIdx.x % 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Rows too long for the registers of one block: passes over memory, the later ones out of L2. A thread meets the same elements in each. It adds up to 2^21
// of them: those of one block of 128 (16) in 32 bits, the blocks in 64. One element an access: 1024 x 32768 bf16 106 us, 128 with the mean. (All in 32 bits, squares of like size came out 1.4e-4 off at 2^24 elements and 2e-2 at 2^31.)
template <int DT>
__global__ void __launch_bounds__(1024) norm8_long_kernel(const __grid_constant__ Norm8Params p) {
    using T = typename Type<DT>::T;
    __shared__ double red[2][32];
    const int row = blockIdx.x;
    wait_for_stream();
    const int seq = p.row_seq[row];
    if (p.dev_mask != nullptr && p.dev_mask[seq] == 0) return;
    auto row_of = [&](const char* base, int64_t i, int64_t stride) { return base == nullptr ? nullptr : reinterpret_cast<const T*>(base) + i * stride; };
    const T *px = row_of(p.x, row, p.x_stride), *pb = row_of(p.branch, row, p.branch_stride), *pw = row_of(p.weight, 0, 0);
    const T *pg = row_of(p.gate, seq, p.mod_stride), *ps = row_of(p.scale, seq, p.mod_stride), *pt = row_of(p.shift, seq, p.mod_stride);
    T* po = p.x_out == nullptr ? nullptr : reinterpret_cast<T*>(p.x_out) + row * p.x_out_stride;
    // without a sign: a step behind the last element passes 2^31
    constexpr uint32_t kStep = 1024 / kLanes * kBlock8;
    const uint32_t dim = p.dim, l = threadIdx.x % kLanes, start = threadIdx.x / kLanes * kBlock8;
    auto value = [&](uint32_t c) {
        const float v = to_float(px[c]);
        return pb == nullptr ? v : fmaf(pg == nullptr ? 1.f : to_float(pg[c]), to_float(pb[c]), v);
    };
    float mean = 0.f;
    if (p.centre) {
        double sum = 0;
        for (uint32_t f = start; f < dim; f += kStep) {
            float part = 0.f;
            for (uint32_t c = f + l; c < min(f + kBlock8, dim); c += kLanes) part += value(c);
            sum += part;
        }
        mean = static_cast<float>(sum_long(sum, red[0]) / p.dim);
    }
    double sq = 0;
    for (uint32_t f = start; f < dim; f += kStep) {
        float part = 0.f;
        for (uint32_t c = f + l; c < min(f + kBlock8, dim); c += kLanes) {
            const float d = value(c) - mean;
            part = fmaf(d, d, part);
        }
        sq += part;
    }
    const float rstd = 1.f / sqrtf(static_cast<float>(sum_long(sq, red[1]) / p.dim) + p.eps);
    // the blocks of a warp go through the loop together
    for (uint32_t f = start, first = threadIdx.x / 32 * (32 / kLanes) * kBlock8; first < dim; f += kStep, first += kStep) {
        float v[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const uint32_t c = f + l + kLanes * e;
            v[e] = 0.f;
            if (c >= dim) continue;
            v[e] = value(c);
            if (po != nullptr) po[c] = from_float<T>(v[e]);
            float y = (v[e] - mean) * rstd;
            if (pw != nullptr) y *= to_float(pw[c]);
            v[e] = fmaf(y, ps == nullptr ? 1.f : 1.f + to_float(ps[c]), pt == nullptr ? 0.f : to_float(pt[c]));
        }
        put16<false>(p.out, row, static_cast<int>(f), l, p.dim, f < dim, v);
    }
}

template <int DT, bool VEC, int NV, int G, int NT>
cudaError_t run_norm8(const Norm8Params& p, cudaStream_t stream) {
    const int per = NT / G;
    return launch_early(norm8_kernel<DT, VEC, NV, G, NT>, (p.rows + per - 1) / per, 1, NT, 0, stream, p);
}

template <int DT, bool VEC>
cudaError_t dispatch_norm8(const Norm8Params& p, cudaStream_t stream) {
    const int per_row = (p.dim + kBlock8 - 1) / kBlock8;
    if (!p.norm) {
        constexpr int per = kQuantThreads / kLanes * kBlocks;
        const int64_t total = static_cast<int64_t>(p.rows) * per_row;
        return launch_early(quantize8_kernel<DT, VEC>, static_cast<unsigned>((total + per - 1) / per), 1, kQuantThreads, 0, stream, p, total, per_row);
    }
    // One access a thread as long as a block has threads for the row: of 4096 elements 256 threads x 1 took 113 us with branch and gate (20926 rows),
    // 128 x 2 took 125; of 1152, 96 x 1 39 us with the branch, 32 x 3 47. Behind 6144 two: 8192 as 256 x 2 94 us (8345 rows), 512 x 1 111.
    const int n = per_row * kLanes;  // accesses of a row
    if (n <= 32) return run_norm8<DT, VEC, 1, 32, 128>(p, stream);
    if (n <= 64) return run_norm8<DT, VEC, 1, 64, 128>(p, stream);
    if (n <= 96) return run_norm8<DT, VEC, 1, 96, 96>(p, stream);
    if (n <= 128) return run_norm8<DT, VEC, 1, 128, 128>(p, stream);
    if (n <= 192) return run_norm8<DT, VEC, 1, 192, 192>(p, stream);
    if (n <= 256) return run_norm8<DT, VEC, 1, 256, 256>(p, stream);
    if (n <= 320) return run_norm8<DT, VEC, 1, 320, 320>(p, stream);
    if (n <= 384) return run_norm8<DT, VEC, 1, 384, 384>(p, stream);
    if (n <= 512) return run_norm8<DT, VEC, 2, 256, 256>(p, stream);
    if (n <= 512 * 2) return run_norm8<DT, VEC, 2, 512, 512>(p, stream);
    return launch_early(norm8_long_kernel<DT>, p.rows, 1, 1024, 0, stream, p);
}

}  // namespace

cudaError_t launch_norm8(const Norm8Params& p, int dtype, bool vectors, cudaStream_t stream) {
    if (p.rows == 0) return cudaSuccess;
    if (dtype == SPECA_BF16) return vectors ? dispatch_norm8<SPECA_BF16, true>(p, stream) : dispatch_norm8<SPECA_BF16, false>(p, stream);
    return vectors ? dispatch_norm8<SPECA_F32, true>(p, stream) : dispatch_norm8<SPECA_F32, false>(p, stream);
}

}  // namespace speca
