// What the row kernels share: storage types, vector accesses, sums over the threads of a row.
#pragma once
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

}  // namespace
}  // namespace speca
