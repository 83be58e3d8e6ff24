// What the 8-bit products on the tensor cores share: waits, loads, block-scaled products, scales in tensor memory.
#pragma once
#include "speca_early.cuh"
#include "speca_matmul8_common.cuh"

namespace speca {
namespace {

constexpr int kRows = 128;  // rows of an operand of one SM, and lanes of tensor memory

__device__ __forceinline__ void fetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// ---- the pair of SMs ----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The first SM's barrier of this name.
template <int CG>
__device__ __forceinline__ uint32_t leaders(uint64_t* bar) {
    uint32_t a = smem_u32(bar);
    if constexpr (CG == 2) asm volatile("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(a));
    return a;
}
// Tells the first SM that this warp's accesses to tensor memory are done. They are (the warp waited for them), and tensor memory is ordered between threads by the
// tcgen05 fences in front of an arrival and behind a wait, whatever the arrival's own strength. No other memory is handed over, so nothing has to be
// released: a release to the cluster waits 1200 cycles for the thread's stores.
template <int CG>
__device__ __forceinline__ void hand_over(uint64_t* bar, int lane) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) {
        if constexpr (CG == 1)
            bar_arrive(bar);
        else
            asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leaders<CG>(bar)) : "memory");
    }
}
// Looks, or waits, for arrivals: from both SMs where there are two. One thread's wait polls: a suspended one wakes up some hundred cycles late.
constexpr uint32_t kPollLimit = 1u << 24;  // some tenths of a second
template <int CG>
__device__ __forceinline__ bool pair_test(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    if constexpr (CG == 1)
        asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok)
                     : "r"(smem_u32(bar)), "r"(parity)
                     : "memory");
    else
        asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok)
                     : "r"(smem_u32(bar)), "r"(parity)
                     : "memory");
    return ok != 0;
}
template <int CG>
__device__ __forceinline__ bool pair_wait(uint64_t* bar, uint32_t parity) {
    for (uint32_t poll = 0; poll < kPollLimit; ++poll)
        if (pair_test<CG>(bar, parity)) return true;
    return false;
}
// A whole warp suspends: where eight or twelve of them polled beside the products, large ones ran 1.3 % slower (power).
template <int CG>
__device__ __forceinline__ bool pair_warp_wait(uint64_t* bar, uint32_t parity) {
    if constexpr (CG == 1) {
        return warp_wait(bar, parity);
    } else {
        for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
            uint32_t ok;
            asm volatile(
                "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                : "=r"(ok)
                : "r"(smem_u32(bar)), "r"(parity)
                : "memory");
            if (__all_sync(0xffffffffu, ok != 0)) return true;
        }
        return false;
    }
}
// A place in a ring.
template <int N>
struct Turn {
    int stage = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++stage == N) stage = 0, phase ^= 1;
    }
};

// ---- tensor cores -------------------------------------------------------------------------------
template <int CG>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}
// Arrives, when all products so far are done, at the barrier of this name in every SM of the tile.
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                     "h"(static_cast<uint16_t>(3))
                     : "memory");
}
// 128 bytes of k a row, with the 128-byte swizzle: 1024 bytes between groups of 8 rows.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
    return static_cast<uint64_t>((addr >> 4) & 0x3fff) | uint64_t(1) << 16 | uint64_t(64) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// e4m3 x e4m3 -> fp32, scales of 8-bit exponents. The scale of block i (0 .. 3) is byte i of a column.
template <int CG, int NT>
__host__ __device__ constexpr uint32_t mma_desc8(uint32_t i) {
    return i << 4 | static_cast<uint32_t>(NT >> 3) << 17 | 1u << 23 | static_cast<uint32_t>(kRows * CG >> 4) << 24 | i << 29;
}
template <int CG>
__device__ __forceinline__ void mma8(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t scale_a, uint32_t scale_b, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(desc), "r"(scale_a), "r"(scale_b), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(desc), "r"(scale_a), "r"(scale_b), "r"(accumulate)
            : "memory");
}

// Scales of four blocks of a row; those of rows that do not exist: 1. An ordinary load behind the wait for the kernel in front, which may be writing them
// when this one begins: the read-only path (__ldg) is for what nobody writes while a kernel runs.
__device__ __forceinline__ uint32_t scale_word(const uint8_t* scales, int64_t stride, int group, int row, int rows) {
    uint32_t word = 0x7f7f7f7fu;
    if (row < rows) asm volatile("ld.global.b32 %0, [%1];" : "=r"(word) : "l"(reinterpret_cast<const uint32_t*>(scales + group * stride) + row) : "memory");
    return word;
}

}  // namespace
}  // namespace speca
