// Matrix products in 8 bits for few rows (single tokens, or short prompts): bound by reading the weights once.
//
// The transposed product, D = W A^T: a block has 128 features as the tensor cores' rows, NR rows of A as their columns, and a share of k.
// The shares of a cluster's blocks are added up through distributed shared memory, in the order of their ranks. Two blocks share an SM; with
// some 100 KB each on its way from memory (a ring of stages of 128 elements of k, filled by the copy engine).
//   warps 0-3  scales into tensor memory, a quarter of the lanes each; then the sums into shared memory
//   warp 4     loads;  warp 5: issues the products;  all eight: the epilogue, a row at a time
// Every wait is bounded, as in the kernel for many rows.
// Measured: weights stream at 6.7 TB/s behind a start and an end of 6 us together (of which an empty launch is 2.5): 1 row x 4096 x 4096 8.2 us, 14336 x 4096
// 14.7, 64 rows 10.0 and 17.1. Tried and not kept: shares sent to the row's block instead of fetched by it (equal or slower), one block an SM with
// twice the stages (17 us for 4096 x 4096 of two shares, 8 us as it is). (With mma.sync in place of the tensor memory's products, 8 rows by 14336 x 4096 took
// 17 us and 32 rows 37.)
#include "speca_matmul8_tensor.cuh"

namespace speca {
namespace {

constexpr int kFewThreads = 256;
constexpr int kLoader = 4, kIssuer = 5;
constexpr uint32_t kMaxRanks = kFewRanks;

template <int NR>
struct FewShape {
    static constexpr uint32_t kBytesW = kRows * 128, kStage = kBytesW + NR * 128;
    static constexpr int kStages = NR <= 16 ? 6 : NR <= 32 ? 5 : NR <= 64 ? 4 : 3;
    // tensor memory: the sums, then two stages of 8 columns of scales (4 for W, 4 for A)
    static constexpr int kScales = NR < 32 ? 32 : NR;
    static constexpr uint32_t kCols = kScales + 16 <= 64 ? 64 : kScales + 16 <= 128 ? 128 : 256;
};
template <int NR>
struct FewSmem {
    uint8_t tiles[FewShape<NR>::kStages][FewShape<NR>::kStage];
    uint64_t full[FewShape<NR>::kStages], empty[FewShape<NR>::kStages];
    uint64_t scales_full[2], scales_used[2], sums_full;
    uint32_t tmem, abort;
};

__device__ __forceinline__ uint32_t cluster_blocks() {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}

template <int DT, int NR>
__global__ void __launch_bounds__(kFewThreads, 2)
    matmul8_few_kernel(const __grid_constant__ Matmul8Params p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w) {
    using S = FewShape<NR>;
    extern __shared__ __align__(1024) char raw[];
    FewSmem<NR>& sm = *reinterpret_cast<FewSmem<NR>*>(raw);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = cluster_rank(), ranks = cluster_blocks();
    const int m_tiles = (p.m + NR - 1) / NR, tile = blockIdx.x / ranks;
    const int m0 = tile % m_tiles * NR, n0 = tile / m_tiles * kRows, rows = min(NR, p.m - m0);
    if (smem_u32(raw) % 1024 != 0) {  // the swizzled tiles rely on it; the same in every block
        if (threadIdx.x == 0) atomicExch(p.gave_up, 1u);
        return;
    }
    if (threadIdx.x == kLoader * 32) {
        for (int i = 0; i < S::kStages; ++i) {
            bar_init(&sm.full[i], 1);
            bar_init(&sm.empty[i], 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(&sm.scales_full[b], 4);  // one arrival per warp
            bar_init(&sm.scales_used[b], 1);
        }
        bar_init(&sm.sums_full, 1);
        sm.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fetch_map(&map_w);
        fetch_map(&map_a);
    }
    wait_for_stream();
    if (p.dev_mask != nullptr) {  // the same in every block of the cluster
        bool live = false;
        for (int r = lane; r < rows; r += 32) live = live || p.dev_mask[p.row_seq[m0 + r]] != 0;
        if (!__any_sync(0xffffffffu, live)) return;
    }
    const int k_blocks = (p.k + kBlock8 - 1) / kBlock8, share = (k_blocks + ranks - 1) / ranks;
    const int begin = min(static_cast<int>(rank) * share, k_blocks), end = min(begin + share, k_blocks);

    const int first_row = rank + ranks * warp;  // of this warp's epilogue
    int seq = first_row < rows ? p.row_seq[m0 + first_row] : 0;

    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    auto load = [&](int kb) {
        bar_expect(&sm.full[stage], S::kStage);
        const uint32_t to = smem_u32(sm.tiles[stage]), bar = smem_u32(&sm.full[stage]);
        load_tile<1>(to, &map_w, kb * kBlock8, n0, bar);
        load_tile<1>(to + S::kBytesW, &map_a, kb * kBlock8, m0, bar);
        if (++stage == S::kStages) stage = 0, phase ^= 1;
    };
    if (warp == kLoader) {
        if (lane == 0)
            for (int kb = begin; kb < min(begin + S::kStages, end); ++kb) load(kb);  // the first stages have room
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(S::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);

    if (warp == kLoader) {
        if (lane == 0) {
            for (int kb = begin + S::kStages; kb < end; ++kb) {
                ok = bar_wait(&sm.empty[stage], phase ^ 1);
                if (!ok) break;
                load(kb);
            }
            if (!ok) sm.abort = 1;
            // Copies in flight must land before the block gives its shared memory back, also where another warp's wait ran out.
            for (int i = 0; i < S::kStages; ++i) bar_wait(&sm.full[i], i < stage ? phase : phase ^ 1);
        }
    } else if (warp == kIssuer) {
        if (elect_one()) {
            Turn<2> held;
            for (int kb = begin; kb < end; ++kb) {
                if (kb == begin || kb % 4 == 0) ok = pair_wait<1>(&sm.scales_full[held.stage], held.phase);
                ok = ok && pair_wait<1>(&sm.full[stage], phase);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = smem_u32(sm.tiles[stage]), scales = tmem + S::kScales + held.stage * 8;
                const uint64_t w = tile_desc(from), a = tile_desc(from + S::kBytesW);
                const uint32_t desc = mma_desc8<1, NR>(0) | static_cast<uint32_t>(kb % 4) << 4 | static_cast<uint32_t>(kb % 4) << 29;
#pragma unroll
                for (int s = 0; s < 4; ++s) mma8<1>(tmem, w + 2 * s, a + 2 * s, desc, scales, scales + 4, kb > begin || s > 0);
                commit<1>(&sm.empty[stage]);
                if (kb % 4 == 3 || kb + 1 == end) {
                    commit<1>(&sm.scales_used[held.stage]);
                    held.next();
                }
                if (++stage == S::kStages) stage = 0, phase ^= 1;
            }
            if (!ok) sm.abort = 1;
            commit<1>(&sm.sums_full);  // also where a wait ran out: what was issued ends before the block does
        }
        __syncwarp();
    } else if (warp < 4) {
        // ---- scales: lane i takes rows i, 32 + i, ...; those of the next group are on their way while this one waits for room ----
        Turn<2> to;
        uint32_t word[8];
        auto fetch = [&](int group) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                word[j] = scale_word(p.w_scales, p.w_scale_stride, group, n0 + 32 * j + lane, p.n);
                word[4 + j] = 32 * j < NR ? scale_word(p.a_scales, p.a_scale_stride, group, m0 + 32 * j + lane, p.m) : 0x7f7f7f7fu;
            }
        };
        const uint32_t first = tmem + (static_cast<uint32_t>(warp * 32) << 16);
        if (begin < end) fetch(begin / 4);
        for (int kb = begin; kb < end; kb = kb / 4 * 4 + 4) {
            ok = pair_warp_wait<1>(&sm.scales_used[to.stage], to.phase ^ 1);
            if (!ok) break;
            tc_fence_after();
            tmem_store4(first + S::kScales + to.stage * 8, word);
            tmem_store4(first + S::kScales + to.stage * 8 + 4, word + 4);
            tmem_wait_store();
            hand_over<1>(&sm.scales_full[to.stage], lane);
            to.next();
            if (kb / 4 * 4 + 4 < end) fetch(kb / 4 + 1);
        }
        // ---- the sums, one feature a lane: [row][feature] where the tiles were ----
        float* const sums = reinterpret_cast<float*>(raw);
        static_assert(NR * kRows * 4 <= sizeof(sm.tiles), "room");
        ok = pair_warp_wait<1>(&sm.sums_full, 0) && ok;
        if (ok) {
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < rows; c += 16) {
                uint32_t x[16];
                tmem_load16(first + c, x);
                tmem_wait_load<16>(x);
#pragma unroll
                for (int e = 0; e < 16; ++e) sums[(c + e) * kRows + warp * 32 + lane] = begin < end ? __uint_as_float(x[e]) : 0.f;
            }
        } else {
            sm.abort = 1;
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(&sm.abort) != 0) atomicExch(p.gave_up, 1u);
    if (ranks > 1) cluster_sync();
    // a row for each warp of the cluster in turn: the shares in the order of their ranks, all asked for at once
    for (int r = rank + ranks * warp; r < rows; r += ranks * 8) {
        const int row = m0 + r;
        const uint32_t at = smem_u32(raw) + (r * kRows + 4 * lane) * 4;
        float x[kMaxRanks][4], v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (uint32_t q = 0; q < kMaxRanks; ++q) {
            if (q >= ranks) break;
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(q));
            asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[q][0]), "=f"(x[q][1]), "=f"(x[q][2]), "=f"(x[q][3]) : "r"(there) : "memory");
        }
        if (r != first_row) seq = p.row_seq[row];
        if (p.dev_mask != nullptr && p.dev_mask[seq] == 0) continue;
#pragma unroll
        for (uint32_t q = 0; q < kMaxRanks; ++q) {
            if (q >= ranks) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[q][e];
        }
        finish_block<DT>(p, row, seq, n0, lane, v);
    }
    __syncwarp();
    __syncthreads();
    if (ranks > 1) cluster_sync();  // the others may still read this block's sums
    if (warp == kLoader) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kCols));
    }
}

template <int DT, int NR>
cudaError_t run_few(const Matmul8Params& p, int ranks, cudaStream_t stream) {
    if (encoder() == nullptr) return cudaErrorNotSupported;
    CUtensorMap a, w;
    if (!encode8(&a, p.a, p.k, p.m, p.a_stride, NR) || !encode8(&w, p.w, p.k, p.n, p.w_stride, kRows)) return cudaErrorNotSupported;
    constexpr int smem = sizeof(FewSmem<NR>);
    static_assert(2 * (smem + 1024) <= 233472, "two blocks to an SM");
    const auto kernel = matmul8_few_kernel<DT, NR>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (static_cast<int64_t>(p.n) + kRows - 1) / kRows * ((p.m + NR - 1) / NR);
    return launch_early(kernel, static_cast<unsigned>(tiles * ranks), static_cast<unsigned>(ranks), kFewThreads, smem, stream, p, a, w);
}

template <int DT>
cudaError_t dispatch_few(const Matmul8Params& p, const FewPlan& plan, cudaStream_t stream) {
    switch (plan.rows) {
        case 16: return run_few<DT, 16>(p, plan.ranks, stream);
        case 32: return run_few<DT, 32>(p, plan.ranks, stream);
        case 64: return run_few<DT, 64>(p, plan.ranks, stream);
        default: return run_few<DT, 128>(p, plan.ranks, stream);
    }
}

}  // namespace

cudaError_t launch_matmul8_few(const Matmul8Params& p, const FewPlan& plan, int dtype, cudaStream_t stream) {
    return dtype == SPECA_BF16 ? dispatch_few<SPECA_BF16>(p, plan, stream) : dispatch_few<SPECA_F32>(p, plan, stream);
}

}  // namespace speca
