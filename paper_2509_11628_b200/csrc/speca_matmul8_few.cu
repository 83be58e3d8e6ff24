// Matrix products in 8 bits for few rows (single tokens): bound by reading the weights once.
//
// A block has 128 features, 16 for each of its 8 warps, and a share of k; the shares of a cluster's blocks are added up through distributed
// shared memory, in the order of their ranks. A ninth warp keeps a ring of stages filled by the copy engine: 128 elements of k of the weights
// and of the rows. (Loads ahead into registers were spilled: 18 us for 6144 x 4096 weights.) Products by mma.sync, 8 rows of A at a
// time: the order of k inside a product is free, so a lane takes the 32 bytes that it reads at once as the operands come, the same of both.
// Sums of 128 products in the tensor cores, then times both scales into the fp32 sum. Every wait is bounded, as in the kernel for many rows.
#include "speca_matmul8_common.cuh"

namespace speca {
namespace {

constexpr int kFewThreads = 288, kFeatures = 128;
constexpr uint32_t kBytesW = kFeatures * 128;
constexpr int kNan = 1 << 20;              // exponent of a scale that is NaN

// NB: rows in eights. Two blocks share an SM.
template <int NB>
struct FewShape {
    static constexpr uint32_t kStage = kBytesW + NB * 1024;
    static constexpr int kStages = NB == 1 ? 6 : NB <= 4 ? 5 : 4;
};
template <int NB>
struct FewSmem {
    uint8_t tiles[FewShape<NB>::kStages][FewShape<NB>::kStage];
    uint64_t full[FewShape<NB>::kStages], empty[FewShape<NB>::kStages];
    uint32_t abort;
};

__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// x * 2^(ea + eb - 254) of two scale bytes, in two steps so that nothing in between leaves the range.
__device__ __forceinline__ float scaled(float x, int ea, int eb) {
    const int e = min(max(ea + eb, 2), 506), h = e >> 1;
    const float y = x * __uint_as_float(static_cast<uint32_t>(h) << 23) * __uint_as_float(static_cast<uint32_t>(e - h) << 23);
    return ea + eb >= kNan ? __uint_as_float(0x7fffffffu) : y;
}
__device__ __forceinline__ int exponent(uint32_t byte) { return byte == 255 ? kNan : static_cast<int>(byte); }

__device__ __forceinline__ uint32_t block_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_blocks() {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}
__device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar))
                 : "memory");
}
// 16-byte piece of a row of a tile, where the 128-byte swizzle put it.
__device__ __forceinline__ uint4 piece(const uint8_t* tile, int row, int i) {
    return *reinterpret_cast<const uint4*>(tile + row * 128 + (i ^ (row % 8)) * 16);
}
// Scales of four blocks of a row; those of rows that do not exist: 1.
__device__ __forceinline__ uint32_t scale_word(const uint8_t* scales, int64_t stride, int group, int row, int rows) {
    return row < rows ? __ldg(reinterpret_cast<const uint32_t*>(scales + group * stride) + row) : 0x7f7f7f7fu;
}

template <int DT, int NB>
__global__ void __launch_bounds__(kFewThreads, 2)
    matmul8_few_kernel(const __grid_constant__ Matmul8Params p, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w) {
    using S = FewShape<NB>;
    extern __shared__ __align__(1024) char raw[];
    FewSmem<NB>& sm = *reinterpret_cast<FewSmem<NB>*>(raw);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const uint32_t rank = block_rank(), ranks = cluster_blocks();
    if (smem_u32(raw) % 1024 != 0) {  // the swizzled tiles rely on it; the same in every block
        if (threadIdx.x == 0) atomicExch(p.gave_up, 1u);
        return;
    }
    if (p.dev_mask != nullptr) {  // the same in every block of the cluster
        bool live = false;
        for (int r = lane; r < p.m; r += 32) live = live || p.dev_mask[p.row_seq[r]] != 0;
        if (!__any_sync(0xffffffffu, live)) return;
    }
    const int k_blocks = (p.k + kBlock8 - 1) / kBlock8, share = (k_blocks + ranks - 1) / ranks;
    const int begin = min(static_cast<int>(rank) * share, k_blocks), end = min(begin + share, k_blocks);
    const int n0 = blockIdx.x / ranks * kFeatures;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            bar_init(&sm.full[i], 1);
            bar_init(&sm.empty[i], 8);  // one arrival per warp
        }
        sm.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();

    float acc[NB][4] = {};
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    if (warp == 8) {
        if (lane == 0) {
            for (int kb = begin; kb < end; ++kb) {
                ok = bar_wait(&sm.empty[stage], phase ^ 1);
                if (!ok) break;
                bar_expect(&sm.full[stage], S::kStage);
                const uint32_t to = smem_u32(sm.tiles[stage]);
                load_box(to, &map_w, kb * kBlock8, n0, &sm.full[stage]);
                load_box(to + kBytesW, &map_a, kb * kBlock8, 0, &sm.full[stage]);
                if (++stage == S::kStages) stage = 0, phase ^= 1;
            }
            if (!ok) {
                sm.abort = 1;
                // copies in flight must land before the block gives its shared memory back
                for (int i = 0; i < S::kStages; ++i) bar_wait(&sm.full[i], i < stage ? phase : phase ^ 1);
            }
        }
    } else {
        const int f0 = n0 + warp * 16 + g;
        uint32_t w_next[2], a_next[NB][2];
        auto fetch = [&](int group) {
            if (group * 4 >= end) return;
            w_next[0] = scale_word(p.w_scales, p.w_scale_stride, group, f0, p.n);
            w_next[1] = scale_word(p.w_scales, p.w_scale_stride, group, f0 + 8, p.n);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                a_next[j][0] = scale_word(p.a_scales, p.a_scale_stride, group, j * 8 + 2 * t, p.m);
                a_next[j][1] = scale_word(p.a_scales, p.a_scale_stride, group, j * 8 + 2 * t + 1, p.m);
            }
        };
        fetch(begin / 4);
        uint32_t w_scale[2] = {}, a_scale[NB][2] = {};
        for (int kb = begin; kb < end; ++kb) {
            if (kb == begin || kb % 4 == 0) {
                w_scale[0] = w_next[0], w_scale[1] = w_next[1];
#pragma unroll
                for (int j = 0; j < NB; ++j) a_scale[j][0] = a_next[j][0], a_scale[j][1] = a_next[j][1];
                fetch(kb / 4 + 1);
            }
            ok = warp_wait(&sm.full[stage], phase);
            if (!ok) break;
            const uint8_t *w = sm.tiles[stage], *a = w + kBytesW;
            const uint4 a0 = piece(w, warp * 16 + g, 2 * t), a1 = piece(w, warp * 16 + g + 8, 2 * t);
            const uint4 a2 = piece(w, warp * 16 + g, 2 * t + 1), a3 = piece(w, warp * 16 + g + 8, 2 * t + 1);
            float part[NB][4];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const uint4 x = piece(a, j * 8 + g, 2 * t), y = piece(a, j * 8 + g, 2 * t + 1);
#pragma unroll
                for (int e = 0; e < 4; ++e) part[j][e] = 0.f;
                mma_e4m3(part[j], a0.x, a1.x, a0.y, a1.y, x.x, x.y);
                mma_e4m3(part[j], a0.z, a1.z, a0.w, a1.w, x.z, x.w);
                mma_e4m3(part[j], a2.x, a3.x, a2.y, a3.y, y.x, y.y);
                mma_e4m3(part[j], a2.z, a3.z, a2.w, a3.w, y.z, y.w);
            }
            __syncwarp();
            if (lane == 0) bar_arrive(&sm.empty[stage]);
            if (++stage == S::kStages) stage = 0, phase ^= 1;
            const int shift = kb % 4 * 8;
            const int e0 = exponent(w_scale[0] >> shift & 255), e1 = exponent(w_scale[1] >> shift & 255);
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int ex = exponent(a_scale[j][0] >> shift & 255), ey = exponent(a_scale[j][1] >> shift & 255);
                acc[j][0] += scaled(part[j][0], e0, ex);
                acc[j][1] += scaled(part[j][1], e0, ey);
                acc[j][2] += scaled(part[j][2], e1, ex);
                acc[j][3] += scaled(part[j][3], e1, ey);
            }
        }
        if (!ok) sm.abort = 1;
    }
    __syncwarp();
    __syncthreads();
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(&sm.abort) != 0) atomicExch(p.gave_up, 1u);
    float* const sums = reinterpret_cast<float*>(raw);  // [8 NB][128], where the tiles were: all of them have been read
    static_assert(8 * NB * kFeatures * 4 <= sizeof(sm.tiles), "room");
    if (warp < 8) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[(j * 8 + 2 * t + i % 2) * kFeatures + warp * 16 + g + 8 * (i / 2)] = acc[j][i];
    }
    __syncthreads();
    cluster_wait();
    // a row for each warp of the cluster in turn: the shares in the order of their ranks
    for (int r = warp < 8 ? rank + ranks * warp : p.m; r < p.m; r += ranks * 8) {
        const int seq = p.row_seq[r];
        if (p.dev_mask != nullptr && p.dev_mask[seq] == 0) continue;
        const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(sums + r * kFeatures + 4 * lane));
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (uint32_t q = 0; q < ranks; ++q) {
            uint32_t there;
            float x[4];
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(q));
            asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(there) : "memory");
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[e];
        }
        finish_block<DT>(p, r, seq, n0, lane, v);
    }
    __syncwarp();
    __syncthreads();
    cluster_wait();  // the others may still read this block's sums
}

template <int DT, int NB>
cudaError_t run_few(const Matmul8Params& p, int sm_count, cudaStream_t stream) {
    if (encoder() == nullptr) return cudaErrorNotSupported;
    CUtensorMap a, w;
    if (!encode8(&a, p.a, p.k, p.m, p.a_stride, 8 * NB) || !encode8(&w, p.w, p.k, p.n, p.w_stride, kFeatures)) return cudaErrorNotSupported;
    constexpr int smem = sizeof(FewSmem<NB>);
    static_assert(2 * (smem + 1024) <= 233472, "two blocks to an SM");
    const auto kernel = matmul8_few_kernel<DT, NB>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    const int64_t blocks = (static_cast<int64_t>(p.n) + kFeatures - 1) / kFeatures;
    const int k_blocks = (p.k + kBlock8 - 1) / kBlock8;
    // shares of k: as many as let all blocks run at once, two to an SM, each with two stages at least
    const int ranks = static_cast<int>(max(int64_t(1), min(min(int64_t(8), 2 * sm_count / blocks), static_cast<int64_t>(k_blocks / 2))));
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(blocks * ranks));
    config.blockDim = dim3(kFewThreads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(ranks);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, p, a, w);
}

template <int DT>
cudaError_t dispatch_few(const Matmul8Params& p, int sm_count, cudaStream_t stream) {
    if (p.m <= 8) return run_few<DT, 1>(p, sm_count, stream);
    if (p.m <= 16) return run_few<DT, 2>(p, sm_count, stream);
    if (p.m <= 32) return run_few<DT, 4>(p, sm_count, stream);
    return run_few<DT, 8>(p, sm_count, stream);
}

}  // namespace

cudaError_t launch_matmul8_few(const Matmul8Params& p, int dtype, int sm_count, cudaStream_t stream) {
    return dtype == SPECA_BF16 ? dispatch_few<SPECA_BF16>(p, sm_count, stream) : dispatch_few<SPECA_F32>(p, sm_count, stream);
}

}  // namespace speca
