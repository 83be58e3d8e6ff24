// Matrix products in 8 bits on the tensor cores: D = A W^T, e4m3 with a power of two as scale per row and 128 elements of k.
//
// The scales go with the operands into the tensor cores (block-scaled tcgen05.mma), so sums over all of k stay in tensor memory in
// fp32. A tile is 128 rows times CG by NT features; with CG = 2 the two SMs of a cluster share it: each holds its 128 rows of A, half of
// the rows of W and its half of the sums, which halves what every SM reads of W. Blocks are persistent over tiles:
//   warps 0-3, 4-7   epilogue of the left and the right half of the columns: one thread per row
//   warp 8           TMA loads of A and W, 128 elements of k a stage
//   warp 9           issues the products (of both SMs, in the first of them)
//   warps 12-15      scales: of 512 elements of k at once, through registers into every quarter of the lanes of tensor memory. (Copied there
//                    from shared memory by the tensor cores themselves they cost 270 cycles of every 2048: 8192 x 8192 x 4096 206 us, 188 without.)
// Sums alternate between two places in tensor memory, so that the epilogue of a tile runs beside the products of the next.
//
// What bounds it: a step of 128 elements of k is 512 cycles of the tensor pipe in a pair (256 x 256) and brings 32 KB into each SM, which takes as
// long (an SM got 90 to 110 GB/s from L2 in every shape tried, 50 to 58 bytes a cycle); tiles of one SM (128 x 128) read as much for half the
// products. Between tiles some 1300 cycles pass while the last sums are read. In a loop the card runs into its power limit (1000 W, 1.4 GHz).
// Measured, e4m3 with bf16 out, in a loop: 4096 x 4608 x 1152 22.9 us (1.90 PFLOP/s; a library's block-scaled product 23.3), 4096 x 1152 x 4608 26.8 (1.62;
// 28.0), 8352 x 14336 x 4096 399 (2.46; 390), 8192^3 422 (2.61; 470), 20928 x 16384 x 4096 1100 (2.55; 1277); 8352 x 14336 x 4096 in a short run 357 (2.74).
// Short k with an activation waits for the epilogue: 4096 x 4608 x 1152 in a graph 19.2 us into bf16, 20 into 8 bits, 22 with GELU into bf16, 27 to 29 with bias and GELU into
// 8 bits; what in it takes the time is not known (the special function unit is busy a quarter of it). Tried there and
// not kept: 16 epilogue warps in place of 8 (28.1 us), exponentials of one pair in 4, 3 or 2 by polynomial (28.3 to 28.9), what the next tile needs asked
// for a tile ahead (30.8 then, 30.1).
#include "speca_matmul8_tensor.cuh"

namespace speca {
namespace {

// Four warpgroups of 128 registers a thread at launch; the epilogue's two take 176, the others give up what they take: 2 x 176 + 2 x 80 = 4 x 128.
constexpr int kThreads = 512, kRegisters = 128;
constexpr int kLoadWarp = 8, kIssueWarp = 9, kScaleWarp = 12;
constexpr uint32_t kTmemCols = 512;
constexpr int kScaleCol = 480;                   // two stages of 16 columns: 4 for A's scales, up to 8 for W's
constexpr uint32_t kStageOut = 32 * 128;
constexpr int kMaxTilesM = 2048;                 // tiles of rows of one launch, listed in shared memory where there is a mask
constexpr int kGroupM = 16;                      // tiles of rows that run beside each other share their features in L2 (8: 3 % slower at large sizes)

template <int CG, int NT>
struct Shape {
    static constexpr int kTileM = kRows * CG;
    static constexpr int kRowsW = NT / CG;       // rows of W that one SM holds
    static constexpr uint32_t kBytesA = kRows * 128, kBytesW = kRowsW * 128, kStage = kBytesA + kBytesW;
    static constexpr int kPartsW = (NT + 127) / 128;
    static constexpr int kStages = 5;            // of 32 KB
    static_assert(kStage == 32768, "128 + 128 rows");
    static constexpr int kCols = NT / 2;         // columns of one epilogue thread
    static_assert(kCols == 64 || kCols == 128, "boxes of 64 or 128 codes");
    // place of the second sums: behind the first, or as far behind as the scales leave room
    static constexpr int kSecond = NT <= kScaleCol - NT ? NT : kScaleCol - NT;
    static constexpr bool kOverlap = kSecond < NT;
};

template <int CG, int NT>
struct Smem {
    using S = Shape<CG, NT>;
    uint8_t tiles[S::kStages][S::kStage];
    uint8_t out[8][kStageOut];   // of each epilogue warp: 32 rows on their way to memory
    float columns[8][2][S::kCols];  // of each epilogue warp: bias and gate of its columns
    uint64_t full[S::kStages], empty[S::kStages];
    uint64_t scales_full[2], scales_used[2];
    uint64_t sums_full[2], sums_free[2], overlap_free[2];
    uint64_t tops[2], drain;
    float top[2][2][kRows];
    uint32_t tmem, abort, n_live;
    uint32_t warp_count[kThreads / 32];
    uint16_t live[kMaxTilesM];
};

// ---- tiles --------------------------------------------------------------------------------------
struct Part {  // what one launch covers
    int m_begin, n_begin;   // first row, first feature
    int m_tiles, n_tiles;
};
struct Place {
    int m, n;  // first row (of the pair) and feature of a tile
};
template <int CG, int NT>
__device__ __forceinline__ Place place(const Part& part, const Smem<CG, NT>& sm, bool masked, int m_tiles, int i) {
    const int per = kGroupM * part.n_tiles, g = i / per, in = i - g * per;
    const int rows = min(kGroupM, m_tiles - g * kGroupM);
    int m = g * kGroupM + in % rows;
    if (masked) m = sm.live[m];
    return Place{part.m_begin + m * Shape<CG, NT>::kTileM, part.n_begin + in / rows * NT};
}
// Whether any row of the tile belongs to an active sequence.
__device__ __forceinline__ bool tile_live(const Matmul8Params& p, int first, int rows) {
    const int last = min(first + rows, p.m) - 1;
    for (int s = p.row_seq[first]; s <= p.row_seq[last]; ++s)
        if (p.dev_mask[s] != 0) return true;
    return false;
}

// ---- epilogue: a warp has 32 rows, one a lane, and takes 32 columns at a time ----
// What the output is: the sums after bias and activation in the layer's type; the same with gate and residual; 8 bits. Each has a kernel of its
// own: the epilogue's code has to stay in the instruction cache (one for all, unrolled over all columns, was three times as slow).
enum Epilogue { kPlain, kResidual, kEight };

// t / (1 + 2^x), two at a time with one reciprocal, 1 / a = b / (a b): the special function unit forms 16 a cycle, and is a quarter busy in a
// product with GELU (4096 x 4608 x 1152; with half of the exponentials as polynomials instead the product took as long). So that
// a b stays finite, also next to a NaN, x is held at 63, where the factor is 2^-63. A little more than that is taken off every factor and none goes below
// zero, so that from there on it is zero, whatever t (NaN of one that is not finite). (Choosing between factor and zero instead took 1.5 % longer.)
__device__ __forceinline__ float factor(float other, float r) {
    float f;
    asm("fma.rn.sat.f32 %0, %1, %2, %3;" : "=f"(f) : "f"(other), "f"(r), "f"(-0x1.0001p-63f));
    return f;
}
__device__ __forceinline__ uint64_t times_sigmoid2(uint64_t t, uint64_t x) {
    float x0, x1, d0, d1, r;
    unpair(x, x0, x1);
    unpair(add2(pair(ex2(fminf(x0, 63.f)), ex2(fminf(x1, 63.f))), pair(1.f, 1.f)), d0, d1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d0 * d1));
    return mul2(t, pair(factor(d1, r), factor(d0, r)));
}
__device__ __forceinline__ void activate32(float (&v)[32], int act) {
    if (act == SPECA_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const uint64_t t = pair(v[e], v[e + 1]);
            unpair(times_sigmoid2(t, mul2(t, fma2(mul2(t, t), pair(kGelu3, kGelu3), pair(kGelu1, kGelu1)))), v[e], v[e + 1]);
        }
    } else if (act == SPECA_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const uint64_t t = pair(v[e], v[e + 1]);
            unpair(times_sigmoid2(t, mul2(t, pair(kSilu1, kSilu1))), v[e], v[e + 1]);
        }
    }
}
// A warp's columns of a row of `n` elements (bias, gate) into its part of shared memory, zeros behind the last; every lane then reads them all.
template <typename T, int N>
__device__ __forceinline__ void stage_columns(float* to, const T* from, int c, int n, int lane) {
#pragma unroll
    for (int i = lane; i < N; i += 32) to[i] = c + i < n ? to_float(from[c + i]) : 0.f;
    __syncwarp();
}
__device__ __forceinline__ void add_columns(float (&v)[32], const float* x) {
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
        const float4 f = *reinterpret_cast<const float4*>(x + e);
        v[e] += f.x, v[e + 1] += f.y, v[e + 2] += f.z, v[e + 3] += f.w;
    }
}

// 32 elements of a lane's own row from column c on, as they lie in memory; zeros behind the last column.
template <typename T>
struct Cols {
    static constexpr int kWords = 8 * sizeof(T);
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const char* base, int64_t row, int64_t stride, int c, int n, bool vectors) {
        const T* from = reinterpret_cast<const T*>(base) + row * stride + c;
        if (vectors && c + 32 <= n) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(from) + i);
                w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            if (c + e >= n) continue;
            if constexpr (sizeof(T) == 4)
                w[e] = __float_as_uint(to_float(from[e]));
            else
                w[e / 2] |= static_cast<uint32_t>(__bfloat16_as_ushort(from[e])) << (e % 2 * 16);
        }
    }
    __device__ __forceinline__ float at(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
};
// 32 columns of a row in the output's type, as they lie in memory.
template <typename T>
__device__ __forceinline__ void pack_row(const float (&v)[32], uint32_t (&w)[8 * sizeof(T)]) {
#pragma unroll
    for (int e = 0; e < static_cast<int>(8 * sizeof(T)); ++e) {
        if constexpr (sizeof(T) == 2)
            w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        else
            w[e] = __float_as_uint(v[e]);
    }
}

// Boxes: 32 rows of PITCH bytes in shared memory, with the swizzle of that width.
template <int PITCH>
__device__ __forceinline__ uint32_t box_piece(int row, int piece) {
    static_assert(PITCH == 64 || PITCH == 128, "a swizzle of this width");
    return row * PITCH + (piece ^ (PITCH == 128 ? row % 8 : row / 2 % 4)) * 16;
}

// N words of this lane's row, from 16-byte piece `first` on.
template <int PITCH, int N>
__device__ __forceinline__ void stage_row(uint8_t* box, int lane, int first, const uint32_t (&w)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
        *reinterpret_cast<uint4*>(box + box_piece<PITCH>(lane, first + i / 4)) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
}
// What the warp staged goes out, row by row.
template <typename T, int PITCH>
__device__ __forceinline__ void write_box(const uint8_t* box, T* out, int64_t stride, int c, int n, int row0, uint32_t live, int lane) {
    constexpr int kBoxCols = PITCH / static_cast<int>(sizeof(T));
    __syncwarp();
#pragma unroll 1
    for (int e = lane; e < kBoxCols && c < n; e += 32) {
        const int byte = e * sizeof(T);
        T* to = out + static_cast<int64_t>(row0) * stride + c + e;
        constexpr int kAtOnce = 8;  // rows
#pragma unroll 1
        for (int r = 0; r < 32; r += kAtOnce) {
            T v[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) v[u] = *reinterpret_cast<const T*>(box + box_piece<PITCH>(r + u, byte / 16) + byte % 16);
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                if ((live >> (r + u) & 1) != 0 && c + e < n) to[(r + u) * stride] = v[u];
        }
    }
    __syncwarp();
}
// The same by the copy engine, all rows together. It leaves out what lies behind the last row, and behind the last column in pieces of 16 bytes
// (what follows a last piece that is cut was overwritten with zeros): so not where it cannot address the output, where a row is not to be written or
// the last piece is cut.
template <typename T>
__device__ __forceinline__ void send_box(const CUtensorMap* map, bool boxed, const uint8_t* box, T* out, int64_t stride, int c, int n, int row0,
                                         uint32_t live, int lane) {
    constexpr int kBoxCols = 128 / static_cast<int>(sizeof(T)), kPiece = 16 / static_cast<int>(sizeof(T));
    if (!boxed || (c + kBoxCols > n && n % kPiece != 0)) return write_box<T, 128>(box, out, stride, c, n, row0, live, lane);
    if (c >= n) return;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(c), "r"(row0), "r"(smem_u32(box))
                     : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}
// The box has been read out of shared memory.
__device__ __forceinline__ void box_read(int lane) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
}

// 32 bytes at once (a whole sector) where rows start on 32.
__device__ __forceinline__ void store32(uint8_t* to, const uint32_t (&w)[8], bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                     "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// Largest finite magnitude of a lane's 32 values; infinities become NaN.
__device__ __forceinline__ float row_top(float (&v)[32]) {
    const float inf = __uint_as_float(0x7f800000u);
    float top[4] = {};
#pragma unroll
    for (int i = 0; i < 32; ++i) top[i % 4] = fmaxf(top[i % 4], fabsf(v[i]));
    float all = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    if (__any_sync(0xffffffffu, all == inf)) {
        all = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (fabsf(v[i]) == inf) v[i] = __uint_as_float(0x7fffffffu);
            all = fmaxf(all, fabsf(v[i]));
        }
    }
    return all;
}

__device__ __forceinline__ void pack_codes(const float (&v)[32], float inv, uint32_t (&w)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = pack_e4m3(v[4 * k] * inv, v[4 * k + 1] * inv, v[4 * k + 2] * inv, v[4 * k + 3] * inv);
}

// ---- the kernel ---------------------------------------------------------------------------------
template <int DT, int CG, int NT, Epilogue E>
__global__ void __cluster_dims__(CG, 1, 1) __launch_bounds__(kThreads, 1)
    matmul8_tc_kernel(const __grid_constant__ Matmul8Params p, const __grid_constant__ Part part, const __grid_constant__ CUtensorMap map_a,
                      const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_out) {
    using S = Shape<CG, NT>;
    using T = typename Type<DT>::T;
    extern __shared__ __align__(1024) char raw[];
    Smem<CG, NT>& sm = *reinterpret_cast<Smem<CG, NT>*>(raw);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = CG == 1 ? 0 : cluster_rank();
    const bool masked = p.dev_mask != nullptr;

    if (smem_u32(raw) % 1024 != 0) {  // the swizzled tiles rely on it; the same in both SMs
        if (threadIdx.x == 0) atomicExch(p.gave_up, 1u);
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            bar_init(&sm.full[i], 1);
            bar_init(&sm.empty[i], 1);
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(&sm.scales_full[b], 4 * CG);   // one arrival per warp
            bar_init(&sm.scales_used[b], 1);
            bar_init(&sm.sums_full[b], 1);
            bar_init(&sm.sums_free[b], 8 * CG);     // one arrival per warp
            bar_init(&sm.overlap_free[b], 4 * CG);
            bar_init(&sm.tops[b], 8);
        }
        bar_init(&sm.drain, 1);
        sm.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fetch_map(&map_a);
        fetch_map(&map_w);
    }
    wait_for_stream();
    if (warp == kLoadWarp) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        }
    }
    // the tiles of rows that hold an active sequence, in order
    int m_tiles = part.m_tiles;
    if (masked) {
        m_tiles = 0;
        for (int first = 0; first < part.m_tiles; first += kThreads) {
            const int i = first + threadIdx.x;
            const bool live = i < part.m_tiles && tile_live(p, part.m_begin + i * S::kTileM, S::kTileM);
            const uint32_t votes = __ballot_sync(0xffffffffu, live);
            if (lane == 0) sm.warp_count[warp] = __popc(votes);
            __syncthreads();
            int before = m_tiles, all = 0;
            for (int k = 0; k < kThreads / 32; ++k) {
                const int n = sm.warp_count[k];
                if (k < warp) before += n;
                all += n;
            }
            if (live) sm.live[before + __popc(votes & ((1u << lane) - 1))] = static_cast<uint16_t>(i);
            m_tiles += all;
            __syncthreads();
        }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();  // the other SM's barriers are there
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sm.tmem);
    const int n_tiles = m_tiles * part.n_tiles, first_tile = blockIdx.x / CG, step = gridDim.x / CG;
    const int k_blocks = (p.k + kBlock8 - 1) / kBlock8;

    if (warp >= kLoadWarp) fewer_registers<80>();
    if (warp == kLoadWarp) {
        // ---- loads: one thread ----
        if (lane == 0) {
            int stage = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int i = first_tile; i < n_tiles && ok; i += step) {
                const Place at = place<CG, NT>(part, sm, masked, m_tiles, i);
                for (int k = 0; k < k_blocks; ++k) {
                    ok = bar_wait(&sm.empty[stage], phase ^ 1);
                    if (!ok) break;
                    if (rank == 0) bar_expect(&sm.full[stage], CG * S::kStage);
                    const uint32_t bar = leaders<CG>(&sm.full[stage]), to = smem_u32(sm.tiles[stage]);
                    load_tile<CG>(to, &map_a, k * kBlock8, at.m + rank * kRows, bar);
                    load_tile<CG>(to + S::kBytesA, &map_w, k * kBlock8, at.n + rank * S::kRowsW, bar);
                    if (++stage == S::kStages) stage = 0, phase ^= 1;
                }
            }
            if (!ok) sm.abort = 1;
            // Copies in flight, those of both SMs, must land before the block gives its shared memory back, also where another warp's wait ran out. The second
            // SM, which cannot wait for the first one's barriers, leaves no sooner than that one does.
            if (rank == 0)
                for (int i = 0; i < S::kStages; ++i) bar_wait(&sm.full[i], i < stage ? phase : phase ^ 1);
            else if (!ok)
                for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
    } else if (warp == kIssueWarp) {
        // ---- products: one thread of the first SM. It looks for the next stage before it issues this one's: a wait that is
        // already satisfied takes some 200 cycles to say so, and a stage's products take 512. ----
        if (rank == 0 && elect_one()) {
            Turn<S::kStages> at;
            Turn<2> held, sums_at;  // scales, sums
            uint32_t overlap_phase[2] = {0, 0};
            bool ok = true, ready = false;
            for (int i = first_tile; i < n_tiles && ok; i += step) {
                const int b = sums_at.stage;
                ok = pair_wait<CG>(&sm.sums_free[b], sums_at.phase ^ 1);
                if (S::kOverlap && i != first_tile && ok) {
                    ok = pair_wait<CG>(&sm.overlap_free[b ^ 1], overlap_phase[b ^ 1]);
                    overlap_phase[b ^ 1] ^= 1;
                }
                const uint32_t sums = tmem + b * S::kSecond;
                for (int k = 0; k < k_blocks && ok; ++k) {
                    if (k % 4 == 0) ok = pair_wait<CG>(&sm.scales_full[held.stage], held.phase);
                    ok = ok && (ready || pair_wait<CG>(&sm.full[at.stage], at.phase));
                    if (!ok) break;
                    const int stage = at.stage;
                    at.next();
                    ready = pair_test<CG>(&sm.full[at.stage], at.phase);
                    tc_fence_after();
                    const uint32_t from = smem_u32(sm.tiles[stage]), scales = tmem + kScaleCol + held.stage * 16;
                    const uint64_t a = tile_desc(from), w = tile_desc(from + S::kBytesA);
                    const uint32_t desc = mma_desc8<CG, NT>(0) | static_cast<uint32_t>(k % 4) << 4 | static_cast<uint32_t>(k % 4) << 29;
#pragma unroll
                    for (int s = 0; s < 4; ++s) mma8<CG>(sums, a + 2 * s, w + 2 * s, desc, scales, scales + 4, k > 0 || s > 0);
                    commit<CG>(&sm.empty[stage]);
                    if (k % 4 == 3 || k + 1 == k_blocks) {
                        commit<CG>(&sm.scales_used[held.stage]);
                        held.next();
                    }
                    if (k + 1 == k_blocks) commit<CG>(&sm.sums_full[b]);
                }
                sums_at.next();
            }
            if (!ok) {
                sm.abort = 1;
                commit<CG>(&sm.drain);  // products in flight must end before tensor memory is given back
                bar_wait(&sm.drain, 0);
            }
        }
        __syncwarp();
    } else if (warp >= kScaleWarp) {
        // ---- scales: lane i takes rows i, 32 + i, ... of a part of 128 rows, each warp for its quarter of the lanes. Those of the next group
        // are on their way from memory while this one waits for room ----
        Turn<2> to;
        uint32_t word[4 * (1 + S::kPartsW)];
        int tile = first_tile, k = 0;
        Place at{0, 0};
        auto fetch = [&] {
            const int a0 = at.m + rank * kRows + lane, w0 = at.n + lane;
#pragma unroll
            for (int j = 0; j < 4; ++j) word[j] = scale_word(p.a_scales, p.a_scale_stride, k / 4, a0 + 32 * j, p.m);
#pragma unroll
            for (int j = 0; j < 4 * S::kPartsW; ++j) word[4 + j] = scale_word(p.w_scales, p.w_scale_stride, k / 4, w0 + 32 * j, p.n);
        };
        bool ok = true;
        if (tile < n_tiles) {
            at = place<CG, NT>(part, sm, masked, m_tiles, tile);
            fetch();
        }
        const uint32_t first = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16) + kScaleCol;
        while (tile < n_tiles) {
            ok = pair_warp_wait<CG>(&sm.scales_used[to.stage], to.phase ^ 1);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int q = 0; q < 1 + S::kPartsW; ++q) tmem_store4(first + to.stage * 16 + 4 * q, word + 4 * q);
            tmem_wait_store();
            hand_over<CG>(&sm.scales_full[to.stage], lane);
            to.next();
            k += 4;
            if (k >= k_blocks) {
                k = 0;
                tile += step;
                if (tile < n_tiles) at = place<CG, NT>(part, sm, masked, m_tiles, tile);
            }
            if (tile < n_tiles) fetch();
        }
        if (!ok) sm.abort = 1;
    } else if (warp < kLoadWarp) {
        // ---- epilogue ----
        more_registers<176>();
        const int half = warp / 4, r = threadIdx.x % 128;
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        int b = 0;
        uint32_t phase = 0;
        bool ok = true;
        uint8_t* const box = sm.out[warp];
        for (int i = first_tile; i < n_tiles; i += step) {
            const Place at = place<CG, NT>(part, sm, masked, m_tiles, i);
            const int row = at.m + rank * kRows + r, row0 = row - lane, n0 = at.n + half * S::kCols;
            bool live = row < p.m;
            int seq = 0;
            if (live && (masked || E == kResidual)) {
                seq = p.row_seq[row];
                live = !masked || p.dev_mask[seq] != 0;
            }
            const uint32_t lives = __ballot_sync(0xffffffffu, live);
            const bool boxed = p.boxes && lives == __ballot_sync(0xffffffffu, row < p.m) && lives != 0;
            // First the columns that the next tile's sums will take: the last of the first place, the first of the second.
            constexpr int kChunks = S::kCols / 32;
            const bool backwards = S::kOverlap && half == 1 && b == 0;
            const uint32_t from = tmem + lanes + b * S::kSecond + half * S::kCols;
            auto chunk = [&](int j) { return 32 * (backwards ? kChunks - 1 - j : j); };
            auto load_chunk = [&](int j, float (&v)[32]) {
                uint32_t bits[32];
                tmem_load32(from + chunk(j), bits);
                tmem_wait_load<32>(bits);
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(bits[e]);
            };
            // before the sums are there: bias, gate (of a warp whose rows belong to one sequence), the residual of the first chunk
            __syncwarp();
            if (p.bias != nullptr) stage_columns<T, S::kCols>(sm.columns[warp][0], reinterpret_cast<const T*>(p.bias), n0, p.n, lane);
            bool one_gate = false;
            Cols<T> residual;
            auto ask = [&](int j) {
                if (p.residual != nullptr && live) residual.load(p.residual, row, p.residual_stride, n0 + chunk(j), p.n, p.vectors);
            };
            if constexpr (E == kResidual) {
                const int s = __shfl_sync(0xffffffffu, seq, lives == 0 ? 0 : __ffs(lives) - 1);
                one_gate = p.gate != nullptr && __all_sync(0xffffffffu, !live || seq == s);
                if (one_gate) stage_columns<T, S::kCols>(sm.columns[warp][1], reinterpret_cast<const T*>(p.gate) + s * p.gate_stride, n0, p.n, lane);
                ask(0);
            }
            ok = pair_warp_wait<CG>(&sm.sums_full[b], phase);
            if (!ok) break;
            tc_fence_after();
            [[maybe_unused]] float held[32], top = 0.f;
#pragma unroll 1
            for (int j = 0; j < kChunks; ++j) {
                const int c = n0 + chunk(j);
                float v[32];
                load_chunk(j, v);
                if (S::kOverlap && j == 0 && half != b) hand_over<CG>(&sm.overlap_free[b], lane);
                if (E != kEight && j == kChunks - 1) hand_over<CG>(&sm.sums_free[b], lane);
                if (p.bias != nullptr) add_columns(v, sm.columns[warp][0] + chunk(j));
                activate32(v, p.act);
                if constexpr (E == kEight) {
                    top = fmaxf(top, row_top(v));
                    // the first stay here, the others wait for the scale where their sums were
                    if (j == 0) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) held[e] = v[e];
                    } else {
                        uint32_t bits[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) bits[e] = __float_as_uint(v[e]);
                        tmem_store32(from + chunk(j), bits);
                    }
                } else {
                    if constexpr (E == kResidual) {
                        if (one_gate) {
                            const float* g = sm.columns[warp][1] + chunk(j);
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                const float4 f = *reinterpret_cast<const float4*>(g + e);
                                v[e] *= f.x, v[e + 1] *= f.y, v[e + 2] *= f.z, v[e + 3] *= f.w;
                            }
                        } else if (p.gate != nullptr && live) {
                            Cols<T> gate;
                            gate.load(p.gate, seq, p.gate_stride, c, p.n, p.vectors);
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] *= gate.at(e);
                        }
                        if (p.residual != nullptr && live) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] += residual.at(e);
                        }
                        if (j + 1 < kChunks) ask(j + 1);
                    }
                    // a box holds 128 bytes a row: one or two chunks
                    constexpr int kPer = 4 / sizeof(T);
                    uint32_t w[8 * sizeof(T)];
                    pack_row<T>(v, w);
                    if (j % kPer == 0) box_read(lane);
                    stage_row<128>(box, lane, chunk(j) / 32 % kPer * 4, w);
                    if (j % kPer == kPer - 1)
                        send_box<T>(&map_out, boxed, box, reinterpret_cast<T*>(p.out), p.out_stride, n0 + chunk(j) / (32 * kPer) * (32 * kPer), p.n,
                                         row0, lives, lane);
                }
            }
            if constexpr (E == kEight) {
                tmem_wait_store();
                if constexpr (S::kCols == 64) {  // a block of 128 columns lies in two threads
                    sm.top[b][half][r] = top;
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sm.tops[b]);
                    ok = warp_wait(&sm.tops[b], phase);
                    if (!ok) break;
                    top = fmaxf(top, sm.top[b][half ^ 1][r]);
                }
                const uint32_t byte = scale_byte(top);
                const float inv = inverse_of(byte);
                if (live && n0 % kBlock8 == 0 && n0 < p.n)
                    p.out8.scales[n0 / (4 * kBlock8) * p.out8.scale_stride + 4 * static_cast<int64_t>(row) + n0 / kBlock8 % 4] =
                        static_cast<uint8_t>(byte);
                // each lane writes its row's codes, 32 bytes at once; where it cannot, through the box, row by row. (Through the copy engine, whose fence
                // waits some hundred cycles, 8192 x 8192 x 1152 with GELU took 107 us, 101 so.)
                const bool direct = p.vectors && n0 + S::kCols <= p.n;
#pragma unroll 1
                for (int j = 0; j < kChunks; ++j) {
                    if (j > 0) load_chunk(j, held);
                    if (j == kChunks - 1) hand_over<CG>(&sm.sums_free[b], lane);
                    uint32_t w[8];
                    pack_codes(held, inv, w);
                    if (!direct)
                        stage_row<S::kCols>(box, lane, chunk(j) / 16, w);
                    else if (live)
                        store32(p.out8.codes + row * p.out8.code_stride + n0 + chunk(j), w, p.wide);
                }
                if (!direct) write_box<uint8_t, S::kCols>(box, p.out8.codes, p.out8.code_stride, n0, p.n, row0, lives, lane);
            }
            if (b == 1) phase ^= 1;
            b ^= 1;
        }
        if (!ok) sm.abort = 1;
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(&sm.abort) != 0) atomicExch(p.gave_up, 1u);
    if constexpr (CG == 2) cluster_sync();  // the other SM may still read, or arrive at, what this one holds
    if (warp == kLoadWarp) {
        tc_fence_after();
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
    }
}

// An output in the layer's type as boxes of 32 rows of 128 bytes.
bool encode_out(CUtensorMap* map, const Matmul8Params& p, int elem) {
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(p.n), static_cast<cuuint64_t>(p.m)};
    const cuuint64_t strides[1] = {p.m > 1 ? static_cast<cuuint64_t>(p.out_stride) * elem : 128};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(128 / elem), 32}, ones[2] = {1, 1};
    return encoder()(map, elem == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, p.out, dims, strides, box, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DT, int CG, int NT>
cudaError_t run(Matmul8Params p, int sm_count, cudaStream_t stream) {
    using S = Shape<CG, NT>;
    if (encoder() == nullptr) return cudaErrorNotSupported;
    CUtensorMap a, w, out = {};
    if (!encode8(&a, p.a, p.k, p.m, p.a_stride, kRows) || !encode8(&w, p.w, p.k, p.n, p.w_stride, S::kRowsW)) return cudaErrorNotSupported;
    p.boxes = p.vectors && p.out != nullptr && encode_out(&out, p, Type<DT>::kBytes);
    constexpr uint32_t smem = sizeof(Smem<CG, NT>);
    static_assert(smem <= 232448 && smem > 116224, "fits one SM, and no two blocks share one (tensor memory)");
    const auto kernel = p.out == nullptr                                  ? matmul8_tc_kernel<DT, CG, NT, kEight>
                        : p.residual != nullptr || p.gate != nullptr ? matmul8_tc_kernel<DT, CG, NT, kResidual>
                                                                     : matmul8_tc_kernel<DT, CG, NT, kPlain>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    // the warps' shares of the registers rely on what the kernel was built with: with fewer they would wait for ever
    cudaFuncAttributes attr;
    static const bool built[3] = {cudaFuncGetAttributes(&attr, matmul8_tc_kernel<DT, CG, NT, kEight>) == cudaSuccess && attr.numRegs >= kRegisters,
                                  cudaFuncGetAttributes(&attr, matmul8_tc_kernel<DT, CG, NT, kResidual>) == cudaSuccess && attr.numRegs >= kRegisters,
                                  cudaFuncGetAttributes(&attr, matmul8_tc_kernel<DT, CG, NT, kPlain>) == cudaSuccess && attr.numRegs >= kRegisters};
    if (!built[0] || !built[1] || !built[2]) return cudaErrorInvalidKernelImage;
    // parts: what the list of tiles holds, and what counts in 32 bits
    constexpr int64_t kMaxN = int64_t(1) << 18;
    for (int64_t m0 = 0; m0 < p.m; m0 += int64_t(kMaxTilesM) * S::kTileM)
        for (int64_t n0 = 0; n0 < p.n; n0 += kMaxN * NT) {
            Part part;
            part.m_begin = static_cast<int>(m0);
            part.n_begin = static_cast<int>(n0);
            part.m_tiles = static_cast<int>((min(p.m - m0, int64_t(kMaxTilesM) * S::kTileM) + S::kTileM - 1) / S::kTileM);
            part.n_tiles = static_cast<int>((min(p.n - n0, kMaxN * NT) + NT - 1) / NT);
            const int64_t tiles = static_cast<int64_t>(part.m_tiles) * part.n_tiles;
            const int blocks = static_cast<int>(min(tiles, static_cast<int64_t>(sm_count / CG))) * CG;
            e = launch_early(kernel, static_cast<unsigned>(blocks), CG, kThreads, smem, stream, p, part, a, w, out);
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

template <int DT>
cudaError_t dispatch(const Matmul8Params& p, Matmul8Kernel kind, int sm_count, cudaStream_t stream) {
    return kind == kOne ? run<DT, 1, 128>(p, sm_count, stream) : run<DT, 2, 256>(p, sm_count, stream);
}

}  // namespace

cudaError_t launch_matmul8(const Matmul8Params& p, int dtype, int sm_count, cudaStream_t stream) {
    if (p.m == 0) return cudaSuccess;
    const Matmul8Plan plan = plan_matmul8(p, dtype, sm_count);
    if (plan.kernel == kFew) return launch_matmul8_few(p, plan.few, dtype, stream);
    return dtype == SPECA_BF16 ? dispatch<SPECA_BF16>(p, plan.kernel, sm_count, stream) : dispatch<SPECA_F32>(p, plan.kernel, sm_count, stream);
}

}  // namespace speca
