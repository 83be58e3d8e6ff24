// Attention of the verification layer in bf16, on the tensor cores (tcgen05, TMA).
//
// A block of 128 packed query rows against tiles of 128 keys: S = Q K^T (fp32, tensor memory), running maximum
// and sum of exp2(scale S - max) per row, P rounded to bf16 back into tensor memory over S, O += P V. A unit
// is two such blocks, which share the K and V tiles and take turns on the tensor cores: while one block's
// products run, the other's exponentials are formed. One unit at a time per SM, blocks persistent over units:
//   warps 0-3, 4-7   softmax and output of block 0 and block 1: one thread per row, its 128 scores in registers
//   warp 8           TMA loads: Q of the unit, then K_0, V_0, K_1, V_1, ... through a ring of tiles
//   warp 9           issues the products (warps 10 and 11 complete the warpgroup)
// Products of one thread run in the order of issue, so S_b(j+1) may overwrite P_b(j) right behind the product
// that reads it, and S_b(j+1) being ready says that O_b is at rest: the softmax threads themselves rescale O in the
// rare tile that raises a row's maximum by more than 2^8 (sums and P are exact to a common factor; it keeps
// P <= 2^8, far inside bf16's range).
// Every wait is bounded. A wait that runs out sets the layer's gave-up flag and ends the block's work.
#include <cuda.h>

#include "speca_attention_common.cuh"

namespace speca {
namespace {

// Three warpgroups of 168 registers a thread at launch; the two that form the softmax take 216 (a row of 128 scores
// and its packed weights stay in registers), the one that loads and issues gives up what they take: 2 x 216 + 72 = 3 x 168.
constexpr int kTcThreads = 384;
constexpr int kBlockRows = 128;
constexpr int kTileKeys = 128;
constexpr uint32_t kPanelBytes = 128 * 128;  // 128 rows of 64 bf16: one 128-byte swizzle span per row
constexpr uint32_t kSpinLimit = 1u << 20;    // polls of one wait; a healthy one ends within a few hundred
constexpr float kRescale = 8.f;              // log2 growth of a row's maximum that is left in P
constexpr uint32_t kTmemCols = 512;          // S_0, S_1 (P over them), O_0, O_1: 128 columns each

// Ring of key and value tiles: what shared memory holds beside Q.
__host__ __device__ constexpr int ring_stages(int panels) { return panels == 2 ? 5 : 8; }

struct Barriers {
    uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2];
    uint64_t kv_full[8], kv_empty[8];
    uint64_t part_done[2], last_set[2];
    uint64_t drain;
    uint32_t tmem;
    uint32_t abort;
    uint32_t last[2];
};
constexpr uint32_t smem_bytes(int panels) {
    return 1024 + (2 + ring_stages(panels)) * panels * kPanelBytes + static_cast<uint32_t>(sizeof(Barriers));
}
static_assert(smem_bytes(2) <= 232448 && smem_bytes(1) > 116224, "fits one SM, and no two blocks share one (tensor memory)");

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// False when the phase did not complete within the limit, or another warp has given up. One thread waits.
__device__ __forceinline__ bool bar_wait(Barriers& b, uint64_t* bar, uint32_t parity) {
    for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
        if (bar_try(bar, parity)) return true;
        if (spin % 256 == 255 && *reinterpret_cast<volatile uint32_t*>(&b.abort) != 0) return false;
    }
    *reinterpret_cast<volatile uint32_t*>(&b.abort) = 1;
    return false;
}
// The same for a whole warp, whose lanes all get one answer and leave together.
__device__ __forceinline__ bool warp_wait(Barriers& b, uint64_t* bar, uint32_t parity) {
    for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
        if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
        if (spin % 256 == 255 && __any_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(&b.abort) != 0)) return false;
    }
    *reinterpret_cast<volatile uint32_t*>(&b.abort) = 1;
    __syncwarp();
    return false;
}
template <int N>
__device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

// ---- tcgen05 ------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Shared-memory operand with the 128-byte swizzle TMA wrote. K-major (Q, K): `stride` = 1024 between groups of
// 8 rows, `lead` unused. MN-major (V): `stride` = 1024 between groups of 8 keys, `lead` between panels of 64 columns.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
    return static_cast<uint64_t>((addr >> 4) & 0x3fff) | static_cast<uint64_t>((lead >> 4) & 0x3fff) << 16 |
           static_cast<uint64_t>((stride >> 4) & 0x3fff) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}
// bf16 x bf16 -> fp32, M = 128.
__host__ __device__ constexpr uint32_t mma_desc(uint32_t n, bool b_mn_major) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (b_mn_major ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a),
        "l"(b), "r"(desc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a),
        "l"(b), "r"(desc), "r"(accumulate)
        : "memory");
}

#define SPECA_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define SPECA_I8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
// 32 columns of this thread's lane (row).
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* x) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
        "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : SPECA_R8(x, 0), SPECA_R8(x, 8), SPECA_R8(x, 16), SPECA_R8(x, 24)
        : "r"(addr));
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t* x) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::SPECA_I8(x, 0),
        SPECA_I8(x, 8), SPECA_I8(x, 16), SPECA_I8(x, 24), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t* x) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : SPECA_R8(x, 0), SPECA_R8(x, 8)
        : "r"(addr));
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t* x) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::SPECA_I8(x, 0),
        SPECA_I8(x, 8), "r"(addr)
        : "memory");
}
// Waits for this warp's loads; the registers they fill pass through, so that no use is scheduled in front of the wait.
#define SPECA_P8(x, i) "+r"(x[i]), "+r"(x[i + 1]), "+r"(x[i + 2]), "+r"(x[i + 3]), "+r"(x[i + 4]), "+r"(x[i + 5]), "+r"(x[i + 6]), "+r"(x[i + 7])
template <int N>
__device__ __forceinline__ void tmem_wait_load(uint32_t* x) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; i += 8) asm volatile("" : SPECA_P8(x, i));
}
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// What a unit asks of its two blocks.
struct Work {
    int kv_len;
    int t0;       // first key tile
    int n[2];     // key tiles of each block
    int rows[2];  // rows of each block
};
__device__ __forceinline__ bool unit_work(const AttnParams& p, const AttnUnit& u, int block_rows, Work& w) {
    if (p.dev_mask != nullptr && p.dev_mask[u.seq] == 0) return false;
    w.kv_len = kv_length(p, u);
    const int tiles = (w.kv_len + kTileKeys - 1) / kTileKeys, share = (tiles + u.n_splits - 1) / u.n_splits;
    w.t0 = u.split * share;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int r0 = u.row0 + b * block_rows;
        w.rows[b] = max(0, min(block_rows, u.q_len * p.group - r0));
        w.n[b] = 0;
        if (w.rows[b] == 0) continue;
        const int seen = visible_keys(p, u, w.kv_len, (r0 + w.rows[b] - 1) / p.group);  // by the block's last row
        w.n[b] = max(0, min(w.t0 + share, (seen + kTileKeys - 1) / kTileKeys) - w.t0);
    }
    return true;
}

struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++stage == stages) {
            stage = 0;
            phase ^= 1;
        }
    }
};

// PANELS: panels of 64 columns that a head spans (head_dim <= 64 or <= 128).
template <int PANELS>
__global__ void __launch_bounds__(kTcThreads, 1)
    attention_bf16_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap map_q,
                          const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    extern __shared__ char smem_raw[];
    constexpr int kStages = ring_stages(PANELS);
    constexpr uint32_t kTileBytes = PANELS * kPanelBytes;
    char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    char* smem_q = smem;                       // two blocks
    char* smem_kv = smem + 2 * kTileBytes;     // the ring
    Barriers& bar = *reinterpret_cast<Barriers*>(smem_kv + kStages * kTileBytes);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int tokens = kBlockRows / p.group, block_rows = tokens * p.group;  // packed rows of a block

    if (threadIdx.x == 0) {
        for (int b = 0; b < 2; ++b) {
            bar_init(&bar.q_full[b], 1);
            bar_init(&bar.q_empty[b], 1);
            bar_init(&bar.s_full[b], 1);
            bar_init(&bar.p_full[b], 4);  // one arrival per warp
            bar_init(&bar.o_full[b], 1);
            bar_init(&bar.part_done[b], 4);
            bar_init(&bar.last_set[b], 1);
        }
        for (int i = 0; i < kStages; ++i) {
            bar_init(&bar.kv_full[i], 1);
            bar_init(&bar.kv_empty[i], 1);
        }
        bar_init(&bar.drain, 1);
        bar.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)), "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bar.tmem);

    if (warp >= 8) fewer_registers<72>();
    if (warp == 8) {
        // ---- loads ----
        if (lane == 0) {
            Ring ring;
            uint32_t q_phase[2] = {0, 0};
            bool ok = true;
            auto load_tile = [&](const CUtensorMap* map, int head, int row) {
                ok = ok && bar_wait(bar, &bar.kv_empty[ring.stage], ring.phase ^ 1);
                if (!ok) return;
                bar_expect(&bar.kv_full[ring.stage], kTileBytes);
                const uint32_t dst = smem_u32(smem_kv) + ring.stage * kTileBytes;
                for (int i = 0; i < PANELS; ++i) tma_load(dst + i * kPanelBytes, map, i * 64, head, row, &bar.kv_full[ring.stage]);
                ring.next(kStages);
            };
            for (int i = blockIdx.x; i < p.n_units && ok; i += gridDim.x) {
                const AttnUnit u = load_unit(p.units, i);
                Work w;
                if (!unit_work(p, u, block_rows, w)) continue;
                const int n = max(w.n[0], w.n[1]);
                for (int b = 0; b < 2 && ok; ++b) {
                    if (w.n[b] > 0) {
                        ok = bar_wait(bar, &bar.q_empty[b], q_phase[b] ^ 1);
                        if (!ok) break;
                        bar_expect(&bar.q_full[b], static_cast<uint32_t>(block_rows) * 128 * PANELS);
                        for (int k = 0; k < PANELS; ++k)
                            tma_load(smem_u32(smem_q) + b * kTileBytes + k * kPanelBytes, &map_q, k * 64, u.kv_head * p.group,
                                     u.q_start + u.row0 / p.group + b * tokens, &bar.q_full[b]);
                        q_phase[b] ^= 1;
                    }
                    if (b == 0 && n > 0) load_tile(&map_k, u.kv_head, u.kv_start + w.t0 * kTileKeys);
                }
                for (int j = 0; j < n && ok; ++j) {
                    const int row = u.kv_start + (w.t0 + j) * kTileKeys;
                    load_tile(&map_v, u.kv_head, row);
                    if (j + 1 < n) load_tile(&map_k, u.kv_head, row + kTileKeys);
                }
            }
            if (!ok) {
                // copies in flight must land before the block gives its shared memory back
                for (int s = 0; s < kStages; ++s)
                    for (uint32_t spin = 0; spin < kSpinLimit; ++spin)
                        if (bar_try(&bar.kv_full[s], s < ring.stage ? ring.phase : ring.phase ^ 1)) break;
                for (int b = 0; b < 2; ++b)
                    for (uint32_t spin = 0; spin < kSpinLimit; ++spin)
                        if (bar_try(&bar.q_full[b], q_phase[b] ^ 1)) break;
            }
        }
    } else if (warp == 9) {
        // ---- products ----
        const int k_steps = (p.head_dim + 15) / 16;
        const uint32_t desc_s = mma_desc(kTileKeys, false), desc_o = mma_desc(16 * k_steps, true);
        Ring ring;
        uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        bool ok = true;
        auto score = [&](int b, int stage) {  // S_b = Q_b K^T
            if (lane == 0) {
                const uint64_t qd = smem_desc(smem_u32(smem_q) + b * kTileBytes, 16, 1024);
                const uint64_t kd = smem_desc(smem_u32(smem_kv) + stage * kTileBytes, 16, 1024);
                for (int k = 0; k < k_steps; ++k) {
                    const uint64_t step = (k / 4) * (kPanelBytes / 16) + (k % 4) * 2;
                    mma_ss(tmem + b * 128, qd + step, kd + step, desc_s, k > 0);
                }
                tc_commit(&bar.s_full[b]);
            }
            __syncwarp();
        };
        for (int i = blockIdx.x; i < p.n_units && ok; i += gridDim.x) {
            const AttnUnit u = load_unit(p.units, i);
            Work w;
            if (!unit_work(p, u, block_rows, w)) continue;
            const int n = max(w.n[0], w.n[1]);
            if (n == 0) continue;
            ok = warp_wait(bar, &bar.kv_full[ring.stage], ring.phase);
            for (int b = 0; b < 2 && ok; ++b) {
                if (w.n[b] == 0) continue;
                ok = warp_wait(bar, &bar.q_full[b], q_phase[b]);
                if (!ok) break;
                q_phase[b] ^= 1;
                tc_fence_after();
                score(b, ring.stage);
                if (w.n[b] == 1 && lane == 0) tc_commit(&bar.q_empty[b]);
            }
            if (!ok) break;
            if (lane == 0) tc_commit(&bar.kv_empty[ring.stage]);
            ring.next(kStages);
            for (int j = 0; j < n && ok; ++j) {
                const int v_stage = ring.stage;
                ok = warp_wait(bar, &bar.kv_full[ring.stage], ring.phase);
                if (!ok) break;
                ring.next(kStages);
                // The last tile may hold other rows behind kv_len. The product stops at the next multiple of 16
                // keys and the rows up to there are cleared: their weight is zero, but zero times NaN is not.
                const int valid = min(kTileKeys, w.kv_len - (w.t0 + j) * kTileKeys), used = (valid + 15) / 16 * 16;
                if (valid < used) {
                    char* v = smem_kv + v_stage * kTileBytes;
                    for (int e = lane; e < (used - valid) * 8 * PANELS; e += 32)
                        *reinterpret_cast<uint4*>(v + (e / 8 % PANELS) * kPanelBytes + (valid + e / (8 * PANELS)) * 128 + e % 8 * 16) =
                            make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                bool have_k = false;
                for (int b = 0; b < 2 && ok; ++b) {
                    if (j >= w.n[b]) continue;
                    ok = warp_wait(bar, &bar.p_full[b], p_phase[b]);
                    if (!ok) break;
                    p_phase[b] ^= 1;
                    tc_fence_after();
                    if (lane == 0) {  // O_b += P_b V
                        const uint64_t vd = smem_desc(smem_u32(smem_kv) + v_stage * kTileBytes, kPanelBytes, 1024);
                        for (int k = 0; k < used / 16; ++k)
                            mma_ts(tmem + 256 + b * 128, tmem + b * 128 + k * 8, vd + k * 128, desc_o, j > 0 || k > 0);
                        if (j + 1 == w.n[b]) tc_commit(&bar.o_full[b]);
                    }
                    __syncwarp();
                    if (j + 1 < w.n[b]) {
                        if (!have_k) ok = warp_wait(bar, &bar.kv_full[ring.stage], ring.phase);
                        if (!ok) break;
                        have_k = true;
                        tc_fence_after();
                        score(b, ring.stage);
                        if (j + 2 == w.n[b] && lane == 0) tc_commit(&bar.q_empty[b]);
                    }
                }
                if (!ok) break;
                if (lane == 0) {
                    tc_commit(&bar.kv_empty[v_stage]);
                    if (j + 1 < n) tc_commit(&bar.kv_empty[ring.stage]);
                }
                if (j + 1 < n) ring.next(kStages);
            }
        }
        if (!ok) {  // products in flight must end before tensor memory is given back
            if (lane == 0) tc_commit(&bar.drain);
            for (uint32_t spin = 0; spin < kSpinLimit; ++spin)
                if (bar_try(&bar.drain, 0)) break;
        }
    } else if (warp < 8) {
        // ---- softmax and output ----
        more_registers<216>();
        const int b = warp / 4;
        const int row = threadIdx.x % 128;
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t tmem_s = tmem + lanes + b * 128, tmem_o = tmem + lanes + 256 + b * 128;
        uint32_t s_phase = 0, o_phase = 0, part_phase = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < p.n_units && ok; i += gridDim.x) {
            const AttnUnit u = load_unit(p.units, i);
            Work w;
            if (!unit_work(p, u, block_rows, w) || w.rows[b] == 0) continue;
            const int pr = u.row0 + b * block_rows + row;  // packed row of the sequence
            const bool live = row < w.rows[b];
            const int limit = live ? visible_keys(p, u, w.kv_len, pr / p.group) : 0;
            // keys that every live row of the block sees: tiles in front of this index need no mask
            const int open = visible_keys(p, u, w.kv_len, (u.row0 + b * block_rows) / p.group);
            float ref = -CUDART_INF_F;  // the maximum that P and the sums refer to
            float l = 0.f;
            for (int j = 0; j < w.n[b]; ++j) {
                const int key0 = (w.t0 + j) * kTileKeys;
                ok = warp_wait(bar, &bar.s_full[b], s_phase);
                if (!ok) break;
                s_phase ^= 1;
                tc_fence_after();
                uint32_t raw[128];
                float* s = reinterpret_cast<float*>(raw);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_load32(tmem_s + c * 32, raw + c * 32);
                tmem_wait_load<128>(raw);
                if (key0 + kTileKeys > open) {
                    const int seen = limit - key0;
#pragma unroll
                    for (int c = 0; c < 128; ++c) s[c] = c < seen ? s[c] : -CUDART_INF_F;
                }
                float top[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int c = 4; c < 128; c += 4)
#pragma unroll
                    for (int k = 0; k < 4; ++k) top[k] = fmaxf(top[k], s[c + k]);
                const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                const bool grow = (m - ref) * p.scale_log2 > kRescale;  // also from -inf, unless m is -inf too
                if (j == 0) {
                    ref = m;
                } else if (__any_sync(0xffffffffu, grow)) {
                    const float next = fmaxf(ref, m);
                    const float f = next == -CUDART_INF_F ? 1.f : ex2((ref - next) * p.scale_log2);
                    ref = next;
                    l *= f;
                    for (int c = 0; c < p.head_dim; c += 16) {
                        uint32_t o[16];
                        tmem_load16(tmem_o + c, o);
                        tmem_wait_load<16>(o);
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                        tmem_store16(tmem_o + c, o);
                    }
                }
                const float shift = ref == -CUDART_INF_F ? 0.f : -ref * p.scale_log2;
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t packed[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        const float e0 = ex2(fmaf(s[h * 64 + 2 * c], p.scale_log2, shift));
                        const float e1 = ex2(fmaf(s[h * 64 + 2 * c + 1], p.scale_log2, shift));
                        packed[c] = pack_bf16(e0, e1);
                        // the sum is over what the product will see: a weight's rounding then divides out where one key dominates
                        sum[0] += __uint_as_float(packed[c] << 16);
                        sum[1] += __uint_as_float(packed[c] & 0xffff0000u);
                    }
                    tmem_store32(tmem_s + h * 32, packed);
                }
                l += sum[0] + sum[1];
                tmem_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&bar.p_full[b]);
            }
            if (!ok) break;
            if (w.n[b] > 0) {
                ok = warp_wait(bar, &bar.o_full[b], o_phase);
                if (!ok) break;
                o_phase ^= 1;
                tc_fence_after();
            }
            const int unit_rows = w.rows[0] + w.rows[1];
            const int64_t pitch = part_row_floats(p.head_dim), split_stride = unit_rows * pitch;
            const int64_t part0 = u.part + b * block_rows * pitch * 4;  // of this block in share 0
            const int tok = u.q_start + pr / p.group, head = u.kv_head * p.group + pr % p.group;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            float* part = reinterpret_cast<float*>(p.parts + part0) + u.split * split_stride + row * pitch;
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.o) + tok * p.o_row + head * p.o_head;
            for (int c = 0; c < p.head_dim; c += 16) {
                uint32_t o[16] = {};
                if (w.n[b] > 0) {
                    tmem_load16(tmem_o + c, o);
                    tmem_wait_load<16>(o);
                }
                if (!live) continue;
                if (u.n_splits > 1) {
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        if (c + k < p.head_dim) *reinterpret_cast<uint4*>(part + c + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    continue;
                }
#pragma unroll
                for (int k = 0; k < 16; k += 8) {
                    if (c + k >= p.head_dim) continue;
                    uint32_t v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = pack_bf16(__uint_as_float(o[k + 2 * e]) * inv, __uint_as_float(o[k + 2 * e + 1]) * inv);
                    *reinterpret_cast<uint4*>(out + c + k) = make_uint4(v[0], v[1], v[2], v[3]);
                }
            }
            tc_fence_before();  // O is read: the next unit's first product may overwrite it once this block's P is there
            if (u.n_splits == 1) {
                if (live && p.lse != nullptr)
                    p.lse[static_cast<int64_t>(head) * p.total_q + tok] =
                        l == 0.f ? -CUDART_INF_F : (ref * p.scale_log2 + log2f(l)) * kLn2;
                continue;
            }
            if (live) {
                part[pitch - 4] = ref * p.scale_log2;
                part[pitch - 3] = l;
            }
            __threadfence();
            __syncwarp();
            if (lane == 0) bar_arrive(&bar.part_done[b]);
            ok = warp_wait(bar, &bar.part_done[b], part_phase);
            if (!ok) break;
            if (row == 0) {
                const uint32_t before = atomicAdd(p.tickets + u.ticket + b, 1u);
                bar.last[b] = before == static_cast<uint32_t>(u.n_splits) - 1;
                if (bar.last[b]) p.tickets[u.ticket + b] = 0;  // ready for the next launch
                bar_arrive(&bar.last_set[b]);
            }
            __syncwarp();
            ok = warp_wait(bar, &bar.last_set[b], part_phase);
            if (!ok) break;
            part_phase ^= 1;
            // read by all four warps before they arrive at part_done again, so before it is set again
            if (*reinterpret_cast<volatile uint32_t*>(&bar.last[b])) {
                __threadfence();
                join_rows<__nv_bfloat16>(p, u, u.row0 + b * block_rows, w.rows[b], part0, split_stride, warp % 4, 4);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(&bar.abort) != 0) atomicExch(p.gave_up, 1u);
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
    }
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
    static const EncodeTiled fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &res) != cudaSuccess ||
            res != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

// [rows, heads, head_dim] as boxes of 64 columns x box_heads x box_rows, columns behind head_dim and rows behind
// the tensor read as zero.
bool encode(CUtensorMap* map, const char* base, int head_dim, int heads, int64_t rows, int64_t row_stride, int64_t head_stride,
            int box_heads, int box_rows) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
    // a dimension of one element is never stepped through: any multiple of 16 will do
    const cuuint64_t strides[2] = {heads > 1 ? static_cast<cuuint64_t>(head_stride) * 2 : 256,
                                   rows > 1 ? static_cast<cuuint64_t>(row_stride) * 2 : 256};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_rows)}, ones[3] = {1, 1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<char*>(base), dims, strides, box, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_attention_bf16(const AttnParams& p, int64_t total_kv, int sm_count, cudaStream_t stream) {
    if (p.n_units == 0) return cudaSuccess;
    if (encoder() == nullptr) return cudaErrorNotSupported;
    CUtensorMap q, k, v;
    // without a single key no tile is loaded: the maps then only have to be valid
    const char* kb = total_kv > 0 ? p.k : p.q;
    const char* vb = total_kv > 0 ? p.v : p.q;
    const int64_t kv_rows = total_kv > 0 ? total_kv : 1;
    if (!encode(&q, p.q, p.head_dim, p.n_heads, p.total_q, p.q_row, p.q_head, p.group, kBlockRows / p.group) ||
        !encode(&k, kb, p.head_dim, p.n_kv_heads, kv_rows, p.k_row, p.k_head, 1, kTileKeys) ||
        !encode(&v, vb, p.head_dim, p.n_kv_heads, kv_rows, p.v_row, p.v_head, 1, kTileKeys))
        return cudaErrorNotSupported;
    const int panels = p.head_dim > 64 ? 2 : 1;
    auto* kernel = panels == 2 ? attention_bf16_kernel<2> : attention_bf16_kernel<1>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes(panels));
    if (e != cudaSuccess) return e;
    kernel<<<p.n_units < sm_count ? p.n_units : sm_count, kTcThreads, smem_bytes(panels), stream>>>(p, q, k, v);
    return cudaGetLastError();
}

}  // namespace speca
