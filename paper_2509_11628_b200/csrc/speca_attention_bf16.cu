// Attention of the verification layer in bf16, on the tensor cores (tcgen05, TMA).
//
// A block of 128 packed query rows against tiles of 128 keys: S = Q K^T (fp32, tensor memory), running maximum
// and sum of exp2(scale S - max) per row, P rounded to bf16 back into tensor memory over S, O += P V. A unit
// is two such blocks, which share the K and V tiles and take turns on the tensor cores: while one block's
// products run, the other's exponentials are formed. One unit at a time per SM, blocks persistent over units:
//   warps 0-3, 4-7   softmax and output of block 0 and block 1: one thread per row, its 128 scores in registers
//   warp 8           TMA loads: Q of the unit, then K_0, V_0, K_1, V_1, ... through a ring of tiles
//   warps 9, 10      issue the products of block 0 and block 1 (warp 11 completes the warpgroup)
// Products of one thread run in the order of issue, so S_b(j+1) may overwrite P_b(j) right behind the product
// that reads it, and S_b(j+1) being ready says that O_b is at rest: the softmax threads themselves rescale O in the
// rare tile that raises a row's largest weight by more than 2^8 (sums and P are exact to a common factor; it keeps
// P <= 2^8, far inside bf16's range). The weights are rounded to bf16 because the tensor cores take them so: an error of up
// to 2^-8 of each, independent from key to key, of which the largest of a tile is taken into the divisor.
// Every wait is bounded. A wait that runs out sets the layer's gave-up flag and ends the block's work.
//
// What bounds it: products and exponentials of a tile take as long as each other (128 x 128 x 128 twice is 1024 cycles of
// the tensor pipe, 128 x 128 exponentials are 1024 of the special function units), and a block's chain
// scores -> weights -> product -> next scores leaves each pipe idle in between: tensor pipe 56 % active, special function
// units 42 %, about 3500 cycles per tile of both blocks. In a loop the card also runs into its power limit
// (990 W, 1740 MHz). Measured: 4608 rows x 24 heads of 128, 250 to 270 us over several cards (0.97 to 1.04 PFLOP/s),
// 20926 rows 4.76 to 5.09 ms (1.05 to 1.12). Tried and not kept, 4608 rows on one card, all under an earlier softmax: 64-key
// tiles with the scores double buffered 238 us, the same with two warpgroups taking turns at the tiles 245, one score buffer
// and P beside it 240 to 265, against 221 of this form.
#include "speca_attention_common.cuh"
#include "speca_tc.cuh"

namespace speca {
namespace {

// Three warpgroups of 168 registers a thread at launch; the two that form the softmax take 216 (a row of 128 scores
// and its packed weights stay in registers), the one that loads and issues gives up what they take: 2 x 216 + 72 = 3 x 168.
// (Two threads per row, 16 softmax warps of 104 registers, measured the same: what the shorter chains gain, telling each
// other the maximum through shared memory costs.)
constexpr int kTcThreads = 384;
constexpr int kLoadWarp = 8, kIssueWarp = 9;
constexpr int kBlockRows = 128;
constexpr int kTileKeys = 128;
constexpr uint32_t kPanelBytes = 128 * 128;  // 128 rows of 64 bf16: one 128-byte swizzle span per row
constexpr float kRescale = 8.f;              // log2 growth of a row's maximum that is left in P
constexpr uint32_t kTmemCols = 512;          // S_0, S_1 (P over them), O_0, O_1: 128 columns each

// Ring of key and value tiles: what shared memory holds beside Q.
__host__ __device__ constexpr int ring_stages(int panels) { return panels == 2 ? 5 : 8; }

struct Barriers {
    uint64_t q_full[2], q_empty[2], s_full[2], p_full[2], o_full[2];
    uint64_t kv_full[8], kv_empty[8];
    uint64_t turn[2], drain[2];
    uint32_t tmem;
    uint32_t abort;
};
constexpr uint32_t smem_bytes(int panels) {
    return (2 + ring_stages(panels)) * panels * kPanelBytes + static_cast<uint32_t>(sizeof(Barriers));
}
static_assert(smem_bytes(2) <= 232448 && smem_bytes(1) > 116224, "fits one SM, and no two blocks share one (tensor memory)");

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
        : "memory");
}

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

__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
// 2^x of a pair without the special function unit, which forms 16 a cycle and SM where the products of a tile leave time
// for just as many: x = n + f, |f| <= 1/2, n by adding 1.5 * 2^23 (its low bits are then n), 2^f by the polynomial of degree 3 of the
// least relative error on [-1/2, 1/2] (Remez exchange; 7.5e-5, a fiftieth of bf16's rounding), n into the exponent. Below
// 2^-125 the weight is zero, as the special function unit gives it below 2^-126; a NaN stays one.
__device__ __forceinline__ void ex2_poly(uint64_t x2, float& e0, float& e1) {
    float x0, x1;
    unpair(x2, x0, x1);
    const uint64_t magic = pair(12582912.f, 12582912.f), minus = pair(-1.f, -1.f);
    const uint64_t t = add2(x2, magic);
    const uint64_t f = add2(x2, fma2(t, minus, magic));
    uint64_t y = fma2(f, pair(0.05517167f, 0.05517167f), pair(0.24261112f, 0.24261112f));
    y = fma2(y, f, pair(0.69326099f, 0.69326099f));
    y = fma2(y, f, pair(0.99992807f, 0.99992807f));
    float t0, t1;
    unpair(t, t0, t1);
    unpair(y, e0, e1);
    e0 = x0 >= -125.f ? __uint_as_float(__float_as_uint(e0) + (__float_as_uint(t0) << 23)) : max_nan(x0, 0.f);
    e1 = x1 >= -125.f ? __uint_as_float(__float_as_uint(e1) + (__float_as_uint(t1) << 23)) : max_nan(x1, 0.f);
}
// Of the pairs, the last of so many by polynomial: 4608 rows x 24 heads of 128 / 16 heads of 64 took 231 / 140 us
// with none, 222 / 127 with one in 8 or 4, 227 / 132 with one in 2.
constexpr int kPolyEvery = 4;
static_assert(kPolyEvery == 4, "the softmax keeps the maximum of the polynomial's keys apart");

// Weights of 64 keys of a row, rounded to bf16, and their sum before the rounding.
__device__ __forceinline__ void weights(const float* s, uint64_t scale2, uint64_t shift2, uint32_t* packed, uint64_t* l) {
#pragma unroll
    for (int c = 0; c < 32; ++c) {
        const uint64_t x2 = fma2(pair(s[2 * c], s[2 * c + 1]), scale2, shift2);
        float e0, e1;
        if (c % kPolyEvery == kPolyEvery - 1) {
            ex2_poly(x2, e0, e1);
        } else {
            unpair(x2, e0, e1);
            e0 = ex2(e0);
            e1 = ex2(e1);
        }
        packed[c] = pack_bf16(e0, e1);
        l[c % 2] = add2(l[c % 2], pair(e0, e1));
    }
}

// What a unit asks of its two blocks. Wide units: two blocks of rows against the same key tiles. Narrow ones (few
// rows against many keys): the same rows twice, each against a share of the keys of its own, so that two chains of
// products and exponentials hide each other's waits there too.
struct Work {
    int kv_len;
    int t0[2];    // first key tile of each block
    int n[2];     // key tiles of each block
    int r0[2];    // first packed row of each block
    int rows[2];  // rows of each block
};
__device__ __forceinline__ bool unit_work(const AttnParams& p, const AttnUnit& u, int block_rows, Work& w) {
    if (p.dev_mask != nullptr && p.dev_mask[u.seq] == 0) return false;
    w.kv_len = kv_length(p, u);
    const int tiles = (w.kv_len + kTileKeys - 1) / kTileKeys, share = (tiles + u.n_splits - 1) / u.n_splits;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int split = u.split + (u.narrow ? b : 0);
        w.r0[b] = u.row0 + (u.narrow ? 0 : b * block_rows);
        w.rows[b] = split < u.n_splits ? max(0, min(block_rows, u.q_len * p.group - w.r0[b])) : 0;
        w.t0[b] = split * share;
        w.n[b] = 0;
        if (w.rows[b] == 0) continue;
        const int seen = visible_keys(p, u, w.kv_len, (w.r0[b] + w.rows[b] - 1) / p.group);  // by the block's last row
        w.n[b] = max(0, min(w.t0[b] + share, (seen + kTileKeys - 1) / kTileKeys) - w.t0[b]);
    }
    return true;
}

// A place in the ring of tiles.
struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ Ring ahead(int k, int stages) const {
        Ring r = *this;
        r.stage += k;
        if (r.stage >= stages) {
            r.stage -= stages;
            r.phase ^= 1;
        }
        return r;
    }
};

// Shared memory of a block: Q of both row blocks, the ring of key and value tiles, the barriers.
template <int PANELS>
struct Smem {
    static constexpr int kStages = ring_stages(PANELS);
    static constexpr uint32_t kTileBytes = PANELS * kPanelBytes;
    char* base;
    __device__ __forceinline__ uint32_t q(int b) const { return smem_u32(base) + b * kTileBytes; }
    __device__ __forceinline__ uint32_t kv(int stage) const { return smem_u32(base) + (2 + stage) * kTileBytes; }
    __device__ __forceinline__ char* kv_ptr(int stage) const { return base + (2 + stage) * kTileBytes; }
    __device__ __forceinline__ Barriers& bar() const { return *reinterpret_cast<Barriers*>(base + (2 + kStages) * kTileBytes); }
};

// ---- loads: one thread. False: a wait ran out ----
template <int PANELS>
__device__ __forceinline__ bool load_tiles(const AttnParams& p, const CUtensorMap& map_q, const CUtensorMap& map_k,
                                           const CUtensorMap& map_v, const Smem<PANELS>& sm) {
    constexpr uint32_t kTileBytes = Smem<PANELS>::kTileBytes;
    constexpr int kStages = Smem<PANELS>::kStages;
    Barriers& bar = sm.bar();
    const int block_rows = kBlockRows / p.group * p.group;
    Ring ring;
    uint32_t q_phase = 0;  // bit b: block b
    bool ok = true;
    auto load_tile = [&](const CUtensorMap& map, int head, int row) {
        if (!bar_wait(&bar.kv_empty[ring.stage], ring.phase ^ 1)) return false;
        bar_expect(&bar.kv_full[ring.stage], kTileBytes);
        for (int i = 0; i < PANELS; ++i)
            tma_load(sm.kv(ring.stage) + i * kPanelBytes, &map, i * 64, head, row, &bar.kv_full[ring.stage]);
        ring = ring.ahead(1, kStages);
        return true;
    };
    for (int i = blockIdx.x; i < p.n_units && ok; i += gridDim.x) {
        const AttnUnit u = load_unit(p.units, i);
        Work w;
        if (!unit_work(p, u, block_rows, w)) continue;
        const int k_head = u.kv_head * p.k_step, v_head = u.kv_head * p.v_step;
        // tiles of block 0's keys and, in a narrow unit, of block 1's
        const int n0 = u.narrow ? w.n[0] : max(w.n[0], w.n[1]), n1 = u.narrow ? w.n[1] : 0;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (w.n[b] > 0 && ok) {
                ok = bar_wait(&bar.q_empty[b], (q_phase >> b & 1) ^ 1);
                if (ok) {
                    bar_expect(&bar.q_full[b], static_cast<uint32_t>(block_rows) * 128 * PANELS);
                    for (int k = 0; k < PANELS; ++k)
                        tma_load(sm.q(b) + k * kPanelBytes, &map_q, k * 64, u.kv_head * p.group,
                                 u.q_start + w.r0[b] / p.group, &bar.q_full[b]);
                    q_phase ^= 1u << b;
                }
            }
            if ((b == 0 ? n0 : n1) > 0) ok = ok && load_tile(map_k, k_head, u.kv_start + w.t0[b] * kTileKeys);
        }
        for (int j = 0; j < max(n0, n1) && ok; ++j) {
            const int row0 = u.kv_start + (w.t0[0] + j) * kTileKeys, row1 = u.kv_start + (w.t0[1] + j) * kTileKeys;
            if (j < n0) ok = load_tile(map_v, v_head, row0);
            if (j < n1) ok = ok && load_tile(map_v, v_head, row1);
            if (j + 1 < n0) ok = ok && load_tile(map_k, k_head, row0 + kTileKeys);
            if (j + 1 < n1) ok = ok && load_tile(map_k, k_head, row1 + kTileKeys);
        }
    }
    if (ok) return true;
    // copies in flight must land before the block gives its shared memory back
    for (int i = 0; i < kStages; ++i) bar_wait(&bar.kv_full[i], i < ring.stage ? ring.phase : ring.phase ^ 1);
    for (int b = 0; b < 2; ++b) bar_wait(&bar.q_full[b], (q_phase >> b & 1) ^ 1);
    return false;
}

// ---- products of row block b: one warp, of which one thread issues. False: a wait ran out ----
template <int STEPS>
__device__ __forceinline__ bool issue_products(const AttnParams& p, const Smem<(STEPS + 3) / 4>& sm, uint32_t tmem, int b) {
    constexpr int kPanels = (STEPS + 3) / 4, kStages = Smem<kPanels>::kStages;
    constexpr uint32_t kDescS = mma_desc(kTileKeys, false), kDescO = mma_desc(16 * STEPS, true);
    Barriers& bar = sm.bar();
    const int block_rows = kBlockRows / p.group * p.group;
    const int part = threadIdx.x % 4;  // the lanes wait for four things at once
    const uint32_t tmem_s = tmem + b * 128, tmem_o = tmem + 256 + b * 128;
    const uint64_t q_desc = smem_desc(sm.q(b), 16, 1024);
    Ring ring;
    uint32_t q_phase = 0, p_phase = 0, turn = 0;
    constexpr int kHandOver = STEPS > 2 ? STEPS - 2 : 0;
    auto score = [&](int stage, bool hand_over) {  // S = Q K^T
        const uint64_t k_desc = smem_desc(sm.kv(stage), 16, 1024);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            if (k == kHandOver && hand_over) bar_arrive(&bar.turn[1 - b]);
            const uint64_t step = (k / 4) * (kPanelBytes / 16) + (k % 4) * 2;
            mma_ss(tmem_s, q_desc + step, k_desc + step, kDescS, k > 0);
        }
        tc_commit(&bar.s_full[b]);
    };
    for (int i = blockIdx.x; i < p.n_units; i += gridDim.x) {
        const AttnUnit u = load_unit(p.units, i);
        Work w;
        if (!unit_work(p, u, block_rows, w)) continue;
        const bool narrow = u.narrow != 0;
        const int own = b == 0 ? w.n[0] : w.n[1], t0 = b == 0 ? w.t0[0] : w.t0[1];
        const int n0 = narrow ? w.n[0] : max(w.n[0], w.n[1]), n1 = narrow ? w.n[1] : 0;  // as loaded
        // a tile that this block has no use for is given back as it arrives
        auto give_back = [&](Ring at) {
            if (!warp_wait(&bar.kv_full[at.stage], at.phase)) return false;
            if (elect_one()) bar_arrive(&bar.kv_empty[at.stage]);
            __syncwarp();
            return true;
        };
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if ((c == 0 ? n0 : n1) == 0) continue;
            if (narrow ? c == b : own > 0) {
                if (!warp_wait(part == 0 ? &bar.q_full[b] : &bar.kv_full[ring.stage], part == 0 ? q_phase : ring.phase)) return false;
                q_phase ^= 1;
                tc_fence_after();
                if (elect_one()) {
                    score(ring.stage, false);
                    if (own == 1) tc_commit(&bar.q_empty[b]);
                    tc_commit(&bar.kv_empty[ring.stage]);
                }
                __syncwarp();
            } else if (!give_back(ring)) {
                return false;
            }
            ring = ring.ahead(1, kStages);
        }
#pragma unroll 1
        for (int j = 0; j < max(n0, n1); ++j) {
            // V_j of block 0's keys, of block 1's, K_j+1 of block 0's, of block 1's, as far as there are such
            const int v0 = j < n0, v1 = j < n1, k0 = j + 1 < n0, k1 = j + 1 < n1;
            const Ring at_v1 = ring.ahead(v0, kStages), at_k0 = ring.ahead(v0 + v1, kStages), at_k1 = ring.ahead(v0 + v1 + k0, kStages);
            const bool second = narrow && b == 1;
            if (j < own) {
                const bool more = j + 1 < own;
                const Ring v_at = second ? at_v1 : ring, k_at = !more ? v_at : second ? at_k1 : at_k0;
                // The last tile may hold other rows behind kv_len. The product stops at the next multiple of 16 keys and the
                // rows up to there are cleared (by both blocks): their weight is zero, but zero times NaN is not.
                const int valid = min(kTileKeys, w.kv_len - (t0 + j) * kTileKeys), steps = (valid + 15) / 16;
                if (valid < steps * 16) {
                    if (!warp_wait(&bar.kv_full[v_at.stage], v_at.phase)) return false;
                    char* v = sm.kv_ptr(v_at.stage) + valid * 128;
                    for (int e = threadIdx.x % 32; e < (steps * 16 - valid) * 8; e += 32)
                        for (int k = 0; k < kPanels; ++k) *reinterpret_cast<uint4*>(v + k * kPanelBytes + e * 16) = make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                // O += P V and the next scores, in turn with the other block
                const uint64_t v_desc = smem_desc(sm.kv(v_at.stage), kPanelBytes, 1024);
                if (!warp_wait(part == 0 ? &bar.p_full[b] : part == 1 ? &bar.turn[b] : &bar.kv_full[part == 2 ? v_at.stage : k_at.stage],
                               part == 0 ? p_phase : part == 1 ? turn : part == 2 ? v_at.phase : k_at.phase))
                    return false;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kTileKeys / 16; ++k)
                        if (k < steps) mma_ts(tmem_o, tmem_s + k * 8, v_desc + k * 128, kDescO, j > 0 || k > 0);
                    if (more) {
                        score(k_at.stage, true);
                        tc_commit(&bar.kv_empty[v_at.stage]);
                        tc_commit(&bar.kv_empty[k_at.stage]);
                        if (j + 2 == own) tc_commit(&bar.q_empty[b]);
                    } else {
                        bar_arrive(&bar.turn[1 - b]);
                        tc_commit(&bar.o_full[b]);
                        tc_commit(&bar.kv_empty[v_at.stage]);
                    }
                }
                __syncwarp();
                p_phase ^= 1;
            } else {
                if (!warp_wait(&bar.turn[b], turn)) return false;
                if (elect_one()) bar_arrive(&bar.turn[1 - b]);
                __syncwarp();
            }
            turn ^= 1;
            const bool back_v = narrow ? (second ? v0 : v1) != 0 : j >= own && v0, back_k = narrow ? (second ? k0 : k1) != 0 : j + 1 >= own && k0;
            if (back_v && !give_back(narrow && !second ? at_v1 : ring)) return false;
            if (back_k && !give_back(narrow && !second ? at_k1 : at_k0)) return false;
            ring = ring.ahead(v0 + v1 + k0 + k1, kStages);
        }
    }
    return true;
}

// STEPS: steps of 16 columns that a head spans.
template <int STEPS>
__global__ void __launch_bounds__(kTcThreads, 1)
    attention_bf16_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap map_q,
                          const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    extern __shared__ __align__(1024) char smem[];
    constexpr int kPanels = (STEPS + 3) / 4;
    const Smem<kPanels> sm{smem};
    Barriers& bar = sm.bar();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int block_rows = kBlockRows / p.group * p.group;  // packed rows of a block

    if (smem_u32(smem) % 1024 != 0) {  // the swizzled tiles rely on it
        if (threadIdx.x == 0) atomicExch(p.gave_up, 1u);
        return;
    }
    if (threadIdx.x == 0) {
        for (int b = 0; b < 2; ++b) {
            bar_init(&bar.q_full[b], 1);
            bar_init(&bar.q_empty[b], 1);
            bar_init(&bar.s_full[b], 1);
            bar_init(&bar.p_full[b], 4);  // one arrival per warp
            bar_init(&bar.o_full[b], 1);
        }
        for (int i = 0; i < sm.kStages; ++i) {
            bar_init(&bar.kv_full[i], 1);
            bar_init(&bar.kv_empty[i], 2);  // one arrival per block
        }
        for (int b = 0; b < 2; ++b) {
            bar_init(&bar.turn[b], 1);
            bar_init(&bar.drain[b], 1);
        }
        bar.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        bar_arrive(&bar.turn[0]);  // block 0 begins
    }
    if (warp == kLoadWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)), "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&bar.tmem);

    if (warp >= kLoadWarp) fewer_registers<72>();
    if (warp == kLoadWarp) {
        if (lane == 0 && !load_tiles<kPanels>(p, map_q, map_k, map_v, sm)) bar.abort = 1;
    } else if (warp == kIssueWarp || warp == kIssueWarp + 1) {
        const int b = warp - kIssueWarp;
        if (!issue_products<STEPS>(p, sm, tmem, b)) {
            bar.abort = 1;
            if (elect_one()) tc_commit(&bar.drain[b]);  // products in flight must end before tensor memory is given back
            warp_wait(&bar.drain[b], 0);
        }
    } else if (warp < kLoadWarp) {
        // ---- softmax and output ----
        more_registers<216>();
        const int b = warp / 4;
        const int row = threadIdx.x % 128;
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t tmem_s = tmem + lanes + b * 128, tmem_o = tmem + lanes + 256 + b * 128;
        uint32_t s_phase = 0, o_phase = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < p.n_units && ok; i += gridDim.x) {
            const AttnUnit u = load_unit(p.units, i);
            Work w;
            if (!unit_work(p, u, block_rows, w)) continue;
            const int n = b == 0 ? w.n[0] : w.n[1], rows = b == 0 ? w.rows[0] : w.rows[1];
            const int t0 = b == 0 ? w.t0[0] : w.t0[1], r0 = b == 0 ? w.r0[0] : w.r0[1];
            if (rows == 0) continue;
            const int pr = r0 + row;  // packed row of the sequence
            const bool live = row < rows;
            const int limit = live ? visible_keys(p, u, w.kv_len, pr / p.group) : 0;
            // keys that every live row of the block sees: tiles in front of this index need no mask
            const int open = visible_keys(p, u, w.kv_len, r0 / p.group);
            float ref = -CUDART_INF_F;  // the maximum that P and the sums refer to
            uint64_t l[2] = {0, 0};   // four running sums in two pairs, joined at the end
            float off = 0.f;          // what the largest weights' rounding added, for the divisor alone
            for (int j = 0; j < n; ++j) {
                const int key0 = (t0 + j) * kTileKeys;
                ok = warp_wait(&bar.s_full[b], s_phase);
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
                float top[4];  // of the pairs by their place in eight keys: the last are the polynomial's
#pragma unroll
                for (int k = 0; k < 4; ++k) top[k] = fmaxf(s[2 * k], s[2 * k + 1]);
#pragma unroll
                for (int c = 8; c < 128; c += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k) top[k] = max3(top[k], s[c + 2 * k], s[c + 2 * k + 1]);
                const float m_ex2 = max3(top[0], top[1], top[2]), m = max3(top[3], m_ex2, m_ex2);
                // Each row goes by its own scores, so that its weights round the same whatever shares the warp. Rows that are not
                // live (other sequences' queries, or what shared memory held) have no say. Also from -inf, unless m is -inf too.
                // (Equal forms of this update took 4.99 to 5.65 ms for 20926 rows x 24 heads on one card; this is among the fastest.)
                const float mine = live ? m : -CUDART_INF_F;
                const bool grow = (mine - ref) * p.scale_log2 > kRescale;
                if (j == 0) {
                    ref = m;
                } else if (__any_sync(0xffffffffu, grow)) {
                    const float next = grow ? mine : ref, f = grow ? ex2((ref - next) * p.scale_log2) : 1.f;
                    ref = next;
                    l[0] = mul2(l[0], pair(f, f));
                    l[1] = mul2(l[1], pair(f, f));
                    off *= f;
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
                const uint64_t scale2 = pair(p.scale_log2, p.scale_log2), shift2 = pair(shift, shift);
                // The sum is over the weights before their rounding to bf16. In the divisor the largest of each tile counts
                // as rounded: where one key dominates, its rounding must divide out. Formed as the stored weight was, since
                // next to a rounding boundary of bf16 the polynomial and the special function unit round apart.
                const float x_top = fmaf(m, p.scale_log2, shift);
                float e_top, e_poly;
                ex2_poly(pair(x_top, x_top), e_poly, e_top);
                e_top = m > m_ex2 ? e_poly : ex2(x_top);
                off += __uint_as_float(pack_bf16(0.f, e_top)) - e_top;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t packed[32];
                    weights(s + h * 64, scale2, shift2, packed, l);
                    tmem_store32(tmem_s + h * 32, packed);
                }
                tmem_wait_store();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(&bar.p_full[b]);
            }
            if (!ok) break;
            if (n > 0) {
                ok = warp_wait(&bar.o_full[b], o_phase);
                if (!ok) break;
                o_phase ^= 1;
                tc_fence_after();
            }
            const int64_t pitch = part_row_floats(p.head_dim);
            const int unit_rows = u.narrow ? rows : w.rows[0] + w.rows[1], split = u.split + (u.narrow ? b : 0);
            const int tok = u.q_start + pr / p.group, head = u.kv_head * p.group + pr % p.group;
            float sums[4];
            unpair(l[0], sums[0], sums[1]);
            unpair(l[1], sums[2], sums[3]);
            const float total = (sums[0] + sums[1]) + (sums[2] + sums[3]);
            const float inv = total == 0.f ? 0.f : 1.f / (total + off);
            float* part = reinterpret_cast<float*>(p.parts + u.part) + (static_cast<int64_t>(split) * unit_rows + pr - u.row0) * pitch;
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.o) + tok * p.o_row + head * p.o_head;
            for (int c = 0; c < p.head_dim; c += 16) {
                uint32_t o[16] = {};
                if (n > 0) {
                    tmem_load16(tmem_o + c, o);
                    tmem_wait_load<16>(o);
                }
                if (!live) continue;
                if (total == 0.f) {  // sees nothing: zero, also where a weight of zero met a value that is not finite
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] = 0;
                }
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
                        total == 0.f ? -CUDART_INF_F : (ref * p.scale_log2 + log2f(total)) * kLn2;
                continue;
            }
            if (live) {
                part[pitch - 4] = ref * p.scale_log2;
                part[pitch - 3] = total;
                part[pitch - 2] = total + off;
            }
        }
        if (!ok) bar.abort = 1;
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *reinterpret_cast<volatile uint32_t*>(&bar.abort) != 0) atomicExch(p.gave_up, 1u);
    if (warp == kLoadWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
    }
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
        !encode(&k, kb, p.head_dim, p.k_step ? p.n_kv_heads : 1, kv_rows, p.k_row, p.k_head, 1, kTileKeys) ||
        !encode(&v, vb, p.head_dim, p.v_step ? p.n_kv_heads : 1, kv_rows, p.v_row, p.v_head, 1, kTileKeys))
        return cudaErrorNotSupported;
    using Kernel = void (*)(AttnParams, CUtensorMap, CUtensorMap, CUtensorMap);
    static const Kernel kernels[] = {attention_bf16_kernel<1>, attention_bf16_kernel<2>, attention_bf16_kernel<3>, attention_bf16_kernel<4>,
                                     attention_bf16_kernel<5>, attention_bf16_kernel<6>, attention_bf16_kernel<7>, attention_bf16_kernel<8>};
    const int steps = (p.head_dim + 15) / 16;
    const Kernel kernel = kernels[steps - 1];
    const uint32_t smem = smem_bytes((steps + 3) / 4);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    kernel<<<p.n_units < sm_count ? p.n_units : sm_count, kTcThreads, smem, stream>>>(p, q, k, v);
    return cudaGetLastError();
}

}  // namespace speca
