// Host side of the verification layer's calls (speca_layer_* in speca.h): the handle, the packing and
// the attention's work list, argument checks and kernel launches.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "speca_layer_handle.h"

using namespace speca;

namespace {

constexpr size_t kAlign = 256;
static_assert(kMaxRows + 65536 <= int64_t(1) << 31 && 2 * 296 * kSimtKeys <= 65536 && 296 * kTcKeys <= 65536, "sums of a count and a tile fit");
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// How the attention of a storage type cuts its work.
struct Tiling {
    int rows;          // most packed rows of a unit
    int narrow;        // a unit of so few rows takes two shares at once
    int keys;          // keys of a tile
    int target;        // units that fill the device: below it, long key ranges are shared out
    int min_share;     // fewest tiles worth a unit of its own
};
// 148 SMs, with two resident blocks each in fp32 and one in bf16.
Tiling tiling(int dtype, int group) {
    if (dtype == SPECA_BF16) return Tiling{2 * tc_block_rows(group), tc_block_rows(group), kTcKeys, 148, 4};
    return Tiling{kSimtRows, 0, kSimtKeys, 296, 4};
}

struct Plan {
    std::vector<AttnUnit> units;
    std::vector<JoinBlock> joins;
    int join_rows = 0;
    std::vector<uint16_t> row_seq;
    std::vector<RopePair> pairs;
    size_t units_off, joins_off, row_seq_off, pairs_off, gave_up_off, parts_off, total;
    int64_t total_q, total_kv;
};

speca_status_t check_offsets(const int64_t* start, int n, int64_t* total) {
    if (start[0] != 0) return SPECA_ERR_SHAPE;
    for (int i = 0; i < n; ++i)
        if (start[i + 1] < start[i] || start[i + 1] > kMaxRows) return SPECA_ERR_SHAPE;
    *total = start[n];
    return SPECA_OK;
}

speca_status_t make_plan_impl(const speca_layer_config_t* c, Plan* P) {
    if (c == nullptr || c->host_q_start == nullptr) return SPECA_ERR_INVALID_ARG;
    if (c->dtype != SPECA_F32 && c->dtype != SPECA_BF16) return SPECA_ERR_INVALID_ARG;
    if (c->n_seqs < 1 || c->n_seqs > SPECA_MAX_SEQS) return SPECA_ERR_SHAPE;
    if (std::isnan(c->scale) || std::isinf(c->scale) || !std::isfinite(c->norm_eps)) return SPECA_ERR_INVALID_ARG;
    const int64_t* qs = c->host_q_start;
    const int64_t* ks = c->host_kv_start != nullptr ? c->host_kv_start : qs;
    speca_status_t st = check_offsets(qs, c->n_seqs, &P->total_q);
    if (st == SPECA_OK) st = check_offsets(ks, c->n_seqs, &P->total_kv);
    if (st != SPECA_OK) return st;
    const bool heads = c->n_heads != 0 || c->n_kv_heads != 0;
    if (heads) {
        if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads != 0) return SPECA_ERR_SHAPE;
        if (c->n_heads / c->n_kv_heads > SPECA_MAX_GROUP || c->n_heads > (1 << 16)) return SPECA_ERR_SHAPE;
        if (c->head_dim < 1 || c->head_dim > SPECA_MAX_HEAD_DIM) return SPECA_ERR_SHAPE;
    }
    if (c->n_axes < 0 || c->n_axes > SPECA_MAX_AXES || (c->n_axes > 0 && !heads)) return SPECA_ERR_SHAPE;
    if (c->n_axes > 0) {
        if (c->pairing != SPECA_ROPE_INTERLEAVED && c->pairing != SPECA_ROPE_HALVES) return SPECA_ERR_INVALID_ARG;
        if (!(c->theta > 0.0) || !std::isfinite(c->theta)) return SPECA_ERR_INVALID_ARG;
        if (c->head_dim % 2 != 0) return SPECA_ERR_SHAPE;
        int sum = 0;
        for (int a = 0; a < c->n_axes; ++a) {
            if (c->axis_dims[a] < 2 || c->axis_dims[a] % 2 != 0 || c->axis_dims[a] > c->head_dim) return SPECA_ERR_SHAPE;
            sum += c->axis_dims[a];
        }
        if (sum > c->head_dim) return SPECA_ERR_SHAPE;
        P->pairs.assign(c->head_dim / 2, RopePair{0.0, -1, 0});
        const double two_pi = 6.283185307179586476925286766559;
        int at = 0;
        for (int a = 0; a < c->n_axes; ++a)
            for (int i = 0; i < c->axis_dims[a] / 2; ++i)
                P->pairs[at++] = RopePair{std::pow(c->theta, -2.0 * i / c->axis_dims[a]) / two_pi, a, 0};
    }
    P->row_seq.resize(static_cast<size_t>(P->total_q));
    for (int s = 0; s < c->n_seqs; ++s)
        std::fill(P->row_seq.begin() + qs[s], P->row_seq.begin() + qs[s + 1], static_cast<uint16_t>(s));

    size_t part_bytes = 0;
    if (heads) {
        const int group = c->n_heads / c->n_kv_heads;
        const Tiling tl = tiling(c->dtype, group);
        const int rows = tl.rows;
        auto blocks = [&](int s) { return ((qs[s + 1] - qs[s]) * group + rows - 1) / rows; };
        auto narrow = [&](int s) { return (qs[s + 1] - qs[s]) * group <= tl.narrow; };
        auto tiles = [&](int s) { return (ks[s + 1] - ks[s] + tl.keys - 1) / tl.keys; };
        // The share of key tiles a unit takes: all of them, unless that leaves SMs idle. Then the smallest
        // share whose units still fit the device at once (more would only add rows to join).
        int64_t longest = 1, whole = 0, n_units = 0;
        for (int s = 0; s < c->n_seqs; ++s) {
            whole += blocks(s) * c->n_kv_heads;
            if (blocks(s) > 0) longest = std::max(longest, tiles(s));
        }
        if (whole > (int64_t(1) << 26)) return SPECA_ERR_SHAPE;
        // shares of a sequence's keys; both halves of a narrow unit are put to use where there are tiles for it
        auto shares = [&](int s, int64_t share) {
            const int64_t n = std::max<int64_t>(1, (tiles(s) + share - 1) / share);
            return n == 1 && narrow(s) && tiles(s) >= 2 * tl.min_share ? 2 : n;
        };
        auto count = [&](int64_t share) {
            int64_t n = 0;
            for (int s = 0; s < c->n_seqs; ++s) {
                n += blocks(s) * c->n_kv_heads * (narrow(s) ? (shares(s, share) + 1) / 2 : shares(s, share));
            }
            return n;
        };
        int64_t share = longest;
        if (whole < tl.target && longest > tl.min_share) {
            int64_t lo = tl.min_share, hi = longest;  // smallest share in [lo, hi] with count <= target
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (count(mid) <= tl.target) hi = mid; else lo = mid + 1;
            }
            share = lo;
        }
        n_units = count(share);
        std::vector<int64_t> cost;
        P->units.reserve(static_cast<size_t>(n_units));
        cost.reserve(static_cast<size_t>(n_units));
        const int64_t row_bytes = part_row_floats(c->head_dim) * 4;
        for (int s = 0; s < c->n_seqs; ++s) {
            const int64_t q_len = qs[s + 1] - qs[s], kv = ks[s + 1] - ks[s], nt = tiles(s);
            const int splits = static_cast<int>(shares(s, share));
            if (q_len * group > kMaxRows) return SPECA_ERR_SHAPE;
            for (int h = 0; h < c->n_kv_heads; ++h)
                for (int64_t r = 0; r < q_len * group; r += rows) {
                    const int64_t n = std::min<int64_t>(rows, q_len * group - r);
                    const int64_t last = (r + n - 1) / group;
                    const int64_t seen = c->causal ? std::max<int64_t>(0, std::min(kv, last + 1 + kv - q_len)) : kv;
                    const int64_t part_nt = (nt + splits - 1) / splits;
                    const int step = narrow(s) && splits > 1 ? 2 : 1;
                    for (int i = 0; i < splits; i += step) {
                        AttnUnit u;
                        u.seq = s;
                        u.kv_head = h;
                        u.row0 = static_cast<int32_t>(r);
                        u.q_len = static_cast<int32_t>(q_len);
                        u.kv_cap = static_cast<int32_t>(kv);
                        u.q_start = static_cast<int32_t>(qs[s]);
                        u.kv_start = static_cast<int32_t>(ks[s]);
                        u.split = i;
                        u.n_splits = splits;
                        u.narrow = step == 2;
                        u.part = static_cast<int64_t>(part_bytes);
                        P->units.push_back(u);
                        cost.push_back(std::max<int64_t>(0, std::min(part_nt, (seen + tl.keys - 1) / tl.keys - i * part_nt)));
                    }
                    if (splits > 1) {
                        P->joins.push_back(JoinBlock{s, h, static_cast<int32_t>(r), static_cast<int32_t>(n), static_cast<int32_t>(qs[s]),
                                                     splits, static_cast<int64_t>(part_bytes)});
                        P->join_rows = std::max(P->join_rows, static_cast<int>(n));
                        part_bytes += static_cast<size_t>(splits * n * row_bytes);
                    }
                }
        }
        // longest first, so that the last units to start are short ones; equal ones keep their order, in
        // which the blocks of one key head follow one another and share its tiles in L2
        std::vector<int32_t> order(P->units.size());
        for (size_t i = 0; i < order.size(); ++i) order[i] = static_cast<int32_t>(i);
        std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return cost[a] > cost[b]; });
        std::vector<AttnUnit> sorted(P->units.size());
        for (size_t i = 0; i < order.size(); ++i) sorted[i] = P->units[order[i]];
        P->units.swap(sorted);
    }
    size_t off = 0;
    P->units_off = off;
    off = align_up(off + P->units.size() * sizeof(AttnUnit), kAlign);
    P->joins_off = off;
    off = align_up(off + P->joins.size() * sizeof(JoinBlock), kAlign);
    P->row_seq_off = off;
    off = align_up(off + P->row_seq.size() * sizeof(uint16_t), kAlign);
    P->pairs_off = off;
    off = align_up(off + P->pairs.size() * sizeof(RopePair), kAlign);
    P->gave_up_off = off;
    off += kAlign;
    P->parts_off = off;
    P->total = off + part_bytes;
    return SPECA_OK;
}

// The C ABI never lets an exception out.
speca_status_t make_plan(const speca_layer_config_t* c, Plan* P) noexcept {
    try {
        return make_plan_impl(c, P);
    } catch (const std::bad_alloc&) {
        return SPECA_ERR_NOMEM;
    } catch (...) {
        return SPECA_ERR_INVALID_ARG;
    }
}

}  // namespace

extern "C" {

speca_status_t speca_layer_workspace_bytes(const speca_layer_config_t* cfg, size_t* out_bytes) {
    if (out_bytes == nullptr) return SPECA_ERR_INVALID_ARG;
    Plan P;
    speca_status_t st = make_plan(cfg, &P);
    if (st == SPECA_OK) *out_bytes = P.total;
    return st;
}

speca_status_t speca_layer_create(const speca_layer_config_t* cfg, speca_layer_t** out) {
    if (out == nullptr) return SPECA_ERR_INVALID_ARG;
    *out = nullptr;
    Plan P;
    speca_status_t st = make_plan(cfg, &P);
    if (st != SPECA_OK) return st;
    if (cfg->workspace == nullptr) return SPECA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(cfg->workspace) % kAlign != 0) return SPECA_ERR_ALIGNMENT;
    if (cfg->workspace_bytes < P.total) return SPECA_ERR_NOMEM;
    int n_dev = 0;
    cudaError_t ce = cudaGetDeviceCount(&n_dev);
    if (ce != cudaSuccess) return SPECA_ERR_CUDA;
    if (cfg->device < 0 || cfg->device >= n_dev) return SPECA_ERR_INVALID_ARG;
    int major = 0;
    cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device);
    if (major != 10) return SPECA_ERR_UNSUPPORTED;  // the kernels are built for sm_100a only
    speca_layer* c = new (std::nothrow) speca_layer();
    if (c == nullptr) return SPECA_ERR_NOMEM;
    c->n_seqs = cfg->n_seqs;
    c->dtype = cfg->dtype;
    c->n_heads = cfg->n_heads;
    c->n_kv_heads = cfg->n_kv_heads;
    c->head_dim = cfg->head_dim;
    c->causal = cfg->causal != 0;
    c->n_axes = cfg->n_axes;
    c->pairing = cfg->pairing;
    for (int a = 0; a < cfg->n_axes; ++a) c->rotated += cfg->axis_dims[a];
    c->device = cfg->device;
    c->total_q = P.total_q;
    c->total_kv = P.total_kv;
    c->n_units = static_cast<int>(P.units.size());
    c->n_joins = static_cast<int>(P.joins.size());
    c->join_rows = P.join_rows;
    c->scale = cfg->scale > 0.f ? cfg->scale : (cfg->head_dim > 0 ? 1.f / std::sqrt(static_cast<float>(cfg->head_dim)) : 1.f);
    c->norm_eps = cfg->norm_eps > 0.f ? cfg->norm_eps : 1e-6f;
    c->ws = static_cast<char*>(cfg->workspace);
    c->units_off = P.units_off;
    c->joins_off = P.joins_off;
    c->row_seq_off = P.row_seq_off;
    c->pairs_off = P.pairs_off;
    c->gave_up_off = P.gave_up_off;
    c->parts_off = P.parts_off;
    cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, c->device);
    DeviceGuard guard(c->device);
    // what is still pending on the memory (its last user's kernels, on any stream) must not land on the lists written here
    ce = guard.ok ? cudaDeviceSynchronize() : cudaErrorInvalidDevice;
    auto upload = [&](size_t off, const void* src, size_t n) {
        if (ce == cudaSuccess && n > 0) ce = cudaMemcpy(c->ws + off, src, n, cudaMemcpyHostToDevice);
    };
    upload(P.units_off, P.units.data(), P.units.size() * sizeof(AttnUnit));
    upload(P.joins_off, P.joins.data(), P.joins.size() * sizeof(JoinBlock));
    upload(P.row_seq_off, P.row_seq.data(), P.row_seq.size() * sizeof(uint16_t));
    upload(P.pairs_off, P.pairs.data(), P.pairs.size() * sizeof(RopePair));
    if (ce == cudaSuccess) ce = cudaMemset(c->ws + P.gave_up_off, 0, sizeof(uint32_t));
    // the copies come from pageable memory: wait, so that work on any stream finds them done
    if (ce == cudaSuccess) ce = cudaDeviceSynchronize();
    if (ce != cudaSuccess) {
        (void)cudaGetLastError();
        delete c;
        return SPECA_ERR_CUDA;
    }
    *out = c;
    return SPECA_OK;
}

speca_status_t speca_layer_destroy(speca_layer_t* c) {
    if (c == nullptr) return SPECA_OK;
    DeviceGuard guard(c->device);
    uint32_t gave_up = 0;
    cudaError_t ce = cudaDeviceSynchronize();
    if (ce == cudaSuccess) ce = cudaMemcpy(&gave_up, c->ws + c->gave_up_off, sizeof gave_up, cudaMemcpyDeviceToHost);
    delete c;
    return ce == cudaSuccess && gave_up == 0 ? SPECA_OK : SPECA_ERR_CUDA;
}

speca_status_t speca_layer_modulate(speca_layer_t* c, int32_t dim, const void* x, int64_t x_stride, const void* branch,
                                    int64_t branch_stride, const void* gate, const void* scale, const void* shift,
                                    int64_t mod_stride, const uint8_t* dev_active_mask, void* x_out, int64_t x_out_stride,
                                    void* y, int64_t y_stride, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    if (dim < 1 || dim > kMaxRows) return fail(c, SPECA_ERR_SHAPE, "modulate: dim outside 1 .. %lld", static_cast<long long>(kMaxRows));
    for (int64_t* s : {&x_stride, &branch_stride, &x_out_stride, &y_stride}) drop_stride(c->total_q, *s);
    drop_stride(c->n_seqs, mod_stride);
    if (c->total_q > 0 && (x == nullptr || y == nullptr)) return fail(c, SPECA_ERR_INVALID_ARG, "modulate: null tensor");
    if (gate != nullptr && branch == nullptr) return fail(c, SPECA_ERR_INVALID_ARG, "modulate: a gate without a branch");
    if (x_stride < 0 || (branch != nullptr && branch_stride < 0) || mod_stride < 0)
        return fail(c, SPECA_ERR_SHAPE, "modulate: negative stride");
    if (c->total_q > 1 && (y_stride < dim || (x_out != nullptr && x_out_stride < dim)))
        return fail(c, SPECA_ERR_SHAPE, "modulate: output rows overlap");
    // in place each thread writes what it alone has read, which takes the same strides
    if (c->total_q > 0 && ((y == x && y_stride != x_stride) || (y == branch && y_stride != branch_stride) || y == x_out ||
                           (x_out == x && x_out_stride != x_stride) ||
                           (x_out != nullptr && x_out == branch && x_out_stride != branch_stride)))
        return fail(c, SPECA_ERR_INVALID_ARG, "modulate: in place needs the strides of the input, and y and x_out apart");
    if (!on_elements(c, x) || !on_elements(c, branch) || !on_elements(c, gate) || !on_elements(c, scale) || !on_elements(c, shift) ||
        !on_elements(c, x_out) || !on_elements(c, y))
        return fail(c, SPECA_ERR_ALIGNMENT, "modulate: a tensor is not aligned to the element size");
    ModulateParams p;
    p.row_seq = reinterpret_cast<const uint16_t*>(c->ws + c->row_seq_off);
    p.dev_mask = dev_active_mask;
    p.x = static_cast<const char*>(x);
    p.branch = static_cast<const char*>(branch);
    p.gate = static_cast<const char*>(gate);
    p.scale = static_cast<const char*>(scale);
    p.shift = static_cast<const char*>(shift);
    p.x_out = static_cast<char*>(x_out);
    p.y = static_cast<char*>(y);
    p.x_stride = x_stride;
    p.branch_stride = branch_stride;
    p.mod_stride = mod_stride;
    p.x_out_stride = x_out_stride;
    p.y_stride = y_stride;
    p.rows = static_cast<int32_t>(c->total_q);
    p.dim = dim;
    p.eps = c->norm_eps;
    const bool wide = dim * elem_size(c) % 16 == 0 && on_16(c, x, x_stride, 0) && on_16(c, branch, branch_stride, 0) &&
                      on_16(c, x_out, x_out_stride, 0) && on_16(c, y, y_stride, 0) &&
                      on_16(c, gate, mod_stride, 0) && on_16(c, scale, mod_stride, 0) && on_16(c, shift, mod_stride, 0);
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    speca_status_t st = check_sticky(c);
    if (st != SPECA_OK) return st;
    cudaError_t e = launch_modulate(p, c->dtype, wide ? static_cast<int>(16 / elem_size(c)) : 1, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SPECA_OK : cuda_fail(c, e, "modulate");
}

speca_status_t speca_layer_rope(speca_layer_t* c, const void* q, int64_t q_row_stride, int64_t q_head_stride, void* q_out,
                                int64_t q_out_row_stride, int64_t q_out_head_stride, const void* k, int64_t k_row_stride,
                                int64_t k_head_stride, void* k_out, int64_t k_out_row_stride, int64_t k_out_head_stride,
                                const float* positions, const void* q_weight, const void* k_weight,
                                const uint8_t* dev_active_mask, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    if (c->n_axes == 0) return fail(c, SPECA_ERR_STATE, "rope: the layer has no rotary axes");
    for (int64_t* s : {&q_row_stride, &q_out_row_stride, &k_row_stride, &k_out_row_stride}) drop_stride(c->total_q, *s);
    for (int64_t* s : {&q_head_stride, &q_out_head_stride}) drop_stride(c->n_heads, *s);
    for (int64_t* s : {&k_head_stride, &k_out_head_stride}) drop_stride(c->n_kv_heads, *s);
    if ((k == nullptr) != (k_out == nullptr)) return fail(c, SPECA_ERR_INVALID_ARG, "rope: k and k_out go together");
    if (c->total_q > 0 && (q == nullptr || q_out == nullptr || positions == nullptr))
        return fail(c, SPECA_ERR_INVALID_ARG, "rope: null tensor");
    if (q_row_stride < 0 || q_head_stride < 0 || k_row_stride < 0 || k_head_stride < 0)
        return fail(c, SPECA_ERR_SHAPE, "rope: negative stride");
    if (meets_itself(c->total_q, q_out_row_stride, c->n_heads, q_out_head_stride, c->head_dim) ||
        (k_out != nullptr && meets_itself(c->total_q, k_out_row_stride, c->n_kv_heads, k_out_head_stride, c->head_dim)))
        return fail(c, SPECA_ERR_SHAPE, "rope: outputs overlap");
    // in place each lane writes what it alone has read, which takes the same strides
    if (c->total_q > 0 && ((q_out == q && (q_out_row_stride != q_row_stride || q_out_head_stride != q_head_stride)) ||
                           (k != nullptr && k_out == k && (k_out_row_stride != k_row_stride || k_out_head_stride != k_head_stride)) ||
                           (k != nullptr && (q_out == k_out || q_out == k || k_out == q))))
        return fail(c, SPECA_ERR_INVALID_ARG, "rope: in place needs the strides of the input, and q and k apart");
    if (!on_elements(c, q) || !on_elements(c, q_out) || !on_elements(c, k) || !on_elements(c, k_out) || !on_elements(c, q_weight) ||
        !on_elements(c, k_weight) || reinterpret_cast<uintptr_t>(positions) % 4 != 0)
        return fail(c, SPECA_ERR_ALIGNMENT, "rope: a tensor is not aligned to the element size");
    RopeParams p;
    p.row_seq = reinterpret_cast<const uint16_t*>(c->ws + c->row_seq_off);
    p.dev_mask = dev_active_mask;
    p.pairs = reinterpret_cast<const RopePair*>(c->ws + c->pairs_off);
    p.q = static_cast<const char*>(q);
    p.k = static_cast<const char*>(k);
    p.q_weight = static_cast<const char*>(q_weight);
    p.k_weight = static_cast<const char*>(k_weight);
    p.q_out = static_cast<char*>(q_out);
    p.k_out = static_cast<char*>(k_out);
    p.positions = positions;
    p.q_row = q_row_stride, p.q_head = q_head_stride, p.qo_row = q_out_row_stride, p.qo_head = q_out_head_stride;
    p.k_row = k_row_stride, p.k_head = k_head_stride, p.ko_row = k_out_row_stride, p.ko_head = k_out_head_stride;
    p.rows = static_cast<int32_t>(c->total_q);
    p.n_heads = c->n_heads;
    p.n_kv_heads = c->n_kv_heads;
    p.head_dim = c->head_dim;
    p.n_axes = c->n_axes;
    p.rotated = c->rotated;
    p.half = c->pairing == SPECA_ROPE_HALVES ? c->rotated / 2 : 0;
    p.eps = c->norm_eps;
    // four pairs as one or two accesses: heads of a multiple of 8 elements and, for HALVES, a multiple of 4 pairs
    const bool vectors = c->head_dim % 8 == 0 && p.half % 4 == 0 && on_16(c, q, q_row_stride, q_head_stride) &&
                         on_16(c, q_out, q_out_row_stride, q_out_head_stride) && on_16(c, k, k_row_stride, k_head_stride) &&
                         on_16(c, k_out, k_out_row_stride, k_out_head_stride) && on_16(c, q_weight, 0, 0) && on_16(c, k_weight, 0, 0);
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    speca_status_t st = check_sticky(c);
    if (st != SPECA_OK) return st;
    cudaError_t e = launch_rope(p, c->dtype, vectors, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SPECA_OK : cuda_fail(c, e, "rope");
}

speca_status_t speca_layer_attention(speca_layer_t* c, const void* q, int64_t q_row_stride, int64_t q_head_stride,
                                     const void* k, int64_t k_row_stride, int64_t k_head_stride, const void* v,
                                     int64_t v_row_stride, int64_t v_head_stride, void* o, int64_t o_row_stride,
                                     int64_t o_head_stride, const int32_t* dev_kv_len, const uint8_t* dev_active_mask,
                                     float* dev_lse, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    if (c->n_heads == 0) return fail(c, SPECA_ERR_STATE, "attention: the layer has no heads");
    if (c->dtype == SPECA_BF16 && c->head_dim % 8 != 0)
        return fail(c, SPECA_ERR_SHAPE, "attention: bf16 heads come in multiples of 8 elements");
    for (int64_t* s : {&q_row_stride, &o_row_stride}) drop_stride(c->total_q, *s);
    for (int64_t* s : {&k_row_stride, &v_row_stride}) drop_stride(c->total_kv, *s);
    for (int64_t* s : {&q_head_stride, &o_head_stride}) drop_stride(c->n_heads, *s);
    for (int64_t* s : {&k_head_stride, &v_head_stride}) drop_stride(c->n_kv_heads, *s);
    if (c->total_q > 0 && (q == nullptr || o == nullptr || (c->total_kv > 0 && (k == nullptr || v == nullptr))))
        return fail(c, SPECA_ERR_INVALID_ARG, "attention: null tensor");
    if (q_row_stride < 0 || q_head_stride < 0 || k_row_stride < 0 || k_head_stride < 0 || v_row_stride < 0 || v_head_stride < 0)
        return fail(c, SPECA_ERR_SHAPE, "attention: negative stride");
    if (meets_itself(c->total_q, o_row_stride, c->n_heads, o_head_stride, c->head_dim))
        return fail(c, SPECA_ERR_SHAPE, "attention: output rows overlap");
    if (c->total_q > 0 && (o == q || o == k || o == v))
        return fail(c, SPECA_ERR_INVALID_ARG, "attention: the output overlaps an input");
    if (!on_elements(c, q) || !on_elements(c, k) || !on_elements(c, v) || !on_elements(c, o) ||
        reinterpret_cast<uintptr_t>(dev_lse) % 4 != 0 || reinterpret_cast<uintptr_t>(dev_kv_len) % 4 != 0)
        return fail(c, SPECA_ERR_ALIGNMENT, "attention: a tensor is not aligned to the element size");
    const bool wide = on_16(c, q, q_row_stride, q_head_stride) && on_16(c, k, k_row_stride, k_head_stride) &&
                      on_16(c, v, v_row_stride, v_head_stride) && on_16(c, o, o_row_stride, o_head_stride);
    if (c->dtype == SPECA_BF16 && !wide)
        return fail(c, SPECA_ERR_ALIGNMENT, "attention: bf16 tensors start on 16 bytes, with strides of multiples of 8 elements");
    if (c->dtype == SPECA_BF16 && ((c->total_q > 1 && q_row_stride == 0) || (c->n_heads > 1 && q_head_stride == 0) ||
                                   (c->total_kv > 1 && (k_row_stride == 0 || v_row_stride == 0))))
        return fail(c, SPECA_ERR_UNSUPPORTED, "attention: the copy engine cannot step by zero over queries or rows");
    AttnParams p;
    p.units = reinterpret_cast<const AttnUnit*>(c->ws + c->units_off);
    p.joins = reinterpret_cast<const JoinBlock*>(c->ws + c->joins_off);
    p.n_units = c->n_units;
    p.n_joins = c->n_joins;
    p.join_rows = c->join_rows;
    p.n_heads = c->n_heads;
    p.n_kv_heads = c->n_kv_heads;
    p.group = c->n_heads / c->n_kv_heads;
    p.head_dim = c->head_dim;
    p.causal = c->causal;
    p.total_q = static_cast<int32_t>(c->total_q);
    p.k_step = k_head_stride != 0;
    p.v_step = v_head_stride != 0;
    p.vectors = wide && c->head_dim % 4 == 0;
    p.scale_log2 = static_cast<float>(c->scale * 1.4426950408889634);
    p.q = static_cast<const char*>(q);
    p.k = static_cast<const char*>(k);
    p.v = static_cast<const char*>(v);
    p.o = static_cast<char*>(o);
    p.q_row = q_row_stride, p.q_head = q_head_stride, p.k_row = k_row_stride, p.k_head = k_head_stride;
    p.v_row = v_row_stride, p.v_head = v_head_stride, p.o_row = o_row_stride, p.o_head = o_head_stride;
    p.dev_kv_len = dev_kv_len;
    p.dev_mask = dev_active_mask;
    p.lse = dev_lse;
    p.parts = c->ws + c->parts_off;
    p.gave_up = reinterpret_cast<uint32_t*>(c->ws + c->gave_up_off);
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    speca_status_t st = check_sticky(c);
    if (st != SPECA_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = c->dtype == SPECA_BF16 ? launch_attention_bf16(p, c->total_kv, c->sm_count, s) : launch_attention_f32(p, s);
    if (e == cudaSuccess) e = launch_attention_join(p, c->dtype, s);
    if (e == cudaErrorNotSupported)
        return fail(c, SPECA_ERR_UNSUPPORTED, "attention: the copy engine cannot address a tensor with these strides");
    return e == cudaSuccess ? SPECA_OK : cuda_fail(c, e, "attention");
}

speca_status_t speca_layer_check(speca_layer_t* c, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint32_t gave_up = 0;
    cudaError_t e = cudaMemcpyAsync(&gave_up, c->ws + c->gave_up_off, sizeof gave_up, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess && gave_up != 0) e = cudaMemsetAsync(c->ws + c->gave_up_off, 0, sizeof gave_up, s);
    if (e != cudaSuccess) return cuda_fail(c, e, "check");
    return gave_up == 0 ? SPECA_OK : fail(c, SPECA_ERR_CUDA, "a kernel gave up on a bounded wait: results since the last check are incomplete");
}

const char* speca_layer_last_error(const speca_layer_t* c) { return c == nullptr ? "" : c->last_error; }

}  // extern "C"
