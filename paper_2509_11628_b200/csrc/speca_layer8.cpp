// Host side of the 8-bit calls (speca_layer_norm8, speca_layer_quantize8, speca_quantize8, speca_layer_matmul8): argument
// checks and kernel launches.
#include <cuda_runtime.h>

#include "speca_layer_handle.h"

using namespace speca;

namespace {

struct Refusal {
    speca_status_t status = SPECA_OK;
    const char* why = "";
};

inline int64_t groups_of(int64_t dim) { return (dim + 4 * kBlock8 - 1) / (4 * kBlock8); }

// A matrix of `rows` x `dim` in 8 bits as a call gets it, with strides that say nothing taken out.
Refusal take(const speca_matrix8_t* m, int64_t rows, int64_t dim, speca_matrix8_t* out) {
    if (m == nullptr) return {SPECA_ERR_INVALID_ARG, "null matrix"};
    *out = *m;
    drop_stride(rows, out->code_stride);
    drop_stride(groups_of(dim), out->scale_stride);
    if (rows > 0 && (out->codes == nullptr || out->scales == nullptr)) return {SPECA_ERR_INVALID_ARG, "null codes or scales"};
    if (rows > 1 && out->code_stride < dim) return {SPECA_ERR_SHAPE, "rows of codes overlap"};
    if (groups_of(dim) > 1 && out->scale_stride < 4 * rows) return {SPECA_ERR_SHAPE, "groups of scales overlap"};
    if (reinterpret_cast<uintptr_t>(out->scales) % 4 != 0 || out->scale_stride % 4 != 0)
        return {SPECA_ERR_ALIGNMENT, "scales start on 4 bytes, in every group"};
    return {};
}

// What the call of a row kernel has besides the rows' own arithmetic.
bool vectors8(const Norm8Params& p, size_t e) {
    auto on = [&](const void* q, int64_t stride) {
        return q == nullptr || (reinterpret_cast<uintptr_t>(q) % 16 == 0 && stride * static_cast<int64_t>(e) % 16 == 0);
    };
    return p.dim % 16 == 0 && on(p.x, p.x_stride) && on(p.branch, p.branch_stride) && on(p.gate, p.mod_stride) &&
           on(p.scale, p.mod_stride) && on(p.shift, p.mod_stride) && on(p.weight, 0) && on(p.x_out, p.x_out_stride) &&
           reinterpret_cast<uintptr_t>(p.out.codes) % 16 == 0 && p.out.code_stride % 16 == 0;
}

Out8 out8(const speca_matrix8_t& m) {
    return Out8{static_cast<uint8_t*>(m.codes), static_cast<uint8_t*>(m.scales), m.code_stride, m.scale_stride};
}

// The rows as they are: shared by the call with a handle and the one without.
Refusal quantize_params(int64_t rows, int64_t dim, const void* x, int64_t x_stride, size_t e, const speca_matrix8_t* out, Norm8Params* p) {
    if (dim < 1 || dim > kMaxRows) return {SPECA_ERR_SHAPE, "dim outside 1 .. SPECA_MAX_ROWS"};
    drop_stride(rows, x_stride);
    if (rows > 0 && x == nullptr) return {SPECA_ERR_INVALID_ARG, "null tensor"};
    if (x_stride < 0) return {SPECA_ERR_SHAPE, "negative stride"};
    if (reinterpret_cast<uintptr_t>(x) % e != 0) return {SPECA_ERR_ALIGNMENT, "a tensor is not aligned to the element size"};
    speca_matrix8_t m;
    const Refusal r = take(out, rows, dim, &m);
    if (r.status != SPECA_OK) return r;
    if (rows > 0 && (m.codes == x || m.scales == x || m.codes == m.scales)) return {SPECA_ERR_INVALID_ARG, "an output overlaps another tensor"};
    *p = Norm8Params{};
    p->x = static_cast<const char*>(x);
    p->x_stride = x_stride;
    p->out = out8(m);
    p->rows = static_cast<int32_t>(rows);
    p->dim = static_cast<int32_t>(dim);
    return {};
}

}  // namespace

extern "C" {

speca_status_t speca_quantize8(int64_t rows, int32_t dim, const void* x, int64_t x_stride, int32_t dtype, const speca_matrix8_t* out,
                               int32_t device, void* stream) {
    if (dtype != SPECA_F32 && dtype != SPECA_BF16) return SPECA_ERR_INVALID_ARG;
    if (rows < 0 || rows > kMaxRows) return SPECA_ERR_SHAPE;
    const size_t e = dtype == SPECA_BF16 ? 2 : 4;
    Norm8Params p;
    const Refusal r = quantize_params(rows, dim, x, x_stride, e, out, &p);
    if (r.status != SPECA_OK) return r.status;
    int n_dev = 0, major = 0;
    if (cudaGetDeviceCount(&n_dev) != cudaSuccess) return SPECA_ERR_CUDA;
    if (device < 0 || device >= n_dev) return SPECA_ERR_INVALID_ARG;
    cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device);
    if (major != 10) return SPECA_ERR_UNSUPPORTED;
    DeviceGuard guard(device);
    if (!guard.ok || cudaGetLastError() != cudaSuccess) return SPECA_ERR_CUDA;
    return launch_norm8(p, dtype, vectors8(p, e), static_cast<cudaStream_t>(stream)) == cudaSuccess ? SPECA_OK : SPECA_ERR_CUDA;
}

speca_status_t speca_layer_quantize8(speca_layer_t* c, int32_t dim, const void* x, int64_t x_stride, const uint8_t* dev_active_mask,
                                     const speca_matrix8_t* out, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    Norm8Params p;
    const Refusal r = quantize_params(c->total_q, dim, x, x_stride, elem_size(c), out, &p);
    if (r.status != SPECA_OK) return fail(c, r.status, "quantize8: %s", r.why);
    p.row_seq = reinterpret_cast<const uint16_t*>(c->ws + c->row_seq_off);
    p.dev_mask = dev_active_mask;
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    speca_status_t st = check_sticky(c);
    if (st != SPECA_OK) return st;
    cudaError_t e = launch_norm8(p, c->dtype, vectors8(p, elem_size(c)), static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SPECA_OK : cuda_fail(c, e, "quantize8");
}

speca_status_t speca_layer_norm8(speca_layer_t* c, int32_t kind, int32_t dim, const void* x, int64_t x_stride, const void* branch,
                                 int64_t branch_stride, const void* gate, const void* scale, const void* shift, int64_t mod_stride,
                                 const void* weight, const uint8_t* dev_active_mask, void* x_out, int64_t x_out_stride,
                                 const speca_matrix8_t* out, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    if (kind != SPECA_NORM_LAYER && kind != SPECA_NORM_RMS) return fail(c, SPECA_ERR_INVALID_ARG, "norm8: unknown kind of norm");
    Norm8Params p;
    const Refusal r = quantize_params(c->total_q, dim, x, x_stride, elem_size(c), out, &p);
    if (r.status != SPECA_OK) return fail(c, r.status, "norm8: %s", r.why);
    drop_stride(c->total_q, branch_stride);
    drop_stride(c->total_q, x_out_stride);
    drop_stride(c->n_seqs, mod_stride);
    if (gate != nullptr && branch == nullptr) return fail(c, SPECA_ERR_INVALID_ARG, "norm8: a gate without a branch");
    if ((branch != nullptr && branch_stride < 0) || mod_stride < 0) return fail(c, SPECA_ERR_SHAPE, "norm8: negative stride");
    if (c->total_q > 1 && x_out != nullptr && x_out_stride < dim) return fail(c, SPECA_ERR_SHAPE, "norm8: output rows overlap");
    // in place each thread writes what it alone has read, which takes the same strides
    if (c->total_q > 0 && ((x_out == x && x_out_stride != p.x_stride) ||
                           (x_out != nullptr && x_out == branch && x_out_stride != branch_stride)))
        return fail(c, SPECA_ERR_INVALID_ARG, "norm8: in place needs the strides of the input");
    if (c->total_q > 0)
        for (const void* q : {static_cast<const void*>(x_out), branch, gate, scale, shift, weight})
            if (q != nullptr && (q == p.out.codes || q == p.out.scales))
                return fail(c, SPECA_ERR_INVALID_ARG, "norm8: the 8-bit output overlaps another tensor");
    if (c->total_q > 0 && x_out != nullptr && (x_out == gate || x_out == scale || x_out == shift || x_out == weight))
        return fail(c, SPECA_ERR_INVALID_ARG, "norm8: x_out overlaps a modulation or the weight");
    if (!on_elements(c, branch) || !on_elements(c, gate) || !on_elements(c, scale) || !on_elements(c, shift) || !on_elements(c, weight) ||
        !on_elements(c, x_out))
        return fail(c, SPECA_ERR_ALIGNMENT, "norm8: a tensor is not aligned to the element size");
    p.row_seq = reinterpret_cast<const uint16_t*>(c->ws + c->row_seq_off);
    p.dev_mask = dev_active_mask;
    p.branch = static_cast<const char*>(branch);
    p.gate = static_cast<const char*>(gate);
    p.scale = static_cast<const char*>(scale);
    p.shift = static_cast<const char*>(shift);
    p.weight = static_cast<const char*>(weight);
    p.x_out = static_cast<char*>(x_out);
    p.branch_stride = branch_stride;
    p.mod_stride = mod_stride;
    p.x_out_stride = x_out_stride;
    p.norm = 1;
    p.centre = kind == SPECA_NORM_LAYER;
    p.eps = c->norm_eps;
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    speca_status_t st = check_sticky(c);
    if (st != SPECA_OK) return st;
    cudaError_t e = launch_norm8(p, c->dtype, vectors8(p, elem_size(c)), static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SPECA_OK : cuda_fail(c, e, "norm8");
}

speca_status_t speca_layer_matmul8(speca_layer_t* c, int32_t n, int32_t k, const speca_matrix8_t* a, const speca_matrix8_t* w,
                                   const void* bias, int32_t activation, const void* residual, int64_t residual_stride,
                                   const void* gate, int64_t gate_stride, const uint8_t* dev_active_mask, void* out,
                                   int64_t out_stride, const speca_matrix8_t* out_8bit, void* stream) {
    if (c == nullptr) return SPECA_ERR_INVALID_ARG;
    if (n < 1 || n > kMaxRows) return fail(c, SPECA_ERR_SHAPE, "matmul8: n outside 1 .. %lld", static_cast<long long>(kMaxRows));
    if (k < 1 || k > SPECA_MAX_K8) return fail(c, SPECA_ERR_SHAPE, "matmul8: k outside 1 .. %d", SPECA_MAX_K8);
    if (activation != SPECA_ACT_NONE && activation != SPECA_ACT_GELU && activation != SPECA_ACT_SILU)
        return fail(c, SPECA_ERR_INVALID_ARG, "matmul8: unknown activation");
    const int64_t m = c->total_q;
    speca_matrix8_t ma, mw, mo{};
    Refusal r = take(a, m, k, &ma);
    if (r.status == SPECA_OK) r = take(w, n, k, &mw);
    if (r.status == SPECA_OK && out_8bit != nullptr) r = take(out_8bit, m, n, &mo);
    if (r.status != SPECA_OK) return fail(c, r.status, "matmul8: %s", r.why);
    if (m > 0 ? (out != nullptr) == (out_8bit != nullptr) : out != nullptr && out_8bit != nullptr)
        return fail(c, SPECA_ERR_INVALID_ARG, "matmul8: one output is expected, in the layer's type or in 8 bits");
    if (out_8bit != nullptr && (residual != nullptr || gate != nullptr))
        return fail(c, SPECA_ERR_INVALID_ARG, "matmul8: an output in 8 bits takes no residual and no gate");
    for (const speca_matrix8_t* q : {&ma, &mw})
        if (reinterpret_cast<uintptr_t>(q->codes) % 16 != 0 || q->code_stride % 16 != 0)
            return fail(c, SPECA_ERR_ALIGNMENT, "matmul8: rows of codes start on 16 bytes");
    drop_stride(m, out_stride);
    drop_stride(m, residual_stride);
    drop_stride(c->n_seqs, gate_stride);
    if (residual_stride < 0 || gate_stride < 0) return fail(c, SPECA_ERR_SHAPE, "matmul8: negative stride");
    if (out != nullptr && m > 1 && out_stride < n) return fail(c, SPECA_ERR_SHAPE, "matmul8: output rows overlap");
    if (!on_elements(c, bias) || !on_elements(c, residual) || !on_elements(c, gate) || !on_elements(c, out))
        return fail(c, SPECA_ERR_ALIGNMENT, "matmul8: a tensor is not aligned to the element size");
    if (m > 0) {
        if (out != nullptr && out == residual && out_stride != residual_stride)
            return fail(c, SPECA_ERR_INVALID_ARG, "matmul8: in place needs the strides of the residual");
        const void* outs[3] = {out, mo.codes, mo.scales};
        for (const void* o : outs)
            for (const void* q : {static_cast<const void*>(ma.codes), static_cast<const void*>(ma.scales), static_cast<const void*>(mw.codes),
                                  static_cast<const void*>(mw.scales), bias, gate})
                if (o != nullptr && o == q) return fail(c, SPECA_ERR_INVALID_ARG, "matmul8: the output overlaps an input");
        if (out_8bit != nullptr && mo.codes == mo.scales) return fail(c, SPECA_ERR_INVALID_ARG, "matmul8: the output's codes and scales overlap");
    }
    Matmul8Params p{};
    p.row_seq = reinterpret_cast<const uint16_t*>(c->ws + c->row_seq_off);
    p.dev_mask = dev_active_mask;
    p.a = static_cast<const uint8_t*>(ma.codes);
    p.w = static_cast<const uint8_t*>(mw.codes);
    p.a_scales = static_cast<const uint8_t*>(ma.scales);
    p.w_scales = static_cast<const uint8_t*>(mw.scales);
    p.a_stride = ma.code_stride;
    p.w_stride = mw.code_stride;
    p.a_scale_stride = ma.scale_stride;
    p.w_scale_stride = mw.scale_stride;
    p.m = static_cast<int32_t>(m);
    p.n = n;
    p.k = k;
    p.bias = static_cast<const char*>(bias);
    p.residual = static_cast<const char*>(residual);
    p.gate = static_cast<const char*>(gate);
    p.out = static_cast<char*>(out);
    p.out8 = out8(mo);
    p.residual_stride = residual_stride;
    p.gate_stride = gate_stride;
    p.out_stride = out_stride;
    p.act = activation;
    auto out_on = [&](int64_t bytes) {
        const void* rows = out != nullptr ? out : mo.codes;
        const int64_t stride = out != nullptr ? out_stride * static_cast<int64_t>(elem_size(c)) : mo.code_stride;
        return reinterpret_cast<uintptr_t>(rows) % bytes == 0 && stride % bytes == 0;
    };
    p.vectors = out_on(16) && on_16(c, bias, 0, 0) && on_16(c, residual, residual_stride, 0) && on_16(c, gate, gate_stride, 0);
    p.wide = out_on(32);
    p.gave_up = reinterpret_cast<uint32_t*>(c->ws + c->gave_up_off);
    DeviceGuard guard(c->device);
    if (!guard.ok) return fail(c, SPECA_ERR_CUDA, "cudaSetDevice failed");
    speca_status_t st = check_sticky(c);
    if (st != SPECA_OK) return st;
    cudaError_t err = launch_matmul8(p, c->dtype, c->sm_count, static_cast<cudaStream_t>(stream));
    if (err == cudaErrorNotSupported)
        return fail(c, SPECA_ERR_UNSUPPORTED, "matmul8: the copy engine cannot address a matrix with this stride");
    return err == cudaSuccess ? SPECA_OK : cuda_fail(c, err, "matmul8");
}

}  // extern "C"
