// The layer's handle and what the checks of its calls share (speca_layer.cpp, speca_layer8.cpp). Host only.
#pragma once
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "speca_layer_internal.h"

struct speca_layer {
    int n_seqs, dtype, n_heads, n_kv_heads, head_dim, causal, n_axes, pairing, rotated, device;
    int64_t total_q, total_kv;
    int n_units, n_joins, join_rows, sm_count;
    float scale, norm_eps;
    char* ws;
    size_t units_off, joins_off, row_seq_off, pairs_off, gave_up_off, parts_off;
    char last_error[256];
};

namespace speca {

// Rows, keys and elements of a row are counted in 32 bits on the device, where they are rounded up to blocks and tiles and
// key ranges end up to a tile per share behind the last key: the limit leaves room for that.
constexpr int64_t kMaxRows = SPECA_MAX_ROWS;

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != dev) ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

inline speca_status_t fail(speca_layer* c, speca_status_t st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(c->last_error, sizeof c->last_error, fmt, ap);
    va_end(ap);
    return st;
}

inline speca_status_t cuda_fail(speca_layer* c, cudaError_t err, const char* what) {
    (void)cudaGetLastError();
    return fail(c, SPECA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(err));
}

// An error left by earlier work on this thread surfaces here, once, before new work is queued.
inline speca_status_t check_sticky(speca_layer* c) {
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SPECA_OK : cuda_fail(c, e, "earlier CUDA error");
}

inline size_t elem_size(const speca_layer* c) { return c->dtype == SPECA_BF16 ? 2 : 4; }

inline bool on_elements(const speca_layer* c, const void* p) { return reinterpret_cast<uintptr_t>(p) % elem_size(c) == 0; }
// The stride of a dimension of one element says nothing: it is taken out of the checks and the addresses.
inline void drop_stride(int64_t count, int64_t& stride) {
    if (count <= 1) stride = 0;
}
// Whether two of rows x heads pieces of `dim` elements with these strides share an element.
inline bool meets_itself(int64_t rows, int64_t row, int64_t heads, int64_t head, int64_t dim) {
    if (rows == 0 || (rows > 1 && row < dim) || (heads > 1 && head < dim)) return rows != 0;
    if (rows <= 1 || heads <= 1) return false;
    using Wide = __int128;
    if (row >= Wide(heads - 1) * head + dim || head >= Wide(rows - 1) * row + dim) return false;
    // pieces of different rows in turn: head j of a row against head 0 of the rows next to it
    for (int64_t j = 1; j < heads; ++j) {
        const Wide at = Wide(j) * head, r = at / row, behind = at - r * row;
        if ((r < rows && behind < dim) || (r + 1 < rows && row - behind < dim)) return true;
    }
    return false;
}
// Rows that start on 16 bytes everywhere: an absent tensor does not stand in the way.
inline bool on_16(const speca_layer* c, const void* p, int64_t s0, int64_t s1) {
    if (p == nullptr) return true;
    const int64_t e = static_cast<int64_t>(elem_size(c));
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && s0 * e % 16 == 0 && s1 * e % 16 == 0;
}

}  // namespace speca
