// Internal declarations shared by the verification layer's host dispatch (speca_layer.cpp) and its
// kernels (speca_layer_rows.cu, speca_attention_*.cu). Not part of the public ABI.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "speca.h"

namespace speca {

// ---- row kernels --------------------------------------------------------------------------------
struct ModulateParams {
    const uint16_t* row_seq;  // sequence of every query row
    const uint8_t* dev_mask;
    const char *x, *branch, *gate, *scale, *shift;
    char *x_out, *y;
    int64_t x_stride, branch_stride, mod_stride, x_out_stride, y_stride;  // elements
    int32_t rows, dim;
    float eps;
};
// `vec`: elements per access (16 bytes of them, or 1 where a pointer, a stride or dim does not allow it)
cudaError_t launch_modulate(const ModulateParams& p, int dtype, int vec, cudaStream_t stream);

// Frequency of one pair of a head in turns (2 pi) per unit of position, and the axis it turns by (-1: kept).
struct RopePair {
    double turns;
    int32_t axis;
    int32_t pad;
};
struct RopeParams {
    const uint16_t* row_seq;
    const uint8_t* dev_mask;
    const RopePair* pairs;  // [head_dim / 2]
    const char *q, *k, *q_weight, *k_weight;
    char *q_out, *k_out;
    const float* positions;
    int64_t q_row, q_head, qo_row, qo_head, k_row, k_head, ko_row, ko_head;  // strides, elements
    int32_t rows, n_heads, n_kv_heads, head_dim, n_axes;
    int32_t rotated;  // elements of a head that turn
    int32_t half;  // HALVES: distance of a pair's elements (R / 2); 0 = INTERLEAVED
    float eps;
};
cudaError_t launch_rope(const RopeParams& p, int dtype, bool vectors, cudaStream_t stream);

// ---- attention ----------------------------------------------------------------------------------
// One unit: a block of packed rows of one (sequence, key head), against one share of the
// sequence's key tiles. Packed row r of a sequence is query r / group, query head kv_head * group + r % group:
// the heads that share a key head share its tiles.
struct AttnUnit {
    int32_t seq, kv_head;
    int32_t row0;     // first packed row
    int32_t q_len, kv_cap;
    int32_t q_start, kv_start;
    int32_t split, n_splits;
    int32_t narrow;   // the unit takes shares split and split + 1 of the keys, for rows of one block
    int64_t part;     // n_splits > 1: byte offset of the partial results of split 0 of this unit's rows
};
static_assert(sizeof(AttnUnit) == 48, "three 16-byte loads");

// Rows whose keys were shared out: their partial results are joined by a launch of its own.
struct JoinBlock {
    int32_t seq, kv_head, row0, rows, q_start, n_splits;
    int64_t part;
};
static_assert(sizeof(JoinBlock) == 32, "two 16-byte loads");

struct AttnParams {
    const AttnUnit* units;
    const JoinBlock* joins;
    int32_t n_units, n_joins, join_rows;  // join_rows: the most rows of a block
    int32_t n_heads, n_kv_heads, group, head_dim;
    int32_t causal, total_q;
    int32_t k_step, v_step;  // 0: all key heads are one in memory, else 1
    int32_t vectors;   // every row starts on 16 bytes and holds a multiple of 4 elements
    float scale_log2;  // scale * log2(e)
    const char *q, *k, *v;
    char* o;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;  // elements
    const int32_t* dev_kv_len;
    const uint8_t* dev_mask;
    float* lse;
    char* parts;        // partial results of shared rows
    uint32_t* gave_up;  // set by a wait that ran out
};
constexpr int kSimtRows = 32, kSimtKeys = 64;  // rows of a unit, keys of a tile
cudaError_t launch_attention_f32(const AttnParams& p, cudaStream_t stream);
// Rows of a unit: two blocks of up to 128, whole queries. NotSupported: the copy engine cannot address a tensor.
__host__ __device__ constexpr int tc_block_rows(int group) { return 128 / group * group; }
constexpr int kTcKeys = 128;
cudaError_t launch_attention_bf16(const AttnParams& p, int64_t total_kv, int sm_count, cudaStream_t stream);

// Joins the partial results of shared rows, behind either attention kernel on the same stream.
cudaError_t launch_attention_join(const AttnParams& p, int dtype, cudaStream_t stream);

// Partial result of one row: head_dim sums, then the running maximum (log2 domain), the sum of the weights and what the
// sums divide by (the same, but for the rounding of the largest weights to bf16).
__host__ __device__ constexpr int64_t part_row_floats(int head_dim) { return (head_dim + 3) / 4 * 4 + 4; }

}  // namespace speca
