// What the 8-bit products share: operands' tensor maps, activations, the epilogue of a warp.
#pragma once
#include "speca_eight_common.cuh"
#include "speca_rows_common.cuh"
#include "speca_tc.cuh"

namespace speca {
namespace {

// GELU and SILU are both t * sigmoid(s) = t / (1 + 2^x), x = -s log2(e); so negative t keep their digits, which 1 + tanh would cost.
// GELU: x = t (kGelu1 + kGelu3 t^2), with 2 sqrt(2 / pi) log2(e) and 0.044715 of it; SILU: x = kSilu1 t.
constexpr float kGelu1 = static_cast<float>(-1.5957691216057308 * 1.4426950408889634), kGelu3 = static_cast<float>(-0.044715 * 1.5957691216057308 * 1.4426950408889634);
constexpr float kSilu1 = -1.4426950408889634f;
__device__ __forceinline__ float times_sigmoid(float t, float x) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return t * r;
}
__device__ __forceinline__ float activate(float t, int act) {
    return act == SPECA_ACT_GELU ? times_sigmoid(t, t * fmaf(t * t, kGelu3, kGelu1)) : act == SPECA_ACT_SILU ? times_sigmoid(t, t * kSilu1) : t;
}

// Four consecutive elements of a row of `n`, from c on, where they exist; zeros elsewhere.
template <typename T>
__device__ __forceinline__ void load4(const char* base, int64_t row, int64_t stride, int c, int n, bool vectors, float (&out)[4]) {
    const T* from = reinterpret_cast<const T*>(base) + row * stride + c;
    if (vectors && c + 4 <= n) {
        const Pack<T, 4> v = *reinterpret_cast<const Pack<T, 4>*>(from);
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = to_float(v.e[e]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = c + e < n ? to_float(from[e]) : 0.f;
}

// The epilogue of one block of 128 columns of row `row`, from column n0 on: lane l holds the sums of columns n0 + 4 l .. + 3.
// The whole warp calls.
template <int DT>
__device__ __forceinline__ void finish_block(const Matmul8Params& p, int row, int seq, int n0, int lane, float (&v)[4]) {
    using T = typename Type<DT>::T;
    const int c = n0 + 4 * lane;
    if (p.bias != nullptr) {
        float b[4];
        load4<T>(p.bias, 0, 0, c, p.n, p.vectors, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += b[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = c + e < p.n ? activate(v[e], p.act) : 0.f;
    if (p.out == nullptr) {
        const uint32_t byte = scale_byte(block_top<4, 16>(v));
        const float inv = inverse_of(byte);
        const uint32_t codes = pack_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        uint8_t* to = p.out8.codes + row * p.out8.code_stride + c;
        if (p.vectors && c + 4 <= p.n) {
            *reinterpret_cast<uint32_t*>(to) = codes;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < p.n) to[e] = static_cast<uint8_t>(codes >> 8 * e);
        }
        if (lane == 0)
            p.out8.scales[n0 / (4 * kBlock8) * p.out8.scale_stride + 4 * static_cast<int64_t>(row) + n0 / kBlock8 % 4] =
                static_cast<uint8_t>(byte);
        return;
    }
    if (p.gate != nullptr) {
        float g[4];
        load4<T>(p.gate, seq, p.gate_stride, c, p.n, p.vectors, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= g[e];
    }
    if (p.residual != nullptr) {
        float r[4];
        load4<T>(p.residual, row, p.residual_stride, c, p.n, p.vectors, r);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += r[e];
    }
    T* to = reinterpret_cast<T*>(p.out) + row * p.out_stride + c;
    if (p.vectors && c + 4 <= p.n) {
        Pack<T, 4> o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o.e[e] = from_float<T>(v[e]);
        *reinterpret_cast<Pack<T, 4>*>(to) = o;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < p.n) to[e] = from_float<T>(v[e]);
    }
}

// [rows, k] bytes as boxes of 128 bytes x box_rows; what lies behind either end reads as zero.
bool encode8(CUtensorMap* map, const uint8_t* base, int k, int rows, int64_t stride, int box_rows) {
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(k), static_cast<cuuint64_t>(rows)};
    // a dimension of one element is never stepped through: any multiple of 16 will do
    const cuuint64_t strides[1] = {rows > 1 ? static_cast<cuuint64_t>(stride) : 128};
    const cuuint32_t box[2] = {128, static_cast<cuuint32_t>(box_rows)}, ones[2] = {1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace speca
