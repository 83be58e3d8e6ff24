// Device code that the attention kernels share: units and visibility.
#pragma once
#include <cuda_bf16.h>
#include <math_constants.h>

#include "speca_layer_internal.h"

namespace speca {
namespace {

__device__ __forceinline__ AttnUnit load_unit(const AttnUnit* units, int i) {
    AttnUnit u;
    const int4* src = reinterpret_cast<const int4*>(units + i);
    int4* dst = reinterpret_cast<int4*>(&u);
#pragma unroll
    for (int k = 0; k < 3; ++k) dst[k] = __ldg(src + k);
    return u;
}

// Keys of the unit's sequence that hold data.
__device__ __forceinline__ int kv_length(const AttnParams& p, const AttnUnit& u) {
    return p.dev_kv_len == nullptr ? u.kv_cap : max(0, min(u.kv_cap, p.dev_kv_len[u.seq]));
}
// Keys that query `i` of the sequence sees: those in front of this index.
__device__ __forceinline__ int visible_keys(const AttnParams& p, const AttnUnit& u, int kv_len, int i) {
    return p.causal ? max(0, kv_len - max(0, u.q_len - 1 - i)) : kv_len;
}

constexpr float kLn2 = 0.6931471805599453f;

}  // namespace
}  // namespace speca
