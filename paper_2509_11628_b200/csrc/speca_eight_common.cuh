// The 8-bit format: blocks of 128 elements with a power of two as scale, e4m3 codes.
#pragma once
#include <stdint.h>

namespace speca {
namespace {

// Scale byte of a block whose largest finite magnitude is `top`: the smallest e with top <= 448 * 2^e, biased by 127, within
// 1..254. 448 = 1.75 * 2^8: eight binades below top's, one more where top's significand exceeds 1.75. Of zeros: 127, a scale of 1.
__device__ __forceinline__ uint32_t scale_byte(float top) {
    const uint32_t u = __float_as_uint(top);
    const int e = static_cast<int>(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
    return top == 0.f ? 127u : static_cast<uint32_t>(max(e, 1));
}
// 1 / scale, exact: 2^(127 - byte). (A byte is at most 254 - 8 + 1 here.)
__device__ __forceinline__ float inverse_of(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return static_cast<uint32_t>(lo) | static_cast<uint32_t>(hi) << 16;
}

// Largest finite magnitude over the lanes that differ in the bits of OVER, of N values a lane each; infinities become NaN, which the
// code for them is. All lanes of the warp take part.
template <int N, int OVER>
__device__ __forceinline__ float block_top(float* v) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, fabsf(v[i]));  // a NaN is passed over
#pragma unroll
    for (int o = OVER; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float inf = __uint_as_float(0x7f800000u);
    if (__any_sync(0xffffffffu, top == inf)) {
        top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (fabsf(v[i]) == inf) v[i] = __uint_as_float(0x7fffffffu);
            top = fmaxf(top, fabsf(v[i]));
        }
#pragma unroll
        for (int o = OVER; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    return top;
}

}  // namespace
}  // namespace speca
