// 4-bit rows for quantised K/V slabs (device side).  With y = x * (1 / channel scale) in fp32 (the reciprocal is the
// caller's), a row's scale is s = max |y| / 7 and an element's code u = clamp(rint(y / s), -7, 7) + 8 in 1 .. 15 (8 in a
// row of zeros); it stands for (u - 8) * s * channel scale.  Both quotients are IEEE divisions, so every
// implementation that divides in fp32 gets the same codes bit for bit (baklava_tree_commit does with BAKLAVA_FLAG_ROW_QUOTIENT).  A byte holds an even channel in its low half
// and the next one in its high half.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace int4q {

// four bf16 values times the reciprocals of their channel scales
__device__ __forceinline__ void scaled4(uint2 raw, float4 inv, float (&y)[4]) {
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.x));
    const float2 b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw.y));
    y[0] = __fmul_rn(a.x, inv.x); y[1] = __fmul_rn(a.y, inv.y);
    y[2] = __fmul_rn(b.x, inv.z); y[3] = __fmul_rn(b.y, inv.w);
}
// bits of the largest magnitude (bits of non-negative floats order like the floats; a NaN comes out on top)
template <int N>
__device__ __forceinline__ uint32_t largest_bits(const float (&y)[N]) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
    return top;
}
__device__ __forceinline__ float row_scale(uint32_t top_bits) { return __fdiv_rn(__uint_as_float(top_bits), 7.0f); }
__device__ __forceinline__ uint32_t code(float y, float s) {
    return s > 0.0f ? (uint32_t)((int)fminf(fmaxf(rintf(__fdiv_rn(y, s)), -7.0f), 7.0f) + 8) : 8u;
}
__device__ __forceinline__ uint32_t codes4(const float (&y)[4], float s) {
    return code(y[0], s) | (code(y[1], s) << 4) | (code(y[2], s) << 8) | (code(y[3], s) << 12);
}

}  // namespace int4q
