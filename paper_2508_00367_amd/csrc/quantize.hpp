// Device code of the 8-bit quantization, shared by the kernels that form 8-bit rows (quantize.hip, residual_norm.hip).
#pragma once

#include <float.h>

#include "common.hpp"

namespace rs {

// The larger magnitude; a NaN on either side stays (fmaxf would drop it).  Magnitudes are non-negative floats: their order is that of
// their bits as unsigned numbers, with the infinity above every number and the NaNs above it.
__device__ __forceinline__ float amax_step(float a, float b) {
    const uint32_t x = __float_as_uint(a), y = __float_as_uint(b) & 0x7fffffffu;
    return __uint_as_float(x > y ? x : y);
}

struct QuantScale {
    float scale, inv;
};
__device__ __forceinline__ QuantScale quant_scale(float amax) {
    if (!(amax <= FLT_MAX)) return {__uint_as_float(0x7fc00000u), 0.f};
    const float scale = fmaxf(amax * (float)(1.0 / 127.0), FLT_MIN);
    return {scale, 1.0f / scale};
}
// (A row that is not finite has inv = 0: infinity and NaN times 0 are NaN, whose conversion gives 0; the other values give 0.)
__device__ __forceinline__ int quant8(float x, QuantScale s) {
    const float r = rintf(x * s.inv);
    return r == r ? (int)r : 0;
}

// Four of them as the bytes of a word.  Rounding by adding 1.5 * 2^23: |x inv| <= 127 (1 + 2^-22), and in that range the sum's
// last bit is 1, so that the add rounds to whole numbers, halves to even, and the integer, in two's complement, is the low byte.
// (A NaN would leave its own low byte: a row that is not finite goes by inv = 0 and gives 0 for all its finite values;
// the products of the others are NaN, and are masked.)
__device__ __forceinline__ uint32_t quant8x4(float a, float b, float c, float d, QuantScale s) {
#pragma clang fp contract(off)  // the product is rounded before the sum
    constexpr float magic = 12582912.0f;
    if (s.inv == 0.f) return 0u;
    const uint32_t x = __float_as_uint(a * s.inv + magic), y = __float_as_uint(b * s.inv + magic);
    const uint32_t z = __float_as_uint(c * s.inv + magic), w = __float_as_uint(d * s.inv + magic);
    // bytes 0 of x, y and of z, w side by side, then the halves
    const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x0c0c0400u), hi = __builtin_amdgcn_perm(w, z, 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

}  // namespace rs
