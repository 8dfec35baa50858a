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
__device__ __forceinline__ float wave_amax(float v) { return lanes_reduce<64>(v, [](float a, float b) { return amax_step(a, b); }); }

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

}  // namespace rs
