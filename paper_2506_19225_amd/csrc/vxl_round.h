// Rounding of results to bf16.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vxl {

// To the nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t f32_to_bf16(float v) {
    uint32_t b = __float_as_uint(v);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0x7fc0;
    b += 0x7fffu + ((b >> 16) & 1u);
    return (uint16_t)(b >> 16);
}

}  // namespace vxl
