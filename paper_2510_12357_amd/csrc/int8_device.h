// Device-side pieces of the 8-bit product: the code of a value, and an output from its exact sum.
#pragma once

#include <math.h>

#include "internal.h"

namespace mm {
namespace {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ void store_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_out(uint16_t* p, float v) { *p = __builtin_bit_cast(uint16_t, (__bf16)v); }

// Codes of a row whose largest magnitude is a: the integer nearest to 127 x / a, ties to even, of the real quotient.
// The fp32 quotient |x| (127 / a) <= 127 is off by at most 127 2^-23 = 1.6e-5, so it decides unless it lies within that of a
// border; there 254 |x| is compared with (2 n + 1) a in 64 bits, where both products are exact (32 bits each).
struct CodeScale {
  float a, inv, up;                       // up: 127 / a stays finite for the smallest a
  __device__ __forceinline__ explicit CodeScale(float amax) {
    up = amax < 0x1p-100f ? 0x1p100f : 1.f;
    a = amax * up;
    inv = a > 0.f ? 127.f / a : 0.f;
  }
  __device__ __forceinline__ int code(float x) const {
    const float v = fabsf(x) * up, t = v * inv;
    float n = rintf(t);
    if (fabsf(t - n) > 0.49996f) {
      n = floorf(t);
      const double d = 254.0 * (double)v - (double)(2.f * n + 1.f) * (double)a;
      if (d > 0.0 || (d == 0.0 && ((int)n & 1))) n += 1.f;
    }
    return (int)copysignf(n, x);
  }
};

// One output from its exact sum; every kernel of the product ends with this, so that its bits do not depend on the kernel.
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale) { return ((float)sum * x_scale) * w_scale; }
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale, float bias) { return fmaf((float)sum * x_scale, w_scale, bias); }

}  // namespace
}  // namespace mm
