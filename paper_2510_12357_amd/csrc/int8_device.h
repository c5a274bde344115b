// Device-side pieces of the 8-bit product: the code of a value, and an output from its exact sum.
#pragma once

#include <math.h>

#include "internal.h"
#include "unaligned.h"

namespace mm {
namespace {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(uint16_t v) { return __uint_as_float((unsigned)v << 16); }
template <typename S> __device__ __forceinline__ S to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t to_out<uint16_t>(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

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

// The values k .. k + N of a row of K floats, zeros behind its end.
template <typename X, int N>
__device__ __forceinline__ void load_floats(const X* row, int k, int K, float (&v)[N]) {
  if (k + N <= K) {
    const Unaligned<X, N> raw = *reinterpret_cast<const Unaligned<X, N>*>(row + k);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_f32(raw.v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = k + i < K ? to_f32(row[k + i]) : 0.f;
  }
}
// The largest magnitude as bits: they compare as the magnitudes do, and a NaN or an infinity is above every number.
template <int N>
__device__ __forceinline__ unsigned magnitude(const float (&v)[N]) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
// What a row's largest magnitude says: its codes and its scale.
struct RowScale {
  unsigned top; bool bad; CodeScale code;
  __device__ __forceinline__ explicit RowScale(unsigned m) : top(m), bad(m >= 0x7f800000u), code(__uint_as_float(m)) {}
  __device__ __forceinline__ float scale() const { return bad ? NAN : __uint_as_float(top) / 127.f; }
};
template <int N>
__device__ __forceinline__ void store_codes(void* p, const RowScale& r, const float (&v)[N]) {
  unsigned w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    w[i] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[i] |= (unsigned)(r.code.code(v[4 * i + j]) & 0xff) << (8 * j);
    w[i] = r.bad ? 0u : w[i];
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) static_cast<unsigned*>(p)[i] = w[i];
}

typedef __attribute__((ext_vector_type(4))) int i32x4;
// The first `left` (1 .. 16) of the 16 codes at p, zeros behind them.
__device__ __forceinline__ i32x4 masked_codes(const int8_t* p, int left) {
  i32x4 v = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = left - 4 * i;
    if (n < 4) v[i] &= n <= 0 ? 0 : (1 << (8 * n)) - 1;
  }
  return v;
}

// One output from its exact sum; every kernel of the product ends with this, so that its bits do not depend on the kernel.
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale) { return ((float)sum * x_scale) * w_scale; }
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale, float bias) { return fmaf((float)sum * x_scale, w_scale, bias); }

}  // namespace
}  // namespace mm
