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
  // as a float without its sign; near: the quotient decides nothing, exact() has to
  __device__ __forceinline__ float quick(float x, bool& near) const {
    const float t = fabsf(x) * up * inv, n = rintf(t);
    near |= fabsf(t - n) > 0.49996f;
    return n;
  }
  __device__ __forceinline__ float exact(float x) const {
    const float v = fabsf(x) * up, t = v * inv;
    float n = rintf(t);
    if (fabsf(t - n) > 0.49996f) {
      n = floorf(t);
      const double d = 254.0 * (double)v - (double)(2.f * n + 1.f) * (double)a;
      if (d > 0.0 || (d == 0.0 && ((int)n & 1))) n += 1.f;
    }
    return n;
  }
};

typedef __attribute__((ext_vector_type(4))) int i32x4;
// 16 bytes of a row's floats as numbers
template <int N> __device__ __forceinline__ void widen(const i32x4 raw, const float*, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __int_as_float(raw[i]);
}
template <int N> __device__ __forceinline__ void widen(const i32x4 raw, const uint16_t*, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __int_as_float(raw[i] << 16); v[2 * i + 1] = __int_as_float(raw[i] & (int)0xffff0000); }
}
// Vector `at`, `at` + per, .. of a row of K floats that starts at any element: the first HELD of them, zeros behind the row's end.  The row's last
// elements, less than a vector, are one thread's; they are read one by one, apart from the others, which are all on their way by then.
template <typename X, int HELD>
struct HeldRow {
  static constexpr int kVec = 16 / sizeof(X);
  i32x4 raw[HELD];
  __device__ __forceinline__ void load(const X* row, int K, int at, int per) {
    const int whole = K / kVec;
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      raw[u] = i32x4{0, 0, 0, 0};
      if (u * per + at < whole) raw[u] = load_unaligned<i32x4>(row + (u * per + at) * kVec);
    }
    const int rest = K - whole * kVec, u_rest = whole / per;
    if (rest && whole - u_rest * per == at) {
      X e[kVec];
#pragma unroll
      for (int i = 0; i < kVec; ++i) e[i] = i < rest ? row[whole * kVec + i] : X(0);
#pragma unroll
      for (int u = 0; u < HELD; ++u) if (u == u_rest) raw[u] = __builtin_bit_cast(i32x4, e);
    }
  }
  __device__ __forceinline__ void values(int u, float (&v)[kVec]) const { widen(raw[u], static_cast<const X*>(nullptr), v); }
};
// Such a vector by itself, from element k on.
template <typename X, int N>
__device__ __forceinline__ void load_floats(const X* row, int k, int K, float (&v)[N]) {
  HeldRow<X, 1> h;
  h.load(row + k, min(max(K - k, 0), N), 0, 1);
  h.values(0, v);
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
  float n[N];
  bool near = false;
#pragma unroll
  for (int i = 0; i < N; ++i) n[i] = r.code.quick(v[i], near);
  if (near) {                                              // about one vector in a thousand
#pragma unroll
    for (int i = 0; i < N; ++i) n[i] = r.code.exact(v[i]);
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    int q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = (int)copysignf(n[4 * i + j], v[4 * i + j]);
    const unsigned w = __builtin_amdgcn_perm((unsigned)q[1], (unsigned)q[0], 0x0c0c0400u) | __builtin_amdgcn_perm((unsigned)q[3], (unsigned)q[2], 0x04000c0cu);
    static_cast<unsigned*>(p)[i] = r.bad ? 0u : w;
  }
}

// The first `left` of 16 codes (all for 16 and more), zeros behind them.
__device__ __forceinline__ i32x4 keep_codes(i32x4 v, int left) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = left - 4 * i;
    if (n < 4) v[i] &= n <= 0 ? 0 : (1 << (8 * n)) - 1;
  }
  return v;
}
__device__ __forceinline__ i32x4 masked_codes(const int8_t* p, int left) { return keep_codes(*reinterpret_cast<const i32x4*>(p), left); }

// One output from its exact sum; every kernel of the product ends with this, so that its bits do not depend on the kernel.  No bias is one of -0,
// which leaves every product as it is, zeros of either sign too.
constexpr float kNoBias = -0.f;
__device__ __forceinline__ float scaled(int sum, float x_scale, float w_scale, float bias) { return fmaf((float)sum * x_scale, w_scale, bias); }

}  // namespace
}  // namespace mm
