// Rotary positions (moe_rope), and new keys and values stored in a paged cache with the rotation on the way (moe_kv_append).
//
// Pairs of channels (a, b) turn by t = pos freq: a' = m (a cos t - b sin t), b' = m (b cos t + a sin t).  A group of lanes takes a token: a lane has
// V pairs of channels, computes their sines and cosines once and turns them in several heads.
#include <algorithm>

#include "internal.h"
#include "unaligned.h"

namespace mm {
namespace {

constexpr int kThreads = 256;
constexpr float kCodeMax = 448.f;          // the largest E4M3 value

// cos and sin of 2 pi times the turns.  What is left of the turns is exact in 64 bits (at 2^20 turns a position and 2^31 positions 2^-2 of the last
// place of fp32's quarter turn would be lost: the bound of the documentation keeps the product's error below 2^-53 of it).  A quarter turn's rest, at
// most 1/2, goes through the Taylor series of sine and cosine to the eleventh and twelfth power: the next terms are below 2^-33.
__device__ __forceinline__ void turn(double turns, float* c, float* s) {
  const double quarters = 4.0 * (turns - floor(turns));
  const double whole = rint(quarters);
  const int n = (int)whole;
  const float x = (float)((quarters - whole) * 1.57079632679489661923);
  const float z = x * x;
  float p = fmaf(z, -2.50521083854417188e-8f, 2.75573192239858907e-6f);
  p = fmaf(z, p, -1.98412698412698413e-4f);
  p = fmaf(z, p, 8.33333333333333333e-3f);
  p = fmaf(z, p, -1.66666666666666667e-1f);
  const float sine = fmaf(x * z, p, x);
  float q = fmaf(z, 2.08767569878680990e-9f, -2.75573192239858907e-7f);
  q = fmaf(z, q, 2.48015873015873016e-5f);
  q = fmaf(z, q, -1.38888888888888889e-3f);
  q = fmaf(z, q, 4.16666666666666667e-2f);
  q = fmaf(z, q, -0.5f);
  const float cosine = fmaf(z, q, 1.f);
  const float u = n & 1 ? cosine : sine, v = n & 1 ? sine : cosine;
  *s = n & 2 ? -u : u;
  *c = (n + 1) & 2 ? -v : v;
}

template <typename X>
__device__ __forceinline__ float widen(X x) { return (float)x; }

template <typename X, int N>
struct Chunk {
  typedef X type __attribute__((ext_vector_type(N)));
  static __device__ __forceinline__ void load(const X* p, float* v) {
    const type x = load_unaligned<type>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = widen<X>(x[i]);
  }
  static __device__ __forceinline__ void store(X* p, const float* v) {
    type x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (X)v[i];
    store_unaligned(p, x);
  }
};
template <typename X>
struct Chunk<X, 1> {
  static __device__ __forceinline__ void load(const X* p, float* v) { v[0] = widen<X>(*p); }
  static __device__ __forceinline__ void store(X* p, const float* v) { *p = (X)v[0]; }
};
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* p, const float* v) {
  if constexpr (N == 1) {
    *p = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[0], 0, false);
  } else if constexpr (N == 2) {
    *reinterpret_cast<uint16_t*>(p) = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[i], v[i + 1], 0, false);
      *reinterpret_cast<int*>(p + i) = __builtin_amdgcn_cvt_pk_fp8_f32(v[i + 2], v[i + 3], lo, true);
    }
  }
}

// X: type of queries, keys and values; V: pairs of a unit, which divides a row's pairs that turn and those that do not; UNITS: units of a lane, a token's lanes
// apart.  C: type of the cache's rows.
template <typename X, typename C, int V, int UNITS, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, const int lanes_log, const int slices) {
  constexpr bool kCodes = sizeof(C) == 1;
  const int lanes = 1 << lanes_log, j = threadIdx.x & (lanes - 1);
  const int units = a.D / (2 * V), half = a.rotary_dim / 2, turning = half / V;
  const unsigned step = gridDim.x * (kThreads >> lanes_log), groups = (unsigned)a.T * (unsigned)slices;      // below 2^31, so that no sum passes 2^32
  for (unsigned at = blockIdx.x * (kThreads >> lanes_log) + (threadIdx.x >> lanes_log); at < groups; at += step) {
    const int t = (int)(at / (unsigned)slices), slice = (int)at - t * slices;
    const int pos = a.pos[t];
    // where the key and value of this token go
    int64_t slot = -1, row = 0;
    if (a.kv_heads && pos >= 0) {
      const int seq = a.seq ? a.seq[t] : t;
      const int page = seq >= 0 && seq < a.n_seqs ? page_of(a.table + seq * a.table_ld, a.table_len, a.n_pages, a.shift, pos) : -1;
      row = pos & ((1 << a.shift) - 1);
      slot = page;
    }
    const int heads = slot >= 0 ? a.heads + 2 * a.kv_heads : a.heads;
    if (slice >= heads) continue;
    float c[UNITS][V], s[UNITS][V];
    int o0[UNITS], o1[UNITS];
    bool turns[UNITS], there[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
      const int u = j + k * lanes;
      there[k] = u < units;
      turns[k] = u < turning;
      o0[k] = turns[k] ? (HALF ? u * V : 2 * u * V) : 2 * u * V;
      o1[k] = turns[k] && HALF ? half + u * V : o0[k] + V;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        c[k][e] = 1.f; s[k][e] = 0.f;
        if (turns[k]) {
          turn((double)pos * (a.freq[u * V + e] * 0.15915494309189533577), &c[k][e], &s[k][e]);
          c[k][e] *= a.mscale; s[k][e] *= a.mscale * a.sign;
        }
      }
    }
    for (int h = slice; h < heads; h += slices) {
      const int kv = h - a.heads;
      const bool value = kv >= a.kv_heads;
      const X* from = kv < 0 ? static_cast<const X*>(a.q) + t * a.q_token + h * a.q_head
                      : value ? static_cast<const X*>(a.v) + t * a.v_token + (kv - a.kv_heads) * a.v_head
                              : static_cast<const X*>(a.k) + t * a.k_token + kv * a.k_head;
      float x[UNITS][2 * V], y[UNITS][2 * V];
#pragma unroll
      for (int k = 0; k < UNITS; ++k) {
        if (!there[k]) continue;
        Chunk<X, V>::load(from + o0[k], x[k]);
        Chunk<X, V>::load(from + o1[k], x[k] + V);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int ia = HALF ? e : 2 * e, ib = HALF ? V + e : 2 * e + 1;
          const float p = x[k][ia], q = x[k][ib];
          const bool moves = turns[k] && !value;
          y[k][ia] = moves ? fmaf(p, c[k][e], -(q * s[k][e])) : p;
          y[k][ib] = moves ? fmaf(q, c[k][e], p * s[k][e]) : q;
        }
      }
      if (kv < 0) {
        X* to = static_cast<X*>(a.q_out) + t * a.out_token + h * a.out_head;
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
          if (!there[k]) continue;
          Chunk<X, V>::store(to + o0[k], y[k]);
          Chunk<X, V>::store(to + o1[k], y[k] + V);
        }
        continue;
      }
      const int head = value ? kv - a.kv_heads : kv;
      C* to = static_cast<C*>(value ? a.v_cache : a.k_cache) + slot * a.page + head * a.head + row * a.row;
      if constexpr (kCodes) {
        unsigned top = 0;
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
          if (!there[k]) continue;
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) top = max(top, __float_as_uint(y[k][e]) & 0x7fffffffu);     // of floats' magnitudes the order is that of their bits
        }
        for (int o = lanes / 2; o; o >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
        const bool finite = top < 0x7f800000u;
        const float most = __uint_as_float(top);
        if (j == 0) {
          float* scales = value ? a.v_scale : a.k_scale;
          scales[((int64_t)slot * a.kv_heads + head) * ((int64_t)1 << a.shift) + row] = finite ? most / kCodeMax : __uint_as_float(0x7fc00000u);
        }
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
          if (!there[k]) continue;
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) y[k][e] = finite && top ? kCodeMax * y[k][e] / most : 0.f;
          store_codes<V>((uint8_t*)to + o0[k], y[k]);
          store_codes<V>((uint8_t*)to + o1[k], y[k] + V);
        }
      } else {
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
          if (!there[k]) continue;
          Chunk<C, V>::store(to + o0[k], y[k]);
          Chunk<C, V>::store(to + o1[k], y[k] + V);
        }
      }
    }
  }
}

template <typename X, typename C, int V, int UNITS>
int launch_units(const RotaryArgs& a, hipStream_t s) {
  const int units = a.D / (2 * V), rows = a.heads + 2 * a.kv_heads;
  int lanes_log = 0;
  while ((UNITS << lanes_log) < units) ++lanes_log;
  const int slices = (int)std::min<int64_t>(rows, std::max<int64_t>(1, (int64_t)(1 << 19) / ((int64_t)a.T << lanes_log)));
  const int per = kThreads >> lanes_log;
  const int blocks = (int)std::min<int64_t>(((int64_t)a.T * slices + per - 1) / per, 1 << 16);
  ProfScope prof(kProfRotary, s);
  if (a.layout == MOE_ROPE_HALF) rotary_kernel<X, C, V, UNITS, true><<<blocks, kThreads, 0, s>>>(a, lanes_log, slices);
  else rotary_kernel<X, C, V, UNITS, false><<<blocks, kThreads, 0, s>>>(a, lanes_log, slices);
  return hip_fail(hipGetLastError(), "rotary_kernel");
}

template <typename X, typename C>
int launch_typed(const RotaryArgs& a, hipStream_t s) {
  // units of V pairs that divide the pairs that turn and those that do not
  const int both = a.rotary_dim / 2 | (a.D - a.rotary_dim) / 2;
  if (both % 8 == 0 && sizeof(X) == 2) return launch_units<X, C, 8, 1>(a, s);
  if (both % 4 == 0) return launch_units<X, C, 4, 1>(a, s);
  if (both % 2 == 0) return launch_units<X, C, 2, 1>(a, s);
  return launch_units<X, C, 1, 2>(a, s);
}

template <typename X>
int launch_from(const RotaryArgs& a, hipStream_t s) {
  switch (a.cache_dtype) {
    case MOE_E4M3: return launch_typed<X, uint8_t>(a, s);
    case MOE_FP32: return launch_typed<X, float>(a, s);
    default: return launch_typed<X, __bf16>(a, s);
  }
}

}  // namespace

int launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  return dtype == MOE_FP32 ? launch_from<float>(a, s) : launch_from<__bf16>(a, s);
}

}  // namespace mm
