// Rotary positions (moe_rope), and new keys and values stored in a paged cache with the rotation on the way (moe_kv_append).
//
// Pairs of channels (a, b) turn by t = pos freq: a' = m (a cos t - b sin t), b' = m (b cos t + a sin t).  A workgroup has a few tokens, works out their sines and cosines
// once, one a thread, into LDS, and turns V pairs a lane of head after head; of a row's lanes each has the same pairs in all heads, so that they stay in registers.
// What bounds it: reading and writing; few tokens, the launch.  4096 tokens of 40 heads of 128 channels, bf16 (84 MB) 16.7 us, 5.0 TB/s; an append of 16384 tokens of 32 + 8 + 8 heads
// (400 MB) 79 us, 5.1 TB/s; of 2111 tokens into 8 bits 9.1 us (copies reach 4.7 TB/s over 84 MB, 5.5 over 400 MB).  With eight sines a lane and head instead, 19.7, 87 and 13.4 us.
#include <algorithm>

#include "internal.h"
#include "unaligned.h"

namespace mm {
namespace {

constexpr int kThreads = 256;
constexpr float kCodeMax = 448.f;          // the largest E4M3 value

// cos and sin of 2 pi times the turns.  What is left of the turns is exact in 64 bits; the turns themselves, a product with two roundings and a rounded constant, are at
// most 3 2^-53 of them off: at 2^20 of them 2^-31 of a turn.  A quarter turn's rest, at most 1/2, goes through the Taylor series of sine and cosine to the eleventh and
// twelfth power: the next terms are below 2^-33.
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
  static __device__ __forceinline__ type load(const X* p) { return load_unaligned<type>(p); }
  static __device__ __forceinline__ void widened(const type& x, float* v) {
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
  typedef X type;
  static __device__ __forceinline__ type load(const X* p) { return *p; }
  static __device__ __forceinline__ void widened(const type& x, float* v) { v[0] = widen<X>(x); }
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

// X: type of queries, keys and values; V: pairs of a unit, which divides a row's pairs that turn and those that do not; UNITS: units of a lane, a row's lanes
// apart.  C: type of the cache's rows.  A workgroup has `tokens` tokens (a power of two) and of each the heads of its part of the grid's second dimension.
constexpr int kAngles = 256;               // of a workgroup
template <typename X, typename C, int V, int UNITS, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a, const int lanes_log, const int tokens, const int heads_each) {
  constexpr bool kCodes = sizeof(C) == 1;
  constexpr int kAhead = sizeof(X) == 4 || kCodes ? 2 : 4;  // heads whose loads are on their way together: registers for more cost waves
  constexpr bool kApart = !HALF && V > 1;                   // a lane's two chunks are half a row apart, each of whole pairs, so that lanes' are neighbours
  typedef Chunk<X, V> Ch;
  __shared__ __attribute__((aligned(16))) float s_cos[kAngles], s_sin[kAngles];
  const int lanes = 1 << lanes_log, j = threadIdx.x & (lanes - 1), row = threadIdx.x >> lanes_log, rows = (kThreads >> lanes_log) / tokens;
  const int units = a.D / (2 * V), half = a.rotary_dim / 2, turning = half / V;
  const int t0 = blockIdx.x * tokens, local = row / rows, t = t0 + local;
  for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
    const int token = i / half;
    float c = 1.f, s = 0.f;
    if (t0 + token < a.T) turn((double)a.pos[t0 + token] * (a.freq[i - token * half] * 0.15915494309189533577), &c, &s);
    s_cos[i] = c * a.mscale;
    s_sin[i] = s * (a.mscale * a.sign);
  }
  // where the key and value of this token go
  int64_t page = -1, slot = 0;
  if (a.kv_heads && t < a.T) {
    const int pos = a.pos[t], seq = a.seq ? a.seq[t] : a.first_seq + t;
    if (pos >= 0 && seq >= 0 && seq < a.n_seqs) page = page_of(a.table + seq * a.table_ld, a.table_len, a.n_pages, a.shift, pos);
    slot = pos & ((1 << a.shift) - 1);
  }
  __syncthreads();
  const int first = blockIdx.y * heads_each, heads = t < a.T ? min(page >= 0 ? a.heads + 2 * a.kv_heads : a.heads, first + heads_each) : 0;
  float c[UNITS][V], s[UNITS][V];
  int o0[UNITS], o1[UNITS];
  bool turns[UNITS][2], there[UNITS];                       // the first half of a lane's pairs, the others
#pragma unroll
  for (int k = 0; k < UNITS; ++k) {
    const int u = j + k * lanes;
    there[k] = u < units;
    turns[k][0] = turns[k][1] = u < turning;
    o0[k] = HALF && u < turning ? u * V : 2 * u * V;
    o1[k] = HALF && u < turning ? half + u * V : o0[k] + V;
    if constexpr (kApart) {
      o0[k] = u * V;
      o1[k] = (units + u) * V;
      turns[k][0] = o0[k] < a.rotary_dim;
      turns[k][1] = there[k] && o1[k] < a.rotary_dim;
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const bool turned = turns[k][2 * e >= V];
      const int angle = local * half + (!kApart ? u * V + e : 2 * e < V ? o0[k] / 2 + e : o1[k] / 2 + e - V / 2);
      c[k][e] = turned ? s_cos[angle] : 1.f;
      s[k][e] = turned ? s_sin[angle] : 0.f;
    }
  }
  for (int h0 = first + row % rows; h0 < heads; h0 += kAhead * rows) {
    typename Ch::type x0[kAhead][UNITS], x1[kAhead][UNITS];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * rows, kv = h - a.heads;
      if (h >= heads) continue;
      const X* from = kv < 0 ? static_cast<const X*>(a.q) + t * a.q_token + h * a.q_head
                      : kv >= a.kv_heads ? static_cast<const X*>(a.v) + t * a.v_token + (kv - a.kv_heads) * a.v_head
                                         : static_cast<const X*>(a.k) + t * a.k_token + kv * a.k_head;
#pragma unroll
      for (int k = 0; k < UNITS; ++k)
        if (there[k]) { x0[i][k] = Ch::load(from + o0[k]); x1[i][k] = Ch::load(from + o1[k]); }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h0 + i * rows, kv = h - a.heads;
      if (h >= heads) continue;
      const bool value = kv >= a.kv_heads;
      float y[UNITS][2 * V];
#pragma unroll
      for (int k = 0; k < UNITS; ++k) {
        if (!there[k]) continue;
        float x[2 * V];
        Ch::widened(x0[i][k], x);
        Ch::widened(x1[i][k], x + V);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int ia = HALF ? e : 2 * e, ib = HALF ? V + e : 2 * e + 1;
          const float p = x[ia], q = x[ib];
          const bool moves = turns[k][2 * e >= V] && !value;
          y[k][ia] = moves ? fmaf(p, c[k][e], -(q * s[k][e])) : p;
          y[k][ib] = moves ? fmaf(q, c[k][e], p * s[k][e]) : q;
        }
      }
      if (kv < 0) {
        X* to = static_cast<X*>(a.q_out) + t * a.out_token + h * a.out_head;
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
          if (!there[k]) continue;
          Ch::store(to + o0[k], y[k]);
          Ch::store(to + o1[k], y[k] + V);
        }
        continue;
      }
      const int head = value ? kv - a.kv_heads : kv;
      C* to = static_cast<C*>(value ? a.v_cache : a.k_cache) + page * a.page + head * a.head + slot * a.row;
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
          scales[((page * a.kv_heads + head) << a.shift) + slot] = finite ? most / kCodeMax : __uint_as_float(0x7fc00000u);
        }
        // quotients by the reciprocal and one step that takes the rest into account; rows of the smallest numbers times 2^64 and of the largest times 2^-64, exactly, so that the
        // reciprocal and 448 y are finite
        const float lift = most < 1e-30f ? 0x1p64f : most > 1e30f ? 0x1p-64f : 1.f, divisor = most * lift, over = 1.f / divisor, by = kCodeMax * lift;
#pragma unroll
        for (int k = 0; k < UNITS; ++k) {
          if (!there[k]) continue;
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) {
            const float n = by * y[k][e], rest = fmaf(by, y[k][e], -n), q = n * over;     // 448 y takes up to three bits more than y
            y[k][e] = finite && top ? fmaf(fmaf(-q, divisor, n) + rest, over, q) : 0.f;
          }
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
  const int units = a.D / (2 * V), heads = a.heads + 2 * a.kv_heads, half = a.rotary_dim / 2;
  int lanes_log = 0;
  while ((UNITS << lanes_log) < units) ++lanes_log;
  const int slots = kThreads >> lanes_log;
  int tokens = 1;
  while (2 * tokens <= slots && 2 * tokens * half <= kAngles && 2 * tokens <= a.T && (a.T / (2 * tokens) >= 1024 || slots / (2 * tokens) >= heads)) tokens *= 2;
  // few tokens: their heads over more workgroups
  const int rows = slots / tokens;
  const int64_t blocks = ((int64_t)a.T + tokens - 1) / tokens;
  const int turns = (heads + rows - 1) / rows, parts = (int)std::max<int64_t>(1, std::min<int64_t>(turns, 1024 / blocks));
  const int heads_each = (turns + parts - 1) / parts * rows;
  ProfScope prof(kProfRotary, s);
  // a grid of 2^32 threads and more would run as what is left of it modulo 2^32
  for (int64_t t = 0; t < a.T; t += (int64_t)tokens << 20) {
    RotaryArgs p = a;
    p.T = (int)std::min<int64_t>(a.T - t, (int64_t)tokens << 20);
    const int64_t x = t * (int64_t)sizeof(X);
    auto moved = [](const void* q, int64_t bytes) { return q ? static_cast<const char*>(q) + bytes : nullptr; };
    p.q = moved(a.q, x * a.q_token); p.k = moved(a.k, x * a.k_token); p.v = moved(a.v, x * a.v_token); p.q_out = const_cast<char*>(moved(a.q_out, x * a.out_token));
    p.pos = a.pos + t;
    p.seq = a.seq ? a.seq + t : nullptr;
    p.first_seq = (int)t;
    const dim3 grid((p.T + tokens - 1) / tokens, (heads + heads_each - 1) / heads_each);
    if (a.layout == MOE_ROPE_HALF) rotary_kernel<X, C, V, UNITS, true><<<grid, kThreads, 0, s>>>(p, lanes_log, tokens, heads_each);
    else rotary_kernel<X, C, V, UNITS, false><<<grid, kThreads, 0, s>>>(p, lanes_log, tokens, heads_each);
  }
  return hip_fail(hipGetLastError(), "rotary_kernel");
}

template <typename X, typename C>
int launch_typed(const RotaryArgs& a, hipStream_t s) {
  // units of V pairs that divide the pairs that turn and those that do not
  const int both = a.rotary_dim / 2 | (a.D - a.rotary_dim) / 2;
  if constexpr (sizeof(X) == 2)
    if (both % 8 == 0) return launch_units<X, C, 8, 1>(a, s);
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
