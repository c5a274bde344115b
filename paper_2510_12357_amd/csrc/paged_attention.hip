// Attention of one new token per sequence over a paged cache (moe_paged_attention).
//
// A workgroup has a part of a sequence's positions, one key head and up to 16 of its query heads; its waves take blocks of the part's positions in turn.
// Scores are the product of a tile of keys (rows: positions) and the queries (columns: heads), so that a lane has four positions of one head, which is where the
// product with the values wants the probabilities: nothing moves between lanes.  That product runs on fp32 matrix instructions, whose operands hold one position a lane: values
// are used as their rows lie in memory, and probabilities are not rounded.
// The maximum that exponentials are taken against follows the scores only when one is 2^8 above it: sums stay far below fp32's range, and most blocks neither exchange
// maxima nor rescale.  Waves' sums are joined in LDS, parts' sums by a second kernel, both in a fixed order.
#include <math.h>

#include "internal.h"
#include "groups.h"

namespace mm {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kSlack = 8.f;                               // how far (log2) scores may be above the maximum in use
constexpr int kMaxPages = kMaxSplit / kMinPage;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// N neighbouring elements of a row of the cache, as they lie there and in fp32
template <typename C, int N> struct Raw;
template <> struct Raw<__bf16, 8> { typedef i32x4 type; };
template <> struct Raw<__bf16, 4> { typedef i32x2 type; };
template <> struct Raw<uint8_t, 8> { typedef i32x2 type; };
template <> struct Raw<uint8_t, 4> { typedef int type; };
struct Eight { f32x4 lo, hi; };
template <> struct Raw<float, 8> { typedef Eight type; };
template <> struct Raw<float, 4> { typedef f32x4 type; };

__device__ __forceinline__ int dword(const i32x4& v, int i) { return v[i]; }
__device__ __forceinline__ int dword(const i32x2& v, int i) { return v[i]; }
__device__ __forceinline__ int dword(int v, int) { return v; }
__device__ __forceinline__ i32x4 zeros(i32x4) { return i32x4{0, 0, 0, 0}; }
__device__ __forceinline__ i32x2 zeros(i32x2) { return i32x2{0, 0}; }
__device__ __forceinline__ int zeros(int) { return 0; }
__device__ __forceinline__ f32x4 zeros(f32x4) { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ Eight zeros(Eight) { return {zeros(f32x4{}), zeros(f32x4{})}; }

template <typename C, int N>
__device__ __forceinline__ float element(const typename Raw<C, N>::type& v, int j) {
  if constexpr (sizeof(C) == 2) {
    const unsigned d = (unsigned)dword(v, j / 2);
    return __uint_as_float(j & 1 ? d & 0xffff0000u : d << 16);
  } else if constexpr (sizeof(C) == 1) {
    switch (j & 3) {                                        // the byte is part of the instruction
      case 0: return __builtin_amdgcn_cvt_f32_fp8(dword(v, j / 4), 0);
      case 1: return __builtin_amdgcn_cvt_f32_fp8(dword(v, j / 4), 1);
      case 2: return __builtin_amdgcn_cvt_f32_fp8(dword(v, j / 4), 2);
      default: return __builtin_amdgcn_cvt_f32_fp8(dword(v, j / 4), 3);
    }
  } else if constexpr (N == 8) {
    return j < 4 ? v.lo[j & 3] : v.hi[j & 3];
  } else {
    return v[j];
  }
}
__device__ __forceinline__ bf16x8 as_bf16(const i32x4& v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ bf16x8 as_bf16(const i32x2& v) { return widen_e4m3(v[0], v[1]); }

__device__ __forceinline__ float lane_max(float v) {        // over the four lanes of a column
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float lane_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float load_query(const AttentionArgs& a, int64_t at) {
  return a.dtype == MOE_FP32 ? static_cast<const float*>(a.q)[at] : (float)static_cast<const __bf16*>(a.q)[at];
}
__device__ __forceinline__ void store_out(const AttentionArgs& a, int64_t at, float v) {
  if (a.dtype == MOE_FP32) static_cast<float*>(a.out)[at] = v;
  else static_cast<__bf16*>(a.out)[at] = (__bf16)v;
}

// C: type of the cache's rows.  A row of the head is CHUNKS chunks of 16 VW channels, VW of them a lane (D below that: RAGGED).  PARTS: bf16 terms of a query,
// 1 of a bf16 one and 3 of an fp32 one, exact; keys of fp32 are multiplied in fp32.
template <typename C, int VW, int CHUNKS, int PARTS, bool RAGGED>
__global__ __launch_bounds__(kThreads) void attention_kernel(const AttentionArgs a) {
  constexpr bool kF32 = sizeof(C) == 4, kCodes = sizeof(C) == 1;
  constexpr int kDims = 16 * VW * CHUNKS;                   // channels that registers are for
  constexpr int kTiles = kF32 || kDims > 128 ? 1 : 2;       // tiles of 16 positions of a block
  constexpr int kBlock = 16 * kTiles;
  constexpr int kSteps = kDims / 32;                        // of the scores' contraction: 32 channels, 8 a lane
  typedef typename Raw<C, VW>::type RawV;
  typedef typename Raw<C, 8>::type RawK;
  __shared__ int s_page[kMaxPages];
  __shared__ __attribute__((aligned(16))) float s_out[kWaves][16][16 * VW];
  __shared__ float s_max[kWaves][16], s_sum[kWaves][16];
  __shared__ int s_bad;

  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n = lane & 15, g = lane >> 4;
  const int tiles = (a.group + kHeadTile - 1) / kHeadTile;
  int at = blockIdx.x;
  const int tile = at % tiles; at /= tiles;
  const int kvh = at % a.kv_heads; at /= a.kv_heads;
  const int part = at % a.parts, b = at / a.parts;

  const Seen seen = seen_by(a.lengths[b], a.max_len, a.window, a.table_len, a.shift);
  const Part p = part_of(seen, a.split, part);
  if (a.parts > 1 && p.begin >= p.end) return;
  const int heads = min(kHeadTile, a.group - tile * kHeadTile), head0 = kvh * a.group + tile * kHeadTile;

  // ---- pages of the part; a number outside the cache spoils the sequence ----
  const int entry0 = p.begin >> a.shift;
  if (tid == 0) s_bad = seen.bad;
  __syncthreads();
  if (p.begin < p.end) {
    const int entries = ((p.begin + a.split - 1) >> a.shift) - entry0 + 1;
    const int32_t* row = a.table + b * a.table_ld;
    for (int i = tid; i < entries; i += kThreads) {
      const int64_t from = (int64_t)(entry0 + i) << a.shift;
      int page = 0;                                         // of positions that are not seen: any
      if (from < p.end && from + ((int64_t)1 << a.shift) > max(p.begin, seen.first)) page = page_of(row, a.table_len, a.n_pages, a.shift, from);
      if (page < 0) { s_bad = 1; page = 0; }
      s_page[i] = page;
    }
  }

  // ---- queries ----
  bf16x8 qf[kF32 ? 1 : PARTS][kSteps];
  float q32[kF32 ? kDims / 4 : 1];
  {
    const int64_t q_at = (int64_t)b * a.q_token + (int64_t)(head0 + min(n, heads - 1)) * a.q_head;
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < kDims / 4; ++i) {
        const int d = 16 * (i / 4) + 4 * g + i % 4;
        q32[i] = n < heads && (!RAGGED || d < a.D) ? load_query(a, q_at + d) : 0.f;
      }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int d = 32 * s + 8 * g + e;
          float q = n < heads && (!RAGGED || d < a.D) ? load_query(a, q_at + d) : 0.f;
#pragma unroll
          for (int t = 0; t < PARTS; ++t) {
            const __bf16 r = (__bf16)q;
            qf[t][s][e] = r;
            q -= (float)r;
          }
        }
    }
  }
  const float to_log2 = a.softcap > 0.f ? a.softcap * kLog2e : a.scale * kLog2e, in_cap = a.softcap > 0.f ? a.scale / a.softcap : 0.f;
  const C* const kbase = static_cast<const C*>(a.k) + (int64_t)kvh * a.head;
  const C* const vbase = static_cast<const C*>(a.v) + (int64_t)kvh * a.head;
  const int mask = (1 << a.shift) - 1;

  float top = -INFINITY, sum = 0.f;
  f32x4 acc[CHUNKS][VW];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int j = 0; j < VW; ++j) acc[c][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  __syncthreads();

  const int first = max(seen.first, p.begin);
  for (int t0 = p.begin + (first - p.begin) / kBlock * kBlock + wave * kBlock; t0 < p.end; t0 += kWaves * kBlock) {
    const bool whole = t0 >= first && t0 + kBlock <= p.end;
    // ---- loads ----
    RawK kr[kTiles][kF32 ? kDims / 8 : kSteps];
    RawV vr[kTiles][4][CHUNKS];
    f32x4 ks[kTiles], vs[kTiles];
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      const int tk = t0 + 16 * u + n;
      const C* krow = kbase + (int64_t)s_page[(tk >> a.shift) - entry0] * a.page + (int64_t)(tk & mask) * a.row;
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < kDims / 16; ++i) {
          const int d = 16 * i + 4 * g;
          const f32x4 x = !RAGGED || d < a.D ? *reinterpret_cast<const f32x4*>(krow + d) : f32x4{0.f, 0.f, 0.f, 0.f};
          if (i % 2) kr[u][i / 2].hi = x; else kr[u][i / 2].lo = x;
        }
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int d = 32 * s + 8 * g;
          kr[u][s] = !RAGGED || d < a.D ? *reinterpret_cast<const RawK*>(krow + d) : zeros(RawK{});
        }
      }
      const int tv = t0 + 16 * u + 4 * g, page = s_page[(tv >> a.shift) - entry0];
      const C* vrow = vbase + (int64_t)page * a.page + (int64_t)(tv & mask) * a.row;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const int d = 16 * VW * c + VW * n;
          vr[u][i][c] = !RAGGED || d < a.D ? *reinterpret_cast<const RawV*>(vrow + (int64_t)i * a.row + d) : zeros(RawV{});
        }
      if constexpr (kCodes) {
        const int64_t sc = (((int64_t)page * a.kv_heads + kvh) << a.shift) + (tv & mask);
        ks[u] = *reinterpret_cast<const f32x4*>(a.k_scale + sc);
        vs[u] = *reinterpret_cast<const f32x4*>(a.v_scale + sc);
      }
    }
    // ---- scores, in units of log 2 ----
    float x[kTiles][4];
    bool there[kTiles][4];
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      f32x4 z = {0.f, 0.f, 0.f, 0.f};
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < kDims / 4; ++i)
          z = __builtin_amdgcn_mfma_f32_16x16x4f32(i % 8 < 4 ? kr[u][i / 8].lo[i % 4] : kr[u][i / 8].hi[i % 4], q32[i], z, 0, 0, 0);
      } else {
#pragma unroll
        for (int t = PARTS - 1; t >= 0; --t)                // small terms first
#pragma unroll
          for (int s = 0; s < kSteps; ++s) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(kr[u][s]), qf[t][s], z, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = z[i];
        if constexpr (kCodes) v *= ks[u][i];
        if (a.softcap > 0.f) v = tanhf(v * in_cap);
        const int t = t0 + 16 * u + 4 * g + i;
        there[u][i] = whole || (t >= first && t < p.end);
        x[u][i] = v;
        most = fmaxf(most, there[u][i] ? v * to_log2 : -INFINITY);
      }
    }
    if (__any(most > top + kSlack)) {
      const float now = lane_max(fmaxf(top, most));
      const float alpha = top == -INFINITY ? 0.f : exp2f(top - now);
      top = now;
      sum *= alpha;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < VW; ++j) acc[c][j] *= alpha;
    }
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float e = there[u][i] ? __builtin_amdgcn_exp2f(fmaf(x[u][i], to_log2, -base)) : 0.f;
        sum += e;
        if constexpr (kCodes) e = there[u][i] ? e * vs[u][i] : 0.f;
        // ---- values: what stands behind the sequence counts as zero, whatever it is ----
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const RawV v = there[u][i] ? vr[u][i][c] : zeros(RawV{});
#pragma unroll
          for (int j = 0; j < VW; ++j) acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(element<C, VW>(v, j), e, acc[c][j], 0, 0, 0);
        }
      }
  }

  // ---- join the waves ----
  sum = lane_sum(sum);
  if (g == 0) { s_max[wave][n] = top; s_sum[wave][n] = sum; }
  __syncthreads();
  auto joined = [&](int head, float* m, float* l) {
    *m = s_max[0][head];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) *m = fmaxf(*m, s_max[w][head]);
    *l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) *l += s_max[w][head] == -INFINITY ? s_sum[w][head] : s_sum[w][head] * exp2f(s_max[w][head] - *m);
  };
  float m, l;
  joined(n, &m, &l);
  const float weight = top == -INFINITY ? (sum == 0.f ? 0.f : sum) : exp2f(top - m);     // a sum without a maximum is NaN
  const bool bad = s_bad;
  const float nan = __uint_as_float(0x7fc00000u);
  const int64_t part_row = ((int64_t)b * a.parts + part) * a.heads + head0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    if (c) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VW; j += 4)
        *reinterpret_cast<f32x4*>(&s_out[wave][n][VW * (4 * g + i) + j]) =
            f32x4{acc[c][j][i], acc[c][j + 1][i], acc[c][j + 2][i], acc[c][j + 3][i]} * weight;
    __syncthreads();
    for (int o = tid; o < 16 * 16 * VW / 4; o += kThreads) {
      const int head = o / (4 * VW), d = o % (4 * VW) * 4, channel = 16 * VW * c + d;
      if (head >= heads || channel >= a.D) continue;
      f32x4 v = *reinterpret_cast<const f32x4*>(&s_out[0][head][d]);
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += *reinterpret_cast<const f32x4*>(&s_out[w][head][d]);
      joined(head, &m, &l);
      if (bad) l = nan;
      if (a.parts > 1) {
        *reinterpret_cast<f32x4*>(a.part_out + (part_row + head) * a.D + channel) = v;
        if (channel == 0) {
          a.part_stat[2 * (part_row + head)] = l == l ? m : nan;      // a sum that is none spoils the whole row
          a.part_stat[2 * (part_row + head) + 1] = l;
        }
      } else {
        const float over = l == 0.f ? 0.f : 1.f / l;
        const int64_t to = (int64_t)b * a.out_token + (int64_t)(head0 + head) * a.out_head + channel;
#pragma unroll
        for (int e = 0; e < 4; ++e) store_out(a, to + e, v[e] * over);
        if (a.lse && channel == 0) a.lse[(int64_t)b * a.heads + head0 + head] = l == 0.f ? -INFINITY : fmaf(m, kLn2, logf(l));
      }
    }
  }
}

// The parts of a row (sequence, head), one wave a row.
__global__ __launch_bounds__(64) void join_kernel(const AttentionArgs a) {
  const int row = blockIdx.x, lane = threadIdx.x, b = row / a.heads, head = row - b * a.heads;
  const Seen seen = seen_by(a.lengths[b], a.max_len, a.window, a.table_len, a.shift);
  const int parts = (seen.end - seen.first / 64 * 64 + a.split - 1) / a.split;
  const int64_t first = (int64_t)b * a.parts * a.heads + head;
  const float* stat = a.part_stat + 2 * first;
  float m = -INFINITY, l = 0.f;
  for (int i = lane; i < parts; i += 64) m = fmaxf(m, stat[2 * (int64_t)i * a.heads]);
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  auto weight = [&](int i) {
    const float pm = stat[2 * (int64_t)i * a.heads];
    return pm == -INFINITY ? 0.f : exp2f(pm - m);
  };
  for (int i = lane; i < parts; i += 64) l += weight(i) == 0.f ? 0.f : weight(i) * stat[2 * (int64_t)i * a.heads + 1];
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
  if (seen.bad) l = __uint_as_float(0x7fc00000u);
  const float over = l == 0.f ? 0.f : 1.f / l;
  for (int d = lane; d < a.D; d += 64) {
    float v = 0.f;
    for (int i = 0; i < parts; ++i) {
      const float w = weight(i);
      if (w != 0.f) v = fmaf(w, a.part_out[(first + (int64_t)i * a.heads) * a.D + d], v);
    }
    store_out(a, (int64_t)b * a.out_token + (int64_t)head * a.out_head + d, v * over);
  }
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : fmaf(m, kLn2, logf(l));
}

template <typename C, int VW, int CHUNKS, int PARTS>
int launch_dims(const AttentionArgs& a, int blocks, hipStream_t s) {
  if (a.D < 16 * VW * CHUNKS) attention_kernel<C, VW, CHUNKS, PARTS, true><<<blocks, kThreads, 0, s>>>(a);
  else attention_kernel<C, VW, CHUNKS, PARTS, false><<<blocks, kThreads, 0, s>>>(a);
  return hip_fail(hipGetLastError(), "attention_kernel");
}
template <typename C, int PARTS>
int launch_parts(const AttentionArgs& a, int blocks, hipStream_t s) {
  if (a.D <= 64) return launch_dims<C, 4, 1, PARTS>(a, blocks, s);
  if (a.D <= 128) return launch_dims<C, 8, 1, PARTS>(a, blocks, s);
  return launch_dims<C, 8, 2, PARTS>(a, blocks, s);
}
template <typename C>
int launch_cache(const AttentionArgs& a, int blocks, hipStream_t s) {
  return a.dtype == MOE_FP32 ? launch_parts<C, 3>(a, blocks, s) : launch_parts<C, 1>(a, blocks, s);
}

}  // namespace

int launch_attention(const AttentionArgs& a, hipStream_t s) {
  ProfScope prof(kProfAttention, s);
  const int blocks = a.B * a.parts * a.kv_heads * ((a.group + kHeadTile - 1) / kHeadTile);
  int rc;
  if (a.cache_dtype == MOE_FP32) rc = launch_parts<float, 1>(a, blocks, s);
  else if (a.cache_dtype == MOE_E4M3) rc = launch_cache<uint8_t>(a, blocks, s);
  else rc = launch_cache<__bf16>(a, blocks, s);
  if (rc || a.parts == 1) return rc;
  join_kernel<<<a.B * a.heads, 64, 0, s>>>(a);
  return hip_fail(hipGetLastError(), "join_kernel");
}

}  // namespace mm
