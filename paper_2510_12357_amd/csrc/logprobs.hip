// Log probabilities of given tokens, entropy, confidence and most probable tokens of output distributions.
//
// One pass over a row.  A wave keeps the best n entries it has seen as a sorted list, entry j in lane j; m is the first of them.  For
// every other entry z, with d = z - m:
//     R += e^d        A += e^d d        so that   log sum = log(1 + R),   entropy = log(1 + R) - A / (1 + R)   where the wave saw the whole row.
// The largest entry itself is in no sum: log p of a nearly certain token is -log(1 + R) with all digits of R.
// A batch of a wave (kPerLane entries per lane) is compared with the list's last entry by one maximum per lane and one ballot.  Only where
// some entry is above it are entries exchanged with the list's, what leaves the list is summed with the batch, and m moves (R and A
// are rescaled); there are about n log(V / n) such entries in a row.  So the ordinary batch costs a difference, an
// exponential and three further operations per entry, and no reference to other lanes.
// Waves of a row (and workgroups, where rows are few) take batches in turn and are joined at the end: sums by the rule of a
// streaming softmax, lists by counting for each candidate how many come before it.
#include "internal.h"
#include "int8_device.h"
#include "route_device.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

constexpr int kList = MOE_MAX_ALTERNATIVES;
constexpr int kPerLaneE = 32;                              // entries of a lane in a batch
constexpr int kBatch = 64 * kPerLaneE;
constexpr int kNone = 0x7fffffff;                          // id of an entry that is not there
constexpr int kMaxParts = 16;                              // workgroups of a row

struct LogprobArgs {
  const void* logits; int64_t ld;
  int V, n_given, n_top, parts;
  const int32_t* tokens;
  float* token_logp; float* entropy; float* conf; int32_t* top_idx; float* top_logp;
  float* ws;                                               // [T][parts] of partial_floats(n) (parts > 1)
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float lane_f(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

// (value, id) in the order value descending, id ascending
__device__ __forceinline__ bool before(float av, int aid, float bv, int bid) { return av > bv || (av == bv && aid < bid); }

// unsigned integers in the order of the floats (no NaN; the zeros are one number)
__device__ __forceinline__ unsigned order_key(float v) {
  const unsigned b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// the largest float below the one of the key
__device__ __forceinline__ float below(unsigned key) { return key == 0x80000000u ? -0x1p-149f : key_value(key - 1); }
constexpr unsigned kKeyNegInf = 0x007fffffu;               // order_key(-inf)

// What a wave (or a workgroup) knows of a row.  list_v / list_id: entry `lane` of the list, -inf / kNone where there is none.
struct Partial { float m, R, A; };

// The state of a wave on its share of a row.
struct Stream {
  float lv = -INFINITY; int lid = kNone;                   // the list, entry j in lane j
  float m = -INFINITY, ref = 0.f;                          // ref: m, or 0 while there is nothing
  float last = -INFINITY;                                  // the list's n-th entry
  float R[4] = {0.f, 0.f, 0.f, 0.f}, A[4] = {0.f, 0.f, 0.f, 0.f};   // four chains each: sums of at most V / 256 links

  // entry (v, id), the same in all lanes, takes its place in the list; returns what leaves it
  __device__ __forceinline__ float insert(float v, int id, int n, int lane) {
    const float out = lane_f(lv, n - 1);
    const float uv = __uint_as_float(__builtin_amdgcn_update_dpp(0x7f800000, __float_as_uint(lv), 0x138, 0xf, 0xf, false));   // of the lane before; +inf in lane 0
    const int uid = __builtin_amdgcn_update_dpp(-1, lid, 0x138, 0xf, 0xf, false);
    const bool b = lane < n && before(v, id, lv, lid), bu = lane > 0 && before(v, id, uv, uid);
    lv = b ? (bu ? uv : v) : lv;
    lid = b ? (bu ? uid : id) : lid;
    return out;
  }

  // entries of x above `thr` change places with the list's.  x_max: the largest of each vector of kVec.
  template <int N, int VEC, typename Id>
  __device__ __forceinline__ void exchange(float (&x)[N], const float (&x_max)[N / VEC], float lane_max, float thr, int n, int lane, Id id_of) {
    const unsigned long long hit = __ballot(lane_max > thr);
    if (__popcll(hit) > n) {
      // Many lanes (the first batch, rising rows): the list's last entry will be at least the n-th largest of the lanes' maxima.  Found in its
      // upper 16 bits by halving; entries below it need not be looked at.
      const unsigned key = order_key(lane_max);
      unsigned t = 0;
#pragma unroll
      for (int bit = 31; bit >= 16; --bit) {
        const unsigned c = t | (1u << bit);
        if (__popcll(__ballot(key >= c)) >= n) t = c;
      }
      if (t > kKeyNegInf) thr = fmaxf(thr, below(t));
    }
#pragma unroll
    for (int u = 0; u < N / VEC; ++u) {
      if (!__ballot(x_max[u] > thr)) continue;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        unsigned long long todo = __ballot(x[u * VEC + e] > thr && x[u * VEC + e] >= last);
        while (todo) {
          const int src = __builtin_ctzll(todo);
          todo &= todo - 1;
          const float v = lane_f(x[u * VEC + e], src);
          const int id = uniform(id_of(u, e, src));
          if (!before(v, id, last, __builtin_amdgcn_readlane(lid, n - 1))) continue;
          const float out = insert(v, id, n, lane);
          if (lane == src) x[u * VEC + e] = out;
          last = lane_f(lv, n - 1);
        }
      }
    }
    const float top = lane_f(lv, 0);
    if (top != m) {
      const float d = m > -INFINITY ? fmaxf(m - top, -200.f) : 0.f, f = __expf(d);
#pragma unroll
      for (int c = 0; c < 4; ++c) { A[c] = f * fmaf(d, R[c], A[c]); R[c] *= f; }
      m = ref = top;
    }
  }

  // d of the lowest values and of -inf is held at -200 beside e^d = 0; a NaN stays one in e^d
  template <int N>
  __device__ __forceinline__ void sum(const float (&x)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float d = x[j] - ref, e = __builtin_amdgcn_exp2f(d * 1.44269504088896341f);
      R[j & 3] += e;
      A[j & 3] = fmaf(e, fmaxf(d, -200.f), A[j & 3]);
    }
  }

  // the list but for its first entry joins the sums; -> the wave's part, the same in all lanes
  __device__ __forceinline__ Partial close(int n, int lane) {
    float r = (R[0] + R[1]) + (R[2] + R[3]), a = (A[0] + A[1]) + (A[2] + A[3]);
    if (lane > 0 && lane < n && lid != kNone) {
      const float d = lv - ref, e = __builtin_amdgcn_exp2f(d * 1.44269504088896341f);
      r += e;
      a = fmaf(e, fmaxf(d, -200.f), a);
    }
    return {m, wave_sum(r), wave_sum(a)};
  }
};

// ---- what is written for a row: lane j < n_top holds the j-th entry (kNone: there is none) ----
struct RowEnd {
  float m, log_sum, sum, A;
  __device__ __forceinline__ RowEnd(Partial p) : m(p.m), log_sum(log1pf(p.R)), sum(1.f + p.R), A(p.A) {
    if (!(fabsf(m) < INFINITY)) log_sum = sum = NAN;
  }
};
template <typename S>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t t, Partial p, float lv, int lid, int lane) {
  const S* row = static_cast<const S*>(a.logits) + t * a.ld;
  const RowEnd r(p);
  if (lane == 0 && a.entropy) a.entropy[t] = r.log_sum - r.A / r.sum;
  if (lane == 0 && a.conf) a.conf[t] = 1.f / r.sum;
  if (lane < a.n_given) {
    const int id = a.tokens[t * a.n_given + lane];
    a.token_logp[t * a.n_given + lane] = id < 0 || id >= a.V ? 0.f : (to_f32(row[id]) - r.m) - r.log_sum;
  }
  if (!a.n_top) return;
  const int found = __popcll(__ballot(lane < a.n_top && lid != kNone));
  if (found < a.n_top) {
    // every entry above -inf is in the list, so the places behind them go to the lowest ids that are not in it (of the first 64: at most
    // 31 are); these are n_top - found <= V - found many
    bool free_id = lane < a.V;
    for (int j = 0; j < found; ++j) free_id &= __builtin_amdgcn_readlane(lid, j) != lane;
    unsigned long long ids = __ballot(free_id);
    for (int j = found; j < a.n_top; ++j) {
      const int id = __builtin_ctzll(ids);
      ids &= ids - 1;
      if (lane == j) lid = id;
    }
  }
  if (lane < a.n_top) {
    a.top_idx[t * a.n_top + lane] = lid;
    a.top_logp[t * a.n_top + lane] = (lv - r.m) - r.log_sum;
  }
}

// ---- joining of parts in LDS ----
constexpr int kMaxLists = 16;
struct Joint {
  float m[kMaxLists], R[kMaxLists], A[kMaxLists];
  float v[kMaxLists * kList]; int id[kMaxLists * kList];   // list w from w * n on
  float cv[kMaxLists * kList]; int cid[kMaxLists * kList]; // candidates
  float ov[kList]; int oid[kList];
  int count;
  unsigned bound;                                          // key of the largest n-th entry of any list so far
};
// One workgroup joins `lists` lists of n entries; the result is for its first wave: lane j has the j-th entry.
__device__ __forceinline__ Partial join(Joint& s, int lists, int n, int tid, int threads, float& lv, int& lid) {
  const int lane = tid & 63;
  if (tid < kList) s.oid[tid] = kNone;
  if (tid < kList) s.ov[tid] = -INFINITY;
  if (tid == 0) s.count = 0;
  float tau = -INFINITY;
  for (int w = 0; w < lists; ++w) tau = fmaxf(tau, s.v[w * n + n - 1]);
  __syncthreads();
  for (int i = tid; i < lists * n; i += threads) {
    if (s.id[i] != kNone && s.v[i] >= tau) {
      const int at = atomicAdd(&s.count, 1);
      s.cv[at] = s.v[i];
      s.cid[at] = s.id[i];
    }
  }
  __syncthreads();
  const int count = s.count;
  for (int i = tid; i < count; i += threads) {
    const float v = s.cv[i];
    const int id = s.cid[i];
    int rank = 0;
    for (int k = 0; k < count; ++k) rank += before(s.cv[k], s.cid[k], v, id);
    if (rank < n) { s.ov[rank] = v; s.oid[rank] = id; }
  }
  __syncthreads();
  Partial p = {0.f, 0.f, 0.f};
  if (tid < 64) {
    lv = lane < n ? s.ov[lane] : -INFINITY;
    lid = lane < n ? s.oid[lane] : kNone;
    const bool in = lane < lists;
    const float mw = in ? s.m[lane] : -INFINITY;
    p.m = wave_max(mw);
    const int first = __builtin_ctzll(__ballot(mw == p.m) | (1ull << 63));
    float r = 0.f, q = 0.f;
    if (in) {
      r = s.R[lane];
      q = s.A[lane];
      if (lane != first) {                                 // its largest entry is one of the others now
        const float d = fmaxf(mw - p.m, -200.f), f = __expf(d);
        q = f * (fmaf(d, r, q) + d);
        r = f * (r + 1.f);
        if (mw == -INFINITY) q = r = s.R[lane] * 0.f;      // nothing in it (or a NaN)
      }
    }
    p.R = wave_sum(r);
    p.A = wave_sum(q);
  }
  return p;
}

__host__ __device__ constexpr int partial_floats(int n) { return 4 + 2 * n; }

// W waves per row part; W == 1: a workgroup is one wave with a row of its own.
template <typename S, int W>
__global__ __launch_bounds__(W * 64) void logprobs_kernel(const LogprobArgs a) {
  constexpr int kVec = 16 / sizeof(S), U = kPerLaneE / kVec;
  __shared__ Joint s;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n = a.n_top > 1 ? a.n_top : 1;
  const int part = a.parts > 1 ? (int)(blockIdx.x % (unsigned)a.parts) : 0;
  const int64_t t = a.parts > 1 ? blockIdx.x / (unsigned)a.parts : blockIdx.x;
  const S* row = static_cast<const S*>(a.logits) + t * a.ld;
  // vectors of 16 bytes on their own alignment; the row starts `shift` entries behind the first one's
  const int shift = (int)(((uintptr_t)row & 15) / sizeof(S));
  const S* base = row - shift;
  const int end = shift + a.V;
  const int batches = (end + kBatch - 1) / kBatch, stride = W * a.parts;
  if (W > 1) {
    if (tid == 0) s.bound = 0;
    __syncthreads();
  }
  auto load = [&](int b, u32x4 (&raw)[U]) {
    const int e0 = b * kBatch;
    if (e0 >= shift && e0 + kBatch <= end) {
      const u32x4* p = reinterpret_cast<const u32x4*>(base + e0) + lane;
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = p[u * 64];
    } else {
      // an edge of the row: only entries of it are read, the others are -inf
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = e0 + (u * 64 + lane) * kVec;
        if (e >= shift && e + kVec <= end) {
          raw[u] = *reinterpret_cast<const u32x4*>(base + e);
        } else {
          constexpr S kNegInf = (S)(sizeof(S) == 2 ? 0xff80 : 0);
          S part[kVec];
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            if constexpr (sizeof(S) == 2) part[i] = kNegInf; else part[i] = -INFINITY;
            if (e + i >= shift && e + i < end) part[i] = base[e + i];
          }
          raw[u] = __builtin_bit_cast(u32x4, part);
        }
      }
    }
  };
  Stream st;
  u32x4 raw[U], next[U];
  int b = part * W + wave;
  if (b < batches) load(b, raw);
  for (; b < batches; b += stride) {
    if (b + stride < batches) load(b + stride, next);
    float x[kPerLaneE], x_max[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(S) == 2) {
          x[u * 8 + 2 * i] = __uint_as_float(raw[u][i] << 16);
          x[u * 8 + 2 * i + 1] = __uint_as_float(raw[u][i] & 0xffff0000u);
        } else {
          x[u * 4 + i] = __uint_as_float(raw[u][i]);
        }
      }
      x_max[u] = x[u * kVec];
#pragma unroll
      for (int e = 1; e < kVec; ++e) x_max[u] = fmaxf(x_max[u], x[u * kVec + e]);
    }
    float top = x_max[0];
#pragma unroll
    for (int u = 1; u < U; ++u) top = fmaxf(top, x_max[u]);
    // A wave's own ids rise, so an entry equal to its list's last comes behind it; one equal to another wave's may come before.
    // What is above m always enters, so that m bounds what is summed.
    float thr = st.last;
    if (W > 1) {
      const unsigned k = *(volatile unsigned*)&s.bound;
      if (k > kKeyNegInf) thr = fmaxf(thr, fminf(below(k), st.m));
    }
    if (__ballot(top > thr)) {
      const float was = st.last;
      st.template exchange<kPerLaneE, kVec>(x, x_max, top, thr, n, lane, [&](int u, int e, int l) { return b * kBatch + (u * 64 + l) * kVec + e - shift; });
      if (W > 1 && st.last > was && lane == 0) atomicMax(&s.bound, order_key(st.last));
    }
    st.sum(x);
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = next[u];
  }
  Partial p = st.close(n, lane);
  if constexpr (W > 1) {
    if (lane == 0) { s.m[wave] = p.m; s.R[wave] = p.R; s.A[wave] = p.A; }
    if (lane < n) { s.v[wave * n + lane] = st.lv; s.id[wave * n + lane] = st.lid; }
    __syncthreads();
    p = join(s, W, n, tid, W * 64, st.lv, st.lid);
    if (wave) return;
  }
  if (a.parts > 1) {
    float* o = a.ws + (t * a.parts + part) * partial_floats(n);
    if (lane == 0) { o[0] = p.m; o[1] = p.R; o[2] = p.A; }
    if (lane < n) { o[4 + lane] = st.lv; o[4 + n + lane] = __int_as_float(st.lid); }
    return;
  }
  write_row<S>(a, t, p, st.lv, st.lid, lane);
}

// Joins the parts of a row.
template <typename S>
__global__ __launch_bounds__(256) void logprobs_join_kernel(const LogprobArgs a) {
  __shared__ Joint s;
  const int tid = threadIdx.x, lane = tid & 63;
  const int n = a.n_top > 1 ? a.n_top : 1;
  const int64_t t = blockIdx.x;
  const float* in = a.ws + t * a.parts * partial_floats(n);
  for (int i = tid; i < a.parts * n; i += 256) {
    const int w = i / n, j = i - w * n;
    s.v[i] = in[w * partial_floats(n) + 4 + j];
    s.id[i] = __float_as_int(in[w * partial_floats(n) + 4 + n + j]);
  }
  if (tid < a.parts) { s.m[tid] = in[tid * partial_floats(n)]; s.R[tid] = in[tid * partial_floats(n) + 1]; s.A[tid] = in[tid * partial_floats(n) + 2]; }
  __syncthreads();
  float lv; int lid;
  const Partial p = join(s, a.parts, n, tid, 256, lv, lid);
  if (tid < 64) write_row<S>(a, t, p, lv, lid, lane);
}

// Waves per row part and parts per row.
struct Split { int waves, parts; };
Split split_of(int T, int V) {
  const int batches = V / kBatch + 1;
  if (T >= 1024) return {1, 1};
  int waves = T >= 256 ? 4 : 16;
  while (waves > 4 && waves > batches) waves /= 2;
  if (batches < 4) waves = 1;
  int parts = 1;
  if (waves == 16) while (parts < kMaxParts && T * parts * 2 <= 256 && batches >= 16 * parts * 2) parts *= 2;
  return {waves, parts};
}

template <typename S>
int launch(const LogprobArgs& a, int T, int waves, hipStream_t s) {
  const dim3 grid((unsigned)T * (unsigned)a.parts);
  switch (waves) {
    case 1: hipLaunchKernelGGL((logprobs_kernel<S, 1>), grid, dim3(64), 0, s, a); break;
    case 4: hipLaunchKernelGGL((logprobs_kernel<S, 4>), grid, dim3(256), 0, s, a); break;
    case 8: hipLaunchKernelGGL((logprobs_kernel<S, 8>), grid, dim3(512), 0, s, a); break;
    default: hipLaunchKernelGGL((logprobs_kernel<S, 16>), grid, dim3(1024), 0, s, a); break;
  }
  int rc = hip_fail(hipGetLastError(), "logprobs_kernel launch");
  if (rc || a.parts == 1) return rc;
  hipLaunchKernelGGL(logprobs_join_kernel<S>, dim3((unsigned)T), dim3(256), 0, s, a);
  return hip_fail(hipGetLastError(), "logprobs_join_kernel launch");
}

}  // namespace

size_t logprobs_workspace_bytes(const moe_logprobs_config& c) {
  const Split sp = split_of(c.T, c.V);
  return sp.parts == 1 ? 0 : align256((size_t)c.T * sp.parts * partial_floats(c.n_top > 1 ? c.n_top : 1) * sizeof(float));
}

int launch_logprobs(const moe_logprobs_config& c, const void* logits, const int32_t* tokens, float* token_logp, float* entropy, float* conf,
                    int32_t* top_idx, float* top_logp, void* ws, hipStream_t s) {
  ProfScope ps(kProfLogprobs, s);
  const Split sp = split_of(c.T, c.V);
  const LogprobArgs a = {logits, c.ld, c.V, c.n_given, c.n_top, sp.parts, tokens, token_logp, entropy, conf, top_idx, top_logp, static_cast<float*>(ws)};
  return c.dtype == MOE_FP32 ? launch<float>(a, c.T, sp.waves, s) : launch<uint16_t>(a, c.T, sp.waves, s);
}

}  // namespace mm
