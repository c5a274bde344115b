// Log probabilities of given tokens, entropy, confidence and most probable tokens of output distributions.
//
// One pass over a row.  A wave keeps the best n entries it has seen as a sorted list, entry j in lane j.  For every other entry z, with
// d = z - ref, ref an entry not far below the wave's largest:
//     R += e^d,    A += e^d d.
// With m the row's largest entry, R and A of all entries but that one, and relative to m:
//     log sum = log(1 + R),    entropy = log(1 + R) - A / (1 + R),    log p of z = (z - m) - log(1 + R).
// The largest entry itself is in no sum, so log p of a nearly certain token, -log(1 + R), has all digits of R.  Entries that equal a wave's
// reference add exactly one each.  Entries that come later may lie up to kLead above it before it moves: each adds e^d with an error of 3 d 2^-24,
// and the sum is brought to m by e^(ref - m) with as much again, 120 2^-24 at most; A is then a difference, A + (ref - m) R, with that error of
// either.  (A row that is constant but for lower first batches; ordinary rows have their largest entry at most a few units above the reference.)
//
// A batch of a wave (kPerLane entries per lane) is compared with the list's last entry by one maximum per lane and one ballot, on the
// differences d, which follow the order of the entries.  Only where one is not below it, entries go to the list, and what the list
// drops is summed.  A lower bound of the n-th entry is known from the start: the n-th of the lanes' maxima over the first batches,
// which wait in registers; about n (1 + log(V / seen)) entries of a row are above what is known when they come.  So the ordinary
// batch costs a difference, a product, an exponential and three and a half further operations per entry, and nothing crosses the
// lanes.  (One multiply-add in place of the difference and the product, on z log2 e - ref log2 e, is no faster, 182 us for 4096 rows of
// 131072 in bf16 either way, and entries that equal the reference then add what the rounded ref log2 e makes of them.)
// Waves of a row (and workgroups, where rows are few) take batches in turn and are joined at the end: sums by the rule of a
// streaming softmax, lists by counting for each candidate how many come before it.  Nothing depends on which wave is first.
// Measured: 4096 rows of 131072 bf16 with 8 alternatives 180 - 191 us (5.6 - 6.0 TB/s; a plain read gets 6.9, and the vector unit issues 0.9 of the time),
// 1999 of 50257 bf16 49 (4.1), 64 of 131072 fp32 with 20 alternatives 20.5 (15.2 with one), one row of 32000 fp32 8.0.
#include <algorithm>

#include "internal.h"
#include "int8_device.h"
#include "route_device.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef unsigned long long u64;

constexpr int kList = MOE_MAX_ALTERNATIVES;
constexpr int kPerLaneB = 16;                              // entries of a lane in a batch
constexpr int kBatch = 64 * kPerLaneB;
constexpr int ring(size_t bytes) { return bytes == 2 ? 4 : 2; }   // batches of a wave in registers or on their way
constexpr int kMaxParts = 16;                              // workgroups of a row, a power of two as the waves are
constexpr float kLead = 20.f;                              // entries may lie this far above the reference: e^20 is far from overflow
constexpr float kFloor = -200.f;                           // d is held here beside e^d = 0

struct LogprobArgs {
  const void* logits; int64_t ld;
  int V, n_given, n_top, parts;
  const int32_t* tokens;
  float* token_logp; float* entropy; float* conf; int32_t* top_idx; float* top_logp;
  u64* ws;                                                 // [T][parts][partial_words(n)] (parts > 1)
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float lane_f(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

// Entries are compared as one integer in the order (value ascending, id descending): the value's bits in the order of the floats (the
// zeros are one number), then the id's complement.  0: no entry.  A NaN never becomes one.
__device__ __forceinline__ unsigned order_key(float v) {
  const unsigned b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 entry_key(float v, int id) { return (u64)order_key(v) << 32 | (unsigned)~id; }
__device__ __forceinline__ float entry_value(u64 k) { return k ? key_value((unsigned)(k >> 32)) : -INFINITY; }
__device__ __forceinline__ int entry_id(u64 k) { return (int)~(unsigned)k; }
constexpr unsigned kKeyNegInf = 0x007fffffu;               // order_key(-inf)
// the largest float below the one of the key; -inf for what lies under all numbers
__device__ __forceinline__ float below(unsigned key) {
  return key <= kKeyNegInf ? -INFINITY : (key == 0x80000000u ? -0x1p-149f : key_value(key - 1));
}
__device__ __forceinline__ u64 lane_key(u64 v, int lane) {
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}

// A lower bound of the n-th largest key of a wave's lanes: its upper 16 bits, by halving.
__device__ __forceinline__ unsigned nth_bound(unsigned key, int n) {
  unsigned t = 0;
#pragma unroll 1
  for (unsigned bit = 0x80000000u; bit >= 0x10000u; bit >>= 1)
    if (__popcll(__ballot(key >= (t | bit))) >= n) t |= bit;
  return t;
}

// e^d, d = 0: exactly 1
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504088896341f); }

// Sums of everything but the entries of a list, relative to ref; ref = -inf: of nothing.
struct Sums {
  float ref, R, A;
  __device__ __forceinline__ void add(float z, float at) {   // -inf adds nothing, a NaN makes R one
    const float d = z - at, e = exp_of(d);
    R += e;
    A = fmaf(e, fmaxf(d, kFloor), A);
  }
  __device__ __forceinline__ Sums seen_from(float m) const {   // m >= ref
    const float d = ref == m ? 0.f : fmaxf(ref - m, kFloor), f = exp_of(d);
    return {m, f * R, f * fmaf(d, R, A)};
  }
};

// The state of a wave on its share of a row.
struct Stream {
  u64 list = 0;                                            // entry j in lane j
  float last = -INFINITY;                                  // the list's n-th entry
  float ref = -INFINITY, limit = -INFINITY;                // limit: ref + kLead
  float at = 0.f;                                          // ref, or 0 while there is nothing
  float R[4] = {0.f, 0.f, 0.f, 0.f}, A[4] = {0.f, 0.f, 0.f, 0.f};   // four chains each: sums of at most V / 256 links

  __device__ __forceinline__ void add(int chain, float d) {
    const float e = exp_of(d);
    float held;                                            // fmaxf would bring a signalling NaN into order first; any NaN is in R already
    asm("v_max_f32 %0, %1, %2" : "=v"(held) : "s"(kFloor), "v"(d));
    R[chain] += e;
    A[chain] = fmaf(e, held, A[chain]);
  }
  __device__ __forceinline__ void refer_to(float top) {
    const float d = fmaxf(ref - top, kFloor), f = exp_of(d);
#pragma unroll
    for (int c = 0; c < 4; ++c) { A[c] = f * fmaf(d, R[c], A[c]); R[c] *= f; }
    ref = at = top;
    limit = top + kLead;
  }

  // Entries of v above thr go to the list, in rounds: in each, every lane's best one that comes before the list's last, lane after lane, and
  // what the list drops for them to the sums at the round's end.  (A round per entry: 4096 rows of 131072 bf16 with 32 alternatives 276 us, so 236; 128 of
  // 151001 fp32 39.2, 32.4.)  id(j): of entry j, rising with j.
  template <int N, typename Id>
  __device__ __forceinline__ void exchange(float (&v)[N], float thr, int n, int lane, Id id) {
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      v[j] += 0.f;                                         // a maximum drops a quiet NaN, but not a signalling one
      top = fmaxf(top, v[j]);
    }
    if (__ballot(top > limit)) refer_to(wave_max(top));
    // many lanes (rising rows): what is below the n-th largest of the lanes' maxima need not be looked at
    if (__popcll(__ballot(top > thr)) > n) thr = fmaxf(thr, below(nth_bound(order_key(top), n)));
    u64 least = lane_key(list, n - 1);
#pragma unroll 1
    while (__ballot(top > thr)) {
      int pos = 0;
#pragma unroll
      for (int j = N - 1; j > 0; --j) pos = v[j] == top ? j : pos;
      pos = v[0] == top ? 0 : pos;
      const u64 key = top > thr ? entry_key(top, id(pos)) : 0;
      u64 hit = __ballot(key > least), taken = 0;
      if (!hit) break;
      float dropped = -INFINITY;                           // what the list dropped for this lane's entry
      int gone = -1;                                       // which entry that was
      const bool drops = least != 0;
      do {
        const int src = __builtin_ctzll(hit);
        const u64 k = lane_key(key, src);
        dropped = lane == src ? entry_value(least) : dropped;
        gone = lane == src ? pos : gone;
        // the entry of the lane before; one above all in lane 0
        const u64 up = (u64)(unsigned)__builtin_amdgcn_update_dpp(-1, (int)(list >> 32), 0x138, 0xf, 0xf, false) << 32 |
                       (unsigned)__builtin_amdgcn_update_dpp(-1, (int)list, 0x138, 0xf, 0xf, false);
        if (k > list && lane < n) list = k > up ? up : k;
        least = lane_key(list, n - 1);
        taken |= 1ull << src;
        hit = __ballot(key > least) & ~taken;
      } while (hit);
      if (least) thr = fmaxf(thr, below((unsigned)(least >> 32)));
      top = -INFINITY;
#pragma unroll
      for (int j = 0; j < N; ++j) { v[j] = gone == j ? -INFINITY : v[j]; top = fmaxf(top, v[j]); }
      if (drops || __popcll(taken) > 1) add(0, dropped - at);
    }
    last = entry_value(least);
  }

  __device__ __forceinline__ Sums sums() const {           // the same in all lanes
    return {ref, wave_sum((R[0] + R[1]) + (R[2] + R[3])), wave_sum((A[0] + A[1]) + (A[2] + A[3]))};
  }
};

// The given token of a lane and its entry.  Two loads that depend on each other: they are issued before the row is read and used behind it.
template <typename S>
struct Given {
  int id;
  bool in;
  S z;
  __device__ __forceinline__ void load_id(const LogprobArgs& a, int64_t t, int lane) {
    id = lane < a.n_given ? a.tokens[t * a.n_given + lane] : -1;
  }
  __device__ __forceinline__ void load_entry(const LogprobArgs& a, const S* row) {
    in = id >= 0 && id < a.V;
    z = row[in ? id : 0];
  }
};

// What is written for a row by one wave: entry j of the list in lane j, s the sums of everything else.
template <typename S>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t t, u64 list, Sums s, const Given<S>& given, int lane) {
  const float m = entry_value(lane_key(list, 0));
  const bool proper = fabsf(m) < INFINITY;
  Sums rest = {m, 0.f, 0.f};
  if (lane > 0) rest.add(entry_value(list), proper ? m : 0.f);
  s = s.seen_from(m);
  const float R = s.R + wave_sum(rest.R), A = s.A + wave_sum(rest.A);
  const float log_sum = proper ? log1pf(R) : NAN, sum = 1.f + R;
  if (lane == 0 && a.entropy) a.entropy[t] = log_sum - A / sum;
  if (lane == 0 && a.conf) a.conf[t] = proper ? 1.f / sum : NAN;
  if (lane < a.n_given) a.token_logp[t * a.n_given + lane] = given.in ? (float)(((double)to_f32(given.z) - m) - log_sum) : 0.f;
  if (!a.n_top) return;
  const int found = __popcll(__ballot(lane < a.n_top && list));
  int id = entry_id(list);
  if (found < a.n_top) {
    // every entry above -inf is in the list, so the places behind them go to the lowest ids that are not in it (of the first 64: at most
    // 31 are); these are n_top - found <= V - found many
    bool free_id = lane < a.V;
    for (int j = 0; j < found; ++j) free_id &= __builtin_amdgcn_readlane(id, j) != lane;
    u64 ids = __ballot(free_id);
    for (int j = found; j < a.n_top; ++j) {
      const int next = __builtin_ctzll(ids);
      ids &= ids - 1;
      if (lane == j) id = next;
    }
  }
  if (lane < a.n_top) {
    a.top_idx[t * a.n_top + lane] = id;
    a.top_logp[t * a.n_top + lane] = (float)(((double)entry_value(list) - m) - log_sum);
  }
}

// ---- joining of lists and sums in LDS ----
constexpr int kMaxLists = 16;
constexpr int kMaxRanked = 256;
struct Joint {
  alignas(16) u64 cand[kMaxLists * kList + 8];            // eight zeros behind the last
  u64 out[kList];
  float ref[kMaxLists], R[kMaxLists], A[kMaxLists];
  int found[kMaxLists], count;
  unsigned low, bound;                                     // keys: lower bounds of the row's n-th entry
  alignas(16) unsigned key[kMaxRanked];
};
__device__ __forceinline__ void open_joint(Joint& s, int tid) {
  if (tid < kList) s.out[tid] = 0;
  if (tid < kMaxRanked) s.key[tid] = 0;                    // no key is 0
  if (tid == 0) { s.count = 0; s.bound = 0; s.low = ~0u; }
}

// A lower bound of the n-th of a workgroup's lane maxima (`waves` waves have one).  The k-th of a wave, k = n / waves, the smallest of the
// waves': k lanes of each are no less, in all about 4 n lanes; their maxima are ranked.
__device__ __forceinline__ unsigned joint_bound(Joint& s, float top, bool any, int waves, int n, int tid) {
  const int lane = tid & 63, k = (n + waves - 1) / waves;
  const unsigned key = order_key(top);
  if (any) {
    const unsigned t = k == 1 ? order_key(wave_max(top)) : nth_bound(key, k);
    if (lane == 0) atomicMin(&s.low, t);
  }
  __syncthreads();
  const unsigned low = s.low;
  const bool in = any && key >= low && key > kKeyNegInf;   // rows that a mask left little of: lanes without an entry are many
  const u64 mask = __ballot(in);
  int at = 0;
  if (mask && lane == 0) at = atomicAdd(&s.count, __popcll(mask));
  at = uniform(at) + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0));
  if (in && at < kMaxRanked) s.key[at] = key;
  __syncthreads();
  const int count = s.count;
  if (count <= kMaxRanked && tid < count) {
    const unsigned mine = s.key[tid];
    int rank = 0;
    for (int i = 0; i < count; i += 16) {
#pragma unroll
      for (int j = 0; j < 16; ++j) rank += s.key[i + j] > mine || (s.key[i + j] == mine && i + j < tid);
    }
    if (rank == n - 1) s.bound = mine;
  }
  __syncthreads();
  return max(low, s.bound);
}

// A wave's list (no gaps) goes behind those of the waves before it: the order of the sums must not depend on who comes first.
__device__ __forceinline__ void put_list(Joint& s, int lists, int w, int n, int lane, u64 list) {
  const int found = __popcll(__ballot(lane < n && list));
  if (lane == 0) s.found[w] = found;
  __syncthreads();
  const int f = lane < lists ? s.found[lane] : 0;
  const int at = wave_reduce(lane < w ? f : 0, 0, [](int x, int y) { return x + y; });
  if (lane < found) s.cand[at + lane] = list;
  if (w == lists - 1 && lane == 0) s.count = at + found;
  if (w == lists - 1 && lane < 8) s.cand[at + found + lane] = 0;
}
// Candidates and sums are in place (no barrier since).  -> for the first wave: the n best, and the sums of everything else.
__device__ __forceinline__ Sums join(Joint& s, int lists, int n, int tid, u64& list) {
  __syncthreads();
  const int count = s.count, lane = tid & 63;
  if (tid < count) {
    const u64 mine = s.cand[tid];
    int rank = 0;
    for (int k = 0; k < count; k += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) rank += s.cand[k + i] > mine;
    }
    if (rank < n) s.out[rank] = mine;
  }
  __syncthreads();
  Sums sum = {-INFINITY, 0.f, 0.f};
  if (tid < 64) {
    list = lane < n ? s.out[lane] : 0;
    const u64 least = lane_key(list, n - 1);
    sum.ref = entry_value(lane_key(list, 0));
    const float at = sum.ref > -INFINITY ? sum.ref : 0.f;
    for (int i = lane; i < count; i += 64) if (s.cand[i] < least) sum.add(entry_value(s.cand[i]), at);
    if (lane < lists) {
      const Sums w = Sums{s.ref[lane], s.R[lane], s.A[lane]}.seen_from(sum.ref);
      sum.R += w.R;
      sum.A += w.A;
    }
    sum.R = wave_sum(sum.R);
    sum.A = wave_sum(sum.A);
  }
  return sum;
}

__host__ __device__ constexpr int partial_words(int n) { return 2 + n; }

// W waves per row part; W == 1: a workgroup is one wave with a row of its own.
template <typename S, int W>
__global__ __launch_bounds__(W * 64) void logprobs_kernel(const LogprobArgs a) {
  constexpr int kVec = 16 / sizeof(S), U = kPerLaneB / kVec, kRing = ring(sizeof(S));
  __shared__ Joint s_joint;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n = a.n_top > 1 ? a.n_top : 1;
  const int part = a.parts > 1 ? (int)(blockIdx.x % (unsigned)a.parts) : 0;
  const int64_t t = a.parts > 1 ? blockIdx.x / (unsigned)a.parts : blockIdx.x;
  const S* row = static_cast<const S*>(a.logits) + t * a.ld;
  // `head` entries up to the first multiple of 16 bytes, `vectors` vectors of 16 bytes in batches, the last of them perhaps not full, and `tail`
  // entries; head and tail are one further batch at the end, one entry a lane.  One wave for a row, many rows or short ones: the last batch
  // and the ends are under way with the others (loaded when they are due: 3000 rows of 1500 bf16 14.3 us, so 12.1; 4096 of 2000 fp32 15.9, 14.8).  Several
  // waves: they are loaded when they are due (otherwise, in the extra code of each copy of a batch, 1 row of 32000 8.0 us, 8.5).
  constexpr bool kAhead = W == 1;
  const int head = min(a.V, (int)((-(uintptr_t)row & 15) / sizeof(S)));
  const int vectors = (a.V - head) / kVec, tail = (a.V - head) % kVec;
  const int full = vectors / (64 * U), batches = kAhead ? (vectors + 64 * U - 1) / (64 * U) : full, stride = W * a.parts, first = part * W + wave;
  const char* body = reinterpret_cast<const char*>(row + head);
  constexpr unsigned kNegInf2 = sizeof(S) == 2 ? 0xff80ff80u : 0xff800000u;
  auto load = [&](int b, u32x4 (&raw)[U]) {                // lanes behind the last vector read that one
    const char* p = body + (int64_t)b * (64 * U * 16);
    const unsigned most = !kAhead || b < full ? ~0u : (unsigned)(vectors - 1 - b * (64 * U)) * 16u;
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + min((unsigned)lane * 16u + u * 1024, most)));
  };
  const int at_end = lane < head ? lane : (lane >= 32 && lane - 32 < tail ? a.V - tail + lane - 32 : -1);
  S end = {};
  if (kAhead && head + tail > 0) end = row[max(at_end, 0)];
  Given<S> given;
  const bool writes = a.parts == 1 && wave == 0;
  if (W > 1 && writes) given.load_id(a, t, lane);
  float x[kPerLaneB];
  auto widen = [&](const u32x4 (&raw)[U], int b) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(S) == 2) {
          x[u * 8 + 2 * i] = __uint_as_float(raw[u][i] << 16);
          x[u * 8 + 2 * i + 1] = __uint_as_float(raw[u][i] & 0xffff0000u);
        } else {
          x[u * 4 + i] = __uint_as_float(raw[u][i]);
        }
      }
    if (kAhead && b >= full) {
#pragma unroll
      for (int j = 0; j < kPerLaneB; ++j) x[j] = (b * U + j / kVec) * 64 + lane < vectors ? x[j] : -INFINITY;
    }
  };
  Stream st;
  float bound = -INFINITY;
  // the batch in x.  rising: its ids lie behind all that the list has
  auto process = [&](bool rising, auto id) {
    const float thr = fmaxf(rising ? st.last : below(order_key(st.last)), bound);
    const float thr_d = fminf(thr > -INFINITY && st.ref > -INFINITY ? thr - st.at : -INFINITY, kLead);
    float d[kPerLaneB], top = -INFINITY;
#pragma unroll
    for (int j = 0; j < kPerLaneB; ++j) { d[j] = x[j] - st.at; top = fmaxf(top, d[j]); }
    if (__ballot(top >= thr_d)) {
      st.exchange(x, thr, n, lane, id);
#pragma unroll
      for (int j = 0; j < kPerLaneB; ++j) d[j] = x[j] - st.at;
    }
#pragma unroll
    for (int j = 0; j < kPerLaneB; ++j) st.add(j & 3, d[j]);
  };
  u32x4 raw[kRing][U];
  const int last = first < batches ? first + (batches - 1 - first) / stride * stride : -1;   // this wave's last batch
  if (last >= 0) {
#pragma unroll
    for (int i = 0; i < kRing; ++i) load(min(first + i * stride, last), raw[i]);
  }
  if (W > 1 && writes) given.load_entry(a, row);
  if (W > 1 ? part * W < batches : last >= 0) {
    float top = -INFINITY;
    if (last >= 0) {
#pragma unroll
      for (int i = 0; i < kRing; ++i) {
        widen(raw[i], min(first + i * stride, last));
#pragma unroll
        for (int j = 0; j < kPerLaneB; ++j) top = fmaxf(top, x[j]);   // a batch that is there twice counts as one
      }
    }
    // A quiet NaN is dropped, a signalling one at the end of the chain is not (earlier it takes what is in front of it along: a lower bound still).  The
    // compiler takes neither for possible.
    asm volatile("" : "+v"(top));
    if (top != top) top = -INFINITY;
    if constexpr (W > 1) {
      open_joint(s_joint, tid);
      if (n == 1) {                                        // an exchange in every wave costs less than the joint bound; four (9.2 us, 12.1 so) do not
        if (last >= 0) bound = below(order_key(wave_max(top)));
      } else {
        __syncthreads();
        bound = below(joint_bound(s_joint, top, last >= 0, min(W, batches - part * W), n, tid));
      }
    } else {
      bound = below(nth_bound(order_key(top), n));
    }
  } else if (W > 1) {
    open_joint(s_joint, tid);
  }
  for (int b = first; b <= last; b += kRing * stride) {
#pragma unroll
    for (int i = 0; i < kRing; ++i) {
      const int at = b + i * stride;
      if (at > last) break;
      widen(raw[i], at);
      load(min(at + kRing * stride, last), raw[i]);
      // a wave's ids rise from batch to batch, so an entry equal to its list's last comes behind it; one equal to another wave's may come before
      process(true, [&](int j) { return head + ((at * U + j / kVec) * 64 + lane) * kVec + j % kVec; });
    }
  }
  if constexpr (kAhead) {
    if (head + tail > 0) {
      x[0] = at_end < 0 ? -INFINITY : to_f32(end);
#pragma unroll
      for (int j = 1; j < kPerLaneB; ++j) x[j] = -INFINITY;
      process(false, [&](int) { return at_end; });
    }
  } else {
    // the batch that is not full, then head and tail
#pragma unroll 1
    for (int b = full + ((first - full) & (stride - 1)); b < full + 2; b += stride) {
      const bool ends = b > full;
      if (ends ? head + tail == 0 : vectors % (64 * U) == 0) continue;
      u32x4 rest[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        rest[u] = u32x4{kNegInf2, kNegInf2, kNegInf2, kNegInf2};
        const int v = (full * U + u) * 64 + lane;
        if (!ends && v < vectors) rest[u] = reinterpret_cast<const u32x4*>(body)[v];
      }
      if (ends && at_end >= 0) {
        if constexpr (sizeof(S) == 2) rest[0][0] = 0xff800000u | row[at_end]; else rest[0][0] = __float_as_uint(row[at_end]);
      }
      widen(rest, full);
      process(false, [&](int j) { return ends ? at_end : head + ((full * U + j / kVec) * 64 + lane) * kVec + j % kVec; });
    }
  }
  Sums sum = st.sums();
  if constexpr (W > 1) {
    Joint& s = s_joint;
    if (lane == 0) { s.ref[wave] = sum.ref; s.R[wave] = sum.R; s.A[wave] = sum.A; }
    put_list(s, W, wave, n, lane, st.list);
    sum = join(s, W, n, tid, st.list);
    if (wave) return;
  }
  if (a.parts > 1) {
    u64* o = a.ws + (t * a.parts + part) * partial_words(n);
    if (lane == 0) { o[0] = (u64)__float_as_uint(sum.R) << 32 | __float_as_uint(sum.ref); o[1] = __float_as_uint(sum.A); }
    if (lane < n) o[2 + lane] = st.list;
    return;
  }
  if constexpr (W == 1) {                                  // other rows' waves hide it
    given.load_id(a, t, lane);
    given.load_entry(a, row);
  }
  write_row<S>(a, t, st.list, sum, given, lane);
}

// Joins the parts of a row: one wave for each.
template <typename S>
__global__ __launch_bounds__(kMaxParts * 64) void logprobs_join_kernel(const LogprobArgs a) {
  __shared__ Joint s;
  const int tid = threadIdx.x, lane = tid & 63, part = uniform(tid >> 6);
  const int n = a.n_top > 1 ? a.n_top : 1;
  const int64_t t = blockIdx.x;
  const u64* in = a.ws + (t * a.parts + part) * partial_words(n);
  Given<S> given;
  if (part == 0) given.load_id(a, t, lane);
  u64 list = lane < n ? in[2 + lane] : 0;
  const u64 w0 = in[0], w1 = in[1];
  if (part == 0) given.load_entry(a, static_cast<const S*>(a.logits) + t * a.ld);
  open_joint(s, tid);
  if (lane == 0) {
    s.ref[part] = __uint_as_float((unsigned)w0);
    s.R[part] = __uint_as_float((unsigned)(w0 >> 32));
    s.A[part] = __uint_as_float((unsigned)w1);
  }
  put_list(s, a.parts, part, n, lane, list);
  const Sums sum = join(s, a.parts, n, tid, list);
  if (tid < 64) write_row<S>(a, t, list, sum, given, lane);
}
static_assert(kMaxParts <= kMaxLists && kList <= 64, "one thread per candidate");

// Waves per row part and parts per row.  us, waves x parts: 4096 rows of 131072 bf16 1x1 206, 4x1 222; 3000 of 50257 bf16 1x1 66.2, 4x1
// 72.4; 2300 of 50257 1x1 62.9, 4x1 57.0; 1999 of 50257 1x1 51.2, 4x1 51.3, 8x1 61.7, of 20000 fp32 1x1 32.0, 4x1 36.1; 1700 of 9000 bf16
// 1x1 18.4, 4x1 23.0; 1200 of 20000 fp32 1x1 29.3, 4x1 25.1; 600 of 56585 bf16 1x1 41.1, 4x1 28.0, 8x1 29.2; 478 of 56585 bf16, 20
// alternatives, 4x1 30.9, 8x1 26.3; 320 of it 4x1 30.0, 8x1 25.4; 300 of 50257 bf16 4x1 21.1, 8x1 18.8, 8x2 24.0; 128 of 151001 fp32 8x1
// 31.4, 8x2 27.2, 8x4 26.8, 8x8 35.0; 64 of 131072 fp32 8x1 35.7, 8x2 27.9, 8x4 22.5, 8x8 23.2; 16 of 131072 fp32 8x1 21.4, 8x4 15.0, 8x8
// 13.2, 8x16 13.5; 8 of 112000 fp32 8x1 17.9, 8x4 13.5, 8x8 12.4; 1 of 131072 bf16 8x1 17.6, 8x4 12.6, 8x8 11.7, 8x16 11.5; 1 of 79984 fp32
// 8x1 13.2, 8x4 11.5, 8x8 11.1; 32 of 50257 fp32 8x1 14.4, 8x2 14.1, 8x4 13.1; 128 of 50257 fp32 8x1 14.9, 8x2 15.7; 1 of 32000 fp32 8x1
// 8.2, 8x2 9.5, 8x4 8.5.  Sixteen waves were slower than eight everywhere (1 of 32000 8.6, 8 of 50257 13.5 against 13.1).
// Not kept, with eight waves: twice as many batches in registers (64 of 131072 fp32 with 20 alternatives 22.7 -> 22.0, with none 16.0 -> 16.9, 300 of
// 50257 bf16 17.0 -> 20.0); batches through LDS, and so one copy of the code instead of one per batch in flight (0.7 to 1 us more for few rows).
struct Split { int waves, parts; };
Split split_of(int T, int V) {
  const int batches = V / kBatch + 1;
  if (T >= 2560 || (T >= 1536 && batches < 32) || batches < 4) return {1, 1};
  if (T > 512 || batches < 8) return {4, 1};
  int parts = 1;
  if (batches >= 64 && T * 2 <= 256) parts = 2;
  if (batches >= 48 && T * 4 <= 256) parts = 4;
  if (batches >= 72 && T * 8 <= 256) parts = 8;
  if (batches >= 256 && T * kMaxParts <= 256) parts = kMaxParts;
  return {8, parts};
}

template <typename S>
int launch_rows(const LogprobArgs& a, int T, int waves, hipStream_t s) {
  const dim3 grid((unsigned)T * (unsigned)a.parts);
  switch (waves) {
    case 1: hipLaunchKernelGGL((logprobs_kernel<S, 1>), grid, dim3(64), 0, s, a); break;
    case 4: hipLaunchKernelGGL((logprobs_kernel<S, 4>), grid, dim3(256), 0, s, a); break;
    default: hipLaunchKernelGGL((logprobs_kernel<S, 8>), grid, dim3(512), 0, s, a); break;
  }
  int rc = hip_fail(hipGetLastError(), "logprobs_kernel launch");
  if (rc || a.parts == 1) return rc;
  hipLaunchKernelGGL(logprobs_join_kernel<S>, dim3((unsigned)T), dim3((unsigned)(a.parts * 64)), 0, s, a);
  return hip_fail(hipGetLastError(), "logprobs_join_kernel launch");
}
template <typename S>
int launch(const LogprobArgs& all, int T, int waves, hipStream_t s) {
  int rc = MOE_OK;
  for (int64_t t = 0; t < T && !rc; t += kLaunchRows) {     // more than one: a wave per row, no workspace
    LogprobArgs a = all;
    if (t) {
      a.logits = static_cast<const S*>(a.logits) + t * a.ld;
      a.tokens += t * a.n_given;                           // 0 where there is none
      a.token_logp += t * a.n_given;
      a.top_idx += t * a.n_top;
      a.top_logp += t * a.n_top;
      if (a.entropy) a.entropy += t;
      if (a.conf) a.conf += t;
    }
    rc = launch_rows<S>(a, (int)std::min<int64_t>(T - t, kLaunchRows), waves, s);
  }
  return rc;
}

}  // namespace

size_t logprobs_workspace_bytes(const moe_logprobs_config& c) {
  const Split sp = split_of(c.T, c.V);
  return sp.parts == 1 ? 0 : align256((size_t)c.T * sp.parts * partial_words(c.n_top > 1 ? c.n_top : 1) * sizeof(u64));
}

int launch_logprobs(const moe_logprobs_config& c, const void* logits, const int32_t* tokens, float* token_logp, float* entropy, float* conf,
                    int32_t* top_idx, float* top_logp, void* ws, hipStream_t s) {
  ProfScope ps(kProfLogprobs, s);
  const Split sp = split_of(c.T, c.V);
  const LogprobArgs a = {logits, c.ld, c.V, c.n_given, c.n_top, sp.parts, tokens, token_logp, entropy, conf, top_idx, top_logp, static_cast<u64*>(ws)};
  return c.dtype == MOE_FP32 ? launch<float>(a, c.T, sp.waves, s) : launch<uint16_t>(a, c.T, sp.waves, s);
}

}  // namespace mm
