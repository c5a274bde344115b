// Attention of one new token per sequence over a paged cache (moe_paged_attention).
//
// What bounds it: reading the keys and values that are seen, once per key head and 16 of its query heads (more heads to a key head read them again, from L2 at best).  The positions of all sequences, for each key head and up to 16 of its query heads, are a
// line of blocks that as many workgroups as run at once share equally (attention_plan.h), whatever the lengths are: 64 sequences of 400 to 8192 positions
// (32 heads on 8 of 128 channels, bf16, 1.1 GB) take 179 us, 6.2 TB/s; with a workgroup for each part of fixed length 191, of which the last ones ran alone.  A workgroup's
// segments are of one sequence and key head each, of which its waves take blocks in turn.
// Scores are the product of a tile of keys (rows: positions) and the queries (columns: heads), so that a lane has four positions of one head, which is where the
// product with the values wants the probabilities: nothing moves between lanes.  Values go into that product from where their rows lie, a lane with the same channels
// of four positions: two halves of different registers make an operand's word.  Keys are loaded by whole rows, too, and change lanes in LDS: straight into the operand's
// layout a load takes half a line of 16 rows, and the same sequences took 221 us.  Both products run on bf16 matrix instructions, exact in the keys, queries and values, and
// probabilities in three bf16 terms; caches in fp32 on fp32 ones.
// A block's keys are loaded again as soon as they are in LDS, its values as soon as they are used: a block and a half of each wave is on its way.  More waves or larger blocks
// did not help (2 or 3 workgroups per CU, 8 or 16 KB a wave: within 1 %), fewer bytes on their way did harm (one workgroup per CU: +15 %).
// Many short sequences are another matter: workgroups of one wave each, which have no waves to join or to wait for (128 sequences of up to 64 15.2 -> 11.0 us, on the long ones 186).
// The maximum that exponentials are taken against follows the scores only when one is 2^8 above it: sums stay far below fp32's range, and most blocks neither exchange
// maxima nor rescale.  Waves' sums are joined in LDS, parts' sums by the last of a unit's workgroups to end or, where parts are many, by a second
// kernel, all in a fixed order.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "groups.h"
#include "unaligned.h"

namespace mm {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kSlack = 8.f;                               // how far (log2) scores may be above the maximum in use
constexpr int kMaxPages = kMaxPiece / kMinPage;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;

// tanh: below 1 by Lambert's continued fraction to its sixth term (2^-29 off), beyond by 1 - 2 / (1 + e^2y).
__device__ __forceinline__ float capped(float y) {
  const float z = y * y;
  const float p = y * fmaf(z, fmaf(z, 21.f, 1260.f), 10395.f), q = fmaf(z, fmaf(z, z + 210.f, 4725.f), 10395.f);
  const float near = p * __builtin_amdgcn_rcpf(q), far = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y * (2.f * kLog2e)));
  return fabsf(y) < 1.f ? near : far;
}

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
  if constexpr (N == 8) return j < 4 ? v.lo[j & 3] : v.hi[j & 3];
  else return v[j];
}
// Element `at` of the operands of four channels from channel j on: bf16 values, or E4M3 codes times `share`, a power of two, widened exactly
template <typename C, typename R>
__device__ __forceinline__ void widen_four(const R& v, int j, int at, bool there, float share, bf16x8* to) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  bf16x2 a, b;
  if constexpr (sizeof(C) == 2) {
    a = __builtin_bit_cast(bf16x2, there ? dword(v, j / 2) : 0);
    b = __builtin_bit_cast(bf16x2, there ? dword(v, j / 2 + 1) : 0);
  } else {
    const unsigned d = there ? (unsigned)dword(v, j / 4) : 0u;
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d, share, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(d, share, true);
  }
  to[0][at] = a[0]; to[1][at] = a[1]; to[2][at] = b[0]; to[3][at] = b[1];
}

// Sums over a wave's lanes up to each, and over all, on the data-parallel primitives: rows of 16, lane 15 of a row into the next one, lane 31 into rows 2 and 3.
__device__ __forceinline__ int wave_sums(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_sums(v), 63); }

__device__ __forceinline__ float lane_max(float v) {        // over the four lanes of a column
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float lane_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
template <typename V>
__device__ __forceinline__ V load_queries(const AttentionArgs& a, int64_t at) {
  if (a.dtype == MOE_FP32) return load_unaligned<V>(static_cast<const float*>(a.q) + at);
  return __builtin_convertvector(load_unaligned<bf16x4>(static_cast<const __bf16*>(a.q) + at), V);
}
// The first head's row of what a workgroup has of a unit that lies in several: of the one that begins there, its last segment, or else of its first one.
__device__ __forceinline__ int64_t part_at(const AttentionArgs& a, int workgroup, bool begins) {
  return (2 * (int64_t)workgroup + begins) * min(a.group, kHeadTile);
}

// Exponentials are at most 2^kSlack, but for rounding, and a sequence sees n of them: times 2^-down, exactly, their sum is at most 1/2, so that no sum of values is larger than the
// largest value, whatever their sizes are.
__device__ __forceinline__ int down_by(const Seen& v) { return (int)kSlack + 1 + (v.end - v.first > 1 ? 32 - __builtin_clz(v.end - v.first - 1) : 0); }
__device__ __forceinline__ float two_to(int n) { return __int_as_float((127 + n) << 23); }
// Four channels of a result: sums v of values times exponentials and 2^-down, the maximum m (log2) that they are taken against and the sum l of the exponentials; without any, zeros.
__device__ __forceinline__ void store_row(const AttentionArgs& a, int b, int head, int channel, f32x4 v, float m, float l, int down) {
  const float over = l == 0.f ? 0.f : two_to(down) / l;
  const int64_t at = (int64_t)b * a.out_token + (int64_t)head * a.out_head + channel;
  v *= over;
  if (a.dtype == MOE_FP32) {
    store_unaligned(static_cast<float*>(a.out) + at, v);
  } else {
    store_unaligned(static_cast<__bf16*>(a.out) + at, __builtin_convertvector(v, bf16x4));
  }
  if (a.lse && channel == 0) a.lse[(int64_t)b * a.heads + head] = l == 0.f ? -INFINITY : fmaf(m, kLn2, logf(l));
}

// Tiles of 16 positions of a wave's block, and waves of a SIMD that the vector registers are shared by: as many as need no spills of them (with 20 the largest bf16 kernel
// took 18 % longer, on half as many workgroups again).  Scalar registers are short in all of these kernels: 55 to 93 of them wait in lanes of vector registers, none that the loop over
// blocks uses, so that it is short sequences that pay for it.
constexpr int block_tiles(size_t bytes, int dims) { return std::clamp(512 / (int)(dims * bytes), 1, 2); }
constexpr int waves_per_simd(size_t bytes, int dims, int parts) {
  if (dims > 128) return bytes < 4 && parts == 1 ? 2 : 1;
  if (dims > 64) return parts == 1 && bytes == 1 ? 3 : 2;
  return parts == 1 && bytes <= 2 ? 4 : 3;
}

// A wave's block of positions, and what its lanes load of it: values of positions 4 g .. 4 g + 3 of a tile, as the product with them wants them, and keys by whole
// rows, 16 bytes a lane, which go through LDS to the lane that has their position in the product with the queries.
template <typename C, int VW, int CHUNKS>
struct Block {
  static constexpr bool kF32 = sizeof(C) == 4, kCodes = sizeof(C) == 1;
  static constexpr int kDims = 16 * VW * CHUNKS;            // channels that registers are for
  static constexpr int kTiles = block_tiles(sizeof(C), kDims);      // tiles of 16 positions: 16 KB of keys and values up to 512 bytes a row
  static constexpr int kPositions = 16 * kTiles;
  static constexpr int kVec = 16 / sizeof(C);               // channels of 16 bytes
  static constexpr int kRowLanes = kDims / kVec;            // lanes of a row of keys
  static constexpr int kLoads = kRowLanes / 4;              // rows of a tile that a lane loads of, and its vectors in the product
  static constexpr int kKeyBytes = kPositions * kRowLanes * 16;
  typedef typename Raw<C, VW>::type RawV;
  typedef typename std::conditional<kF32, f32x4, i32x4>::type RawK;
  RawK k[kTiles][kLoads];
  RawV v[kTiles][4][CHUNKS];
  float scale;                                              // of a key (lanes below 32) or value: position lane % 32; through LDS to the lanes that multiply by it
  // where vector c of row r of a tile is in LDS: eight rows' vectors of the same c fall on different banks
  static __device__ __forceinline__ int place(int r, int c) {
    constexpr int kRows = kRowLanes < 16 ? 16 / kRowLanes : 1;        // of 256 bytes, all banks
    return (r * kRowLanes + (c ^ (r / kRows & (kRowLanes < 16 ? kRowLanes - 1 : 15)))) * 16;
  }
};
// Loads past the caches: keys and values are read once (64 sequences as above: with ordinary loads 214 us, then 191).
template <typename T>
__device__ __forceinline__ T load_once(const T* p) { return __builtin_nontemporal_load(p); }
__device__ __forceinline__ Eight load_once(const Eight* p) { return {load_once(&p->lo), load_once(&p->hi)}; }

// What workgroups hand to each other through memory goes past their XCDs' caches.
typedef __attribute__((ext_vector_type(2))) float f32x2;
__device__ __forceinline__ void hand_over(float* p, f32x2 v) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 taken_over(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// kWaves: of a workgroup.  C: type of the cache's rows.  A row of the head is CHUNKS chunks of 16 VW channels, VW of them a lane (D below that: RAGGED).  PARTS: bf16 terms of a query,
// 1 of a bf16 one and 3 of an fp32 one, exact; keys of fp32 are multiplied in fp32.
template <typename C, int VW, int CHUNKS, int PARTS, bool RAGGED, int kWaves>
__global__ __launch_bounds__(64 * kWaves, waves_per_simd(sizeof(C), 16 * VW * CHUNKS, PARTS)) void attention_kernel(const AttentionArgs a) {
  typedef Block<C, VW, CHUNKS> Blk;
  constexpr int kThreads = 64 * kWaves;
  constexpr bool kF32 = Blk::kF32, kCodes = Blk::kCodes;
  constexpr int kDims = Blk::kDims, kTiles = Blk::kTiles, kBlock = Blk::kPositions, kVec = Blk::kVec, kLoads = Blk::kLoads;
  constexpr int kSteps = kDims / 32;                        // of the scores' contraction: 32 channels, 8 a lane
  __shared__ int s_page[kMaxPages];
  // keys of the waves' blocks, in the end their sums
  constexpr int kOutBytes = 16 * 16 * VW * 4, kWaveBytes = Blk::kKeyBytes > kOutBytes ? Blk::kKeyBytes : kOutBytes;
  __shared__ __attribute__((aligned(16))) char s_mem[kWaves * kWaveBytes];
  __shared__ float s_max[kWaves][16], s_sum[kWaves][16];
  __shared__ __attribute__((aligned(16))) float s_scale[kCodes ? kWaves : 1][2][32];
  __shared__ int s_bad, s_last;
  fetch_arguments<sizeof(AttentionArgs)>();

  const int tiles = (a.group + kHeadTile - 1) / kHeadTile, units = a.kv_heads * tiles;
  int workgroup;
  auto seen_with = [&](int length) { return seen_by(length, a.max_len, a.window, a.table_len, a.shift); };
  auto seen_of = [&](int b) { return seen_with(uniform(a.lengths[b])); };       // b: the same in all lanes

  // ---- the line: its length, and the sequence in which this workgroup's share begins; every wave by itself ----
  int cursor, finish, each, b = 0, line = 0, length = 0;
  {
    const int lane = threadIdx.x & 63;
    auto length_of = [&](int i) { return i < a.B ? a.lengths[i] : 0; };
    auto on_line = [&](int length) { return line_places(blocks_of(seen_with(length)), a.align) * units; };
    const int first_64 = length_of(lane);
    int total = on_line(first_64);
    for (int i = lane + 64; i < a.B; i += 64) total += on_line(a.lengths[i]);
    total = wave_total(total);
    each = places_each(total, a.workgroups, a.align, kLeast);
    // neighbours on the line run on the same XCD of the 8 that take workgroups in turn: tiles of a large group read the same keys and values.  The grid is whole eights.
    const int active = (total + each - 1) / each, run = (active + 7) / 8;
    workgroup = blockIdx.x / 8 < run ? blockIdx.x % 8 * run + blockIdx.x / 8 : active;
    cursor = min(total, min(workgroup, active) * each);
    finish = min(total, cursor + each);
    if (a.started && blockIdx.x == 0 && threadIdx.x == 0) a.started[4 * a.workgroups] = active;
    if (cursor < finish)
      for (;; b += 64) {                                    // ends at the sequence that holds the place
        const int there = b ? length_of(b + lane) : first_64, n = on_line(there), upto = line + wave_sums(n);
        const uint64_t behind = __ballot(cursor < upto);
        if (behind) {
          const int at = __builtin_ctzll(behind);
          line = __builtin_amdgcn_readlane(upto - n, at);
          length = __builtin_amdgcn_readlane(there, at);
          b += at;
          break;
        }
        line = __builtin_amdgcn_readlane(upto, 63);
      }
  }
  // ---- sequences without anything to see, or of a length that there is not: pieces of their rows to each workgroup ----
  constexpr int kRowPiece = 4 * kThreads;
  const int row_vecs = a.heads * (a.D / 4), pieces = (row_vecs + kRowPiece - 1) / kRowPiece;
  for (int64_t e = blockIdx.x; e < (int64_t)a.B * pieces; e += gridDim.x) {
    const int sequence = (int)(e / pieces), from = (int)(e % pieces) * kRowPiece;
    const Seen v = seen_of(sequence);
    if (v.first < v.end) continue;
    const float l = v.bad ? __uint_as_float(0x7fc00000u) : 0.f;
    for (int i = from + threadIdx.x; i < min(from + kRowPiece, row_vecs); i += kThreads)
      store_row(a, sequence, i / (a.D / 4), i % (a.D / 4) * 4, f32x4{0.f, 0.f, 0.f, 0.f}, -INFINITY, l, 0);
  }
  if (cursor >= finish) return;
  if (a.started && threadIdx.x < 4) a.started[4 * workgroup + threadIdx.x] = 0;
  int listed_b = -1, listed_from = 0, listed_to = 0;        // whose pages' numbers are in LDS

  // ================= the segments of the share =================
  while (true) {
  // what follows from the lane is worked out anew for each segment: held over all of them it would not leave registers enough
  const int wave = uniform(threadIdx.x >> 6);
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, n = lane & 15, g = lane >> 4;
  const Seen seen = seen_with(length);
  const int next_length = a.lengths[min(b + 1, a.B - 1)];   // on its way meanwhile
  const Segment seg = segment_at(line, blocks_of(seen), a.align, cursor, finish, each);
  if (seg.blocks) {
  const int tile = seg.unit % tiles, kvh = seg.unit / tiles;
  const int heads = min(kHeadTile, a.group - tile * kHeadTile), head0 = kvh * a.group + tile * kHeadTile;
  const int32_t* const row = a.table + b * a.table_ld;
  bf16x8 qf[kF32 ? 1 : PARTS][kSteps];
  float q32[kF32 ? kDims / 4 : 1];
  {
    const int64_t q_at = (int64_t)b * a.q_token + (int64_t)(head0 + min(n, heads - 1)) * a.q_head;
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < kDims / 4; i += 4) {
        const int d = 4 * i + 4 * g;
        const f32x4 q = n < heads && (!RAGGED || d < a.D) ? load_queries<f32x4>(a, q_at + d) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; ++e) q32[i + e] = q[e];
      }
    } else {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = kCodes ? 64 * (s / 2) + 16 * g + 8 * (s % 2) : 32 * s + 8 * g;      // the order of the keys' vectors
        const bool there = n < heads && (!RAGGED || d < a.D);
        if constexpr (PARTS == 1) {
          qf[0][s] = there ? load_unaligned<bf16x8>(static_cast<const __bf16*>(a.q) + q_at + d) : bf16x8{};
        } else {
          f32x8 q = there ? load_unaligned<f32x8>(static_cast<const float*>(a.q) + q_at + d) : f32x8{};
#pragma unroll
          for (int t = 0; t < PARTS; ++t) {
            qf[t][s] = __builtin_convertvector(q, bf16x8);
            q -= __builtin_convertvector(qf[t][s], f32x8);
          }
        }
      }
    }
  }
  const float to_log2 = a.scale * kLog2e;
  const int down = down_by(seen);
  const float share = two_to(-down);
  const C* const kbase = static_cast<const C*>(a.k) + (int64_t)kvh * a.head;
  const C* const vbase = static_cast<const C*>(a.v) + (int64_t)kvh * a.head;
  const int mask = (1 << a.shift) - 1;
  char* const keys = s_mem + wave * kWaveBytes;

  float top = -INFINITY, sum = 0.f;
  f32x4 acc[CHUNKS][VW];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int j = 0; j < VW; ++j) acc[c][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  bool bad = false;

  // ---- pieces of the segment, as long as LDS has room for their pages' numbers ----
  const int segment_begin = (seen.first / kSpan + seg.block) * kSpan, segment_end = (int)min((int64_t)seen.end, (int64_t)segment_begin + (int64_t)seg.blocks * kSpan);
  for (int piece = segment_begin; piece < segment_end; piece += kMaxPiece) {
  const struct { int begin, end; } p = {piece, (int)min((int64_t)segment_end, (int64_t)piece + kMaxPiece)};
  const int first = max(seen.first, p.begin), entry0 = p.begin >> a.shift, entries = (((p.end - 1) | (kSpan - 1)) >> a.shift) - entry0 + 1;
  __syncthreads();
  if (b != listed_b || p.begin != listed_from || p.end != listed_to) {      // the next key head's are the same
  listed_b = b; listed_from = p.begin; listed_to = p.end;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  for (int i = tid; i < entries; i += kThreads) {
    const int64_t from = (int64_t)(entry0 + i) << a.shift;
    int page = 0;                                           // of positions that are not seen: any
    if (from < p.end && from + ((int64_t)1 << a.shift) > first) page = page_of(row, a.table_len, a.n_pages, a.shift, from);
    if (page < 0) { s_bad = 1; page = 0; }                  // a number outside the cache spoils the sequence
    s_page[i] = page;
  }
  __syncthreads();
  }
  bad |= s_bad;

  Blk r;
  // The queries are here before the loop begins, so that no wait for them stands in it.
  if constexpr (kF32) {
#pragma unroll
    for (int i = 0; i < kDims / 4; ++i) asm volatile("" : "+v"(q32[i]));
  } else {
#pragma unroll
    for (int t = 0; t < PARTS; ++t)
#pragma unroll
      for (int s = 0; s < kSteps; ++s) asm volatile("" : "+v"(qf[t][s]));
  }
  // Behind the part's end every lane reads the first row: a load in a branch would make each wait behind it one for all loads on their way.
  auto load_keys = [&](int t0) {
    const bool any = t0 < p.end;
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
#pragma unroll
      for (int s = 0; s < kLoads; s += kLoads < 4 ? kLoads : 4) {
        const int tk = t0 + 16 * u + lane / Blk::kRowLanes * kLoads + s, c = lane % Blk::kRowLanes * kVec;
        const C* krow = kbase + (any ? (int64_t)s_page[any ? (tk >> a.shift) - entry0 : 0] * a.page + (int64_t)(tk & mask) * a.row + c : 0);
#pragma unroll
        for (int i = 0; i < (kLoads < 4 ? kLoads : 4); ++i)
          r.k[u][s + i] = !RAGGED || c < a.D ? load_once(reinterpret_cast<const typename Blk::RawK*>(krow + i * a.row)) : typename Blk::RawK{0, 0, 0, 0};
      }
    }
    if constexpr (kCodes) {
      const int ts = t0 + lane % kBlock;
      const int64_t at = any ? (((int64_t)s_page[(ts >> a.shift) - entry0] * a.kv_heads + kvh) << a.shift) + (ts & mask) : 0;
      r.scale = load_once((lane < 32 ? a.k_scale : a.v_scale) + at);
    }
  };
  auto load_values = [&](int t0) {
    const bool any = t0 < p.end;
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      const int tv = t0 + 16 * u + 4 * g;
      const int64_t page = s_page[any ? (tv >> a.shift) - entry0 : 0];
      const C* vrow = vbase + (any ? page * a.page + (int64_t)(tv & mask) * a.row + VW * n : 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const int d = 16 * VW * c;
          r.v[u][i][c] = !RAGGED || d + VW * n < a.D ? load_once(reinterpret_cast<const typename Blk::RawV*>(vrow + i * a.row + d)) : zeros(typename Blk::RawV{});
        }
    }
  };
  auto use = [&](int t0, int next) {
    // ---- scores, in units of log 2 ----
    const bool whole = t0 >= first && t0 + kBlock <= p.end;
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int s = 0; s < kLoads; ++s) *reinterpret_cast<typename Blk::RawK*>(keys + u * 16 * Blk::kRowLanes * 16 + Blk::place(lane / Blk::kRowLanes * kLoads + s, lane % Blk::kRowLanes)) = r.k[u][s];
    f32x4 ks[kTiles], vs[kTiles];
    if constexpr (kCodes) s_scale[wave][lane / 32][lane % 32] = r.scale;
    asm volatile("" ::: "memory");                          // other lanes' writes: a wave's LDS operations run in order
    if constexpr (kCodes) {
#pragma unroll
      for (int u = 0; u < kTiles; ++u) {
        ks[u] = *reinterpret_cast<const f32x4*>(&s_scale[wave][0][16 * u + 4 * g]);
        vs[u] = *reinterpret_cast<const f32x4*>(&s_scale[wave][1][16 * u + 4 * g]);
      }
    }
    load_keys(next);
    float x[kTiles][4];
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < kTiles; ++u) {
      f32x4 z = {0.f, 0.f, 0.f, 0.f};
      typename Blk::RawK kf[kLoads];
#pragma unroll
      for (int s = 0; s < kLoads; ++s) kf[s] = *reinterpret_cast<const typename Blk::RawK*>(keys + u * 16 * Blk::kRowLanes * 16 + Blk::place(n, 4 * s + g));
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < kDims / 4; ++i) z = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[i / 4][i % 4], q32[i], z, 0, 0, 0);
      } else {
#pragma unroll
        for (int t = PARTS - 1; t >= 0; --t)                // small terms first
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            bf16x8 key;
            if constexpr (kCodes) key = widen_e4m3(kf[s / 2][s % 2 * 2], kf[s / 2][s % 2 * 2 + 1]);
            else key = __builtin_bit_cast(bf16x8, kf[s]);
            z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, qf[t][s], z, 0, 0, 0);
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = z[i];
        if constexpr (kCodes) v *= ks[u][i];
        x[u][i] = v * to_log2;
      }
    }
    if (a.softcap > 0.f) {
      const float cap = a.softcap * kLog2e, per = 1.f / cap;
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[u][i] = cap * capped(x[u][i] * per);
    }
    auto hidden = [&](int u, int i) { const int t = t0 + 16 * u + 4 * g + i; return t < first || t >= p.end; };
    if (!whole) {                                           // what is not seen counts as nothing, whatever it is
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[u][i] = hidden(u, i) ? -INFINITY : x[u][i];
    }
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, x[u][i]);
    if (__any(most > top + kSlack)) {
      const float now = lane_max(fmaxf(top, most));
      const float alpha = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - now);
      top = now;
      sum *= alpha;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < VW; ++j) acc[c][j] *= alpha;
    }
    const float base = top == -INFINITY ? 0.f : top;
    float e[kTiles][4];
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        e[u][i] = __builtin_amdgcn_exp2f(x[u][i] - base);
        sum += e[u][i];
      }
    if (!whole) {
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool no = hidden(u, i);
          if constexpr (kCodes) vs[u][i] = no ? 0.f : vs[u][i];
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c) r.v[u][i][c] = no ? zeros(typename Blk::RawV{}) : r.v[u][i][c];
        }
    }
#pragma unroll
    for (int u = 0; u < kTiles; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) e[u][i] *= kCodes ? vs[u][i] : share;         // 8-bit values have it in their conversion, so that weights of small rows stay normal numbers
    // ---- values ----
    if constexpr (kF32) {
#pragma unroll
      for (int u = 0; u < kTiles; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < VW; ++j)
              acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(element<C, VW>(r.v[u][i][c], j), e[u][i], acc[c][j], 0, 0, 0);
    } else {
      // position 4 g + i of tile u is operand element 4 (u % 2) + i of lane group g in both; probabilities in three bf16 terms, which hold all of their 24 bits (of
      // 122880 bf16 results over 200 positions 39 are not the nearest ones to the definition's in 64 bits, with two terms 195, with sums in fp32 of torch 47)
#pragma unroll
      for (int u0 = 0; u0 < kTiles; u0 += 2) {
        constexpr int kTerms = 3;
        f32x8 w;
        bf16x8 term[kTerms];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) w[4 * u + i] = u0 + u < kTiles ? e[u0 + u < kTiles ? u0 + u : 0][i] : 0.f;
#pragma unroll
        for (int t = 0; t < kTerms; ++t) {
          term[t] = __builtin_convertvector(w, bf16x8);
          w -= __builtin_convertvector(term[t], f32x8);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
          for (int j = 0; j < VW; j += 4) {
            bf16x8 value[4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) widen_four<C>(r.v[u0 + u < kTiles ? u0 + u : 0][i][c], j, 4 * u + i, u0 + u < kTiles, share, value);
#pragma unroll
            for (int t = kTerms - 1; t >= 0; --t)           // small terms first
#pragma unroll
              for (int o = 0; o < 4; ++o) acc[c][j + o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value[o], term[t], acc[c][j + o], 0, 0, 0);
          }
      }
    }
    load_values(next);
  };

  // ---- the piece's blocks in turn over the waves; keys of the next one are loaded as soon as this one's are used, and values ----
  constexpr int kStride = kWaves * kBlock;
  int t0 = p.begin + (first - p.begin) / kBlock * kBlock + wave * kBlock;
  if (t0 < p.end) { load_keys(t0); load_values(t0); }
  for (; t0 < p.end; t0 += kStride) use(t0, t0 + kStride);
  }

  // ---- join the waves ----
  {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, n = lane & 15, g = lane >> 4;
  sum = lane_sum(sum);
  if (g == 0) { s_max[wave][n] = top; s_sum[wave][n] = sum; }
  __syncthreads();
  const float nan = __uint_as_float(0x7fc00000u);
  auto joined = [&](int head, float* m, float* l) {
    *m = s_max[0][head];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) *m = fmaxf(*m, s_max[w][head]);
    *l = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) *l += s_max[w][head] == -INFINITY ? s_sum[w][head] : s_sum[w][head] * __builtin_amdgcn_exp2f(s_max[w][head] - *m);
    if (bad) *l = nan;
  };
  float m, l;
  joined(n, &m, &l);
  const float weight = top == -INFINITY ? (sum == 0.f ? 0.f : sum) : __builtin_amdgcn_exp2f(top - m);     // a sum without a maximum is NaN
  const int64_t part_row = part_at(a, workgroup, seg.block == 0);
  // where four channels of a head's sums are in LDS: the same ones of the 16 heads fall on different banks
  auto sums_at = [](int head, int quad) { return 16 * (head * 4 * VW + (quad ^ (head & (4 * VW - 1)))); };
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    if (c) __syncthreads();
    if (n < heads) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < VW; j += 4)
          *reinterpret_cast<f32x4*>(keys + sums_at(n, (VW * (4 * g + i) + j) / 4)) =
              f32x4{acc[c][j][i], acc[c][j + 1][i], acc[c][j + 2][i], acc[c][j + 3][i]} * weight;
    }
    __syncthreads();
    for (int o = tid; o < heads * 4 * VW; o += kThreads) {
      const int head = o / (4 * VW), quad = o % (4 * VW), channel = 16 * VW * c + 4 * quad;
      if (head >= heads || channel >= a.D) continue;
      f32x4 v = *reinterpret_cast<const f32x4*>(s_mem + sums_at(head, quad));
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += *reinterpret_cast<const f32x4*>(s_mem + w * kWaveBytes + sums_at(head, quad));
      joined(head, &m, &l);
      if (seg.parts > 1) {
        float* to = a.part_out + (part_row + head) * a.D + channel;
        const f32x2 stat = {l == l ? m : nan, l};           // a sum that is none spoils the whole row
        if (a.counters) {
          hand_over(to, f32x2{v[0], v[1]});
          hand_over(to + 2, f32x2{v[2], v[3]});
          if (channel == 0) hand_over(a.part_stat + 2 * (part_row + head), stat);
        } else {
          *reinterpret_cast<f32x4*>(to) = v;
          if (channel == 0) *reinterpret_cast<f32x2*>(a.part_stat + 2 * (part_row + head)) = stat;
        }
      } else {
        store_row(a, b, head0 + head, channel, v, m, l, down);
      }
    }
  }
  if (seg.parts > 1 && a.counters) {
    // ---- the last of a unit's parts to end joins them, in their order ----
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // what was handed over is there
    __syncthreads();
    if (tid == 0) {
      int* counter = a.counters + seg.workgroup;
      const int ended = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
      if (ended == seg.parts) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);     // as the next call finds it
      s_last = ended == seg.parts;
    }
    __syncthreads();
    if (s_last) {
      const int vecs = a.D / 4;
      for (int o = tid; o < heads * vecs; o += kThreads) {
        const int head = o / vecs, channel = o % vecs * 4;
        float most = -INFINITY, l = 0.f;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        constexpr int kAhead = 8;
        for (int i0 = 0; i0 < seg.parts; i0 += kAhead) {
          f32x2 st[kAhead], lo[kAhead], hi[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            const int part = min(i0 + i, seg.parts - 1);
            const int64_t at = part_at(a, seg.workgroup + part, part == 0) + head;
            st[i] = taken_over(a.part_stat + 2 * at);
            lo[i] = taken_over(a.part_out + at * a.D + channel);
            hi[i] = taken_over(a.part_out + at * a.D + channel + 2);
          }
          float now = most;
#pragma unroll
          for (int i = 0; i < kAhead; ++i) now = fmaxf(now, st[i][0]);
          const float alpha = most == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(most - now);
          most = now;
          l = l == l ? l * alpha : l;
          v *= alpha;
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            const float w = i0 + i >= seg.parts || st[i][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[i][0] - most);
            if (i0 + i < seg.parts) l += w * st[i][1];
            v += w * f32x4{lo[i][0], lo[i][1], hi[i][0], hi[i][1]};
          }
        }
        store_row(a, b, head0 + head, channel, v, most, l, down);
      }
    }
  }
  if (seg.parts > 1 && seg.block == 0 && a.started && tid < 4) a.started[4 * workgroup + tid] = tid == 0 ? seg.parts : tid == 1 ? b : tid == 2 ? seg.unit : down;
  }

  __syncthreads();
  }
  cursor += seg.length;
  if (cursor >= finish) break;
  const int behind = line + line_places(blocks_of(seen), a.align) * units;
  if (cursor >= behind) {
    line = behind;
    ++b;
    length = uniform(next_length);
    while (blocks_of(seen_with(length)) == 0) length = uniform(a.lengths[++b]);
  }
  }
}

// The same of units of many parts: a workgroup for each workgroup of the first kernel in which a unit begins that ends in another one, and for each of its heads; four channels
// a thread, the parts in turn over the threads of a channel.  512 threads, both kernels
// together: 21.3 us for 32 heads over 16000 positions (24.8 with 1024 threads, 20.8 with 256), 91.5 over 131072 (93.4 with 1024, 93.3 with 256).
constexpr int kJoinThreads = 512;
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const AttentionArgs a) {
  __shared__ float s_top[kJoinThreads / 64];
  __shared__ __attribute__((aligned(16))) f32x4 s_v[kJoinThreads];
  __shared__ float s_l[kJoinThreads];
  const int tid = threadIdx.x, workgroup = blockIdx.x, parts = workgroup < a.started[4 * a.workgroups] ? a.started[4 * workgroup] : 0, b = a.started[4 * workgroup + 1], unit = a.started[4 * workgroup + 2], down = a.started[4 * workgroup + 3];
  const int tiles = (a.group + kHeadTile - 1) / kHeadTile, tile = unit % tiles, h = blockIdx.y, head = unit / tiles * a.group + tile * kHeadTile + h;
  if (parts == 0 || h >= a.group - tile * kHeadTile) return;
  auto at = [&](int part) { return part_at(a, workgroup + part, part == 0) + h; };
  float m = -INFINITY;
  for (int i = tid; i < parts; i += kJoinThreads) m = fmaxf(m, a.part_stat[2 * at(i)]);
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) s_top[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / 64; ++w) m = fmaxf(m, s_top[w]);
  const int vecs = a.D / 4, turns = kJoinThreads / vecs, turn = tid / vecs, d = tid % vecs * 4;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  if (turn < turns) {
#pragma unroll 8
    for (int i = turn; i < parts; i += turns) {
      const f32x2 st = *reinterpret_cast<const f32x2*>(a.part_stat + 2 * at(i));
      const float w = st[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[0] - m);
      l += w * st[1];
      v += w * *reinterpret_cast<const f32x4*>(a.part_out + at(i) * a.D + d);
    }
  }
  s_v[tid] = v;
  s_l[tid] = l;
  __syncthreads();
  if (tid >= vecs) return;
  for (int t = 1; t < turns; ++t) { v += s_v[t * vecs + tid]; l += s_l[t * vecs + tid]; }
  store_row(a, b, head, d, v, m, l, down);
}

template <typename C, int VW, int CHUNKS, int PARTS, bool RAGGED>
int launch_waves(const AttentionArgs& a, hipStream_t s) {
  const int grid = (a.workgroups + 7) / 8 * 8;
  if (a.waves == 1) attention_kernel<C, VW, CHUNKS, PARTS, RAGGED, 1><<<grid, 64, 0, s>>>(a);
  else attention_kernel<C, VW, CHUNKS, PARTS, RAGGED, kMostWaves><<<grid, 64 * kMostWaves, 0, s>>>(a);
  return hip_fail(hipGetLastError(), "attention_kernel");
}
template <typename C, int VW, int CHUNKS, int PARTS>
int launch_dims(const AttentionArgs& a, hipStream_t s) {
  return a.D < 16 * VW * CHUNKS ? launch_waves<C, VW, CHUNKS, PARTS, true>(a, s) : launch_waves<C, VW, CHUNKS, PARTS, false>(a, s);
}
template <typename C, int PARTS>
int launch_parts(const AttentionArgs& a, hipStream_t s) {
  if (a.D <= 64) return launch_dims<C, 4, 1, PARTS>(a, s);
  if (a.D <= 128) return launch_dims<C, 8, 1, PARTS>(a, s);
  return launch_dims<C, 8, 2, PARTS>(a, s);
}
template <typename C>
int launch_cache(const AttentionArgs& a, hipStream_t s) {
  return a.dtype == MOE_FP32 ? launch_parts<C, 3>(a, s) : launch_parts<C, 1>(a, s);
}

}  // namespace

int attention_slots(int cache_dtype, int D, int dtype) {
  const size_t bytes = cache_dtype == MOE_FP32 ? 4 : cache_dtype == MOE_E4M3 ? 1 : 2;
  return device_cu_count() * waves_per_simd(bytes, D <= 64 ? 64 : D <= 128 ? 128 : 256, bytes == 4 || dtype == MOE_BF16 ? 1 : 3);
}

int launch_attention(const AttentionArgs& a, hipStream_t s) {
  ProfScope prof(kProfAttention, s);
  int rc;
  if (a.cache_dtype == MOE_FP32) rc = launch_parts<float, 1>(a, s);
  else if (a.cache_dtype == MOE_E4M3) rc = launch_cache<uint8_t>(a, s);
  else rc = launch_cache<__bf16>(a, s);
  if (rc || !a.started) return rc;
  join_kernel<<<dim3(a.workgroups, std::min(a.group, kHeadTile)), kJoinThreads, 0, s>>>(a);
  return hip_fail(hipGetLastError(), "join_kernel");
}

}  // namespace mm
