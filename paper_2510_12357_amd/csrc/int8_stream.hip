// The 8-bit product for up to 64 tokens: every weight is read once, so memory sets the pace, and for small weights the latency of a launch.
//
// A workgroup of eight waves, one per CU, keeps the codes of all tokens in its registers: `split` waves share K, each holding its part of it, and
// weights are all that streams.  A wave goes through blocks of 16 weight rows in chunks of 256 k, by a ring of four chunks of its own in LDS, which
// loads fill past the registers, sixteen lanes reading 256 bytes of a row; the ring runs on from block to block.  (Operands straight from memory
// into registers, in the matrix instruction's order, touch a row per lane, 64 lines an instruction, and the address units set the pace: 64 x 131072 x
// 4096 took 227 us so.  With the codes loaded beside every chunk 180, in tiles of 128 rows that share them in LDS 135 - 144; chunks of 128 bytes of 32
// rows instead of 256 of 16 cost 9 % with 16 tokens.)  Waves that share K add their sums of integers up in LDS, exactly, one barrier a
// block; without a split there is no barrier.
// Measured: 64 x 131072 x 4096 102 us (5.5 TB/s of weights and outputs), 16 x 131072 x 4096 91 (5.9), 8 x 131072 x 16384 332 (6.5), 1 x 32000 x 2048 with its
// quantisation 13.4 (4.9), 8 x 2048 x 2048 6.5; a plain read gets 6.9.
// Where the codes come from: the caller's rows; the workspace of moe_linear_int8, in the order of the matrix instruction's lanes, so that a load is
// 1 KB in one piece; or float tokens that every workgroup quantises for itself, which saves a launch in front of this one
// (both ways measured: int8_route.cpp).
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "groups.h"
#include "int8_device.h"
#include "unaligned.h"

namespace mm {
namespace {

typedef __attribute__((address_space(3))) void lds_void;

constexpr int kWavesS = kStreamWaves, kThreadsS = kWavesS * 64;
constexpr int kRing = 4, kRowBytes = kStreamChunk, kStage = 16 * kRowBytes, kRingBytes = kWavesS * kRing * kStage;
constexpr int kSteps = kRowBytes / 64;                     // matrix instructions (16 x 16 x 64) of a chunk
constexpr int kMaxRows = 512;                              // weight rows of a workgroup: their scales and biases are kept in LDS
constexpr int kScaleBytes = 2 * kMaxRows * 4;
constexpr int code_pitch(int K) { return ((K + 15) / 16 | 1) * 16; }   // bytes of a token's codes in LDS: 16 tokens start at 16 different banks
constexpr int code_bytes(int T, int K) { return T * code_pitch(K) + kRowBytes; }   // a chunk may reach behind the last token's
constexpr int sum_bytes(int TB, int split) { return split > 1 ? 2 * (kWavesS / split) * TB * 1024 : 0; }

enum Tokens { kRows, kLanes, kFloats };                    // where codes come from, as above
struct FloatTokens { const void* x; int64_t ldx; };

// At most N loads of this wave in flight.  An asm block, so that no load moves across it; the LDS accesses below are asm blocks too, because the
// compiler would wait for every load into LDS in front of its own.
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void read4(i32x4 (&v)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3) {
  asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]) : "v"(a0), "v"(a1), "v"(a2), "v"(a3) : "memory");
}
__device__ __forceinline__ float read_float(unsigned at) {
  float v;
  asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(at) : "memory");
  return v;
}
// The sums of a block of 16 tokens: four words of 64 lanes each, one behind the other.
// reads a sum and leaves zeros behind
__device__ __forceinline__ i32x4 take_sum(unsigned at) {
  typedef __attribute__((ext_vector_type(2))) int i32x2;
  i32x2 lo, hi;
  asm volatile("ds_read2st64_b32 %0, %2 offset0:0 offset1:1\n\tds_read2st64_b32 %1, %2 offset0:2 offset1:3\n\ts_waitcnt lgkmcnt(0)\n\t"
               "ds_write2st64_b32 %2, %3, %3 offset0:0 offset1:1\n\tds_write2st64_b32 %2, %3, %3 offset0:2 offset1:3"
               : "=&v"(lo), "=&v"(hi) : "v"(at), "v"(0) : "memory");
  return i32x4{lo[0], lo[1], hi[0], hi[1]};
}
// adds the result of a matrix instruction that may have just been issued
__device__ __forceinline__ void add_sum(unsigned at, i32x4 v) {
  asm volatile("s_nop 15\n\tds_add_u32 %0, %1\n\tds_add_u32 %0, %2 offset:256\n\tds_add_u32 %0, %3 offset:512\n\tds_add_u32 %0, %4 offset:768"
               :: "v"(at), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]) : "memory");
}

// TB: blocks of 16 tokens, 1, 2 or 4.  X: type of float tokens.
template <typename S, Tokens FROM, typename X, int TB>
__global__ __launch_bounds__(kThreadsS) __attribute__((amdgpu_waves_per_eu(2, 2))) void int8_stream_kernel(const Int8Args a, const FloatTokens f, const int split,
                                                                                                          const int turns) {
  constexpr int kChunks = stream_chunks(TB);
  extern __shared__ __attribute__((aligned(1024))) char s_mem[];   // the rings, scales and biases, sums, codes of float tokens
  __shared__ unsigned s_max[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int c = lane & 15, g = lane >> 4;                  // token (or weight row) and group of 16 k of a lane's operand
  const int part = wave & (split - 1), group = wave / split, groups = kWavesS / split;
  const int row0 = blockIdx.x * turns * groups * 16;       // turn j of this wave's group: rows row0 + 16 (j groups + group) ..
  const int rows = min(a.N - row0, turns * groups * 16);
  const int Kw = (a.K + 15) & ~15;                         // behind K, the tokens' codes are zero
  const int chunks = (Kw + kRowBytes - 1) / kRowBytes, first = chunks * part / split, n = chunks * (part + 1) / split - first;
  const unsigned lds0 = (unsigned)(size_t)s_mem, scales_at = lds0 + kRingBytes, sums_at = scales_at + kScaleBytes;

  // ---- float tokens: `per` threads for one, in turn for each of its vectors, of which they hold the first ones.  Loads end in order: these first ----
  constexpr int kVec = 16 / sizeof(X), kHeld = 4;
  int per = kThreadsS;
  while (per > 32 && per * a.T > kThreadsS) per >>= 1;
  const int ft = tid / per, fat = tid % per;
  const X* const frow = static_cast<const X*>(f.x) + (int64_t)min(ft, a.T - 1) * f.ldx;
  HeldRow<X, kHeld> held;
  if constexpr (FROM == kFloats) held.load(frow, a.K, fat, per);

  // ---- codes of the wave's part of K ----
  i32x4 xf[kChunks][TB][kSteps];
  if constexpr (FROM != kFloats) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (i >= n) break;
#pragma unroll
      for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int step = (first + i) * kSteps + s;
          if constexpr (FROM == kLanes) {
            xf[i][b][s] = *reinterpret_cast<const i32x4*>(a.x + ((int64_t)step * a.lane_blocks + min(b, a.lane_blocks - 1)) * 1024 + lane * 16);
          } else {
            const int8_t* row = a.x + (int64_t)min(16 * b + c, a.T - 1) * a.ldx;
            const int k = 64 * step + 16 * g;
            xf[i][b][s] = masked_codes(row + (k < a.K ? k : 0), a.K - k);
          }
        }
    }
  }

  // ---- weights: buffer loads into LDS, rows and columns that do not exist are out of range ----
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w + (int64_t)row0 * a.ldw, (unsigned)((rows - 1) * (int)a.ldw + Kw));
  char* const ring = s_mem + wave * (kRing * kStage);
  int load_turn = 0, load_chunk = 0, load_stage = 0;       // what is loaded next
  auto load = [&]() {
    const int row = 16 * (load_turn * groups + group) + g, k0 = (first + load_chunk) * kRowBytes;
    const bool there = n > 0 && load_turn < turns;         // behind the last block: zeros, without memory traffic
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int r = row + 4 * p, k = k0 + (c ^ (4 * p + g)) * 16;
      const unsigned off = there && r < rows && k < Kw ? (unsigned)r * (unsigned)a.ldw + (unsigned)k : kOob;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void*)(ring + load_stage * kStage + p * 1024), 16, (int)off, 0, 0, kStreamOnce);
    }
    load_stage = (load_stage + 1) & (kRing - 1);
    load_chunk = load_chunk + 1 >= n ? 0 : load_chunk + 1;
    load_turn += load_chunk == 0;
  };
  // scales and biases of the rows, the latter kNoBias where there are none; sums start from zero
  float ws0[2] = {0.f, kNoBias};
  if (tid < rows) { ws0[0] = a.w_scale[row0 + tid]; if (a.bias) ws0[1] = a.bias[row0 + tid]; }
  static_assert(kMaxRows <= kThreadsS, "one row a thread");
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i) load();
  asm volatile("ds_write_b32 %0, %1\n\tds_write_b32 %0, %2 offset:%3" :: "v"(scales_at + 4u * tid), "v"(ws0[0]), "v"(ws0[1]), "n"(4 * kMaxRows) : "memory");
  for (int i = tid * 16; i < sum_bytes(TB, split); i += kThreadsS * 16) {
    const i32x4 zero = {0, 0, 0, 0};
    asm volatile("ds_write_b128 %0, %1" :: "v"(sums_at + (unsigned)i), "v"(zero) : "memory");
  }
  if constexpr (FROM == kFloats) {
    const int pitch = code_pitch(a.K);
    char* const codes = s_mem + kRingBytes + kScaleBytes + sum_bytes(TB, split);
    if (tid < 16) s_max[tid] = 0;
    lds_barrier();
    unsigned top = 0;
    float v[kVec];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) { held.values(u, v); top = max(top, magnitude(v)); }
    for (int k = (kHeld * per + fat) * kVec; k < a.K; k += per * kVec) {
      load_floats(frow, k, a.K, v);
      top = max(top, magnitude(v));
    }
    for (int o = min(per, 64) / 2; o; o >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    if ((fat & 63) == 0 && ft < a.T) atomicMax(&s_max[ft], top);
    lds_barrier();
    if (ft < a.T) {
      const RowScale code(s_max[ft]);
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
        const int k = (u * per + fat) * kVec;
        if (k < Kw) { held.values(u, v); store_codes(codes + ft * pitch + k, code, v); }
      }
      for (int k = (kHeld * per + fat) * kVec; k < Kw; k += per * kVec) {
        load_floats(frow, k, a.K, v);
        store_codes(codes + ft * pitch + k, code, v);
      }
    }
    lds_barrier();
    // behind Kw stands anything: weights are zero there
    const unsigned at = (unsigned)(size_t)codes + (unsigned)(min(c, a.T - 1) * pitch + first * kRowBytes + 16 * g);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (i >= n) break;
      const unsigned k = at + (unsigned)(i * kRowBytes);
      read4(xf[i][0], k, k + 64u, k + 128u, k + 192u);
    }
  } else {
    lds_barrier();
  }
  // token scales of the sums that this wave finishes: tokens 16 b + 4 g + v
  float xs[TB][4];
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int t = 16 * b + 4 * g + v;
      if constexpr (FROM == kFloats) xs[b][v] = t < a.T ? RowScale(s_max[t]).scale() : 0.f;
      else xs[b][v] = a.x_scale[min(t, a.T - 1)];
    }

  const unsigned wlane = lds0 + (unsigned)(wave * (kRing * kStage) + c * kRowBytes);
  unsigned w_at[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) w_at[s] = wlane + (unsigned)(((4 * s + g) ^ c) * 16);
  auto finish = [&](int turn, int b, const i32x4& sum) {
    const int r = 16 * (turn * groups + group) + c;
    const float ws = read_float(scales_at + 4u * (unsigned)r), bias = read_float(scales_at + 4u * (unsigned)(kMaxRows + r));
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int t = 16 * b + 4 * g + v;
      if (t < a.T && r < rows)
        static_cast<S*>(a.out)[(int64_t)t * a.ldo + row0 + r] = to_out<S>(scaled(sum[v], xs[b][v], ws, bias));
    }
  };
  int stage = 0;
  for (int turn = 0; turn < turns; ++turn) {
    i32x4 acc[TB] = {};
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (i >= n) break;
      wait_loads<(kRing - 2) * 4>();                       // the loads behind this chunk's are those of the two after it
      i32x4 w[kSteps];
      const unsigned s = (unsigned)(stage * kStage);
      read4(w, w_at[0] + s, w_at[1] + s, w_at[2] + s, w_at[3] + s);
      stage = (stage + 1) & (kRing - 1);
      load();
#pragma unroll
      for (int q = 0; q < kSteps; ++q)
#pragma unroll
        for (int b = 0; b < TB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(xf[i][b][q], w[q], acc[b], 0, 0, 0);
    }
    if (split == 1) {
#pragma unroll
      for (int b = 0; b < TB; ++b) finish(turn, b, acc[b]);
    } else {
      // Two sets of sums in turn: one is finished, and left at zero, while the other is added to; the barrier of a turn is behind the
      // finishing of the one before.
      const unsigned at = sums_at + (unsigned)(((turn & 1) * groups + group) * TB * 1024 + lane * 4);
      if (n > 0) {
#pragma unroll
        for (int b = 0; b < TB; ++b) add_sum(at + b * 1024u, acc[b]);
      }
      lds_barrier();
#pragma unroll
      for (int b = 0; b < TB; ++b)
        if ((b & (split - 1)) == part) finish(turn, b, take_sum(at + b * 1024u));
    }
  }
  wait_loads<0>();                                         // the loads behind the last chunk end before the workgroup does
}

// Waves that share K: as few as their registers allow, more while the rows do not give every wave of the chip a block.
struct Shape { int split, turns; };
Shape shape_of(int T, int N, int K) {
  const int tb = T <= 16 ? 1 : (T <= 32 ? 2 : 4);
  const int blocks = (N + 15) / 16, chunks = (K + kRowBytes - 1) / kRowBytes, cus = device_cu_count();
  int split = 1;
  while (split * stream_chunks(tb) < chunks) split *= 2;
  while (split < kWavesS && split < chunks && (int64_t)blocks * split < (int64_t)cus * kWavesS) split *= 2;
  if (tb == 4 && split == 2) split = 4;                    // the sums of four groups of 64 tokens have no room in LDS
  const int groups = kWavesS / split;
  int turns = (blocks + cus * groups - 1) / (cus * groups);
  if (turns > kMaxRows / (16 * groups)) turns = kMaxRows / (16 * groups);
  return {split, turns};
}

template <typename S, Tokens FROM, typename X, int TB>
int launch_t(const Int8Args& a, const FloatTokens& f, hipStream_t s) {
  const Shape sh = shape_of(a.T, a.N, a.K);
  const int rows = 16 * (kWavesS / sh.split) * sh.turns;
  constexpr int kFixed = kRingBytes + kScaleBytes, kMost = FROM == kFloats ? sum_bytes(1, 2) + kMaxFused + 16 * 31 + kRowBytes : sum_bytes(TB, TB == 4 ? 4 : 2);
  static_assert(kFixed + kMost + 64 <= 163840, "LDS of a CU");
  const int lds = kFixed + sum_bytes(TB, sh.split) + (FROM == kFloats ? code_bytes(a.T, a.K) : 0);
  static std::atomic<int> ready{0};
  if (!ready.load(std::memory_order_relaxed)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_stream_kernel<S, FROM, X, TB>), hipFuncAttributeMaxDynamicSharedMemorySize, kFixed + kMost) != hipSuccess)
      return hip_fail(hipGetLastError(), "int8_stream_kernel: LDS size attribute");
    ready.store(1, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL((int8_stream_kernel<S, FROM, X, TB>), dim3((unsigned)((a.N + rows - 1) / rows)), dim3(kThreadsS), (size_t)lds, s, a, f, sh.split, sh.turns);
  return hip_fail(hipGetLastError(), "int8_stream_kernel launch");
}
template <typename S, Tokens FROM>
int launch_b(const Int8Args& a, hipStream_t s) {
  const FloatTokens none = {nullptr, 0};
  if (a.T <= 16) return launch_t<S, FROM, float, 1>(a, none, s);
  return a.T <= 32 ? launch_t<S, FROM, float, 2>(a, none, s) : launch_t<S, FROM, float, 4>(a, none, s);
}
template <typename S>
int launch_s(const Int8Args& a, hipStream_t s) { return a.lane_blocks ? launch_b<S, kLanes>(a, s) : launch_b<S, kRows>(a, s); }
template <typename X>
int launch_x(const Int8Args& a, const FloatTokens& f, hipStream_t s) {
  return a.out_dtype == MOE_FP32 ? launch_t<float, kFloats, X, 1>(a, f, s) : launch_t<uint16_t, kFloats, X, 1>(a, f, s);
}

}  // namespace

int launch_int8_stream(const Int8Args& a, hipStream_t s) { return a.out_dtype == MOE_FP32 ? launch_s<float>(a, s) : launch_s<uint16_t>(a, s); }

size_t int8_lane_codes_bytes(int T, int K) { return (size_t)((T + 15) / 16 * 16) * ((K + kRowBytes - 1) / kRowBytes * kRowBytes); }

int launch_int8_stream_float(const Int8Args& a, const void* x, int x_dtype, int64_t ldx, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  const FloatTokens f = {x, ldx};
  return x_dtype == MOE_FP32 ? launch_x<float>(a, f, s) : launch_x<uint16_t>(a, f, s);
}

}  // namespace mm
