// The 8-bit product for up to 32 tokens: every weight is read once, so memory sets the pace, and for small weights the latency of a launch.
//
// A wave has 16 weight rows and all tokens, and a ring of kRing chunks of 256 k of its own in LDS, which loads fill past the registers: sixteen lanes
// read 256 bytes of a row.  (Operands straight into registers, in the matrix instruction's order, touch a row per lane: 64 lines an instruction,
// and the address units set the pace; 64 x 131072 x 4096 took 227 us so.)  Nothing is shared between waves, so there is no barrier in the
// loop.  The tokens' codes come into registers, as far ahead as the weights, because loads end in order.  The four waves of a
// workgroup have weight rows of their own, or, where rows are few, share them and split K; their sums of integers are joined in LDS, exactly.
// Where the codes come from: the caller's rows; the workspace of moe_linear_int8, in the order of the matrix instruction's lanes, so that a load is
// 1 KB in one piece; or float tokens that every workgroup quantises for itself while its first weights are on their way, up to a
// size where that costs less than a launch in front of this one.
#include <atomic>
#include <type_traits>

#include "internal.h"
#include "groups.h"
#include "int8_device.h"
#include "unaligned.h"

namespace mm {
namespace {

typedef __attribute__((address_space(3))) void lds_void;

constexpr int kRing = 4, kRowBytes = 256, kStage = 16 * kRowBytes;
constexpr int kSteps = kRowBytes / 64;                     // matrix instructions (16 x 16 x 64) of a chunk
constexpr int kRingBytes = 4 * kRing * kStage;             // of a workgroup
constexpr int kMaxFused = 16384;                           // elements of float tokens that every workgroup quantises
constexpr int code_pitch(int K) { return (K + 255) / 256 * 256 + 16; }   // bytes of a token's codes in LDS: 16 tokens start at 16 different banks

// At most N loads of this wave in flight.  An asm block, so that no load moves across it.
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

enum Tokens { kRows, kLanes, kFloats };                    // where codes come from, as above

struct FloatTokens { const void* x; int64_t ldx; };

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// a lane's weights of one chunk
__device__ __forceinline__ void read_weights(i32x4 (&w)[4], const unsigned (&at)[4], unsigned stage) {
  asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]) : "v"(at[0] + stage), "v"(at[1] + stage), "v"(at[2] + stage), "v"(at[3] + stage) : "memory");
}
// and, from LDS, its codes
__device__ __forceinline__ void read_codes(i32x4 (&x)[4], unsigned at) {
  asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:64\n\tds_read_b128 %2, %4 offset:128\n\tds_read_b128 %3, %4 offset:192\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]) : "v"(at) : "memory");
}

// TB: blocks of 16 tokens, 1 or 2.  X: type of float tokens.
template <typename S, Tokens FROM, typename X, int TB>
__global__ __launch_bounds__(256) void int8_stream_kernel(const Int8Args a, const FloatTokens f, const int split) {
  extern __shared__ __attribute__((aligned(1024))) char s_mem[];   // the rings, later partial sums; codes of float tokens
  __shared__ unsigned s_max[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int c = lane & 15, g = lane >> 4;                  // token (or weight row) and group of 16 k of a lane's operand
  const int part = wave & (split - 1), group = wave / split;
  const int n0 = uniform((blockIdx.x * (4 / split) + group) * 16);
  const bool idle = n0 >= a.N;                             // past the last row: keeps the barriers only
  const int chunks = (a.K16 + kRowBytes - 1) / kRowBytes;
  const int begin = idle ? 0 : chunks * part / split, end = idle ? 0 : chunks * (part + 1) / split;

  // ---- weights: buffer loads into LDS, rows and columns that do not exist are out of range ----
  const int rows = idle ? 1 : min(a.N - n0, 16);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w + (int64_t)(idle ? 0 : n0) * a.ldw, (unsigned)((rows - 1) * (int)a.ldw + a.K16));
  char* const ring = s_mem + wave * (kRing * kStage);
  unsigned woff[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int r = 4 * p + (lane >> 4);
    woff[p] = r < rows ? (unsigned)r * (unsigned)a.ldw : kOob;
  }
  auto load_w = [&](int stage, int k) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const unsigned at = (unsigned)(k * kRowBytes) + (unsigned)((lane & 15) ^ (4 * p + (lane >> 4))) * 16u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void*)(ring + stage * kStage + p * 1024), 16, (int)(at < (unsigned)a.K16 ? woff[p] + at : kOob), 0, 0,
                                               kStreamOnce);
    }
  };
  unsigned w_at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w_at[i] = (unsigned)(size_t)ring + (unsigned)(c * kRowBytes + ((4 * i + g) ^ c) * 16);

  // ---- tokens.  What stands behind K16 meets weights of zero; it only has to be there.  So do tokens behind T, which are not stored ----
  const int pitch = code_pitch(a.K);
  i32x4 xf[kRing][TB][kSteps];
  const unsigned x_at = (unsigned)(size_t)s_mem + (unsigned)(kRingBytes + min(c, a.T - 1) * pitch + 16 * g);   // (kFloats)
  const char* xrow[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b)
    xrow[b] = reinterpret_cast<const char*>(a.x) + (FROM == kRows ? (int64_t)min(16 * b + c, a.T - 1) * a.ldx : b * 1024 + lane * 16);
  auto load_x = [&](int d, int k) {
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      if constexpr (FROM == kFloats) { read_codes(xf[d][b], x_at + (unsigned)(k * kRowBytes)); continue; }
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const int at = k * kRowBytes + 64 * i + 16 * g;
        if constexpr (FROM == kLanes) xf[d][b][i] = *reinterpret_cast<const i32x4*>(xrow[b] + (int64_t)(k * kSteps + i) * (TB * 1024));
        else xf[d][b][i] = *reinterpret_cast<const i32x4*>(xrow[b] + ((unsigned)at < (unsigned)a.K16 ? at : 0));   // a row holds 16 codes at least
      }
    }
  };

  i32x4 acc[TB] = {};
  auto multiply = [&](int d, const i32x4 (&w)[4]) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(xf[d][b][i], w[i], acc[b], 0, 0, 0);
  };
  constexpr bool kAhead = FROM != kFloats;                 // codes in LDS are read when they are used
  auto first_loads = [&]() {                               // chunks that are not there fill their stage with zeros
#pragma unroll
    for (int d = 0; d < kRing - 1; ++d) { load_w(d, begin + d < end ? begin + d : 1 << 20); if (kAhead) load_x(d, max(min(begin + d, chunks - 1), 0)); }
  };
  if constexpr (FROM == kFloats) {
    // `per` threads for a token, in turn for each of its vectors, of which they hold the first kHeld.  Loads end in order: the tokens' first.
    constexpr int kVec = 16 / sizeof(X), kHeld = 8;
    int per = 256;
    while (per > 16 && per * a.T > 256) per >>= 1;
    const int t = tid / per, at = tid % per;
    const X* row = static_cast<const X*>(f.x) + (int64_t)min(t, a.T - 1) * f.ldx;
    HeldRow<X, kHeld> held;
    held.load(row, a.K, at, per);
    if (tid < 16) s_max[tid] = 0;
    asm volatile("" ::: "memory");
    first_loads();
    lds_barrier();
    unsigned top = 0;
    float v[kVec];
#pragma unroll
    for (int u = 0; u < kHeld; ++u) if (u * per * kVec < a.K) { held.values(u, v); top = max(top, magnitude(v)); }
    for (int k = (kHeld * per + at) * kVec; k < a.K; k += per * kVec) {
      load_floats(row, k, a.K, v);
      top = max(top, magnitude(v));
    }
    for (int o = min(per, 64) / 2; o; o >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    if ((at & 63) == 0 && t < a.T) atomicMax(&s_max[t], top);
    lds_barrier();
    if (t < a.T) {                                         // up to K16: there weights may be anything
      const RowScale code(s_max[t]);
      char* const codes = s_mem + kRingBytes + t * pitch;
#pragma unroll
      for (int u = 0; u < kHeld; ++u) {
        const int k = (u * per + at) * kVec;
        if (k < a.K16) { held.values(u, v); store_codes(codes + k, code, v); }
      }
      for (int k = (kHeld * per + at) * kVec; k < a.K16; k += per * kVec) {
        load_floats(row, k, a.K, v);
        store_codes(codes + k, code, v);
      }
    }
    lds_barrier();
  } else {
    first_loads();
  }

  // The chunk in stage d.  In flight behind it: the chunks up to kRing - 2 further on, and their tokens' codes.
  constexpr int kPer = 4 + (kAhead ? TB * kSteps : 0);
  static_assert((kRing - 2) * kPer < 64, "what the wait can count");
  i32x4 w[4];
  int k = begin;
  for (; k + 2 * kRing - 2 < end; k += kRing) {
#pragma unroll
    for (int d = 0; d < kRing; ++d) {
      constexpr int kLast = kRing - 1;
      wait_loads<(kRing - 2) * kPer>();
      read_weights(w, w_at, d * kStage);
      load_w((d + kLast) % kRing, k + d + kLast);
      if (kAhead) load_x((d + kLast) % kRing, k + d + kLast); else load_x(d, k + d);
      multiply(d, w);
    }
  }
  // the last chunks, fewer than 2 kRing - 1
#pragma unroll
  for (int d = 0; d < 2 * kRing - 2; ++d) {
    if (k + d < end) {
      if (k + d + kRing - 2 < end) wait_loads<(kRing - 2) * kPer>();
      else wait_loads<0>();
      read_weights(w, w_at, d % kRing * kStage);
      if (k + d + kRing - 1 < end) { load_w((d + kRing - 1) % kRing, k + d + kRing - 1); if (kAhead) load_x((d + kRing - 1) % kRing, k + d + kRing - 1); }
      if (!kAhead) load_x(d % kRing, k + d);
      multiply(d % kRing, w);
    }
  }
  if (FROM == kRows && a.k_tail && part == split - 1 && !idle) {
    // the last K % 16 codes, in the lanes of the first group
    const i32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = zero;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) xf[0][b][i] = zero;
      if (g == 0) xf[0][b][0] = masked_codes(reinterpret_cast<const int8_t*>(xrow[b]) + a.K16, a.k_tail);
    }
    if (g == 0) w[0] = *reinterpret_cast<const i32x4*>(a.w + (int64_t)min(n0 + c, a.N - 1) * a.ldw + a.K16);
    multiply(0, w);
  }

  if (split > 1) {
    __syncthreads();                                       // the rings have been read
    i32x4* sums = reinterpret_cast<i32x4*>(s_mem);
#pragma unroll
    for (int b = 0; b < TB; ++b) sums[(wave * TB + b) * 64 + lane] = acc[b];
    __syncthreads();
    if (part) return;
    for (int s = 1; s < split; ++s)
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[b] += sums[((wave + s) * TB + b) * 64 + lane];
  }
  if (idle) return;
  // a lane's column is a weight row, accumulator v of block b token 16 b + 4 (l / 16) + v
  float xs = 0.f;
  if (lane < a.T) {
    if constexpr (FROM == kFloats) xs = RowScale(s_max[lane & 15]).scale();
    else xs = a.x_scale[lane];
  }
  const int n = n0 + c;
  const float ws = a.w_scale[min(n, a.N - 1)], bias = a.bias ? a.bias[min(n, a.N - 1)] : 0.f;
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int t = 16 * b + 4 * g + v;
      const float s = __shfl(xs, t);
      if (t < a.T && n < a.N)
        static_cast<S*>(a.out)[(int64_t)t * a.ldo + n] = to_out<S>(a.bias ? scaled(acc[b][v], s, ws, bias) : scaled(acc[b][v], s, ws));
    }
}

// K over as many waves of a workgroup as it takes to have two workgroups for every CU, a wave keeping two chunks at least
int split_of(int N, int K) {
  const int blocks = (N + 15) / 16, chunks = (K + kRowBytes - 1) / kRowBytes;
  int split = 1;
  while (split < 4 && blocks * split < 2048 && chunks >= 2 * split) split *= 2;
  return split;
}

template <typename S, Tokens FROM, typename X, int TB>
int launch_t(const Int8Args& a, const FloatTokens& f, hipStream_t s) {
  const int split = split_of(a.N, a.K), rows = 16 * (4 / split);
  const int lds = kRingBytes + (FROM == kFloats ? a.T * code_pitch(a.K) : 0);
  static std::atomic<int> ready{0};
  if (!ready.load(std::memory_order_relaxed)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_stream_kernel<S, FROM, X, TB>), hipFuncAttributeMaxDynamicSharedMemorySize,
                            kRingBytes + (FROM == kFloats ? kMaxFused + 16 * (kRowBytes + 16) : 0)) != hipSuccess)
      return hip_fail(hipGetLastError(), "int8_stream_kernel: LDS size attribute");
    ready.store(1, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL((int8_stream_kernel<S, FROM, X, TB>), dim3((unsigned)((a.N + rows - 1) / rows)), dim3(256), (size_t)lds, s, a, f, split);
  return hip_fail(hipGetLastError(), "int8_stream_kernel launch");
}
template <typename S>
int launch_s(const Int8Args& a, bool in_lanes, hipStream_t s) {
  const FloatTokens none = {nullptr, 0};
  if (in_lanes) return a.T <= 16 ? launch_t<S, kLanes, float, 1>(a, none, s) : launch_t<S, kLanes, float, 2>(a, none, s);
  return a.T <= 16 ? launch_t<S, kRows, float, 1>(a, none, s) : launch_t<S, kRows, float, 2>(a, none, s);
}
template <typename X>
int launch_x(const Int8Args& a, const FloatTokens& f, hipStream_t s) {
  return a.out_dtype == MOE_FP32 ? launch_t<float, kFloats, X, 1>(a, f, s) : launch_t<uint16_t, kFloats, X, 1>(a, f, s);
}

}  // namespace

int launch_int8_stream(const Int8Args& a, bool in_lanes, hipStream_t s) {
  return a.out_dtype == MOE_FP32 ? launch_s<float>(a, in_lanes, s) : launch_s<uint16_t>(a, in_lanes, s);
}

bool int8_quantises_itself(int T, int K) { return T <= 16 && (int64_t)T * K <= kMaxFused; }
size_t int8_lane_codes_bytes(int T, int K) { return (size_t)(T <= 16 ? 16 : 32) * ((K + kRowBytes - 1) / kRowBytes * kRowBytes); }

int launch_int8_stream_float(const Int8Args& a, const void* x, int x_dtype, int64_t ldx, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  const FloatTokens f = {x, ldx};
  return x_dtype == MOE_FP32 ? launch_x<float>(a, f, s) : launch_x<uint16_t>(a, f, s);
}

}  // namespace mm
