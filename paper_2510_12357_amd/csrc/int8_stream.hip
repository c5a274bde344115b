// The 8-bit product for up to 64 tokens: every weight is read once, so memory sets the pace, and for small weights the latency of a launch.
//
// A wave has R blocks of 16 weight rows and all tokens (TB blocks of 16) and goes through K in steps of 64, operands straight from memory
// into registers, D steps ahead: a load of a weight block is 16 rows x 64 bytes, the next step's the other half of those lines.  The four waves of a
// workgroup have weight rows of their own, or, where rows are few, share them and split K; their sums of integers are joined in LDS, exactly.
// Float tokens (moe_linear_int8) are quantised by every workgroup for itself while its first weights are on their way, up to a size
// where that costs less than a launch in front of this one.
#include <algorithm>

#include "internal.h"
#include "int8_device.h"
#include "route_device.h"
#include "unaligned.h"

namespace mm {
namespace {

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct FloatTokens { const void* x; int64_t ldx; };

constexpr int kMaxFused = 16384;        // elements of float tokens that every workgroup quantises
constexpr int code_pitch(int K) { return (K + 63) / 64 * 64 + 16; }   // bytes of a token's codes in LDS: 16 tokens start at 16 different banks

// X: the tokens' float type, or int8_t for codes
template <typename S, typename X, int TB, int R>
__global__ __launch_bounds__(256) void int8_stream_kernel(const Int8Args a, const FloatTokens f, const int split) {
  constexpr bool kFused = !std::is_same_v<X, int8_t>;
  constexpr int D = R + TB <= 3 ? 8 : 4;
  extern __shared__ __attribute__((aligned(16))) char s_mem[];   // codes of float tokens, then the partial sums
  __shared__ unsigned s_max[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), g = lane >> 4, c = lane & 15;
  const int part = wave & (split - 1), group = wave / split;
  const int n0 = uniform((blockIdx.x * (4 / split) + group) * (16 * R));
  const bool idle = n0 >= a.N;                             // past the last row: keeps the barriers only
  const int whole = a.K16 >> 6;                            // steps of four whole vectors
  const int begin = idle ? 0 : (int)((int64_t)whole * part / split), end = idle ? 0 : (int)((int64_t)whole * (part + 1) / split);

  const char* wbase = reinterpret_cast<const char*>(a.w) + (int64_t)min(n0, a.N - 1) * a.ldw;
  unsigned woff[R], xoff[TB];
#pragma unroll
  for (int r = 0; r < R; ++r) woff[r] = (unsigned)max(min(16 * r + c, a.N - 1 - n0), 0) * (unsigned)a.ldw + 16u * g;
  const int pitch = kFused ? code_pitch(a.K) : 0;
#pragma unroll
  for (int b = 0; b < TB; ++b) xoff[b] = (unsigned)min(16 * b + c, a.T - 1) * (kFused ? (unsigned)pitch : (unsigned)a.ldx) + 16u * g;

  i32x4 acc[R][TB];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[r][b] = i32x4{0, 0, 0, 0};
  i32x4 wf[D][R], xf[D][TB];
  auto load_w = [&](int d, int k) {
#pragma unroll
    for (int r = 0; r < R; ++r) wf[d][r] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wbase + (int64_t)k * 64 + woff[r]));
  };
  auto load_x = [&](int d, int k) {
#pragma unroll
    for (int b = 0; b < TB; ++b) xf[d][b] = *reinterpret_cast<const i32x4*>((kFused ? s_mem : reinterpret_cast<const char*>(a.x)) + (int64_t)k * 64 + xoff[b]);
  };
  auto multiply = [&](int d) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[r][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[d][r], xf[d][b], acc[r][b], 0, 0, 0);
  };
#pragma unroll
  for (int d = 0; d < D; ++d) if (begin + d < end) { load_w(d, begin + d); if (!kFused) load_x(d, begin + d); }

  if constexpr (kFused) {
    // `per` threads for a token, in turn for each of its vectors
    constexpr int kVec = 16 / sizeof(X);
    int per = 256;
    while (per > 16 && per * a.T > 256) per >>= 1;
    const int t = tid / per, at = tid % per;
    const X* row = static_cast<const X*>(f.x) + (int64_t)min(t, a.T - 1) * f.ldx;
    if (tid < 16) s_max[tid] = 0;
    __syncthreads();
    unsigned top = 0;
    for (int k = at * kVec; k < a.K; k += per * kVec) {
      float v[kVec];
      load_floats(row, k, a.K, v);
      top = max(top, magnitude(v));
    }
    for (int o = min(per, 64) / 2; o; o >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    if ((at & 63) == 0 && t < a.T) atomicMax(&s_max[t], top);
    __syncthreads();
    if (t < a.T) {
      const RowScale code(s_max[t]);
      for (int k = at * kVec; k < pitch - 16; k += per * kVec) {
        float v[kVec];
        load_floats(row, k, a.K, v);
        store_codes(s_mem + t * pitch + k, code, v);
      }
    }
    __syncthreads();
#pragma unroll
    for (int d = 0; d < D; ++d) if (begin + d < end) load_x(d, begin + d);
  }

  int k = begin;
  for (; k + 2 * D <= end; k += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      multiply(d);
      load_w(d, k + d + D);
      load_x(d, k + d + D);
    }
  }
#pragma unroll
  for (int d = 0; d < D; ++d) {
    if (k + d < end) {
      multiply(d);
      if (k + d + D < end) { load_w(d, k + d + D); load_x(d, k + d + D); }
    }
  }
#pragma unroll
  for (int d = 0; d < D; ++d) if (k + d + D < end) multiply(d);
  if (part == split - 1 && !idle && ((a.K16 & 63) || a.k_tail)) {
    // the last step: vectors beyond K are zero, one may count in part
    const int left = (a.K16 & 63) + a.k_tail - 16 * g;
    const i32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < R; ++r) wf[0][r] = left > 0 ? *reinterpret_cast<const i32x4*>(wbase + (int64_t)whole * 64 + woff[r]) : zero;
#pragma unroll
    for (int b = 0; b < TB; ++b)
      xf[0][b] = left > 0 ? masked_codes(reinterpret_cast<const int8_t*>((kFused ? s_mem : reinterpret_cast<const char*>(a.x)) + (int64_t)whole * 64 + xoff[b]), min(left, 16)) : zero;
    multiply(0);
  }

  if (split > 1) {
    i32x4* sums = reinterpret_cast<i32x4*>(s_mem + (kFused ? a.T * pitch : 0));
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int b = 0; b < TB; ++b) sums[((wave * R + r) * TB + b) * 64 + lane] = acc[r][b];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        if (((r * TB + b) & (split - 1)) != part) continue;
        i32x4 sum = {0, 0, 0, 0};
        for (int w = 0; w < split; ++w) sum += sums[(((group * split + w) * R + r) * TB + b) * 64 + lane];
        acc[r][b] = sum;
      }
  }
  if (idle) return;
  // accumulator v of lane l is weight row 4*(l/16) + v, token l%16
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int n = n0 + 16 * r + 4 * g;
    float ws[4], bias[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int i = min(n + v, a.N - 1);
      ws[v] = a.w_scale[i];
      bias[v] = a.bias ? a.bias[i] : 0.f;
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const int t = 16 * b + c;
      if (((r * TB + b) & (split - 1)) != part || t >= a.T) continue;
      float xs;
      if constexpr (kFused) xs = RowScale(s_max[t]).scale();
      else xs = a.x_scale[t];
      S* p = static_cast<S*>(a.out) + (int64_t)t * a.ldo + n;
      Unaligned<S, 4> o;
#pragma unroll
      for (int v = 0; v < 4; ++v) o.v[v] = to_out<S>(a.bias ? scaled(acc[r][b][v], xs, ws[v], bias[v]) : scaled(acc[r][b][v], xs, ws[v]));
      if (n + 3 < a.N) {
        *reinterpret_cast<Unaligned<S, 4>*>(p) = o;
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) if (n + v < a.N) p[v] = o.v[v];
      }
    }
  }
}

// R blocks of weight rows per wave, K split over `split` waves.
struct Shape { int r, split; };
Shape shape_of(int T, int N, int K) {
  const int rows16 = (N + 15) / 16;
  const int r = rows16 >= 4096 ? 4 : 1;
  int split = 4;
  while (split > 1 && (rows16 / r) * split > 8192) split >>= 1;
  return {r, split};
}

template <typename S, typename X, int TB, int R>
int launch_t(const Int8Args& a, const FloatTokens& f, int split, hipStream_t s) {
  constexpr bool kFused = !std::is_same_v<X, int8_t>;
  const int rows = 16 * R * (4 / split);
  const size_t lds = (kFused ? (size_t)a.T * code_pitch(a.K) : 0) + (split > 1 ? 4 * R * TB * 1024 : 0);
  hipLaunchKernelGGL((int8_stream_kernel<S, X, TB, R>), dim3((unsigned)((a.N + rows - 1) / rows)), dim3(256), lds, s, a, f, split);
  return hip_fail(hipGetLastError(), "int8_stream_kernel launch");
}
template <typename S, typename X, int TB>
int launch_r(const Int8Args& a, const FloatTokens& f, hipStream_t s) {
  const Shape sh = shape_of(a.T, a.N, a.K);
  return sh.r == 4 ? launch_t<S, X, TB, 4>(a, f, sh.split, s) : launch_t<S, X, TB, 1>(a, f, sh.split, s);
}
template <typename X, int TB>
int launch_s(const Int8Args& a, const FloatTokens& f, hipStream_t s) {
  return a.out_dtype == MOE_FP32 ? launch_r<float, X, TB>(a, f, s) : launch_r<uint16_t, X, TB>(a, f, s);
}

}  // namespace

int launch_int8_stream(const Int8Args& a, hipStream_t s) {
  const FloatTokens none = {nullptr, 0};
  switch ((a.T + 15) / 16) {
    case 1: return launch_s<int8_t, 1>(a, none, s);
    case 2: return launch_s<int8_t, 2>(a, none, s);
    case 3: return launch_s<int8_t, 3>(a, none, s);
    default: return launch_s<int8_t, 4>(a, none, s);
  }
}

bool int8_quantises_itself(int T, int K) { return T <= 16 && (int64_t)T * K <= kMaxFused; }

int launch_int8_stream_float(const Int8Args& a, const void* x, int x_dtype, int64_t ldx, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  const FloatTokens f = {x, ldx};
  return x_dtype == MOE_FP32 ? launch_s<float, 1>(a, f, s) : launch_s<uint16_t, 1>(a, f, s);
}

}  // namespace mm
