// Rows of floats -> 8-bit codes and one scale per row (moe_quantize_rows).
//
// A workgroup per row, which it holds in registers between the largest magnitude and the codes (what does not fit is read twice), so that
// the bound is memory: each value is read once.  One wave where it holds a row by itself, four where not.
#include "internal.h"
#include "route_device.h"
#include "int8_device.h"

namespace mm {
namespace {

constexpr int kHeld = 4;                                   // vectors of 16 bytes that a thread holds

template <typename X, int THREADS>
__global__ __launch_bounds__(THREADS) void quantize_kernel(const X* __restrict__ x, int K, int64_t ldx, int8_t* __restrict__ q, int64_t ldq,
                                                           float* __restrict__ scale, int lane_blocks) {
  constexpr int kVec = 16 / sizeof(X);
  __shared__ unsigned s_max[THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const X* row = x + (int64_t)blockIdx.x * ldx;
  HeldRow<X, kHeld> held;
  held.load(row, K, tid, THREADS);
  unsigned top = 0;
  float v[kVec];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) { held.values(u, v); top = max(top, magnitude(v)); }
  for (int k = (kHeld * THREADS + tid) * kVec; k < K; k += THREADS * kVec) {
    load_floats(row, k, K, v);
    top = max(top, magnitude(v));
  }
  top = wave_reduce(top, 0u, [](unsigned a, unsigned b) { return max(a, b); });
  if constexpr (THREADS > 64) {
    if (lane == 0) s_max[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, s_max[w]);
  }
  const RowScale r(top);
  int8_t* out = q + (lane_blocks ? (int64_t)(blockIdx.x / 16 * 1024 + blockIdx.x % 16 * 16) : (int64_t)blockIdx.x * ldq);
  auto place = [&](int k) { return lane_blocks ? (k >> 6) * lane_blocks * 1024 + ((k >> 4) & 3) * 256 + (k & 15) : k; };
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int k = (u * THREADS + tid) * kVec;
    held.values(u, v);
    if (k < ldq) store_codes(out + place(k), r, v);
  }
  for (int k = (kHeld * THREADS + tid) * kVec; k < ldq; k += THREADS * kVec) {
    load_floats(row, k, K, v);
    store_codes(out + place(k), r, v);
  }
  if (tid == 0) scale[blockIdx.x] = r.scale();
}

template <typename X>
int launch(const void* x, int rows, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int lane_blocks, hipStream_t s) {
  constexpr int kHeldByWave = 64 * kHeld * (16 / sizeof(X));
  if (K <= kHeldByWave)
    hipLaunchKernelGGL((quantize_kernel<X, 64>), dim3((unsigned)rows), dim3(64), 0, s, static_cast<const X*>(x), K, ldx, q, ldq, scale, lane_blocks);
  else
    hipLaunchKernelGGL((quantize_kernel<X, 256>), dim3((unsigned)rows), dim3(256), 0, s, static_cast<const X*>(x), K, ldx, q, ldq, scale, lane_blocks);
  return hip_fail(hipGetLastError(), "quantize_kernel launch");
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int rows, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int lane_blocks, hipStream_t s) {
  ProfScope ps(kProfQuantize, s);
  return dtype == MOE_FP32 ? launch<float>(x, rows, K, ldx, q, ldq, scale, lane_blocks, s) : launch<uint16_t>(x, rows, K, ldx, q, ldq, scale, lane_blocks, s);
}

}  // namespace mm
