// Rows of floats -> 8-bit codes and one scale per row (moe_quantize_rows).
//
// A workgroup per row, which it holds in registers between the largest magnitude and the codes (up to 8192 values; what does not fit is read
// twice), so that each value is read once.  What bounds it: the launch up to some hundred rows, then memory and the vector unit, which quotients and codes
// take 19 instructions an element, 20 thousand cycles a SIMD for 4096 x 4096 of either type, 0.76 of its busy cycles with bf16 and 0.60 with fp32 (counters).
// 4096 x 4096 fp32 17.2 us (4.9 TB/s), bf16 14.1 (3.6 TB/s); 4096 x 8192 fp32 33.5 (with half of a row held 39.8); 64 x 4096 bf16 3.4.
#include <algorithm>

#include "internal.h"
#include "route_device.h"
#include "int8_device.h"

namespace mm {
namespace {

constexpr int held(int threads, size_t bytes) { return threads == 64 || bytes == 2 ? 4 : 8; }   // vectors of 16 bytes that a thread holds

template <typename X, int THREADS>
__global__ __launch_bounds__(THREADS) void quantize_kernel(const X* __restrict__ x, int K, int64_t ldx, int8_t* __restrict__ q, int64_t ldq,
                                                           float* __restrict__ scale, int lane_blocks) {
  constexpr int kVec = 16 / sizeof(X);
  __shared__ unsigned s_max[THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int kHeld = held(THREADS, sizeof(X));
  const X* row = x + (int64_t)blockIdx.x * ldx;
  HeldRow<X, kHeld> in;
  in.load(row, K, tid, THREADS);
  unsigned top = 0;
  float v[kVec];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) { in.values(u, v); top = max(top, magnitude(v)); }
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
    in.values(u, v);
    if (k < ldq) store_codes(out + place(k), r, v);
  }
  for (int k = (kHeld * THREADS + tid) * kVec; k < ldq; k += THREADS * kVec) {
    load_floats(row, k, K, v);
    store_codes(out + place(k), r, v);
  }
  if (tid == 0) scale[blockIdx.x] = r.scale();
}

// One wave where it holds a row by itself, four where not, and for few rows of more than 512 bf16 values, where a wave's own time shows.  us, one / four
// waves, bf16: 333 x 300 3.1 / 3.1, 333 x 1000 3.6 / 3.2, 333 x 1971 5.5 / 3.3, 1000 x 1500 5.4 / 4.2, 4000 x 1000 6.1 / 7.4, 4000 x 1971 10.0 / 9.4, 40000 x 1971 53 / 69;
// fp32: 333 x 1000 2.9 / 3.0, 4000 x 1000 5.8 / 7.4.
template <typename X>
int launch(const void* x, int rows, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int lane_blocks, hipStream_t s) {
  constexpr int kHeldByWave = 64 * held(64, sizeof(X)) * (16 / sizeof(X));
  const bool one_wave = K <= kHeldByWave && !(sizeof(X) == 2 && K > 512 && rows <= 2048);
  for (int64_t r = 0; r < rows; r += kLaunchRows) {        // more than one: rows of codes, for lane_blocks are of 64 tokens at most
    const dim3 grid((unsigned)std::min<int64_t>(rows - r, kLaunchRows));
    const X* xr = static_cast<const X*>(x) + r * ldx;
    if (one_wave)
      hipLaunchKernelGGL((quantize_kernel<X, 64>), grid, dim3(64), 0, s, xr, K, ldx, q + r * ldq, ldq, scale + r, lane_blocks);
    else
      hipLaunchKernelGGL((quantize_kernel<X, 256>), grid, dim3(256), 0, s, xr, K, ldx, q + r * ldq, ldq, scale + r, lane_blocks);
    const int rc = hip_fail(hipGetLastError(), "quantize_kernel launch");
    if (rc) return rc;
  }
  return MOE_OK;
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int rows, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int lane_blocks, hipStream_t s) {
  ProfScope ps(kProfQuantize, s);
  return dtype == MOE_FP32 ? launch<float>(x, rows, K, ldx, q, ldq, scale, lane_blocks, s) : launch<uint16_t>(x, rows, K, ldx, q, ldq, scale, lane_blocks, s);
}

}  // namespace mm
