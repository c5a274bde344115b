// Rows of floats -> 8-bit codes and one scale per row (moe_quantize_rows).
#include "internal.h"
#include "route_device.h"
#include "int8_device.h"

namespace mm {
namespace {

// One workgroup per row, two sweeps: the largest magnitude, then the codes.
template <typename S>
__global__ __launch_bounds__(256) void quantize_kernel(const S* __restrict__ x, int K, int64_t ldx, int8_t* __restrict__ q, int64_t ldq,
                                                       float* __restrict__ scale) {
  __shared__ unsigned s_max[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const S* row = x + (int64_t)blockIdx.x * ldx;
  // magnitudes compare as their bits do, and a NaN or an infinity is above every number
  unsigned top = 0;
  for (int k = tid; k < K; k += 256) top = max(top, __float_as_uint(to_f32(row[k])) & 0x7fffffffu);
  top = wave_reduce(top, 0u, [](unsigned a, unsigned b) { return max(a, b); });
  if (lane == 0) s_max[wave] = top;
  __syncthreads();
  top = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
  const bool bad = top >= 0x7f800000u;
  const float a = __uint_as_float(top);
  const CodeScale c(a);
  int8_t* out = q + (int64_t)blockIdx.x * ldq;
  for (int k = tid; k < ldq; k += 256) out[k] = k < K && !bad ? (int8_t)c.code(to_f32(row[k])) : (int8_t)0;
  if (tid == 0) scale[blockIdx.x] = bad ? NAN : a / 127.f;
}

}  // namespace

int launch_quantize_rows(const void* x, int dtype, int rows, int K, int64_t ldx, int8_t* q, int64_t ldq, float* scale, hipStream_t s) {
  ProfScope ps(kProfQuantize, s);
  if (dtype == MOE_FP32)
    hipLaunchKernelGGL(quantize_kernel<float>, dim3((unsigned)rows), dim3(256), 0, s, static_cast<const float*>(x), K, ldx, q, ldq, scale);
  else
    hipLaunchKernelGGL(quantize_kernel<uint16_t>, dim3((unsigned)rows), dim3(256), 0, s, static_cast<const uint16_t*>(x), K, ldx, q, ldq, scale);
  return hip_fail(hipGetLastError(), "quantize_kernel launch");
}

}  // namespace mm
