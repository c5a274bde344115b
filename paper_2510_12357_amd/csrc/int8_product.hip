// out[t][n] = x_scale[t] w_scale[n] sum_k x[t][k] w[n][k] + bias[n] on the matrix cores' 8-bit integers.
#include "internal.h"
#include "int8_device.h"

namespace mm {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

// The 16 codes from column k on, zeros from column K on.
__device__ __forceinline__ i32x4 codes16(const int8_t* row, int k, int K) {
  if (k >= K) return i32x4{0, 0, 0, 0};
  i32x4 v = *reinterpret_cast<const i32x4*>(row + k);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int left = K - k - 4 * i;
    if (left < 4) v[i] &= left <= 0 ? 0 : (1 << (8 * left)) - 1;
  }
  return v;
}

// One wave per 32 weight rows x 32 tokens, operands straight from memory.
template <typename S>
__global__ __launch_bounds__(64) void product_kernel(const Int8Args a) {
  const int lane = threadIdx.x, r = lane & 31, h = lane >> 5;
  const int n0 = blockIdx.x * 32, t0 = blockIdx.y * 32;
  const int t = min(t0 + r, a.T - 1);
  const int8_t* wrow = a.w + (int64_t)min(n0 + r, a.N - 1) * a.ldw;
  const int8_t* xrow = a.x + (int64_t)t * a.ldx;
  i32x16 acc = {};
  for (int k = 0; k < a.K; k += 32) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(codes16(wrow, k + 16 * h, a.K), codes16(xrow, k + 16 * h, a.K), acc, 0, 0, 0);
  if (t0 + r >= a.T) return;
  const float xs = a.x_scale[t];
  S* out = static_cast<S*>(a.out) + (int64_t)t * a.ldo;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int n = n0 + 8 * (v >> 2) + 4 * h + (v & 3);
    if (n < a.N) store_out(out + n, a.bias ? scaled(acc[v], xs, a.w_scale[n], a.bias[n]) : scaled(acc[v], xs, a.w_scale[n]));
  }
}

}  // namespace

int launch_int8_product(const Int8Args& a, hipStream_t s) {
  ProfScope ps(kProfInt8Product, s);
  const dim3 grid((unsigned)((a.N + 31) / 32), (unsigned)((a.T + 31) / 32));
  if (a.out_dtype == MOE_FP32) hipLaunchKernelGGL(product_kernel<float>, grid, dim3(64), 0, s, a);
  else hipLaunchKernelGGL(product_kernel<uint16_t>, grid, dim3(64), 0, s, a);
  return hip_fail(hipGetLastError(), "product_kernel launch");
}

}  // namespace mm
