// Log probabilities of given tokens, entropy, confidence and most probable tokens of output distributions.
#include "internal.h"
#include "int8_device.h"
#include "route_device.h"

namespace mm {
namespace {

struct LogprobArgs {
  const void* logits; int64_t ld;
  int V, n_given, n_top;
  const int32_t* tokens;
  float* token_logp; float* entropy; float* conf; int32_t* top_idx; float* top_logp;
};

// (value, id) in the order value descending, id ascending
struct Ranked { float v; int id; };
__device__ __forceinline__ bool before(Ranked a, Ranked b) { return a.v > b.v || (a.v == b.v && a.id < b.id); }
__device__ __forceinline__ float ordered(float z) { return z == z ? z : -INFINITY; }

// One workgroup per row; the row is read once for the maximum, once for the sums and once per alternative.
constexpr int kThreads = 256, kWaves = kThreads / 64;
template <typename S>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const LogprobArgs a) {
  __shared__ float s_f[kWaves][2];
  __shared__ Ranked s_r[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t t = blockIdx.x;
  const S* row = static_cast<const S*>(a.logits) + t * a.ld;
  float m = -INFINITY;
  for (int v = tid; v < a.V; v += kThreads) m = fmaxf(m, ordered(to_f32(row[v])));
  m = wave_max(m);
  if (lane == 0) s_f[wave][0] = m;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_f[w][0]);
  __syncthreads();
  float rest = 0.f, spread = 0.f, count = 0.f;
  for (int v = tid; v < a.V; v += kThreads) {
    const float d = to_f32(row[v]) - m;
    if (d == 0.f) { count += 1.f; continue; }
    const float e = expf(d);
    rest += e;
    spread += e * fmaxf(d, -200.f);
  }
  rest = wave_sum(rest); spread = wave_sum(spread); count = wave_sum(count);
  __shared__ float s_c[kWaves];
  if (lane == 0) { s_f[wave][0] = rest; s_f[wave][1] = spread; s_c[wave] = count; }
  __syncthreads();
  rest = spread = count = 0.f;
  for (int w = 0; w < kWaves; ++w) { rest += s_f[w][0]; spread += s_f[w][1]; count += s_c[w]; }
  const float sum = count + rest;
  float log_sum = logf(count) + log1pf(rest / count);
  if (!(fabsf(m) < INFINITY)) log_sum = NAN;
  if (tid == 0 && a.entropy) a.entropy[t] = log_sum - spread / sum;
  if (tid == 0 && a.conf) a.conf[t] = log_sum == log_sum ? 1.f / sum : NAN;
  for (int g = tid; g < a.n_given; g += kThreads) {
    const int id = a.tokens[t * a.n_given + g];
    a.token_logp[t * a.n_given + g] = id < 0 || id >= a.V ? 0.f : (to_f32(row[id]) - m) - log_sum;
  }
  Ranked last = {INFINITY, -1};
  for (int j = 0; j < a.n_top; ++j) {
    Ranked best = {-INFINITY, 0x7fffffff};
    for (int v = tid; v < a.V; v += kThreads) {
      const Ranked c = {ordered(to_f32(row[v])), v};
      if (before(last, c) && before(c, best)) best = c;
    }
    for (int o = 32; o; o >>= 1) {
      const Ranked c = {__shfl_xor(best.v, o), __shfl_xor(best.id, o)};
      if (before(c, best)) best = c;
    }
    __syncthreads();
    if (lane == 0) s_r[wave] = best;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) if (before(s_r[w], best)) best = s_r[w];
    last = best;
    if (tid == 0) { a.top_idx[t * a.n_top + j] = best.id; a.top_logp[t * a.n_top + j] = (to_f32(row[best.id]) - m) - log_sum; }
  }
}

}  // namespace

size_t logprobs_workspace_bytes(const moe_logprobs_config&) { return 0; }

int launch_logprobs(const moe_logprobs_config& c, const void* logits, const int32_t* tokens, float* token_logp, float* entropy, float* conf,
                    int32_t* top_idx, float* top_logp, void*, hipStream_t s) {
  ProfScope ps(kProfLogprobs, s);
  const LogprobArgs a = {logits, c.ld, c.V, c.n_given, c.n_top, tokens, token_logp, entropy, conf, top_idx, top_logp};
  if (c.dtype == MOE_FP32) hipLaunchKernelGGL(logprobs_kernel<float>, dim3((unsigned)c.T), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(logprobs_kernel<uint16_t>, dim3((unsigned)c.T), dim3(kThreads), 0, s, a);
  return hip_fail(hipGetLastError(), "logprobs_kernel launch");
}

}  // namespace mm
