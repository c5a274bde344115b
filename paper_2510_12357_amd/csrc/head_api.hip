// C-ABI entry points of the output head: host-side validation and kernel sequencing (int8_quantize.hip,
// int8_product.hip, logprobs.hip).
#include "internal.h"

namespace mm {
namespace {

constexpr int64_t kMaxLd = 1 << 22;      // rows of a tile stay below 2 GiB, so that 32 bits address them
constexpr int64_t kAnyLd = INT64_MAX;    // float tokens are read row by row, in 64 bits

int check_ld(const char* what, int64_t ld, int64_t least, int64_t multiple, int64_t most = kMaxLd) {
  if (ld < least) return fail(MOE_E_SHAPE, "%s = %lld is below the row length %lld", what, (long long)ld, (long long)least);
  if (ld % multiple) return fail(MOE_E_UNSUPPORTED, "%s = %lld must be a multiple of %lld", what, (long long)ld, (long long)multiple);
  if (ld >= most) return fail(MOE_E_UNSUPPORTED, "%s = %lld reaches %lld", what, (long long)ld, (long long)most);
  return MOE_OK;
}
bool float_type(int dtype) { return dtype == MOE_BF16 || dtype == MOE_FP32; }
int64_t code_ld(int K) { return ((int64_t)K + 15) / 16 * 16; }

// codes: moe_matmul_int8, whose x has the row length of codes
int resolve(const moe_int8_config* cfg, bool codes, moe_int8_config* c) {
  if (!cfg) return fail(MOE_E_BADARG, "config is NULL");
  *c = *cfg;
  if (c->T < 0 || c->N <= 0 || c->K <= 0) return fail(MOE_E_SHAPE, "T=%d N=%d K=%d", c->T, c->N, c->K);
  if (c->K > MOE_INT8_MAX_K) return fail(MOE_E_UNSUPPORTED, "K=%d above %d", c->K, MOE_INT8_MAX_K);
  if (!float_type(c->out_dtype)) return fail(MOE_E_BADARG, "out_dtype %d", c->out_dtype);
  if (!codes && !float_type(c->x_dtype)) return fail(MOE_E_BADARG, "x_dtype %d", c->x_dtype);
  if (c->ldx < 0 || c->ldw < 0 || c->ldo < 0) return fail(MOE_E_BADARG, "negative leading dimension");
  if (c->reserved) return fail(MOE_E_BADARG, "reserved field is %d", c->reserved);
  if (!c->ldx) c->ldx = c->K;
  if (!c->ldw) c->ldw = c->K;
  if (!c->ldo) c->ldo = c->N;
  int rc = check_ld("ldx", c->ldx, c->K, codes ? 16 : 1, codes ? kMaxLd : kAnyLd);
  if (!rc) rc = check_ld("ldw", c->ldw, c->K, 16);
  if (!rc) rc = check_ld("ldo", c->ldo, c->N, 1);
  return rc;
}

int check_aligned(const char* call, const char* what, const void* p, unsigned to) {
  if (!p) return fail(MOE_E_BADARG, "%s: %s is NULL", call, what);
  if ((uintptr_t)p & (to - 1)) return fail(MOE_E_BADARG, "%s: %s is not %u-byte aligned", call, what, to);
  return MOE_OK;
}
unsigned type_bytes(int dtype) { return dtype == MOE_FP32 ? 4 : 2; }

int check_product(const char* call, const moe_int8_config& c, const int8_t* w, const float* w_scale, const float* bias, const void* out) {
  int rc = check_aligned(call, "w", w, 16);
  if (!rc) rc = check_aligned(call, "w_scale", w_scale, 4);
  if (!rc && bias) rc = check_aligned(call, "bias", bias, 4);
  return rc ? rc : check_aligned(call, "out", out, type_bytes(c.out_dtype));
}

// workspace of moe_linear_int8: the codes, in rows or in the order of the streaming kernel's lanes, then the scales
int lane_blocks(const moe_int8_config& c) { return int8_streams(c.T, c.K) && !int8_quantises_itself(c.T, c.K) ? (c.T + 15) / 16 : 0; }
size_t codes_bytes(const moe_int8_config& c) { return align256(lane_blocks(c) ? int8_lane_codes_bytes(c.T, c.K) : (size_t)c.T * code_ld(c.K)); }

int resolve(const moe_logprobs_config* cfg, moe_logprobs_config* c) {
  if (!cfg) return fail(MOE_E_BADARG, "config is NULL");
  *c = *cfg;
  if (c->T < 0 || c->V <= 0) return fail(MOE_E_SHAPE, "T=%d V=%d", c->T, c->V);
  if (!float_type(c->dtype)) return fail(MOE_E_BADARG, "dtype %d", c->dtype);
  if (c->n_given < 0 || c->n_top < 0 || c->ld < 0) return fail(MOE_E_BADARG, "n_given=%d n_top=%d ld=%lld", c->n_given, c->n_top, (long long)c->ld);
  if (c->reserved) return fail(MOE_E_BADARG, "reserved field is %d", c->reserved);
  if (c->n_top > c->V) return fail(MOE_E_SHAPE, "n_top=%d of %d tokens", c->n_top, c->V);
  if (c->n_top > MOE_MAX_ALTERNATIVES) return fail(MOE_E_UNSUPPORTED, "n_top=%d above %d", c->n_top, MOE_MAX_ALTERNATIVES);
  if (c->n_given > MOE_MAX_GIVEN) return fail(MOE_E_UNSUPPORTED, "n_given=%d above %d", c->n_given, MOE_MAX_GIVEN);
  if (!c->ld) c->ld = c->V;
  return check_ld("ld", c->ld, c->V, 1);
}

}  // namespace
}  // namespace mm

using namespace mm;

extern "C" int moe_quantize_rows(const void* x, int32_t dtype, int32_t rows, int32_t K, int64_t ldx, int8_t* q, int64_t ldq, float* scale,
                                 void* stream) {
  const char* call = "moe_quantize_rows";
  if (!float_type(dtype)) return fail(MOE_E_BADARG, "%s: dtype %d", call, dtype);
  if (rows < 0 || K <= 0) return fail(MOE_E_SHAPE, "%s: rows=%d K=%d", call, rows, K);
  if (ldx < 0 || ldq < 0) return fail(MOE_E_BADARG, "%s: negative leading dimension", call);
  if (K > MOE_INT8_MAX_K) return fail(MOE_E_UNSUPPORTED, "%s: K=%d above %d", call, K, MOE_INT8_MAX_K);
  if (!ldx) ldx = K;
  if (!ldq) ldq = K;
  int rc = check_ld("ldx", ldx, K, 1);
  if (!rc) rc = check_ld("ldq", ldq, K, 16);
  if (rc || rows == 0) return rc;
  rc = check_aligned(call, "x", x, type_bytes(dtype));
  if (!rc) rc = check_aligned(call, "q", q, 16);
  if (!rc) rc = check_aligned(call, "scale", scale, 4);
  if (rc) return rc;
  return launch_quantize_rows(x, dtype, rows, K, ldx, q, ldq, scale, 0, static_cast<hipStream_t>(stream));
}

extern "C" int moe_matmul_int8(const moe_int8_config* cfg, const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale,
                               const float* bias, void* out, void* stream) {
  const char* call = "moe_matmul_int8";
  moe_int8_config c;
  int rc = resolve(cfg, true, &c);
  if (rc || c.T == 0) return rc;
  rc = check_aligned(call, "x", x, 16);
  if (!rc) rc = check_aligned(call, "x_scale", x_scale, 4);
  if (!rc) rc = check_product(call, c, w, w_scale, bias, out);
  if (rc) return rc;
  const Int8Args a = {c.T, c.N, c.K, c.out_dtype, c.K & ~15, c.K & 15, 0, c.ldx, c.ldw, c.ldo, x, x_scale, w, w_scale, bias, out};
  return launch_int8_product(a, static_cast<hipStream_t>(stream));
}

extern "C" size_t moe_linear_int8_workspace_bytes(const moe_int8_config* cfg) {
  moe_int8_config c;
  if (resolve(cfg, false, &c)) return 0;
  return codes_bytes(c) + align256((size_t)c.T * sizeof(float));
}

extern "C" int moe_linear_int8(const moe_int8_config* cfg, const void* x, const int8_t* w, const float* w_scale, const float* bias, void* out,
                               void* ws, size_t ws_bytes, void* stream) {
  const char* call = "moe_linear_int8";
  moe_int8_config c;
  int rc = resolve(cfg, false, &c);
  if (rc || c.T == 0) return rc;
  rc = check_aligned(call, "x", x, type_bytes(c.x_dtype));
  if (!rc) rc = check_product(call, c, w, w_scale, bias, out);
  if (rc) return rc;
  const size_t need = codes_bytes(c) + align256((size_t)c.T * sizeof(float));
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_E_WORKSPACE, "%s: workspace %p of %zu bytes (need %zu, 256-byte aligned)", call, ws, ws_bytes, need);
  int8_t* q = static_cast<int8_t*>(ws);
  float* scale = reinterpret_cast<float*>(q + codes_bytes(c));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Int8Args a = {c.T, c.N, c.K, c.out_dtype, (int)code_ld(c.K), 0, lane_blocks(c), code_ld(c.K), c.ldw, c.ldo, q, scale, w, w_scale, bias, out};
  if (int8_quantises_itself(c.T, c.K)) return launch_int8_stream_float(a, x, c.x_dtype, c.ldx, s);
  rc = launch_quantize_rows(x, c.x_dtype, c.T, c.K, c.ldx, q, code_ld(c.K), scale, a.lane_blocks, s);
  return rc ? rc : launch_int8_product(a, s);
}

extern "C" size_t moe_token_logprobs_workspace_bytes(const moe_logprobs_config* cfg) {
  moe_logprobs_config c;
  return resolve(cfg, &c) || c.T == 0 ? 0 : logprobs_workspace_bytes(c);
}

extern "C" int moe_token_logprobs(const moe_logprobs_config* cfg, const void* logits, const int32_t* tokens, float* token_logp, float* entropy,
                                  float* conf, int32_t* top_idx, float* top_logp, void* ws, size_t ws_bytes, void* stream) {
  const char* call = "moe_token_logprobs";
  moe_logprobs_config c;
  int rc = resolve(cfg, &c);
  if (rc || c.T == 0) return rc;
  rc = check_aligned(call, "logits", logits, type_bytes(c.dtype));
  if (!rc && c.n_given) rc = check_aligned(call, "tokens", tokens, 4);
  if (!rc && c.n_given) rc = check_aligned(call, "token_logp", token_logp, 4);
  if (!rc && c.n_top) rc = check_aligned(call, "top_idx", top_idx, 4);
  if (!rc && c.n_top) rc = check_aligned(call, "top_logp", top_logp, 4);
  if (!rc && entropy) rc = check_aligned(call, "entropy", entropy, 4);
  if (!rc && conf) rc = check_aligned(call, "conf", conf, 4);
  if (rc) return rc;
  const size_t need = logprobs_workspace_bytes(c);
  if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
    return fail(MOE_E_WORKSPACE, "%s: workspace %p of %zu bytes (need %zu, 256-byte aligned)", call, ws, ws_bytes, need);
  return launch_logprobs(c, logits, tokens, token_logp, entropy, conf, top_idx, top_logp, ws, static_cast<hipStream_t>(stream));
}
