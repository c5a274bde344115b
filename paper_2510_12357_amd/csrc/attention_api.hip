// C-ABI entry points of the attention step: host-side validation and kernel sequencing (rotary.hip, paged_attention.hip).
#include <math.h>

#include "internal.h"

namespace mm {
namespace {

bool float_type(int dtype) { return dtype == MOE_BF16 || dtype == MOE_FP32; }
unsigned type_bytes(int dtype) { return dtype == MOE_FP32 ? 4 : dtype == MOE_E4M3 ? 1 : 2; }

int check_aligned(const char* call, const char* what, const void* p, unsigned to) {
  if (!p) return fail(MOE_E_BADARG, "%s: %s is NULL", call, what);
  if ((uintptr_t)p & (to - 1)) return fail(MOE_E_BADARG, "%s: %s is not %u-byte aligned", call, what, to);
  return MOE_OK;
}

int resolve_table(const char* call, int64_t rows, int table_len, int64_t* ld) {
  if (table_len < 1) return fail(MOE_E_SHAPE, "%s: table rows of %d entries", call, table_len);
  if (*ld < 0) return fail(MOE_E_BADARG, "%s: negative stride of the table", call);
  if (!*ld || rows <= 1) *ld = table_len;
  if (*ld < table_len) return fail(MOE_E_SHAPE, "%s: rows of the table overlap (stride %lld)", call, (long long)*ld);
  if (*ld >= ((int64_t)1 << 46) / (rows > 0 ? rows : 1)) return fail(MOE_E_UNSUPPORTED, "%s: stride of the table reaches too far", call);
  return MOE_OK;
}

// The kernels count a token's heads, their channels and those of its keys and values in 32 bits.
int check_heads(const char* call, int64_t heads, int D) {
  return heads * D < (int64_t)1 << 29 ? MOE_OK : fail(MOE_E_UNSUPPORTED, "%s: %lld heads of %d channels", call, (long long)heads, D);
}

// Strides of [n, heads, D], 0 = dense: neither heads nor tokens overlap, whichever of the two is the outer one.
int resolve_strides(const char* call, const char* what, int64_t n, int64_t heads, int64_t D, int64_t* token, int64_t* head) {
  if (*token < 0 || *head < 0) return fail(MOE_E_BADARG, "%s: negative stride of %s", call, what);
  if (!*head) *head = D;
  if (!*token) *token = heads * *head;
  if (n <= 1) *token = heads * *head > *token ? heads * *head : *token;
  if (heads <= 1) *head = *head < D ? D : *head;
  constexpr int64_t kFar = (int64_t)1 << 46;            // so that no product below leaves 64 bits
  if (*token >= kFar / (n > 0 ? n : 1) || *head >= kFar / (heads > 0 ? heads : 1)) return fail(MOE_E_UNSUPPORTED, "%s: strides of %s reach too far", call, what);
  if (*head < D || (*token < (heads - 1) * *head + D && (*token < D || *head < (n - 1) * *token + D)))
    return fail(MOE_E_SHAPE, "%s: rows of %s overlap (strides %lld, %lld)", call, what, (long long)*token, (long long)*head);
  return MOE_OK;
}

int check_rotation(const char* call, int D, int rotary_dim, int layout, float mscale) {
  if (rotary_dim < 0 || rotary_dim > D || rotary_dim % 2) return fail(MOE_E_SHAPE, "%s: rotary_dim=%d of D=%d", call, rotary_dim, D);
  if (layout != MOE_ROPE_HALF && layout != MOE_ROPE_INTERLEAVED) return fail(MOE_E_BADARG, "%s: layout %d", call, layout);
  if (!isfinite(mscale)) return fail(MOE_E_BADARG, "%s: mscale is not finite", call);
  return MOE_OK;
}

int resolve(const char* call, const moe_kv_cache* cache, moe_kv_cache* c) {
  if (!cache) return fail(MOE_E_BADARG, "%s: cache is NULL", call);
  *c = *cache;
  if (c->n_pages <= 0 || c->heads <= 0 || c->D <= 0) return fail(MOE_E_SHAPE, "%s: cache of %d pages, %d heads, D=%d", call, c->n_pages, c->heads, c->D);
  if (page_shift(c->page_size) < 0 || c->page_size > 1 << 20) return fail(MOE_E_UNSUPPORTED, "%s: page_size %d is no power of two from 4 to 2^20", call, c->page_size);
  if (c->D % 16 || c->D > MOE_MAX_HEAD_DIM) return fail(MOE_E_UNSUPPORTED, "%s: D=%d of a cache is no multiple of 16 up to %d", call, c->D, MOE_MAX_HEAD_DIM);
  if (!float_type(c->dtype) && c->dtype != MOE_E4M3) return fail(MOE_E_BADARG, "%s: cache dtype %d", call, c->dtype);
  if (c->reserved) return fail(MOE_E_BADARG, "%s: reserved field is %d", call, c->reserved);
  if (c->page < 0 || c->head < 0 || c->row < 0) return fail(MOE_E_BADARG, "%s: negative stride of the cache", call);
  if (int rc = check_heads(call, c->heads, c->D)) return rc;
  const int64_t D = c->D, n = c->page_size, h = c->heads, whole = 16 / type_bytes(c->dtype), far = (int64_t)1 << 46;
  if (!c->row) c->row = D;
  if (!c->head) c->head = n * c->row;
  if (!c->page) c->page = h * c->head > n * c->row ? h * c->head : n * c->row;
  if (c->n_pages == 1 && c->page < far / 2 && c->head < far / 2 / h && c->row < far / 2 / n) c->page = h * c->head + n * c->row;      // there is no next page
  if (c->row % whole || c->head % whole || c->page % whole) return fail(MOE_E_UNSUPPORTED, "%s: strides of the cache are no whole 16 bytes", call);
  if (c->page >= far / c->n_pages || c->head >= far / h || c->row >= far / n) return fail(MOE_E_UNSUPPORTED, "%s: strides of the cache reach too far", call);
  const bool heads_outside = c->row >= D && c->head >= (n - 1) * c->row + D, rows_outside = c->head >= D && c->row >= (h - 1) * c->head + D;
  if (!heads_outside && !rows_outside) return fail(MOE_E_SHAPE, "%s: rows of the cache overlap (strides %lld, %lld)", call, (long long)c->head, (long long)c->row);
  if (c->page < (h - 1) * c->head + (n - 1) * c->row + D) return fail(MOE_E_SHAPE, "%s: pages of the cache overlap (stride %lld)", call, (long long)c->page);
  return MOE_OK;
}
int check_cache_pointers(const char* call, const moe_kv_cache& c) {
  int rc = check_aligned(call, "cache.k", c.k, 16);
  if (!rc) rc = check_aligned(call, "cache.v", c.v, 16);
  if (!rc && c.dtype == MOE_E4M3) rc = check_aligned(call, "cache.k_scale", c.k_scale, 16);
  if (!rc && c.dtype == MOE_E4M3) rc = check_aligned(call, "cache.v_scale", c.v_scale, 16);
  if (!rc && (c.k == c.v || (c.dtype == MOE_E4M3 && c.k_scale == c.v_scale))) rc = fail(MOE_E_BADARG, "%s: keys and values are the same memory", call);
  return rc;
}

int resolve(const char* call, const moe_attention_config* cfg, const moe_kv_cache& cache, moe_attention_config* c, AttentionPlan* plan) {
  if (!cfg) return fail(MOE_E_BADARG, "%s: config is NULL", call);
  *c = *cfg;
  if (c->B < 0 || c->heads <= 0) return fail(MOE_E_SHAPE, "%s: B=%d heads=%d", call, c->B, c->heads);
  if (c->heads % cache.heads) return fail(MOE_E_SHAPE, "%s: %d query heads on %d key heads", call, c->heads, cache.heads);
  if (int rc = check_heads(call, c->heads, cache.D)) return rc;
  if (!float_type(c->dtype)) return fail(MOE_E_BADARG, "%s: dtype %d", call, c->dtype);
  if (c->max_len < 0 || c->window < 0) return fail(MOE_E_BADARG, "%s: max_len=%d window=%d", call, c->max_len, c->window);
  if (c->max_len > INT32_MAX - 2 * kMaxPiece) return fail(MOE_E_UNSUPPORTED, "%s: max_len=%d", call, c->max_len);
  if (!isfinite(c->scale) || !isfinite(c->softcap) || c->softcap < 0) return fail(MOE_E_BADARG, "%s: scale %g softcap %g", call, c->scale, c->softcap);
  if (fabsf(c->scale) > 1e30f || c->softcap > 1e30f || (c->softcap > 0 && c->softcap < 1e-30f)) return fail(MOE_E_UNSUPPORTED, "%s: scale %g softcap %g", call, c->scale, c->softcap);
  if (int rc = resolve_table(call, c->B, c->table_len, &c->table_ld)) return rc;
  if (int rc = resolve_strides(call, "q", c->B, c->heads, cache.D, &c->q_token, &c->q_head)) return rc;
  if (int rc = resolve_strides(call, "out", c->B, c->heads, cache.D, &c->out_token, &c->out_head)) return rc;
  const int64_t span = (int64_t)c->table_len << page_shift(cache.page_size);
  if (span < c->max_len) c->max_len = (int)span;           // longer sequences are behind their table row
  *plan = plan_attention(c->B, cache.heads, c->heads / cache.heads, c->max_len, c->window, attention_slots(cache.dtype, cache.D, c->dtype), device_cu_count());
  if (!plan->fits) return fail(MOE_E_UNSUPPORTED, "%s: %d sequences of up to %d positions on %d heads are too many", call, c->B, c->max_len, c->heads);
  return MOE_OK;
}
static_assert(kMostWorkgroups * sizeof(int32_t) == MOE_ATTENTION_COUNTERS, "the header's size");
// Workspace: of each workgroup two segments' sums and their statistics, and what the second kernel needs.
struct Workspace {
  size_t stat, started, bytes;
  Workspace(const moe_attention_config& c, const moe_kv_cache& cache, const AttentionPlan& p) {
    const size_t rows = (size_t)p.workgroups * 2 * (c.heads / cache.heads < kHeadTile ? c.heads / cache.heads : kHeadTile);
    stat = align256(rows * cache.D * sizeof(float));
    started = stat + align256(rows * 2 * sizeof(float));
    bytes = p.split && p.workgroups > 1 ? started + align256(((size_t)p.workgroups * 4 + 1) * sizeof(int32_t)) : 0;
  }
};

}  // namespace
}  // namespace mm

using namespace mm;

extern "C" int moe_rope(const moe_rope_config* cfg, const void* x, const int32_t* pos, const double* freq, void* out, void* stream) {
  const char* call = "moe_rope";
  if (!cfg) return fail(MOE_E_BADARG, "%s: config is NULL", call);
  moe_rope_config c = *cfg;
  if (c.T < 0 || c.heads <= 0 || c.D <= 0) return fail(MOE_E_SHAPE, "%s: T=%d heads=%d D=%d", call, c.T, c.heads, c.D);
  if (c.D % 2 || c.D > MOE_MAX_HEAD_DIM) return fail(MOE_E_UNSUPPORTED, "%s: D=%d is no even number up to %d", call, c.D, MOE_MAX_HEAD_DIM);
  if (!float_type(c.dtype)) return fail(MOE_E_BADARG, "%s: dtype %d", call, c.dtype);
  if (c.inverse != 0 && c.inverse != 1) return fail(MOE_E_BADARG, "%s: inverse is %d", call, c.inverse);
  int rc = check_heads(call, c.heads, c.D);
  if (!rc) rc = check_rotation(call, c.D, c.rotary_dim, c.layout, c.mscale);
  if (!rc) rc = resolve_strides(call, "x", c.T, c.heads, c.D, &c.x_token, &c.x_head);
  if (!rc) rc = resolve_strides(call, "out", c.T, c.heads, c.D, &c.out_token, &c.out_head);
  if (rc || c.T == 0) return rc;
  rc = check_aligned(call, "x", x, type_bytes(c.dtype));
  if (!rc) rc = check_aligned(call, "pos", pos, 4);
  if (!rc && c.rotary_dim) rc = check_aligned(call, "freq", freq, 8);
  if (!rc) rc = check_aligned(call, "out", out, type_bytes(c.dtype));
  if (rc) return rc;
  if (x == out && (c.x_token != c.out_token || c.x_head != c.out_head)) return fail(MOE_E_BADARG, "%s: in place with other strides", call);
  RotaryArgs a = {};
  a.T = c.T; a.heads = c.heads; a.D = c.D; a.rotary_dim = c.rotary_dim; a.layout = c.layout; a.mscale = c.mscale; a.sign = c.inverse ? -1.f : 1.f;
  a.q = x; a.q_out = out; a.q_token = c.x_token; a.q_head = c.x_head; a.out_token = c.out_token; a.out_head = c.out_head;
  a.pos = pos; a.freq = freq;
  return launch_rotary(a, c.dtype, static_cast<hipStream_t>(stream));
}

extern "C" int moe_kv_append(const moe_append_config* cfg, const moe_kv_cache* cache, const void* q, const void* k, const void* v, const int32_t* pos,
                             const int32_t* seq, const int32_t* table, const double* freq, void* q_out, void* stream) {
  const char* call = "moe_kv_append";
  moe_kv_cache kv;
  int rc = resolve(call, cache, &kv);
  if (rc) return rc;
  if (!cfg) return fail(MOE_E_BADARG, "%s: config is NULL", call);
  moe_append_config c = *cfg;
  if (c.T < 0 || c.heads < 0 || c.n_seqs < 0) return fail(MOE_E_SHAPE, "%s: T=%d heads=%d n_seqs=%d", call, c.T, c.heads, c.n_seqs);
  if (!float_type(c.dtype)) return fail(MOE_E_BADARG, "%s: dtype %d", call, c.dtype);
  rc = check_heads(call, c.heads, kv.D);
  if (!rc) rc = check_rotation(call, kv.D, c.rotary_dim, c.layout, c.mscale);
  if (!rc) rc = resolve_table(call, c.n_seqs, c.table_len, &c.table_ld);
  if (!rc) rc = resolve_strides(call, "k", c.T, kv.heads, kv.D, &c.k_token, &c.k_head);
  if (!rc) rc = resolve_strides(call, "v", c.T, kv.heads, kv.D, &c.v_token, &c.v_head);
  if (!rc && c.heads) rc = resolve_strides(call, "q", c.T, c.heads, kv.D, &c.q_token, &c.q_head);
  if (!rc && c.heads) rc = resolve_strides(call, "q_out", c.T, c.heads, kv.D, &c.out_token, &c.out_head);
  if (rc || c.T == 0) return rc;
  const unsigned b = type_bytes(c.dtype);
  rc = check_cache_pointers(call, kv);
  if (!rc && c.heads) rc = check_aligned(call, "q", q, b);
  if (!rc) rc = check_aligned(call, "k", k, b);
  if (!rc) rc = check_aligned(call, "v", v, b);
  if (!rc) rc = check_aligned(call, "pos", pos, 4);
  if (!rc && seq) rc = check_aligned(call, "seq", seq, 4);
  if (!rc) rc = check_aligned(call, "table", table, 4);
  if (!rc && c.rotary_dim) rc = check_aligned(call, "freq", freq, 8);
  if (!rc && c.heads) rc = check_aligned(call, "q_out", q_out, b);
  if (rc) return rc;
  if (c.heads && q == q_out && (c.q_token != c.out_token || c.q_head != c.out_head)) return fail(MOE_E_BADARG, "%s: in place with other strides", call);
  RotaryArgs a = {};
  a.T = c.T; a.heads = c.heads; a.kv_heads = kv.heads; a.D = kv.D; a.rotary_dim = c.rotary_dim; a.layout = c.layout; a.mscale = c.mscale; a.sign = 1.f;
  a.q = q; a.k = k; a.v = v; a.q_out = q_out;
  a.q_token = c.q_token; a.q_head = c.q_head; a.k_token = c.k_token; a.k_head = c.k_head; a.v_token = c.v_token; a.v_head = c.v_head;
  a.out_token = c.out_token; a.out_head = c.out_head;
  a.pos = pos; a.seq = seq; a.table = table; a.freq = freq;
  a.n_seqs = c.n_seqs; a.table_len = c.table_len; a.table_ld = c.table_ld; a.n_pages = kv.n_pages; a.shift = page_shift(kv.page_size); a.cache_dtype = kv.dtype;
  a.page = kv.page; a.head = kv.head; a.row = kv.row;
  a.k_cache = kv.k; a.v_cache = kv.v; a.k_scale = kv.k_scale; a.v_scale = kv.v_scale;
  return launch_rotary(a, c.dtype, static_cast<hipStream_t>(stream));
}

extern "C" size_t moe_paged_attention_workspace_bytes(const moe_attention_config* cfg, const moe_kv_cache* cache) {
  const char* call = "moe_paged_attention_workspace_bytes";
  moe_kv_cache kv;
  moe_attention_config c;
  AttentionPlan p;
  if (resolve(call, cache, &kv) || resolve(call, cfg, kv, &c, &p)) return 0;
  return Workspace(c, kv, p).bytes;
}

extern "C" int moe_paged_attention(const moe_attention_config* cfg, const moe_kv_cache* cache, const void* q, const int32_t* table,
                                   const int32_t* lengths, void* out, float* lse, void* ws, size_t ws_bytes, int32_t* counters, void* stream) {
  const char* call = "moe_paged_attention";
  moe_kv_cache kv;
  moe_attention_config c;
  AttentionPlan p;
  int rc = resolve(call, cache, &kv);
  if (!rc) rc = resolve(call, cfg, kv, &c, &p);
  if (rc || c.B == 0) return rc;
  rc = check_cache_pointers(call, kv);
  if (!rc) rc = check_aligned(call, "q", q, type_bytes(c.dtype));
  if (!rc) rc = check_aligned(call, "table", table, 4);
  if (!rc) rc = check_aligned(call, "lengths", lengths, 4);
  if (!rc) rc = check_aligned(call, "out", out, type_bytes(c.dtype));
  if (!rc && lse) rc = check_aligned(call, "lse", lse, 4);
  if (!rc && counters) rc = check_aligned(call, "counters", counters, 4);
  if (rc) return rc;
  // a workgroup would store over what another one reads; strides of what there is only one of do not matter
  if (q == out && ((c.B > 1 && c.q_token != c.out_token) || (c.heads > 1 && c.q_head != c.out_head))) return fail(MOE_E_BADARG, "%s: in place with other strides", call);
  const Workspace w(c, kv, p);
  const size_t need = w.bytes;
  if (need && (!ws || ((uintptr_t)ws & 255) || ws_bytes < need))
    return fail(MOE_E_WORKSPACE, "%s: workspace %p of %zu bytes (need %zu, 256-byte aligned)", call, ws, ws_bytes, need);
  AttentionArgs a = {};
  a.B = c.B; a.heads = c.heads; a.kv_heads = kv.heads; a.group = c.heads / kv.heads; a.D = kv.D; a.dtype = c.dtype; a.cache_dtype = kv.dtype;
  a.max_len = c.max_len; a.window = c.window; a.table_len = c.table_len; a.table_ld = c.table_ld; a.n_pages = kv.n_pages; a.shift = page_shift(kv.page_size);
  a.workgroups = p.workgroups; a.waves = p.waves; a.align = p.align; a.scale = c.scale; a.softcap = c.softcap;
  a.q_token = c.q_token; a.q_head = c.q_head; a.out_token = c.out_token; a.out_head = c.out_head;
  a.page = kv.page; a.head = kv.head; a.row = kv.row;
  a.q = q; a.table = table; a.lengths = lengths; a.k = kv.k; a.v = kv.v; a.k_scale = kv.k_scale; a.v_scale = kv.v_scale;
  a.out = out; a.lse = lse;
  if (need) {
    char* const at = static_cast<char*>(ws);
    a.part_out = static_cast<float*>(ws);
    a.part_stat = reinterpret_cast<float*>(at + w.stat);
    if (p.few_parts) a.counters = counters;
    if (!a.counters) a.started = reinterpret_cast<int32_t*>(at + w.started);
  }
  return launch_attention(a, static_cast<hipStream_t>(stream));
}
