// C entry points of the LLM task's side (argument checks and the launch plan; the kernels are in cache.hip and
// cache_attention.hip).
#include <algorithm>
#include <cmath>
#include <string>

#include "cache.h"

using namespace cs;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }

cs_status invalid(const char* who, const char* what) { return fail(CS_ERR_INVALID_ARG, std::string(who) + ": " + what); }
cs_status unsupported(const char* who, const char* what) { return fail(CS_ERR_UNSUPPORTED, std::string(who) + ": " + what); }

// rows of heads x dim elements, `row` elements apart
cs_status check_rows(const char* who, const void* p, int64_t row, int64_t heads, int64_t dim, int size) {
  if (!p || !aligned16(p)) return invalid(who, "NULL or misaligned rows");
  if (row < heads * dim || row > (int64_t)1 << 40) return invalid(who, "rows overlap or lie too far apart");
  if (row * size % 16) return unsupported(who, "rows must be multiples of 16 bytes apart");
  return CS_OK;
}

constexpr int64_t MAX_ROWS = (int64_t)1 << 31;
constexpr int32_t MAX_HEADS = 1024;

cs_status check_cache(const char* who, const cs_cache_config* c) {
  if (!c) return invalid(who, "NULL configuration");
  if (c->struct_size != sizeof(cs_cache_config)) return invalid(who, "config.struct_size mismatch");
  if (c->n_kv_heads <= 0 || c->head_dim <= 0 || c->page_tokens <= 0 || c->n_pages <= 0) return invalid(who, "configuration sizes");
  if (c->n_kv_heads > MAX_HEADS) return unsupported(who, "at most 1024 key/value heads");
  if (c->head_dim != 64 && c->head_dim != 128) return unsupported(who, "head_dim must be 64 or 128");
  if (c->page_tokens % 32 || c->page_tokens > 1 << 20) return unsupported(who, "page_tokens must be a multiple of 32, at most 2^20");
  if (c->n_pages > 0x7fffffff) return unsupported(who, "at most 2^31 - 1 pages");
  return CS_OK;
}

cs_status check_batch(const char* who, const cs_cache_config* c, const cs_cache_batch* b, int32_t n_heads) {
  if (cs_status st = check_cache(who, c)) return st;
  if (!b) return invalid(who, "NULL batch");
  if (b->struct_size != sizeof(cs_cache_batch)) return invalid(who, "batch.struct_size mismatch");
  if (b->n_seqs < 0 || b->n_queries < 0 || b->max_queries < 0 || b->max_keys < 0 || b->table_width < 0) return invalid(who, "negative size");
  if (b->n_queries >= MAX_ROWS || b->max_keys > (int64_t)1 << 30) return unsupported(who, "at most 2^31 - 1 queries and 2^30 keys");
  if (n_heads <= 0 || n_heads % c->n_kv_heads) return invalid(who, "n_heads must be a positive multiple of n_kv_heads");
  if (n_heads > MAX_HEADS) return unsupported(who, "at most 1024 heads");
  if ((int64_t)b->max_queries * (n_heads / c->n_kv_heads) >= MAX_ROWS - 64) return unsupported(who, "too many queries in a sequence");
  return CS_OK;
}

CacheAttnArgs attention_args(const cs_cache_config* c, const cs_cache_batch* b, int32_t n_heads) {
  CacheAttnArgs a = {};
  a.shape = cache_shape(*c);
  a.n_seqs = b->n_seqs;
  a.n_queries = b->n_queries;
  a.max_queries = (int32_t)(b->max_queries < b->n_queries ? b->max_queries : b->n_queries);
  a.max_keys = b->max_keys;
  a.table_width = b->table_width;
  a.n_heads = n_heads;
  a.group = n_heads / c->n_kv_heads;
  return a;
}

cs_status cache_rows(const char* who, const cs_cache_config* c, const void* pool, const void* k, int64_t k_row, const void* v, int64_t v_row,
                     int32_t dtype, const int64_t* slots, int64_t n_rows, int32_t* err_flag, CacheRows& a) {
  if (cs_status st = check_cache(who, c)) return st;
  if (dtype != CS_F32 && dtype != CS_BF16) return invalid(who, "dtype");
  if (n_rows < 0) return invalid(who, "negative size");
  if (n_rows >= MAX_ROWS) return unsupported(who, "at most 2^31 - 1 rows");
  if (n_rows == 0) return CS_OK;
  if (!pool || !aligned16(pool)) return invalid(who, "NULL or misaligned pool");
  if (!slots || !aligned8(slots) || !aligned4(err_flag)) return invalid(who, "NULL or misaligned slots or flag");
  const int size = dtype == CS_BF16 ? 2 : 4;
  if (cs_status st = check_rows(who, k, k_row, c->n_kv_heads, c->head_dim, size)) return st;
  if (cs_status st = check_rows(who, v, v_row, c->n_kv_heads, c->head_dim, size)) return st;
  a = CacheRows{static_cast<unsigned char*>(const_cast<void*>(pool)), const_cast<void*>(k), const_cast<void*>(v), k_row, v_row, slots, n_rows,
                cache_shape(*c), err_flag};
  return CS_OK;
}

cs_status qk_norm_rope(const cs_qk_config* c, const void* q, int64_t q_row, const void* k, int64_t k_row, void* q_out, int64_t q_out_row,
                       void* k_out, int64_t k_out_row, int32_t dtype, const float* q_gain, const float* k_gain, const float* cos_sin,
                       const int32_t* positions, int64_t n_rows, int32_t* err_flag, void* stream) {
  const char* who = "cs_qk_norm_rope";
  if (!c) return invalid(who, "NULL configuration");
  if (c->struct_size != sizeof(cs_qk_config)) return invalid(who, "config.struct_size mismatch");
  if (dtype != CS_F32 && dtype != CS_BF16) return invalid(who, "dtype");
  if (c->n_heads < 0 || c->n_kv_heads < 0 || c->n_heads + (int64_t)c->n_kv_heads <= 0) return invalid(who, "heads");
  if (c->n_heads > MAX_HEADS || c->n_kv_heads > MAX_HEADS) return unsupported(who, "at most 1024 heads");
  if (c->head_dim <= 0 || c->rotary_dim <= 0 || c->rotary_dim > c->head_dim) return invalid(who, "head_dim, rotary_dim");
  if (c->head_dim % 16 || c->rotary_dim % 16 || c->head_dim > 256)
    return unsupported(who, "head_dim and rotary_dim must be multiples of 16, head_dim at most 256");
  if (c->axes < 1 || c->axes > 3) return invalid(who, "axes");
  const int half = c->rotary_dim / 2;
  int64_t sum = 0;
  for (int x = 0; x < 3; ++x) {
    if (c->sections[x] < 0 || (x >= c->axes && c->sections[x])) return invalid(who, "sections");
    sum += c->sections[x];
  }
  if (sum != half) return invalid(who, "sections must sum to rotary_dim / 2");
  if (c->interleaved != 0 && c->interleaved != 1) return invalid(who, "interleaved must be 0 or 1");
  // (pair 3 (n - 1) + x is the last one of axis x; it has to be a pair)
  if (c->interleaved && (c->axes != 3 || 3 * c->sections[1] - 2 >= half || 3 * c->sections[2] - 1 >= half))
    return invalid(who, "interleaved sections need three axes, the second and third no larger than a third of the pairs");
  if (!(c->eps >= 0)) return invalid(who, "eps");
  if (c->n_positions <= 0 || c->n_positions > (int64_t)1 << 31) return invalid(who, "n_positions");
  if (n_rows < 0) return invalid(who, "negative size");
  if (n_rows >= MAX_ROWS) return unsupported(who, "at most 2^31 - 1 rows");
  if (n_rows == 0) return CS_OK;
  const int size = dtype == CS_BF16 ? 2 : 4;
  if (c->n_heads) {
    if (cs_status st = check_rows(who, q, q_row, c->n_heads, c->head_dim, size)) return st;
    if (cs_status st = check_rows(who, q_out, q_out_row, c->n_heads, c->head_dim, size)) return st;
  }
  if (c->n_kv_heads) {
    if (cs_status st = check_rows(who, k, k_row, c->n_kv_heads, c->head_dim, size)) return st;
    if (cs_status st = check_rows(who, k_out, k_out_row, c->n_kv_heads, c->head_dim, size)) return st;
  }
  const bool norm = q_gain || k_gain;
  if (norm && ((c->n_heads && !q_gain) || (c->n_kv_heads && !k_gain))) return invalid(who, "one gain without the other");
  if (!aligned16(q_gain) || !aligned16(k_gain)) return invalid(who, "misaligned gains");
  if (!cos_sin || !aligned16(cos_sin) || !positions || !aligned4(positions) || !aligned4(err_flag))
    return invalid(who, "NULL or misaligned table, positions or flag");
  QkArgs a = {};
  a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
  a.q_row = q_row; a.k_row = k_row; a.q_out_row = q_out_row; a.k_out_row = k_out_row;
  a.norm = norm; a.q_gain = q_gain; a.k_gain = k_gain; a.cos_sin = cos_sin; a.positions = positions;
  a.n_rows = n_rows; a.n_positions = c->n_positions;
  a.n_heads = c->n_heads; a.n_kv_heads = c->n_kv_heads; a.head_dim = c->head_dim; a.half = half; a.axes = c->axes;
  if (c->interleaved) {
    a.end0 = a.end1 = half;
    a.lim1 = 3 * c->sections[1]; a.lim2 = 3 * c->sections[2];
  } else {
    a.end0 = c->sections[0]; a.end1 = c->sections[0] + c->sections[1];
    a.lim1 = a.lim2 = 0;
  }
  a.eps = c->eps; a.err = err_flag;
  return launch_qk_norm_rope(a, dtype, static_cast<hipStream_t>(stream));
}

cs_status attention_cache(const cs_cache_config* c, const void* pool, const cs_cache_batch* b, const void* q, int64_t q_row, void* out,
                          int64_t out_row, int32_t n_heads, float scale, int32_t causal, void* workspace, size_t workspace_bytes,
                          int32_t* err_flag, void* stream) {
  const char* who = "cs_attention_cache";
  if (cs_status st = check_batch(who, c, b, n_heads)) return st;
  if (causal != 0 && causal != 1) return invalid(who, "causal must be 0 or 1");
  if (!(scale - scale == 0)) return invalid(who, "scale must be finite");
  if (b->n_seqs == 0 || b->n_queries == 0 || b->max_queries == 0) return CS_OK;
  if (cs_status st = check_rows(who, q, q_row, n_heads, c->head_dim, 2)) return st;
  if (cs_status st = check_rows(who, out, out_row, n_heads, c->head_dim, 2)) return st;
  if (!pool || !aligned16(pool)) return invalid(who, "NULL or misaligned pool");
  if (!b->cu_queries || !b->n_keys || (!b->page_table && b->table_width) || !aligned4(b->cu_queries) || !aligned4(b->n_keys) ||
      !aligned4(b->page_table) || !aligned4(err_flag))
    return invalid(who, "NULL or misaligned lengths, page table or flag");
  CacheAttnArgs a = attention_args(c, b, n_heads);
  size_t need = 0;
  if (cs_status st = plan_cache_attention(a, need)) return st;
  if (need && (!workspace || !aligned16(workspace))) return invalid(who, "NULL or misaligned workspace");
  if (workspace_bytes < need)
    return fail(CS_ERR_WORKSPACE, std::string(who) + ": needs " + std::to_string(need) + " bytes of workspace, got " + std::to_string(workspace_bytes));
  a.pool = static_cast<const unsigned char*>(pool);
  a.q = static_cast<const bf16_t*>(q); a.q_row = q_row;
  a.out = static_cast<bf16_t*>(out); a.out_row = out_row;
  a.cu = b->cu_queries; a.n_keys = b->n_keys; a.table = b->page_table;
  // (a scale of zero as one too small to matter: -inf, a masked score, stays what it is)
  a.scale_log2 = std::max(std::fabs(scale) * 1.4426950408889634f, 1e-30f);
  a.q_sign = scale < 0 ? 0x80008000u : 0;
  a.causal = causal; a.err = err_flag;
  return launch_cache_attention(a, workspace, static_cast<hipStream_t>(stream));
}

}  // namespace

extern "C" {

cs_status cs_qk_norm_rope(const cs_qk_config* config, const void* q, int64_t q_row, const void* k, int64_t k_row, void* q_out,
                          int64_t q_out_row, void* k_out, int64_t k_out_row, int32_t dtype, const float* q_gain, const float* k_gain,
                          const float* cos_sin, const int32_t* positions, int64_t n_rows, int32_t* err_flag, void* stream) try {
  return qk_norm_rope(config, q, q_row, k, k_row, q_out, q_out_row, k_out, k_out_row, dtype, q_gain, k_gain, cos_sin, positions, n_rows,
                      err_flag, stream);
}
CS_CATCH_ALL("cs_qk_norm_rope")

cs_status cs_cache_query(const cs_cache_config* config, size_t* page_bytes, size_t* pool_bytes) try {
  if (cs_status st = check_cache("cs_cache_query", config)) return st;
  const size_t page = (size_t)cache_shape(*config).head_bytes * (size_t)config->n_kv_heads;
  if (page_bytes) *page_bytes = page;
  if (pool_bytes) *pool_bytes = page * (size_t)config->n_pages;
  return CS_OK;
}
CS_CATCH_ALL("cs_cache_query")

cs_status cs_cache_write(const cs_cache_config* config, void* pool, const void* k, int64_t k_row, const void* v, int64_t v_row, int32_t dtype,
                         const int64_t* slots, int64_t n_rows, int32_t* err_flag, void* stream) try {
  CacheRows a = {};
  if (cs_status st = cache_rows("cs_cache_write", config, pool, k, k_row, v, v_row, dtype, slots, n_rows, err_flag, a)) return st;
  return n_rows ? launch_cache_write(a, dtype, static_cast<hipStream_t>(stream)) : CS_OK;
}
CS_CATCH_ALL("cs_cache_write")

cs_status cs_cache_read(const cs_cache_config* config, const void* pool, const int64_t* slots, int64_t n_rows, void* k, int64_t k_row, void* v,
                        int64_t v_row, int32_t dtype, int32_t* err_flag, void* stream) try {
  CacheRows a = {};
  if (cs_status st = cache_rows("cs_cache_read", config, pool, k, k_row, v, v_row, dtype, slots, n_rows, err_flag, a)) return st;
  return n_rows ? launch_cache_read(a, dtype, static_cast<hipStream_t>(stream)) : CS_OK;
}
CS_CATCH_ALL("cs_cache_read")

cs_status cs_attention_cache_query(const cs_cache_config* config, const cs_cache_batch* batch, int32_t n_heads, size_t* workspace_bytes) try {
  if (!workspace_bytes) return invalid("cs_attention_cache_query", "NULL argument");
  if (cs_status st = check_batch("cs_attention_cache_query", config, batch, n_heads)) return st;
  const CacheAttnArgs a = attention_args(config, batch, n_heads);
  return plan_cache_attention(a, *workspace_bytes);
}
CS_CATCH_ALL("cs_attention_cache_query")

cs_status cs_attention_cache(const cs_cache_config* config, const void* pool, const cs_cache_batch* batch, const void* q, int64_t q_row, void* out,
                             int64_t out_row, int32_t n_heads, float scale, int32_t causal, void* workspace, size_t workspace_bytes,
                             int32_t* err_flag, void* stream) try {
  return attention_cache(config, pool, batch, q, q_row, out, out_row, n_heads, scale, causal, workspace, workspace_bytes, err_flag, stream);
}
CS_CATCH_ALL("cs_attention_cache")

}  // extern "C"
