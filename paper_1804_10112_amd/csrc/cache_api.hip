// C ABI entry points of the paged cache, of attention over it and of the rules on logits: checks of the arguments and dispatch.
// Host code only.
#include "common.hpp"

namespace spt {

// implemented in the kernel translation units
size_t cache_extend_workspace(const spt_cache* c);
spt_status cache_extend_dispatch(const spt_cache* c, const int32_t* add, int32_t* refused, void* ws, hipStream_t s);
spt_status cache_free_dispatch(const spt_cache* c, const int32_t* new_len, hipStream_t s);
spt_status cache_fork_dispatch(const spt_cache* c, int n, const int32_t* parents, const int32_t* children, hipStream_t s);
spt_status cache_write_dispatch(const spt_cache* c, int layer, const int32_t* first, int total, const void* k, const void* v,
                                int64_t token_stride, int64_t head_stride, hipStream_t s);
spt_status cache_compact_dispatch(const spt_cache* c, const int32_t* first, const spt_tensor* keep, hipStream_t s);
size_t cache_attention_workspace(const spt_cache* c, int32_t q_heads);
spt_status cache_attention_dispatch(const spt_cache* c, int32_t layer, const int32_t* first, int32_t total, const spt_tensor* tree,
                                    const void* q, int32_t q_heads, int64_t q_token_stride, int64_t q_head_stride, float scale,
                                    void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse, void* ws,
                                    hipStream_t s);
spt_status adjust_logits_dispatch(int32_t dtype, int64_t R, int64_t V, const void* logits, int64_t logits_stride,
                                  const spt_logit_rules* rules, void* out, int64_t out_stride, hipStream_t s);

// Limits that keep grids and 32-bit indices of the kernels in range.
constexpr int64_t kMaxRows = 1 << 20, kMaxTokens = 1 << 24, kMaxForks = 1 << 16, kMaxStride = int64_t(1) << 40, kMaxInPage = int64_t(1) << 33,
                  kMaxColumns = 1 << 27;

// Of a scale: times log2(e) it is still a number. With an infinity scores of 0 would become NaN, with NaN hidden ones too.
constexpr float kMostScale = 0x1p127f;

static bool narrow_type(int32_t dtype, const char* what) {
  if (dtype == SPT_F32 || dtype == SPT_F16 || dtype == SPT_BF16) return true;
  if (dtype == SPT_F64)
    fail(SPT_ERR_UNSUPPORTED, "%s: SPT_F64 is not supported (SPT_F32, SPT_F16, SPT_BF16 are)", what);
  else
    fail(SPT_ERR_INVALID_ARG, "%s: unknown dtype %d", what, dtype);
  return false;
}

static spt_status narrow_status(int32_t dtype) { return dtype == SPT_F64 ? SPT_ERR_UNSUPPORTED : SPT_ERR_INVALID_ARG; }

static bool odd_address(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

static bool stride_ok(int64_t stride, int32_t dtype) {
  return stride >= 0 && stride < kMaxStride && stride % (dtype == SPT_F32 ? 4 : 8) == 0;
}

static spt_status cache_ok(const spt_cache* c, const char* what) {
  if (!c) return fail(SPT_ERR_INVALID_ARG, "%s: null cache", what);
  if (!narrow_type(c->dtype, what)) return narrow_status(c->dtype);
  if (c->layers < 1 || c->heads < 1 || c->layers > 65536 || c->heads > 65535)
    return fail(SPT_ERR_INVALID_ARG, "%s: layers %d or heads %d out of range", what, c->layers, c->heads);
  if (c->width < 8 || c->width > 256 || c->width % 8 != 0)
    return fail(SPT_ERR_UNSUPPORTED, "%s: width %d is not a multiple of 8 from 8 to 256", what, c->width);
  if (c->page < 1 || c->page > 65536 || (c->page & (c->page - 1)) != 0)
    return fail(SPT_ERR_UNSUPPORTED, "%s: page %d is not a power of two from 1 to 65536", what, c->page);
  if (static_cast<int64_t>(c->layers) * c->heads > 65536)
    return fail(SPT_ERR_UNSUPPORTED, "%s: %d layers of %d heads, at most 65536 in all", what, c->layers, c->heads);
  if (c->rows < 0 || c->row_pages < 0 || c->pages < 0 || c->pages >= INT32_MAX)
    return fail(SPT_ERR_INVALID_ARG, "%s: rows, row_pages or pages out of range", what);
  if (c->rows > kMaxRows) return fail(SPT_ERR_UNSUPPORTED, "%s: %d rows, at most %lld", what, c->rows, (long long)kMaxRows);
  if (static_cast<int64_t>(c->rows) * (static_cast<int64_t>(c->row_pages) + 1) >= INT32_MAX ||
      static_cast<int64_t>(c->row_pages) * c->page >= INT32_MAX - 65536)
    return fail(SPT_ERR_UNSUPPORTED, "%s: a table of %d rows of %d pages of %d slots is beyond int32", what, c->rows, c->row_pages,
                c->page);
  if (!stride_ok(c->layer_stride, c->dtype) || !stride_ok(c->page_stride, c->dtype) || !stride_ok(c->slot_stride, c->dtype) ||
      !stride_ok(c->head_stride, c->dtype))
    return fail(SPT_ERR_INVALID_ARG, "%s: the cache's strides must not be negative and must be multiples of 16 bytes", what);
  if (c->page_stride >= kMaxInPage || c->slot_stride >= kMaxInPage || c->head_stride >= kMaxInPage)
    return fail(SPT_ERR_UNSUPPORTED, "%s: a page, slot or head stride of 2^33 elements or more", what);
  if (c->pages > 0 && (!c->K || !c->V || !c->refs)) return fail(SPT_ERR_INVALID_ARG, "%s: K, V or refs is null", what);
  if (odd_address(c->K) || odd_address(c->V)) return fail(SPT_ERR_INVALID_ARG, "%s: K or V is not 16-byte aligned", what);
  if (c->rows > 0 && (!c->len || (!c->table && c->row_pages > 0)))
    return fail(SPT_ERR_INVALID_ARG, "%s: table or len is null", what);
  return SPT_OK;
}

// A CSR matrix of N rows of which only the structure counts.
static spt_status pattern_ok(const spt_tensor* t, int64_t N, const char* what, const char* name) {
  spt_tensor p = *t;
  p.dtype = SPT_F32;
  p.vals = &p;  // never read; the host check asks for a pointer
  const Format f = recognize(&p);
  if (f == Format::Invalid) return SPT_ERR_INVALID_ARG;
  if (f != Format::CSR) return fail(SPT_ERR_UNSUPPORTED, "%s: %s must be CSR", what, name);
  if (p.level[0].N != N)
    return fail(SPT_ERR_INVALID_ARG, "%s: %s has %lld rows, not %lld", what, name, (long long)p.level[0].N, (long long)N);
  if (p.nvals >= INT32_MAX) return fail(SPT_ERR_UNSUPPORTED, "%s: %s has entries beyond int32", what, name);
  return SPT_OK;
}

static spt_status ws_ok(const void* ws, size_t given, size_t needed, const char* what) {
  if (reinterpret_cast<uintptr_t>(ws) % 256 != 0) return fail(SPT_ERR_INVALID_ARG, "workspace pointer is not 256-byte aligned");
  if (!ws || given < needed) return fail(SPT_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", what, needed, ws ? given : 0);
  return SPT_OK;
}

}  // namespace spt

using namespace spt;

extern "C" {

size_t spt_cache_workspace_bytes(int32_t op, const spt_cache* c, int32_t q_heads) {
  clear_error();
  if (cache_ok(c, "cache_workspace_bytes") != SPT_OK) return 0;
  size_t n = 0;
  if (op == SPT_CACHE_EXTEND) {
    n = cache_extend_workspace(c);
  } else if (op == SPT_CACHE_ATTENTION) {
    if (q_heads < 1 || q_heads > 65535 || q_heads % c->heads != 0) {
      fail(SPT_ERR_INVALID_ARG, "cache_workspace_bytes: q_heads %d is not a multiple of the cache's %d heads, up to 65535", q_heads,
           c->heads);
      return 0;
    }
    n = cache_attention_workspace(c, q_heads);
  } else {
    fail(SPT_ERR_INVALID_ARG, "cache_workspace_bytes: unknown op %d", op);
    return 0;
  }
  return n < 256 ? 256 : n;
}

spt_status spt_cache_extend(const spt_cache* c, const int32_t* add, int32_t* refused_dev, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  spt_status st = cache_ok(c, "cache_extend");
  if (st != SPT_OK) return st;
  if (!refused_dev || (!add && c->rows > 0)) return fail(SPT_ERR_INVALID_ARG, "cache_extend: add or refused_dev is null");
  st = ws_ok(ws, ws_bytes, cache_extend_workspace(c), "cache_extend");
  if (st != SPT_OK) return st;
  return cache_extend_dispatch(c, add, refused_dev, ws, static_cast<hipStream_t>(stream));
}

spt_status spt_cache_free(const spt_cache* c, const int32_t* new_len, void* stream) {
  clear_error();
  const spt_status st = cache_ok(c, "cache_free");
  if (st != SPT_OK) return st;
  if (c->rows == 0) return SPT_OK;
  if (!new_len) return fail(SPT_ERR_INVALID_ARG, "cache_free: new_len is null");
  return cache_free_dispatch(c, new_len, static_cast<hipStream_t>(stream));
}

spt_status spt_cache_fork(const spt_cache* c, int64_t n, const int32_t* parents, const int32_t* children, void* stream) {
  clear_error();
  const spt_status st = cache_ok(c, "cache_fork");
  if (st != SPT_OK) return st;
  if (n < 0) return fail(SPT_ERR_INVALID_ARG, "cache_fork: n = %lld is negative", (long long)n);
  if (n > kMaxForks) return fail(SPT_ERR_UNSUPPORTED, "cache_fork: n = %lld, at most %lld", (long long)n, (long long)kMaxForks);
  if (n == 0) return SPT_OK;
  if (!parents || !children) return fail(SPT_ERR_INVALID_ARG, "cache_fork: parents or children is null");
  return cache_fork_dispatch(c, static_cast<int>(n), parents, children, static_cast<hipStream_t>(stream));
}

spt_status spt_cache_write(const spt_cache* c, int32_t layer, const int32_t* first, int64_t T, const void* k, const void* v,
                           int64_t token_stride, int64_t head_stride, void* stream) {
  clear_error();
  const spt_status st = cache_ok(c, "cache_write");
  if (st != SPT_OK) return st;
  if (layer < 0 || layer >= c->layers) return fail(SPT_ERR_INVALID_ARG, "cache_write: layer %d of %d", layer, c->layers);
  if (T < 0) return fail(SPT_ERR_INVALID_ARG, "cache_write: T = %lld is negative", (long long)T);
  if (T > kMaxTokens) return fail(SPT_ERR_UNSUPPORTED, "cache_write: T = %lld, at most %lld", (long long)T, (long long)kMaxTokens);
  if (T == 0 || c->rows == 0 || c->pages == 0) return SPT_OK;
  if (!first || !k || !v) return fail(SPT_ERR_INVALID_ARG, "cache_write: first, k or v is null");
  if (odd_address(k) || odd_address(v)) return fail(SPT_ERR_INVALID_ARG, "cache_write: k or v is not 16-byte aligned");
  if (!stride_ok(token_stride, c->dtype) || !stride_ok(head_stride, c->dtype))
    return fail(SPT_ERR_INVALID_ARG, "cache_write: strides must not be negative and must be multiples of 16 bytes");
  return cache_write_dispatch(c, layer, first, static_cast<int>(T), k, v, token_stride, head_stride,
                              static_cast<hipStream_t>(stream));
}

spt_status spt_cache_compact(const spt_cache* c, const int32_t* first, const spt_tensor* keep, void* stream) {
  clear_error();
  spt_status st = cache_ok(c, "cache_compact");
  if (st != SPT_OK) return st;
  if (!keep) return fail(SPT_ERR_INVALID_ARG, "cache_compact: keep is null");
  st = pattern_ok(keep, c->rows, "cache_compact", "keep");
  if (st != SPT_OK) return st;
  if ((keep->level[1].flags & (SPT_ORDERED | SPT_UNIQUE)) != (SPT_ORDERED | SPT_UNIQUE))
    return fail(SPT_ERR_UNSUPPORTED, "cache_compact: the columns of keep must be ordered and unique");
  if (c->rows == 0) return SPT_OK;
  if (!first) return fail(SPT_ERR_INVALID_ARG, "cache_compact: first is null");
  return cache_compact_dispatch(c, first, keep, static_cast<hipStream_t>(stream));
}

spt_status spt_cache_attention(const spt_cache* c, int32_t layer, const int32_t* first, int64_t T, const spt_tensor* tree,
                               const void* q, int32_t q_heads, int64_t q_token_stride, int64_t q_head_stride, float scale, void* out,
                               int64_t out_token_stride, int64_t out_head_stride, float* lse, void* ws, size_t ws_bytes,
                               void* stream) {
  clear_error();
  spt_status st = cache_ok(c, "cache_attention");
  if (st != SPT_OK) return st;
  if (layer < 0 || layer >= c->layers) return fail(SPT_ERR_INVALID_ARG, "cache_attention: layer %d of %d", layer, c->layers);
  if (T < 0) return fail(SPT_ERR_INVALID_ARG, "cache_attention: T = %lld is negative", (long long)T);
  if (T > kMaxTokens) return fail(SPT_ERR_UNSUPPORTED, "cache_attention: T = %lld, at most %lld", (long long)T, (long long)kMaxTokens);
  if (q_heads < 1 || q_heads > 65535 || q_heads % c->heads != 0)
    return fail(SPT_ERR_INVALID_ARG, "cache_attention: q_heads %d is not a multiple of the cache's %d heads, up to 65535", q_heads,
                c->heads);
  if (!(scale >= -kMostScale && scale <= kMostScale))
    return fail(SPT_ERR_INVALID_ARG, "cache_attention: scale %g is not a number from -2^127 to 2^127", static_cast<double>(scale));
  if (T * (q_heads / c->heads) >= INT32_MAX - 256)
    return fail(SPT_ERR_UNSUPPORTED, "cache_attention: %lld tokens of %d query heads for each head of K", (long long)T,
                q_heads / c->heads);
  if (tree) {
    st = pattern_ok(tree, T, "cache_attention", "tree");
    if (st != SPT_OK) return st;
  }
  st = ws_ok(ws, ws_bytes, spt_cache_workspace_bytes(SPT_CACHE_ATTENTION, c, q_heads), "cache_attention");
  if (st != SPT_OK) return st;
  if (T == 0 || c->rows == 0) return SPT_OK;
  if (!first || !q || !out) return fail(SPT_ERR_INVALID_ARG, "cache_attention: first, q or out is null");
  if (odd_address(q) || odd_address(out)) return fail(SPT_ERR_INVALID_ARG, "cache_attention: q or out is not 16-byte aligned");
  if (!stride_ok(q_token_stride, c->dtype) || !stride_ok(q_head_stride, c->dtype) || !stride_ok(out_token_stride, c->dtype) ||
      !stride_ok(out_head_stride, c->dtype))
    return fail(SPT_ERR_INVALID_ARG, "cache_attention: strides must not be negative and must be multiples of 16 bytes");
  return cache_attention_dispatch(c, layer, first, static_cast<int32_t>(T), tree, q, q_heads, q_token_stride, q_head_stride, scale,
                                  out, out_token_stride, out_head_stride, lse, ws, static_cast<hipStream_t>(stream));
}

spt_status spt_adjust_logits(int32_t dtype, int64_t R, int64_t V, const void* logits, int64_t logits_stride,
                             const spt_logit_rules* rules, void* out, int64_t out_stride, void* stream) {
  clear_error();
  if (!narrow_type(dtype, "adjust_logits")) return narrow_status(dtype);
  if (!rules) return fail(SPT_ERR_INVALID_ARG, "adjust_logits: null rules");
  if (R < 0 || V < 0 || V >= INT32_MAX || rules->sequences < 0)
    return fail(SPT_ERR_INVALID_ARG, "adjust_logits: %lld rows of %lld columns, %lld sequences", (long long)R, (long long)V,
                (long long)rules->sequences);
  if (R > kMaxTokens || rules->sequences > kMaxTokens)
    return fail(SPT_ERR_UNSUPPORTED, "adjust_logits: %lld rows, %lld sequences, at most %lld", (long long)R,
                (long long)rules->sequences, (long long)kMaxTokens);
  if (V > kMaxColumns)
    return fail(SPT_ERR_UNSUPPORTED, "adjust_logits: %lld columns, at most %lld", (long long)V, (long long)kMaxColumns);
  if (!rules->first && R != rules->sequences)
    return fail(SPT_ERR_INVALID_ARG, "adjust_logits: %lld rows of %lld sequences need first", (long long)R,
                (long long)rules->sequences);
  if (logits_stride < V || out_stride < V || logits_stride >= kMaxStride || out_stride >= kMaxStride)
    return fail(SPT_ERR_INVALID_ARG, "adjust_logits: a row stride is below the column count or too large");
  spt_status st = SPT_OK;
  if (rules->seen && (st = pattern_ok(rules->seen, rules->sequences, "adjust_logits", "seen")) != SPT_OK) return st;
  if (rules->tree && (st = pattern_ok(rules->tree, R, "adjust_logits", "tree")) != SPT_OK) return st;
  if (rules->tree && !rules->drafts) return fail(SPT_ERR_INVALID_ARG, "adjust_logits: a tree without drafts");
  if (rules->bias) {
    if ((st = pattern_ok(rules->bias, rules->sequences, "adjust_logits", "bias")) != SPT_OK) return st;
    if (rules->bias->dtype != SPT_F32) return fail(SPT_ERR_UNSUPPORTED, "adjust_logits: bias must be SPT_F32");
    if (!(rules->bias->level[1].flags & SPT_UNIQUE))
      return fail(SPT_ERR_UNSUPPORTED, "adjust_logits: the columns of bias must be unique");
    if (!rules->bias->vals && rules->bias->nvals > 0) return fail(SPT_ERR_INVALID_ARG, "adjust_logits: bias has no values");
  }
  if (rules->allowed && (rules->allowed_stride < (V + 31) / 32 || rules->allowed_stride >= kMaxStride))
    return fail(SPT_ERR_INVALID_ARG, "adjust_logits: allowed_stride %lld is below the %lld words of a row",
                (long long)rules->allowed_stride, (long long)((V + 31) / 32));
  if (R == 0 || V == 0 || rules->sequences == 0) return SPT_OK;
  if (!logits || !out) return fail(SPT_ERR_INVALID_ARG, "adjust_logits: logits or out is null");
  const uintptr_t size = dtype == SPT_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % size || reinterpret_cast<uintptr_t>(out) % size)
    return fail(SPT_ERR_INVALID_ARG, "adjust_logits: logits or out is not aligned to its values");
  if (logits == out && logits_stride != out_stride)
    return fail(SPT_ERR_INVALID_ARG, "adjust_logits: logits and out are one array with two strides");
  return adjust_logits_dispatch(dtype, R, V, logits, logits_stride, rules, out, out_stride, static_cast<hipStream_t>(stream));
}

}  // extern "C"
