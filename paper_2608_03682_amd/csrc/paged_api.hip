// C entry points of the paged key/value cache: every check that the host can make,
// then one launch (attention: two where the keys are split over blocks).
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "errors.hpp"
#include "paged.hpp"
#include "paged_host.hpp"

using namespace phyai;

namespace phyai {

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
void req(bool ok, const char* m) {
  if (!ok) fail(PHYAI_EINVAL, m);
}
// Lengths, scales and the status word; the status takes atomics, which fault elsewhere.
void words(std::initializer_list<const void*> ps) {
  for (const void* p : ps) req((reinterpret_cast<uintptr_t>(p) & 3u) == 0, "lengths, scales and status must be 4-byte aligned");
}
int elem_bytes(int dtype) { return dtype == PHYAI_DTYPE_F32 ? 4 : (dtype == PHYAI_DTYPE_BF16 ? 2 : 1); }

// Sizes small enough that no product below, and no row number of a kernel, leaves
// 31 bits (63 where it is an offset).
constexpr int kMaxRequests = 4096, kMaxRows = 1 << 20, kMaxHeads = 1024, kMaxLayers = 1024;
constexpr int64_t kMaxStride = int64_t(1) << 40;

int row_kind(int dtype) {
  req(dtype == PHYAI_DTYPE_F32 || dtype == PHYAI_DTYPE_BF16, "rows must be F32 or BF16");
  return dtype == PHYAI_DTYPE_F32 ? PAGED_F32 : PAGED_BF16;
}

void check_sizes(int batch, int rows, int dim) {
  req(batch >= 1 && batch <= kMaxRequests, "batch out of range 1..4096");
  req(rows >= 1 && rows <= kMaxRows, "rows out of range 1..2^20");
  req(dim == 64 || dim == 128 || dim == 256, "head_dim must be 64, 128 or 256");
  req((int64_t)batch * rows <= INT32_MAX / 2, "batch * rows out of range");
}

// A block of 256 threads takes one or two tokens, and a launch has fewer than 2^32 threads.
void check_tokens(int batch, int rows) {
  req((int64_t)batch * rows <= (1 << 24), "batch * rows out of range 1..2^24");
}

HeadRows head_rows(const phyai_head_rows* h, int dtype, const char* what) {
  const int es = elem_bytes(dtype);
  const std::string w = what;
  if (!h || !h->data) fail(PHYAI_EINVAL, w + " must not be NULL");
  if (!aligned16(h->data)) fail(PHYAI_EINVAL, w + " must be 16-byte aligned");
  if (h->n_heads < 1 || h->n_heads > kMaxHeads) fail(PHYAI_EINVAL, w + ": n_heads out of range 1..1024");
  for (int64_t s : {h->batch_stride, h->token_stride, h->head_stride})
    if (s < 0 || s > kMaxStride || s * es % 16 != 0)
      fail(PHYAI_EINVAL, w + ": strides must be >= 0 and multiples of 16 bytes");
  return HeadRows{h->data, h->batch_stride, h->token_stride, h->head_stride, h->n_heads};
}

// Rows that are written: no two of them at one place because of a missing stride.
HeadRows out_rows(const phyai_head_rows* h, int dtype, const char* what, int batch, int rows, int dim) {
  const HeadRows o = head_rows(h, dtype, what);
  if ((batch > 1 && o.b < dim) || (rows > 1 && o.t < dim) || (o.n > 1 && o.h < dim))
    fail(PHYAI_EINVAL, std::string(what) + ": rows that are written overlap (a stride below head_dim)");
  return o;
}

// base^(-2i/D) turns over 2 pi as 64-bit fractions.  The powers are multiplied up in
// long double (64-bit mantissa): 128 factors lose 2^-55 of the value at most.
bool rope_freq(float base, int D, RopeFreq& f) {
  for (auto& x : f.f) x = 0;
  req(base == 0.f || (std::isfinite(base) && base >= 1.f), "rope_base must be 0 or a number >= 1");
  if (base == 0.f) return false;
  const long double step = powl(static_cast<long double>(base), -2.0L / D);
  long double w = 0.15915494309189533576888376337251436L;      // 1 / 2 pi
  for (int i = 0; i < D / 2; ++i, w *= step) f.f[i] = static_cast<uint64_t>(w * 18446744073709551616.0L);
  return true;
}

}  // namespace

PagePool page_pool(const phyai_paged_cache* c, int layer) {
  req(c, "cache must not be NULL");
  req(c->dtype == PHYAI_DTYPE_F32 || c->dtype == PHYAI_DTYPE_BF16 || c->dtype == PHYAI_DTYPE_FP8E4M3,
      "cache dtype must be F32, BF16 or FP8E4M3");
  req(c->k && c->v && c->page_table, "cache pools and page table must not be NULL");
  req(aligned16(c->k) && aligned16(c->v), "cache pools must be 16-byte aligned");
  words({c->page_table, c->k_scale, c->v_scale});
  req(c->dtype != PHYAI_DTYPE_FP8E4M3 || (c->k_scale && c->v_scale), "an FP8E4M3 cache needs k_scale and v_scale");
  req(c->n_layers >= 1 && c->n_layers <= kMaxLayers, "cache n_layers out of range 1..1024");
  req(c->n_kv_heads >= 1 && c->n_kv_heads <= kMaxHeads, "cache n_kv_heads out of range 1..1024");
  check_sizes(c->batch, 1, c->head_dim);
  req(c->page_size >= 16 && c->page_size <= 4096 && (c->page_size & (c->page_size - 1)) == 0,
      "page_size must be a power of two, 16..4096");
  req(c->n_pages >= 1, "n_pages < 1");
  req(c->max_pages >= 1 && c->table_stride >= c->max_pages, "max_pages < 1 or table_stride < max_pages");
  req((int64_t)c->max_pages * c->page_size <= (1 << 30), "more than 2^30 tokens of a request");
  req(layer >= 0 && layer < c->n_layers, "layer out of range");
  const int es = elem_bytes(c->dtype);
  for (int64_t s : {c->layer_stride, c->page_stride, c->token_stride, c->head_stride})
    req(s >= 0 && s <= kMaxStride && s * es % 16 == 0, "cache strides must be >= 0 and multiples of 16 bytes");
  const int D = c->head_dim;
  req((c->n_layers == 1 || c->layer_stride >= D) && (c->n_pages == 1 || c->page_stride >= D) && c->token_stride >= D &&
          (c->n_kv_heads == 1 || c->head_stride >= D), "cache rows overlap (a stride below head_dim)");
  // lanes address inside a page with 32 bits
  req(c->token_stride * es <= (int64_t(1) << 30) / c->page_size, "a page's tokens span more than 2^30 bytes");
  PagePool p{};
  p.k = static_cast<char*>(c->k) + layer * c->layer_stride * es;
  p.v = static_cast<char*>(c->v) + layer * c->layer_stride * es;
  p.k_scale = c->k_scale;
  p.v_scale = c->v_scale;
  p.table = c->page_table;
  p.page_bytes = c->page_stride * es;
  p.head_bytes = c->head_stride * es;
  p.layer_bytes = c->layer_stride * es;
  p.token_bytes = static_cast<int>(c->token_stride * es);
  p.page_shift = __builtin_ctz(static_cast<unsigned>(c->page_size));
  p.n_pages = c->n_pages;
  p.max_pages = c->max_pages;
  p.table_stride = c->table_stride;
  return p;
}

int pool_kind(const phyai_paged_cache* c) {
  return c->dtype == PHYAI_DTYPE_F32 ? PAGED_F32 : (c->dtype == PHYAI_DTYPE_BF16 ? PAGED_BF16 : PAGED_FP8);
}

void enqueue_norm_rope(const phyai_head_rows* q, const phyai_head_rows* k, const phyai_head_rows* q_out,
                       const phyai_head_rows* k_out, const float* q_gain, const float* k_gain, float eps,
                       float rope_base, const int32_t* past_len, const int32_t* new_len, int batch, int rows,
                       int head_dim, int dtype, int32_t* status, hipStream_t s) {
  const int kind = row_kind(dtype);
  check_sizes(batch, rows, head_dim);
  check_tokens(batch, rows);
  req(q || k, "q and k are both NULL");
  NormRopeArgs a{};
  if (q) {
    a.q = head_rows(q, dtype, "q");
    a.q_out = out_rows(q_out, dtype, "q_out", batch, rows, head_dim);
    req(a.q.n == a.q_out.n, "q_out has another number of heads than q");
  }
  if (k) {
    a.k = head_rows(k, dtype, "k");
    a.k_out = out_rows(k_out, dtype, "k_out", batch, rows, head_dim);
    req(a.k.n == a.k_out.n, "k_out has another number of heads than k");
  }
  req(std::isfinite(eps) && eps >= 0.f, "eps must be 0 or a positive number");
  req(eps > 0.f || (!q_gain && !k_gain), "gains need eps > 0");
  req(aligned16(q_gain) && aligned16(k_gain), "gains must be 16-byte aligned");
  req((q || !q_gain) && (k || !k_gain), "a gain without its rows");
  a.rope = rope_freq(rope_base, head_dim, a.freq);
  a.norm = eps > 0.f;
  words({past_len, new_len, status});
  req(a.norm || a.rope, "eps and rope_base are both 0: nothing to do");
  a.q_gain = q_gain;
  a.k_gain = k_gain;
  a.past_len = past_len;
  a.new_len = new_len;
  a.status = status;
  a.B = batch;
  a.M = rows;
  a.eps = eps;
  norm_rope(a, head_dim, kind, s);
  HIPC(hipGetLastError());
}

void enqueue_append(const phyai_paged_cache* cache, int layer, const phyai_head_rows* k, const phyai_head_rows* v,
                    float rope_base, const int32_t* past_len, const int32_t* new_len, int rows, int dtype,
                    int32_t* status, hipStream_t s) {
  PagedAppendArgs a{};
  a.pool = page_pool(cache, layer);
  const int kind = row_kind(dtype);
  req((kind == PAGED_F32) == (cache->dtype == PHYAI_DTYPE_F32), "an F32 cache takes F32 rows, BF16 and FP8E4M3 caches BF16 rows");
  check_sizes(cache->batch, rows, cache->head_dim);
  check_tokens(cache->batch, rows);
  a.k = head_rows(k, dtype, "k");
  a.v = head_rows(v, dtype, "v");
  req(a.k.n == cache->n_kv_heads && a.v.n == cache->n_kv_heads, "k and v must have the cache's n_kv_heads heads");
  req(past_len, "past_len must not be NULL");
  words({past_len, new_len, status});
  a.rope = rope_freq(rope_base, cache->head_dim, a.freq);
  a.past_len = past_len;
  a.new_len = new_len;
  a.status = status;
  a.B = cache->batch;
  a.M = rows;
  paged_append(a, cache->head_dim, pool_kind(cache), s);
  HIPC(hipGetLastError());
}

namespace {

// What the size and place of the split depend on.
PagedAttnArgs attention_plan(const phyai_paged_cache* cache, int n_q_heads, int rows, int max_kv_len, int window,
                             int64_t& floats) {
  check_sizes(cache->batch, rows, cache->head_dim);
  req(n_q_heads >= 1 && n_q_heads <= kMaxHeads && n_q_heads % cache->n_kv_heads == 0,
      "query heads must be a multiple of n_kv_heads, at most 1024");
  req(max_kv_len >= 1 && (int64_t)max_kv_len <= (int64_t)cache->max_pages * cache->page_size,
      "max_kv_len out of range 1..max_pages * page_size");
  PagedAttnArgs a{};
  a.B = cache->batch;
  a.M = rows;
  a.nkv = cache->n_kv_heads;
  a.G = n_q_heads / cache->n_kv_heads;
  a.max_kv = max_kv_len;
  a.window = window;
  req((int64_t)a.B * n_q_heads * rows <= INT32_MAX / 2, "batch * rows * query heads out of range");
  floats = paged_attention_plan(a, cache->head_dim, pool_kind(cache));
  return a;
}

}  // namespace

int64_t attention_workspace(const phyai_paged_cache* cache, int n_q_heads, int rows, int max_kv_len) {
  (void)page_pool(cache, 0);
  int64_t floats = 0;
  attention_plan(cache, n_q_heads, rows, max_kv_len, 0, floats);
  return floats * 4;
}

void enqueue_attention(const phyai_paged_cache* cache, int layer, const phyai_head_rows* q, const phyai_head_rows* out,
                       const int32_t* kv_len, const int32_t* new_len, int max_kv_len, float scale, int causal,
                       int window, int rows, int dtype, void* workspace, int64_t workspace_bytes, int32_t* status,
                       hipStream_t s) {
  const PagePool pool = page_pool(cache, layer);
  const int kind = row_kind(dtype);
  req((kind == PAGED_F32) == (cache->dtype == PHYAI_DTYPE_F32), "an F32 cache takes F32 rows, BF16 and FP8E4M3 caches BF16 rows");
  check_sizes(cache->batch, rows, cache->head_dim);
  const HeadRows hq = head_rows(q, dtype, "q");
  const HeadRows ho = out_rows(out, dtype, "out", cache->batch, rows, cache->head_dim);
  req(hq.n == ho.n, "out has another number of heads than q");
  req(kv_len, "kv_len must not be NULL");
  words({kv_len, new_len, status});
  req(std::isfinite(scale) && scale > 0.f, "scale must be a positive number");
  req(causal == 0 || causal == 1, "causal must be 0 or 1");
  req(window >= 0 && (window == 0 || causal), "window must be >= 0, and 0 without a causal mask");
  int64_t floats = 0;
  PagedAttnArgs a = attention_plan(cache, hq.n, rows, max_kv_len, window, floats);
  req(floats == 0 || (workspace && aligned16(workspace)), "workspace must be given and 16-byte aligned");
  req(workspace_bytes >= floats * 4, "workspace too small: ask phyai_paged_attention_workspace");
  a.pool = pool;
  a.q = hq;
  a.out = ho;
  a.kv_len = kv_len;
  a.new_len = new_len;
  a.status = status;
  a.causal = causal;
  a.scale = scale;
  a.part = static_cast<float*>(workspace);
  a.ml = reinterpret_cast<float2*>(a.part + floats / (cache->head_dim + 2) * cache->head_dim);
  paged_attention(a, cache->head_dim, pool_kind(cache), s);
  HIPC(hipGetLastError());
}

}  // namespace phyai

extern "C" {

int phyai_qk_norm_rope(const phyai_head_rows* q, const phyai_head_rows* k, const phyai_head_rows* q_out,
                       const phyai_head_rows* k_out, const float* q_gain, const float* k_gain, float eps,
                       float rope_base, const int32_t* past_len, const int32_t* new_len, int32_t batch, int32_t rows,
                       int32_t head_dim, int32_t dtype, int32_t* status, void* stream) {
  return run_guarded([&] {
    enqueue_norm_rope(q, k, q_out, k_out, q_gain, k_gain, eps, rope_base, past_len, new_len, batch, rows, head_dim,
                      dtype, status, static_cast<hipStream_t>(stream));
  });
}

int phyai_paged_append(const phyai_paged_cache* cache, int32_t layer, const phyai_head_rows* k,
                       const phyai_head_rows* v, float rope_base, const int32_t* past_len, const int32_t* new_len,
                       int32_t rows, int32_t dtype, int32_t* status, void* stream) {
  return run_guarded([&] {
    enqueue_append(cache, layer, k, v, rope_base, past_len, new_len, rows, dtype, status,
                   static_cast<hipStream_t>(stream));
  });
}

int phyai_paged_attention(const phyai_paged_cache* cache, int32_t layer, const phyai_head_rows* q,
                          const phyai_head_rows* out, const int32_t* kv_len, const int32_t* new_len,
                          int32_t max_kv_len, float scale, int32_t causal, int32_t window, int32_t rows, int32_t dtype,
                          void* workspace, int64_t workspace_bytes, int32_t* status, void* stream) {
  return run_guarded([&] {
    enqueue_attention(cache, layer, q, out, kv_len, new_len, max_kv_len, scale, causal, window, rows, dtype, workspace,
                      workspace_bytes, status, static_cast<hipStream_t>(stream));
  });
}

int64_t phyai_paged_attention_workspace(const phyai_paged_cache* cache, int32_t n_q_heads, int32_t rows,
                                        int32_t max_kv_len) {
  int64_t bytes = 0;
  const int rc = run_guarded([&] { bytes = attention_workspace(cache, n_q_heads, rows, max_kv_len); });
  return rc == PHYAI_OK ? bytes : rc;
}

int phyai_paged_gather(const phyai_paged_cache* cache, const int32_t* kv_len, void* out, int32_t rows, int32_t* status,
                       void* stream) {
  return run_guarded([&] {
    PagedGatherArgs a{};
    a.pool = page_pool(cache, 0);
    check_sizes(cache->batch, rows, cache->head_dim);
    req(kv_len && out, "kv_len and out must not be NULL");
    req(aligned16(out), "out must be 16-byte aligned");
    words({kv_len, status});
    req((int64_t)cache->n_layers * 2 * cache->batch <= 65535, "n_layers * 2 * batch out of range 1..65535");
    a.kv_len = kv_len;
    a.out = out;
    a.status = status;
    a.layers = cache->n_layers;
    a.B = cache->batch;
    a.rows = rows;
    a.nkv = cache->n_kv_heads;
    a.D = cache->head_dim;
    paged_gather(a, pool_kind(cache), static_cast<hipStream_t>(stream));
    HIPC(hipGetLastError());
  });
}

}  // extern "C"
