// C-ABI layer of the inference calls: argument checks, the rotary plan and the page bookkeeping (host integers), dispatch to the
// kernels.  No device memory is allocated here and nothing synchronises.
#include <cmath>
#include <cstring>

#include "api_checks.h"
#include "paged.h"

using namespace mmsp;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 26;          // rows of a call

mmsp_status check_rotary(const mmsp_rotary* r) {
  if (r == nullptr) return fail(MMSP_ERR_INVALID_ARG, "rotary is NULL");
  if (r->head_dim != 64 && r->head_dim != 128) return fail(MMSP_ERR_UNSUPPORTED, "rotary head_dim=%d: only 64 and 128 have kernels", r->head_dim);
  if (r->n_axes < 1 || r->n_axes > kMaxAxes) return fail(MMSP_ERR_INVALID_ARG, "n_axes=%d is not in [1, %d]", r->n_axes, kMaxAxes);
  for (int i = 0; i < r->head_dim / 2; ++i)
    if (r->axis[i] >= r->n_axes) return fail(MMSP_ERR_INVALID_ARG, "axis[%d]=%d is not below n_axes=%d", i, r->axis[i], r->n_axes);
  return MMSP_OK;
}

mmsp_status check_positions(const mmsp_rotary* r, int64_t n_rows, const int32_t* positions, int64_t pos_stride) {
  if (positions == nullptr) return fail(MMSP_ERR_INVALID_ARG, "positions is NULL");
  if (r->n_axes > 1 && pos_stride < n_rows)
    return fail(MMSP_ERR_INVALID_ARG, "pos_stride=%lld is smaller than the %lld rows", (long long)pos_stride, (long long)n_rows);
  return MMSP_OK;
}

RotaryArgs rotary_args(const mmsp_rotary* r, const int32_t* positions, int64_t pos_stride, bool inverse) {
  RotaryArgs a;
  memcpy(a.turns, r->turns, sizeof(a.turns));
  memcpy(a.axis, r->axis, sizeof(a.axis));
  a.positions = positions; a.pos_stride = pos_stride; a.n_axes = r->n_axes; a.inverse = inverse;
  return a;
}

mmsp_status check_heads(const mmsp_heads* h, int32_t d, const char* which, int i) {
  if (h->data == nullptr || !aligned16(h->data)) return fail(MMSP_ERR_INVALID_ARG, "%s[%d].data must be non-NULL and 16-byte aligned", which, i);
  if (h->n_heads <= 0 || h->n_heads > 65536) return fail(MMSP_ERR_INVALID_ARG, "%s[%d].n_heads=%d is not in [1, 65536]", which, i, h->n_heads);
  if (h->dtype != MMSP_BF16 && h->dtype != MMSP_F32) return fail(MMSP_ERR_INVALID_ARG, "%s[%d].dtype=%d is not MMSP_BF16 or MMSP_F32", which, i, h->dtype);
  if (h->tok_stride < d || h->head_stride < d || h->tok_stride % 8 || h->head_stride % 8)
    return fail(MMSP_ERR_INVALID_ARG, "%s[%d]: strides must be >= head_dim and multiples of 8 elements", which, i);
  return MMSP_OK;
}

mmsp_status check_pool(const mmsp_shape* s, const mmsp_cache* c) {
  if (c == nullptr) return fail(MMSP_ERR_INVALID_ARG, "cache is NULL");
  if (c->n_pages < 0 || (c->n_pages > 0 && (c->k == nullptr || c->v == nullptr)))
    return fail(MMSP_ERR_INVALID_ARG, "n_pages=%d is negative, or k or v is NULL", c->n_pages);
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(MMSP_ERR_INVALID_ARG, "the cache's k and v must be 16-byte aligned");
  if (c->page_size <= 0 || c->page_size % 16 != 0) return fail(MMSP_ERR_INVALID_ARG, "page_size=%d must be a positive multiple of 16", c->page_size);
  const int64_t d = s->head_dim;
  if (c->page_stride < d || c->tok_stride < d || c->head_stride < d || c->page_stride % 8 || c->tok_stride % 8 || c->head_stride % 8)
    return fail(MMSP_ERR_INVALID_ARG, "the cache's strides must be >= head_dim and multiples of 8 elements");
  if (c->tok_stride > (1 << 23)) return fail(MMSP_ERR_INVALID_ARG, "token strides above 2^23 elements are not supported");
  return MMSP_OK;
}

mmsp_status check_cache(const mmsp_shape* s, const mmsp_cache* c) {
  mmsp_status st = check_pool(s, c);
  if (st != MMSP_OK) return st;
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > kMaxExtent)
    return fail(MMSP_ERR_INVALID_ARG, "max_pages=%d x page_size=%d is not in [1, 2^30] tokens", c->max_pages, c->page_size);
  if (c->n_seqs < 0 || c->n_rows < 0 || c->n_rows > kMaxRows || c->n_seqs > kMaxRows)
    return fail(MMSP_ERR_INVALID_ARG, "n_seqs=%d and n_rows=%d must be in [0, 2^26]", c->n_seqs, c->n_rows);
  if (c->most_new < 0) return fail(MMSP_ERR_INVALID_ARG, "most_new=%d is negative", c->most_new);
  if (c->cu_new == nullptr && c->n_rows != c->n_seqs)
    return fail(MMSP_ERR_INVALID_ARG, "without cu_new every sequence has one row: n_rows=%d, n_seqs=%d", c->n_rows, c->n_seqs);
  if (c->n_seqs > 0 && (c->page_table == nullptr || c->lengths == nullptr))
    return fail(MMSP_ERR_INVALID_ARG, "page_table and lengths must be non-NULL");
  if (c->table_stride < c->max_pages) return fail(MMSP_ERR_INVALID_ARG, "table_stride=%lld is smaller than max_pages=%d", (long long)c->table_stride, c->max_pages);
  return MMSP_OK;
}

CacheArgs cache_args(const mmsp_cache* c) {
  CacheArgs a;
  a.k = reinterpret_cast<char*>(c->k); a.v = reinterpret_cast<char*>(c->v);
  a.page_stride = c->page_stride; a.tok_stride = c->tok_stride; a.head_stride = c->head_stride;
  a.table = c->page_table; a.table_stride = c->table_stride; a.lengths = c->lengths; a.cu_new = c->cu_new;
  a.n_pages = c->n_pages; a.page_size = c->page_size; a.max_pages = c->max_pages; a.n_seqs = c->n_seqs; a.n_rows = c->n_rows; a.most_new = c->most_new;
  a.page_div = fast_div(c->page_size);
  return a;
}

CacheAttnArgs attn_args(const mmsp_shape* s, const mmsp_cache* c) {
  CacheAttnArgs a;
  memset(&a, 0, sizeof(a));
  a.cache = cache_args(c);
  a.q_ts = s->q_tok_stride; a.q_hs = s->q_head_stride; a.lse_hs = s->lse_head_stride;
  a.Hq = s->n_q_heads; a.Hkv = s->n_kv_heads; a.group = s->n_q_heads / s->n_kv_heads; a.d = s->head_dim;
  a.group_div = fast_div(a.group);
  a.scale = s->softmax_scale;
  return a;
}

// ---- page bookkeeping ----

int64_t pages_for(const mmsp_pages* p, int64_t tokens) { return (tokens + p->page_size - 1) / p->page_size; }

mmsp_status check_pages(const mmsp_pages* p) {
  if (p == nullptr || p->refs == nullptr || p->free_pages == nullptr) return fail(MMSP_ERR_INVALID_ARG, "pages, refs or free_pages is NULL");
  if (p->n_pages <= 0 || p->page_size <= 0) return fail(MMSP_ERR_INVALID_ARG, "n_pages=%d and page_size=%d must be positive", p->n_pages, p->page_size);
  if (p->n_free < 0 || p->n_free > p->n_pages) return fail(MMSP_ERR_INVALID_ARG, "n_free=%d is not in [0, %d]", p->n_free, p->n_pages);
  return MMSP_OK;
}

// The first `tokens` tokens of a row: the row has entries for them, and every page of this pool among them is in use.
mmsp_status check_row(const mmsp_pages* p, const int32_t* row, int32_t max_pages, int64_t tokens) {
  if (row == nullptr) return fail(MMSP_ERR_INVALID_ARG, "row is NULL");
  if (max_pages < 0 || tokens < 0 || tokens > kMaxExtent || pages_for(p, tokens) > max_pages)
    return fail(MMSP_ERR_INVALID_ARG, "%lld tokens do not fit a row of %d pages of %d", (long long)tokens, max_pages, p->page_size);
  for (int64_t i = 0; i < pages_for(p, tokens); ++i)
    if (row[i] >= 0 && (row[i] >= p->n_pages || p->refs[row[i]] <= 0))
      return fail(MMSP_ERR_INVALID_ARG, "entry %lld of the row is page %d, which is not in use", (long long)i, row[i]);
  return MMSP_OK;
}

}  // namespace

extern "C" {

mmsp_status mmsp_rotary_plan(int32_t head_dim, double theta, int32_t n_axes, const int32_t* sections, mmsp_rotary* rotary) {
  if (sections == nullptr || rotary == nullptr) return fail(MMSP_ERR_INVALID_ARG, "sections or rotary is NULL");
  if (head_dim != 64 && head_dim != 128) return fail(MMSP_ERR_UNSUPPORTED, "rotary head_dim=%d: only 64 and 128 have kernels", head_dim);
  if (!(theta >= 1.0) || !std::isfinite(theta)) return fail(MMSP_ERR_INVALID_ARG, "theta must be finite and >= 1");
  if (n_axes < 1 || n_axes > kMaxAxes) return fail(MMSP_ERR_INVALID_ARG, "n_axes=%d is not in [1, %d]", n_axes, kMaxAxes);
  int64_t sum = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (sections[a] < 0) return fail(MMSP_ERR_INVALID_ARG, "sections[%d]=%d is negative", a, sections[a]);
    sum += sections[a];
  }
  if (sum != head_dim / 2) return fail(MMSP_ERR_INVALID_ARG, "the sections sum to %lld, not to head_dim / 2 = %d", (long long)sum, head_dim / 2);
  memset(rotary, 0, sizeof(*rotary));
  rotary->head_dim = head_dim;
  rotary->n_axes = n_axes;
  constexpr double kTurn = 0.15915494309189533577;      // 1 / (2 pi)
  for (int i = 0, a = 0, left = sections[0]; i < head_dim / 2; ++i, --left) {
    while (left == 0) left = sections[++a];
    rotary->axis[i] = (uint8_t)a;
    rotary->turns[i] = (uint64_t)std::ldexp(std::pow(theta, -2.0 * i / head_dim) * kTurn, 64);   // below 2^62
  }
  return MMSP_OK;
}

mmsp_status mmsp_rotary_apply(const mmsp_rotary* rotary, int64_t n_rows, const int32_t* positions, int64_t pos_stride,
                              int32_t n_tensors, const mmsp_heads* x, const mmsp_heads* y, int inverse, void* hip_stream) {
  mmsp_status st = check_rotary(rotary);
  if (st != MMSP_OK) return st;
  if (n_rows < 0 || n_rows > kMaxRows) return fail(MMSP_ERR_INVALID_ARG, "n_rows=%lld is not in [0, 2^26]", (long long)n_rows);
  if (n_tensors < 1 || n_tensors > 2) return fail(MMSP_ERR_INVALID_ARG, "n_tensors=%d is not 1 or 2", n_tensors);
  if (x == nullptr || y == nullptr) return fail(MMSP_ERR_INVALID_ARG, "x or y is NULL");
  st = check_positions(rotary, n_rows, positions, pos_stride);
  if (st != MMSP_OK) return st;
  HeadsArgs t[2] = {};
  for (int i = 0; i < n_tensors; ++i) {
    st = check_heads(&x[i], rotary->head_dim, "x", i);
    if (st == MMSP_OK) st = check_heads(&y[i], rotary->head_dim, "y", i);
    if (st != MMSP_OK) return st;
    if (x[i].n_heads != y[i].n_heads) return fail(MMSP_ERR_INVALID_ARG, "x[%d] has %d heads, y[%d] %d", i, x[i].n_heads, i, y[i].n_heads);
    if (x[i].dtype != x[0].dtype || y[i].dtype != y[0].dtype) return fail(MMSP_ERR_INVALID_ARG, "the tensors of a call must have the same types");
    if (x[i].data == y[i].data && (x[i].dtype != y[i].dtype || x[i].tok_stride != y[i].tok_stride || x[i].head_stride != y[i].head_stride))
      return fail(MMSP_ERR_INVALID_ARG, "in place, x[%d] and y[%d] must have the same strides and dtype", i, i);
    t[i] = {reinterpret_cast<const char*>(x[i].data), reinterpret_cast<char*>(y[i].data), x[i].tok_stride, x[i].head_stride, y[i].tok_stride, y[i].head_stride,
            x[i].n_heads};
  }
  if (x[0].dtype == MMSP_BF16 && y[0].dtype == MMSP_F32) return fail(MMSP_ERR_UNSUPPORTED, "bf16 to f32 has no kernel");
  return device_result(launch_rotary(rotary_args(rotary, positions, pos_stride, inverse != 0), t, n_tensors, (int)n_rows, rotary->head_dim, x[0].dtype, y[0].dtype,
                                     reinterpret_cast<hipStream_t>(hip_stream)),
                       "rotary_apply");
}

mmsp_status mmsp_cache_append(const mmsp_shape* shape, const mmsp_cache* cache, const mmsp_rotary* rotary, const int32_t* positions, int64_t pos_stride,
                              const void* q, const void* k, const void* v, void* q_out, void* hip_stream) {
  mmsp_status st = check_shape(shape);
  if (st == MMSP_OK) st = check_cache(shape, cache);
  if (st != MMSP_OK) return st;
  if (rotary != nullptr) {
    st = check_rotary(rotary);
    if (st == MMSP_OK) st = check_positions(rotary, cache->n_rows, positions, pos_stride);
    if (st != MMSP_OK) return st;
    if (rotary->head_dim != shape->head_dim) return fail(MMSP_ERR_INVALID_ARG, "rotary has head_dim %d, the shape %d", rotary->head_dim, shape->head_dim);
  }
  if (k == nullptr || v == nullptr || (q_out != nullptr && q == nullptr)) return fail(MMSP_ERR_INVALID_ARG, "k, v, and q where q_out is given, must be non-NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)) return fail(MMSP_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
  AppendArgs a;
  a.cache = cache_args(cache);
  a.q = reinterpret_cast<const char*>(q); a.k = reinterpret_cast<const char*>(k); a.v = reinterpret_cast<const char*>(v); a.q_out = reinterpret_cast<char*>(q_out);
  a.q_ts = shape->q_tok_stride; a.q_hs = shape->q_head_stride; a.kv_ts = shape->kv_tok_stride; a.kv_hs = shape->kv_head_stride;
  a.out_ts = q_out == q ? a.q_ts : (int64_t)shape->n_q_heads * shape->head_dim;
  a.out_hs = q_out == q ? a.q_hs : shape->head_dim;
  a.Hq = q_out != nullptr ? shape->n_q_heads : 0; a.Hkv = shape->n_kv_heads;
  RotaryArgs r;
  if (rotary != nullptr) r = rotary_args(rotary, positions, pos_stride, false);
  return device_result(launch_append(a, rotary != nullptr ? &r : nullptr, shape->head_dim, shape->io_dtype, reinterpret_cast<hipStream_t>(hip_stream)), "cache_append");
}

size_t mmsp_cache_workspace_bytes(const mmsp_shape* shape, const mmsp_cache* cache) {
  if (check_shape(shape) != MMSP_OK || check_cache(shape, cache) != MMSP_OK || cache->n_seqs == 0) return 0;
  return (size_t)cache_attn_workspace_bytes(attn_args(shape, cache), shape->io_dtype);
}

mmsp_status mmsp_cache_attn(const mmsp_shape* shape, const mmsp_cache* cache, const void* q, void* o_final, float* o, float* lse,
                            void* workspace, size_t workspace_bytes, void* hip_stream) {
  mmsp_status st = check_shape(shape);
  if (st == MMSP_OK) st = check_cache(shape, cache);
  if (st != MMSP_OK) return st;
  if (q == nullptr) return fail(MMSP_ERR_INVALID_ARG, "q is NULL");
  if (o_final == nullptr && o == nullptr && lse == nullptr) return fail(MMSP_ERR_INVALID_ARG, "nothing to do: o_final, o and lse are all NULL");
  if (!aligned16(q) || !aligned16(o_final) || !aligned16(o)) return fail(MMSP_ERR_INVALID_ARG, "q, o_final and o must be 16-byte aligned");
  if (lse != nullptr && shape->lse_head_stride < cache->n_rows)
    return fail(MMSP_ERR_INVALID_ARG, "lse_head_stride=%lld is smaller than the %d rows", (long long)shape->lse_head_stride, cache->n_rows);
  if ((int64_t)cache->n_rows * shape->n_q_heads > (1 << 23))
    return fail(MMSP_ERR_UNSUPPORTED, "%d rows x %d heads: more than 2^23 are not supported", cache->n_rows, shape->n_q_heads);
  if (cache->n_rows == 0 || cache->n_seqs == 0) return MMSP_OK;
  CacheAttnArgs a = attn_args(shape, cache);
  if (cache_attn_tiles(a, shape->io_dtype) > 0x1p30)
    return fail(MMSP_ERR_UNSUPPORTED, "%d sequences of up to %d pages of %d tokens and %d KV heads are too much for a call", cache->n_seqs, cache->max_pages,
                cache->page_size, shape->n_kv_heads);
  const size_t need = (size_t)cache_attn_workspace_bytes(a, shape->io_dtype);
  if (workspace == nullptr || workspace_bytes < need)
    return fail(MMSP_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes given, %zu needed (mmsp_cache_workspace_bytes)", workspace_bytes, need);
  if (!aligned16(workspace)) return fail(MMSP_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  a.q = q; a.o_final = o_final; a.o = o; a.lse = lse;
  a.ws = reinterpret_cast<char*>(workspace);
  return device_result(launch_cache_attn(a, shape->io_dtype, reinterpret_cast<hipStream_t>(hip_stream)), "cache_attn");
}

mmsp_status mmsp_cache_copy_pages(const mmsp_shape* shape, const mmsp_cache* cache, int32_t n_layers, int64_t layer_stride,
                                  const mmsp_page_copy* copies, int32_t n_copies, void* hip_stream) {
  mmsp_status st = check_shape(shape);
  if (st == MMSP_OK) st = check_pool(shape, cache);
  if (st != MMSP_OK) return st;
  if (n_layers < 0 || n_copies < 0) return fail(MMSP_ERR_INVALID_ARG, "n_layers=%d or n_copies=%d is negative", n_layers, n_copies);
  if (n_layers > 1 && layer_stride % 8 != 0) return fail(MMSP_ERR_INVALID_ARG, "layer_stride=%lld must be a multiple of 8 elements", (long long)layer_stride);
  if (n_copies > 0 && copies == nullptr) return fail(MMSP_ERR_INVALID_ARG, "copies is NULL");
  const int elt = shape->io_dtype == MMSP_BF16 ? 2 : 4;
  const double pieces = (double)cache->page_size * shape->n_kv_heads * shape->head_dim * elt / 16;
  if (pieces > (1 << 28) || pieces * 2 * n_layers >= 0x1p32)   // a grid has fewer than 2^32 threads
    return fail(MMSP_ERR_UNSUPPORTED, "pages of %d tokens x %d heads in %d layers are too large for a launch", cache->page_size, shape->n_kv_heads, n_layers);
  return device_result(launch_copy_pages(cache_args(cache), n_layers, layer_stride, shape->n_kv_heads, shape->head_dim, elt, reinterpret_cast<const int32_t*>(copies),
                                         n_copies, reinterpret_cast<hipStream_t>(hip_stream)),
                       "cache_copy_pages");
}

mmsp_status mmsp_pages_init(mmsp_pages* p) {
  if (p == nullptr) return fail(MMSP_ERR_INVALID_ARG, "pages is NULL");
  p->n_free = 0;
  mmsp_status st = check_pages(p);
  if (st != MMSP_OK) return st;
  for (int32_t i = 0; i < p->n_pages; ++i) {
    p->refs[i] = 0;
    p->free_pages[i] = p->n_pages - 1 - i;
  }
  p->n_free = p->n_pages;
  return MMSP_OK;
}

mmsp_status mmsp_pages_grow(mmsp_pages* p, int32_t* row, int32_t max_pages, int64_t n_old, int64_t n_new, mmsp_page_copy* copy, int32_t* n_copies) {
  mmsp_status st = check_pages(p);
  if (st == MMSP_OK) st = check_row(p, row, max_pages, n_old);
  if (st != MMSP_OK) return st;
  if (copy == nullptr || n_copies == nullptr) return fail(MMSP_ERR_INVALID_ARG, "copy or n_copies is NULL");
  if (n_new < n_old || n_new > kMaxExtent || pages_for(p, n_new) > max_pages)
    return fail(MMSP_ERR_INVALID_ARG, "%lld tokens are fewer than %lld or do not fit a row of %d pages of %d", (long long)n_new, (long long)n_old, max_pages, p->page_size);
  const int64_t have = pages_for(p, n_old), want = pages_for(p, n_new);
  const bool partly = n_old % p->page_size != 0 && n_new > n_old;
  const int32_t last = partly ? row[have - 1] : -1;
  const bool own_copy = last >= 0 && p->refs[last] > 1;
  if (want - have + own_copy > p->n_free)
    return fail(MMSP_ERR_NO_PAGES, "%lld pages needed, %d of %d are free", (long long)(want - have + own_copy), p->n_free, p->n_pages);
  *n_copies = 0;
  auto take = [&] {
    const int32_t page = p->free_pages[--p->n_free];
    p->refs[page] = 1;
    return page;
  };
  if (own_copy) {
    row[have - 1] = take();
    --p->refs[last];
    *copy = {last, row[have - 1], (int32_t)(n_old % p->page_size)};
    *n_copies = 1;
  }
  for (int64_t i = have; i < want; ++i) row[i] = take();
  return MMSP_OK;
}

mmsp_status mmsp_pages_fork(mmsp_pages* p, const int32_t* row, int32_t max_pages, int64_t n_tokens, int32_t* new_row) {
  mmsp_status st = check_pages(p);
  if (st == MMSP_OK) st = check_row(p, row, max_pages, n_tokens);
  if (st != MMSP_OK) return st;
  if (new_row == nullptr || new_row == row) return fail(MMSP_ERR_INVALID_ARG, "new_row is NULL or row itself");
  const int64_t have = pages_for(p, n_tokens);
  for (int64_t i = 0; i < have; ++i) {
    new_row[i] = row[i];
    if (row[i] >= 0) ++p->refs[row[i]];
  }
  for (int64_t i = have; i < max_pages; ++i) new_row[i] = -1;
  return MMSP_OK;
}

mmsp_status mmsp_pages_free(mmsp_pages* p, int32_t* row, int32_t max_pages, int64_t n_tokens) {
  mmsp_status st = check_pages(p);
  if (st == MMSP_OK) st = check_row(p, row, max_pages, n_tokens);
  if (st != MMSP_OK) return st;
  const int64_t have = pages_for(p, n_tokens);
  const int32_t n_free = p->n_free;
  for (int64_t i = have - 1; i >= 0; --i) {             // the first page is given out next
    if (row[i] < 0) continue;
    if (--p->refs[row[i]] == 0) p->free_pages[p->n_free++] = row[i];
    if (p->refs[row[i]] < 0) {                          // the row names a page more often than it is held: nothing is let go of
      const int32_t page = row[i];
      for (int64_t j = i; j < have; ++j)
        if (row[j] >= 0) ++p->refs[row[j]];
      p->n_free = n_free;
      return fail(MMSP_ERR_INVALID_ARG, "page %d is in the row more often than it is held", page);
    }
  }
  for (int64_t i = 0; i < have; ++i) row[i] = -1;
  return MMSP_OK;
}

mmsp_status mmsp_pages_compact(mmsp_pages* p, int32_t* rows, int64_t row_stride, int32_t max_pages, int32_t n_seqs, const int64_t* n_tokens,
                               mmsp_page_copy* copies, int32_t* n_copies, int32_t* n_used) {
  mmsp_status st = check_pages(p);
  if (st != MMSP_OK) return st;
  if (n_seqs < 0 || (n_seqs > 0 && (rows == nullptr || n_tokens == nullptr)) || copies == nullptr || n_copies == nullptr || n_used == nullptr)
    return fail(MMSP_ERR_INVALID_ARG, "n_seqs=%d is negative, or an argument is NULL", n_seqs);
  if (row_stride < max_pages) return fail(MMSP_ERR_INVALID_ARG, "row_stride=%lld is smaller than max_pages=%d", (long long)row_stride, max_pages);
  for (int32_t s = 0; s < n_seqs; ++s) {
    st = check_row(p, rows + s * row_stride, max_pages, n_tokens[s]);
    if (st != MMSP_OK) return st;
  }
  auto each_entry = [&](auto f) {
    for (int32_t s = 0; s < n_seqs; ++s)
      for (int64_t i = 0, have = pages_for(p, n_tokens[s]); i < have; ++i)
        if (rows[s * row_stride + i] >= 0) f(rows[s * row_stride + i]);
  };
  // do the rows account for every reference, and no more?
  each_entry([&](int32_t page) { --p->refs[page]; });
  bool agree = true;
  for (int32_t i = 0; i < p->n_pages; ++i) agree = agree && p->refs[i] == 0;
  each_entry([&](int32_t page) { ++p->refs[page]; });
  if (!agree) return fail(MMSP_ERR_INVALID_ARG, "the rows do not name every page in use as often as it is held");
  int32_t used = 0;
  for (int32_t i = 0; i < p->n_pages; ++i) used += p->refs[i] > 0;
  // the k-th page in use behind the border moves into the k-th hole before it; the new ids are kept where the list of free pages was
  int32_t* const now = p->free_pages;
  int32_t hole = 0, n = 0;
  for (int32_t i = 0; i < p->n_pages; ++i) now[i] = i;
  for (int32_t i = used; i < p->n_pages; ++i) {
    if (p->refs[i] == 0) continue;
    while (p->refs[hole] > 0) ++hole;
    now[i] = hole;
    copies[n++] = {i, hole, p->page_size};
    ++hole;
  }
  each_entry([&](int32_t& page) { page = now[page]; });
  for (int32_t i = 0; i < n; ++i) {
    p->refs[copies[i].dst] = p->refs[copies[i].src];
    p->refs[copies[i].src] = 0;
  }
  p->n_free = p->n_pages - used;
  for (int32_t i = 0; i < p->n_free; ++i) p->free_pages[i] = p->n_pages - 1 - i;
  *n_copies = n;
  *n_used = used;
  return MMSP_OK;
}

}  // extern "C"
