// C ABI of the operators for drafted trees, page selection and eviction over a
// paged key/value cache: every argument is checked here, before anything is
// launched.
#include "span.h"

#include "paged_check.h"

using namespace dex;

namespace {

// What the attention calls share.
const char *attention_fault(int dtype, int head_dim, int n_heads, int n_kv_heads, int n, int draft, float scale,
                            int n_pages, int page_size, int n_seqs, int max_pages) {
  if (const char *why = cache_fault(dtype, head_dim, n_pages, n_kv_heads, page_size)) return why;
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return why;
  if (head_dim != 32 && head_dim != 64 && head_dim != 128) return "head_dim is not 32, 64 or 128";
  if (n_heads < n_kv_heads || n_heads % n_kv_heads || n_heads / n_kv_heads > 64)
    return "n_heads is not a multiple of n_kv_heads, up to 64 times it";
  if (n_heads > 8192) return "n_heads is over 8192";
  if (n < 0 || n > (1 << 20)) return "the number of rows or trees is not 0 to 2^20";
  if ((int64_t)n * draft * n_heads > (1 << 30)) return "too many rows for one call";
  if (!std::isfinite(scale)) return "scale is not finite";
  return nullptr;
}
const char *attention_arrays(int dtype, const void *q, const void *k, const void *v, const void *table, const void *len,
                             const void *out, const void *seq, const void *lse) {
  if (!q || !k || !v || !table || !len || !out) return "queries, pages, table, lengths or out are NULL";
  if (!aligned(k, 16) || !aligned(v, 16)) return "the pages are not 16-byte aligned";
  if (!words(seq, len, table, lse) || !aligned(q, elem(dtype)) || !aligned(out, elem(dtype))) return kType;
  return nullptr;
}

SpanArgs span_args(int head_dim, int n_heads, int n_kv_heads, int n, int draft, const int32_t *seq, const int32_t *len,
                   int max_len, float scale, const void *q, int64_t q_row, int64_t q_head, const void *k_pages,
                   const void *v_pages, int n_pages, int page_size, const int32_t *table, int n_seqs, int max_pages,
                   void *out, int64_t out_row, int64_t out_head, float *lse, void *work) {
  SpanArgs a{};
  a.q = q; a.q_row = q_row; a.q_head = q_head; a.k = k_pages; a.v = v_pages;
  a.map = PageMap{table, n_seqs, max_pages, n_pages, n_kv_heads, page_shift(page_size)};
  a.seq = seq; a.len = len; a.n = n; a.draft = draft; a.n_heads = n_heads; a.head_dim = head_dim;
  a.max_len = a.most = max_len; a.scale = scale;
  a.out = out; a.out_row = out_row; a.out_head = out_head; a.lse = lse; a.work = work;
  return a;
}

int words_of(int draft) { return (draft + 63) / 64; }
bool known_sizes(int dtype, int n, int n_heads, int n_kv_heads, int head_dim) {
  return known(dtype) && n >= 0 && n <= (1 << 20) && n_heads >= 1 && n_heads <= 8192 && n_kv_heads >= 1 &&
         n_kv_heads <= n_heads && (head_dim == 32 || head_dim == 64 || head_dim == 128);
}
const char kWork[] = "the work memory is NULL or not 16-byte aligned";
const char kDraft[] = "draft is not 1 to 256";
const char kTrees[] = "n_trees is not 0 to 2^20";
const char kThreads[] = "a launch would have 2^32 threads or more: too many rows, trees or sequences for one call";

// The limits of weigh and select, keys and pages of all rows and kv heads (max_len at
// most 2^30).
bool too_many_keys(int n_rows, int n_kv_heads, int max_len) {
  return (int64_t)n_rows * n_kv_heads * (max_len / 256 + 1) > (1ll << 30);
}
bool too_many_pages(int n_rows, int n_kv_heads, int max_len, int page_size) {
  return (int64_t)n_rows * n_kv_heads * (max_len / page_size + 128) > (1ll << 33);
}

}  // namespace

extern "C" {

dex_status dex_tree_mask(const int32_t *parent, int32_t n_trees, int32_t draft, uint64_t *mask, int32_t *depth,
                         void *stream) {
  static const char fn[] = "dex_tree_mask";
  REFUSE_IF(n_trees < 0 || n_trees > (1 << 20), kTrees);
  REFUSE_IF(draft < 1 || draft > kMaxDraft, kDraft);
  if (n_trees == 0) return DEX_OK;
  REFUSE_IF(!parent || !mask, "an array is NULL");
  REFUSE_IF(!words(parent, depth) || !aligned(mask, 8), kType);
  const TreeMaskArgs a{parent, n_trees, draft, mask, words_of(draft), depth};
  return launched(fn, launch_tree_mask(a, (hipStream_t)stream));
}

dex_status dex_tree_accept(const int32_t *parent, const int32_t *token, const int32_t *target, const int32_t *n_draft,
                           const int32_t *root, int32_t n_trees, int32_t draft, int32_t *path, int32_t *count,
                           int32_t *next, void *stream) {
  static const char fn[] = "dex_tree_accept";
  REFUSE_IF(n_trees < 0 || n_trees > (1 << 20), kTrees);
  REFUSE_IF(draft < 1 || draft > kMaxDraft, kDraft);
  if (n_trees == 0) return DEX_OK;
  REFUSE_IF(!parent || !token || !target || !path || !count || !next, "an array is NULL");
  REFUSE_IF(!words(parent, token, target, n_draft, root, path, count, next), kType);
  const TreeAcceptArgs a{parent, token, target, n_draft, root, n_trees, draft, path, count, next};
  return launched(fn, launch_tree_accept(a, (hipStream_t)stream));
}

int64_t dex_pages_tree_attention_work(int32_t dtype, int32_t n_trees, int32_t draft, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t head_dim, int32_t max_len) {
  if (!known_sizes(dtype, n_trees, n_heads, n_kv_heads, head_dim) || draft < 1 || draft > kMaxDraft || max_len < 0) return 0;
  return (int64_t)span_work(dtype, n_trees, draft, n_heads, n_kv_heads, head_dim, max_len, true, false);
}

dex_status dex_pages_tree_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_trees,
                                    int32_t draft, const int32_t *tree_seq, const int32_t *tree_len,
                                    const int32_t *tree_draft, int32_t max_len, float scale, const void *q, int64_t q_row,
                                    int64_t q_head, const uint64_t *mask, const void *k_pages, const void *v_pages,
                                    int32_t n_pages, int32_t page_size, const int32_t *table, int32_t n_seqs,
                                    int32_t max_pages, void *out, int64_t out_row, int64_t out_head, float *lse,
                                    void *work, void *stream) {
  static const char fn[] = "dex_pages_tree_attention";
  REFUSE_IF(draft < 1 || draft > kMaxDraft, kDraft);
  if (const char *why = attention_fault(dtype, head_dim, n_heads, n_kv_heads, n_trees, draft, scale, n_pages, page_size,
                                        n_seqs, max_pages))
    return refuse(fn, why);
  REFUSE_IF(max_len < 0 || max_len > (1 << 30), "max_len is not 0 to 2^30");
  if (n_trees == 0) return DEX_OK;
  if (const char *why = attention_arrays(dtype, q, k_pages, v_pages, table, tree_len, out, tree_seq, lse))
    return refuse(fn, why);
  REFUSE_IF(!mask, "mask is NULL");
  REFUSE_IF(!aligned(mask, 8) || !words(tree_draft), kType);
  REFUSE_IF(overlaps((int64_t)n_trees * draft, out_row, n_heads, out_head, head_dim), kOverlap);
  SpanArgs a = span_args(head_dim, n_heads, n_kv_heads, n_trees, draft, tree_seq, tree_len, max_len, scale, q, q_row, q_head,
                         k_pages, v_pages, n_pages, page_size, table, n_seqs, max_pages, out, out_row, out_head, lse, work);
  a.mask = mask; a.words = words_of(draft); a.n_draft = tree_draft;
  REFUSE_IF(!span_fits(dtype, a), kThreads);
  REFUSE_IF(span_work(dtype, n_trees, draft, n_heads, n_kv_heads, head_dim, max_len, true, false) > 0 &&
                (!work || !aligned(work, 16)), kWork);
  return launched(fn, launch_span(dtype, a, (hipStream_t)stream));
}

int64_t dex_pages_sparse_attention_work(int32_t dtype, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads,
                                        int32_t head_dim, int32_t n_columns, int32_t page_size) {
  if (!known_sizes(dtype, n_rows, n_heads, n_kv_heads, head_dim) || n_columns < 1 || page_shift(page_size) < 0 ||
      (int64_t)n_columns * page_size > (1 << 30))
    return 0;
  return (int64_t)span_work(dtype, n_rows, 1, n_heads, n_kv_heads, head_dim, n_columns * page_size, false, false);
}

dex_status dex_pages_sparse_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t n_rows, const int32_t *row_seq, const int32_t *row_len, float scale,
                                      const void *q, int64_t q_row, int64_t q_head, const int32_t *columns,
                                      int32_t n_columns, const void *k_pages, const void *v_pages, int32_t n_pages,
                                      int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages,
                                      void *out, int64_t out_row, int64_t out_head, float *lse, void *work,
                                      void *stream) {
  static const char fn[] = "dex_pages_sparse_attention";
  if (const char *why = attention_fault(dtype, head_dim, n_heads, n_kv_heads, n_rows, 1, scale, n_pages, page_size, n_seqs,
                                        max_pages))
    return refuse(fn, why);
  REFUSE_IF(n_columns < 1 || (int64_t)n_columns * page_size > (1 << 30), "n_columns is below 1, or over 2^30 / page_size");
  if (n_rows == 0) return DEX_OK;
  if (const char *why = attention_arrays(dtype, q, k_pages, v_pages, table, row_len, out, row_seq, lse)) return refuse(fn, why);
  REFUSE_IF(!columns, "columns is NULL");
  REFUSE_IF(!words(columns), kType);
  REFUSE_IF(overlaps(n_rows, out_row, n_heads, out_head, head_dim), kOverlap);
  SpanArgs a = span_args(head_dim, n_heads, n_kv_heads, n_rows, 1, row_seq, row_len, 1 << 30, scale, q, q_row, q_head, k_pages,
                         v_pages, n_pages, page_size, table, n_seqs, max_pages, out, out_row, out_head, lse, work);
  a.columns = columns; a.n_cols = n_columns; a.most = n_columns * page_size;
  REFUSE_IF(!span_fits(dtype, a), kThreads);
  REFUSE_IF(span_work(dtype, n_rows, 1, n_heads, n_kv_heads, head_dim, a.most, false, false) > 0 &&
                (!work || !aligned(work, 16)), kWork);
  return launched(fn, launch_span(dtype, a, (hipStream_t)stream));
}

int64_t dex_pages_weigh_work(int32_t dtype, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                             int32_t max_len) {
  if (!known_sizes(dtype, n_rows, n_heads, n_kv_heads, head_dim) || max_len < 0 || max_len > (1 << 30) ||
      too_many_keys(n_rows, n_kv_heads, max_len) || (int64_t)n_rows * n_heads > (1 << 30))
    return 0;
  return (int64_t)span_work(dtype, n_rows, 1, n_heads, n_kv_heads, head_dim, max_len, false, true);
}

dex_status dex_pages_weigh(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_rows,
                           const int32_t *row_seq, const int32_t *row_len, int32_t max_len, float scale, const void *q,
                           int64_t q_row, int64_t q_head, const float *weight, int64_t weight_ld, float *weight_out,
                           int64_t weight_out_ld, const void *k_pages, const void *v_pages, int32_t n_pages,
                           int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages, void *out,
                           int64_t out_row, int64_t out_head, float *lse, void *work, void *stream) {
  static const char fn[] = "dex_pages_weigh";
  if (const char *why = attention_fault(dtype, head_dim, n_heads, n_kv_heads, n_rows, 1, scale, n_pages, page_size, n_seqs,
                                        max_pages))
    return refuse(fn, why);
  REFUSE_IF(max_len < 0 || max_len > (1 << 30), "max_len is not 0 to 2^30");
  REFUSE_IF(too_many_keys(n_rows, n_kv_heads, max_len), "too many keys for one call");
  if (n_rows == 0) return DEX_OK;
  if (const char *why = attention_arrays(dtype, q, k_pages, v_pages, table, row_len, out, row_seq, lse)) return refuse(fn, why);
  REFUSE_IF(!weight || !weight_out, "weight or weight_out is NULL");
  REFUSE_IF(!words(weight, weight_out), kType);
  REFUSE_IF(weight_ld < max_len || weight_out_ld < max_len, "a row of the weights is shorter than max_len");
  REFUSE_IF(weight == weight_out && weight_ld != weight_out_ld, "weight_out is weight with another stride");
  REFUSE_IF(overlaps(n_rows, out_row, n_heads, out_head, head_dim), kOverlap);
  SpanArgs a = span_args(head_dim, n_heads, n_kv_heads, n_rows, 1, row_seq, row_len, max_len, scale, q, q_row, q_head,
                         k_pages, v_pages, n_pages, page_size, table, n_seqs, max_pages, out, out_row, out_head, lse, work);
  a.weight = weight; a.weight_ld = weight_ld; a.weight_out = weight_out; a.weight_out_ld = weight_out_ld;
  REFUSE_IF(!span_fits(dtype, a), kThreads);
  REFUSE_IF(!work || !aligned(work, 16), kWork);
  return launched(fn, launch_span(dtype, a, (hipStream_t)stream));
}

dex_status dex_pages_keep(int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_pages, int32_t n_kv_heads,
                          int32_t page_size, void *k_pool, void *v_pool, const int32_t *table, int32_t n_seqs,
                          int32_t max_pages, const int32_t *to_table, int32_t to_pages, const int32_t *first,
                          const int32_t *index, int64_t index_layer, int64_t index_seq, int64_t index_head,
                          int32_t capacity, const int32_t *count, void *stream) {
  static const char fn[] = "dex_pages_keep";
  if (const char *why = cache_fault(dtype, head_dim, n_pages, n_kv_heads, page_size)) return refuse(fn, why);
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return refuse(fn, why);
  REFUSE_IF(head_dim * elem(dtype) % 16, "a head's row is not a multiple of 16 bytes");
  REFUSE_IF(n_layers < 1 || (int64_t)n_layers * n_kv_heads > (1 << 20), "n_layers is not 1 to 2^20 / n_kv_heads");
  REFUSE_IF((int64_t)n_layers * n_kv_heads * n_seqs * (head_dim * elem(dtype) / 16) > (1 << 30), "too many rows for one call");
  REFUSE_IF(to_table && (to_pages < 1 || (int64_t)to_pages * page_size > (1 << 30)),
            "to_pages is below 1, or ends past position 2^30");
  REFUSE_IF(capacity < 0 || capacity > (1 << 30), "capacity is not 0 to 2^30");
  REFUSE_IF(index_layer < 0 || index_seq < 0 || index_head < 0, "a stride of the index is below 0");
  if (capacity == 0) return DEX_OK;
  REFUSE_IF(!k_pool || !v_pool || !table || !index || !count, "pools, table, index or count are NULL");
  REFUSE_IF(!aligned(k_pool, 16) || !aligned(v_pool, 16), "the pools are not 16-byte aligned");
  REFUSE_IF(!words(table, to_table, first, index, count), kType);
  KeepArgs a{};
  a.k = k_pool; a.v = v_pool; a.n_layers = n_layers; a.row_bytes = (int)(head_dim * elem(dtype));
  a.map = PageMap{table, n_seqs, max_pages, n_pages, n_kv_heads, page_shift(page_size)};
  a.to = to_table; a.to_pages = to_pages; a.first = first; a.index = index; a.index_layer = index_layer;
  a.index_seq = index_seq; a.index_head = index_head; a.capacity = capacity; a.count = count;
  REFUSE_IF(!keep_fits(a), kThreads);
  return launched(fn, launch_keep(a, (hipStream_t)stream));
}

dex_status dex_pages_trim(const int32_t *table, const int32_t *ref, const int32_t *length, int32_t n_seqs,
                          int32_t max_pages, int32_t n_pages, int32_t page_size, int32_t *table_out, int32_t *ref_out,
                          void *stream) {
  static const char fn[] = "dex_pages_trim";
  REFUSE_IF(!table || !ref || !length || !table_out || !ref_out, "an array is NULL");
  REFUSE_IF(n_pages < 1 || n_pages > (1 << 30), "n_pages is not 1 to 2^30");
  REFUSE_IF(page_shift(page_size) < 0, "page_size is not a power of two up to 1024");
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return refuse(fn, why);
  REFUSE_IF(!words(table, ref, length, table_out, ref_out), kType);
  const TrimArgs a{table, ref, length, table_out, ref_out, n_seqs, max_pages, n_pages, page_shift(page_size)};
  return launched(fn, launch_trim(a, (hipStream_t)stream));
}

dex_status dex_pages_bounds(int32_t dtype, int32_t head_dim, const void *k_pages, int32_t n_pages, int32_t n_kv_heads,
                            int32_t page_size, const int32_t *table, int32_t n_seqs, int32_t max_pages,
                            const int32_t *length, int32_t n_new, void *bounds, void *stream) {
  static const char fn[] = "dex_pages_bounds";
  if (const char *why = cache_fault(dtype, head_dim, n_pages, n_kv_heads, page_size)) return refuse(fn, why);
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return refuse(fn, why);
  REFUSE_IF(head_dim != 32 && head_dim != 64 && head_dim != 128, "head_dim is not 32, 64 or 128");
  REFUSE_IF(n_new < 0, "n_new is below 0");
  const int64_t most = (int64_t)max_pages * page_size;
  if (n_new > most) n_new = (int32_t)most;
  REFUSE_IF(((int64_t)n_new / page_size + 2) * n_kv_heads * n_seqs > (1ll << 30), "too many pages for one call");
  if (n_new == 0) return DEX_OK;
  REFUSE_IF(!k_pages || !table || !length || !bounds, "an array is NULL");
  REFUSE_IF(!aligned(k_pages, 16) || !aligned(bounds, 16), "the pages or their bounds are not 16-byte aligned");
  REFUSE_IF(!words(table, length), kType);
  BoundsArgs a{};
  a.k = k_pages; a.map = PageMap{table, n_seqs, max_pages, n_pages, n_kv_heads, page_shift(page_size)};
  a.len = length; a.head_dim = head_dim; a.n_new = n_new; a.bounds = bounds;
  REFUSE_IF(!bounds_fits(a), kThreads);
  return launched(fn, launch_bounds(dtype, a, (hipStream_t)stream));
}

int64_t dex_pages_select_work(int32_t n_rows, int32_t n_kv_heads, int32_t page_size, int32_t max_len) {
  if (n_rows < 0 || n_rows > (1 << 20) || n_kv_heads < 1 || n_kv_heads > 4096 || page_shift(page_size) < 0 || max_len < 0 ||
      max_len > (1 << 30) || too_many_pages(n_rows, n_kv_heads, max_len, page_size))
    return 0;
  return (int64_t)select_work(n_rows, n_kv_heads, page_shift(page_size), max_len);
}

dex_status dex_pages_select(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_rows,
                            const int32_t *row_seq, const int32_t *row_len, int32_t max_len, const void *q, int64_t q_row,
                            int64_t q_head, const void *bounds, int32_t n_pages, int32_t page_size, const int32_t *table,
                            int32_t n_seqs, int32_t max_pages, int32_t n_select, int32_t sinks, int32_t recent,
                            int32_t *columns, void *work, void *stream) {
  static const char fn[] = "dex_pages_select";
  if (const char *why = attention_fault(dtype, head_dim, n_heads, n_kv_heads, n_rows, 1, 1.f, n_pages, page_size, n_seqs,
                                        max_pages))
    return refuse(fn, why);
  REFUSE_IF(max_len < 0 || max_len > (1 << 30), "max_len is not 0 to 2^30");
  REFUSE_IF(sinks < 0 || recent < 0 || sinks > (1 << 30) || recent > (1 << 30), "sinks or recent is not 0 to 2^30");
  REFUSE_IF(n_select < 1 || n_select > (1 << 30) || n_select < (int64_t)sinks + recent, "n_select is below 1 or sinks + recent");
  REFUSE_IF(too_many_pages(n_rows, n_kv_heads, max_len, page_size), "too many pages for one call");
  if (n_rows == 0) return DEX_OK;
  REFUSE_IF(!q || !bounds || !table || !row_len || !columns, "queries, bounds, table, lengths or columns are NULL");
  REFUSE_IF(!aligned(bounds, 16), "the bounds are not 16-byte aligned");
  REFUSE_IF(!words(row_seq, row_len, table, columns) || !aligned(q, elem(dtype)), kType);
  REFUSE_IF(max_len > 0 && (!work || !aligned(work, 16)), kWork);
  SelectArgs a{};
  a.q = q; a.q_row = q_row; a.q_head = q_head; a.bounds = bounds;
  a.map = PageMap{table, n_seqs, max_pages, n_pages, n_kv_heads, page_shift(page_size)};
  a.seq = row_seq; a.len = row_len; a.n_rows = n_rows; a.n_heads = n_heads; a.head_dim = head_dim; a.max_len = max_len;
  a.n_select = n_select; a.sinks = sinks; a.recent = recent; a.columns = columns; a.work = work;
  REFUSE_IF(!select_fits(dtype, a), kThreads);
  return launched(fn, launch_select(dtype, a, (hipStream_t)stream));
}

dex_status dex_pages_evict(const float *weight, int64_t weight_ld, int32_t n_seqs, int32_t n_kv_heads, int32_t capacity,
                           const int32_t *length, int32_t budget, int32_t sinks, int32_t recent, int32_t *index,
                           int32_t *count, float *weight_out, int64_t weight_out_ld, void *stream) {
  static const char fn[] = "dex_pages_evict";
  REFUSE_IF(n_seqs < 0 || n_seqs > (1 << 20), "n_seqs is not 0 to 2^20");
  REFUSE_IF(n_kv_heads < 1 || n_kv_heads > 4096, "n_kv_heads is not 1 to 4096");
  REFUSE_IF((int64_t)n_seqs * n_kv_heads > (1 << 30), "too many rows for one call");
  REFUSE_IF(capacity < 1 || capacity > (1 << 30), "capacity is not 1 to 2^30");
  REFUSE_IF(sinks < 0 || recent < 0 || sinks > (1 << 30) || recent > (1 << 30), "sinks or recent is not 0 to 2^30");
  REFUSE_IF(budget < 1 || budget > (1 << 30) || budget < (int64_t)sinks + recent, "budget is below 1 or sinks + recent");
  if (n_seqs == 0) return DEX_OK;
  REFUSE_IF(weight_ld < capacity || weight_out_ld < capacity, "a row of the weights is shorter than capacity");
  REFUSE_IF(!weight || !length || !index || !count || !weight_out, "an array is NULL");
  REFUSE_IF(weight == weight_out && weight_ld != weight_out_ld, "weight_out is weight with another stride");
  REFUSE_IF(!words(weight, length, index, count, weight_out), kType);
  EvictArgs a{};
  a.weight = weight; a.weight_out = weight_out; a.weight_ld = weight_ld; a.weight_out_ld = weight_out_ld;
  a.capacity = capacity; a.len = length; a.n = n_seqs; a.heads = n_kv_heads; a.budget = budget; a.sinks = sinks;
  a.recent = recent; a.index = index; a.count = count;
  REFUSE_IF(!evict_fits(a), kThreads);
  return launched(fn, launch_evict(a, (hipStream_t)stream));
}

}  // extern "C"
