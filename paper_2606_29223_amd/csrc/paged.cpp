// C ABI of the operators over a paged key/value cache: every argument is
// checked here, before anything is launched.
#include <cmath>

#include "dex.h"
#include "paged_check.h"

using namespace dex;

extern "C" {

dex_status dex_rotary_turns(int32_t scaling, int32_t rot_dim, double theta, double factor, double original, double slow,
                            double fast, double *turns) {
  static const char fn[] = "dex_rotary_turns";
  REFUSE_IF(!turns, "turns is NULL");
  REFUSE_IF(scaling < DEX_ROTARY_PLAIN || scaling > DEX_ROTARY_BANDS, "unknown scaling");
  REFUSE_IF(rot_dim < 2 || rot_dim % 2 || rot_dim > 1024, "rot_dim is not even, 2 to 1024");
  REFUSE_IF(!(theta > 0) || !std::isfinite(theta), "theta is not a positive number");
  REFUSE_IF(scaling != DEX_ROTARY_PLAIN && (!(factor > 0) || !std::isfinite(factor)), "factor is not a positive number");
  REFUSE_IF(scaling == DEX_ROTARY_BASE && rot_dim == 2, "a changed base has no effect on one pair");
  REFUSE_IF(scaling == DEX_ROTARY_BANDS && (!(original > 0) || !std::isfinite(original)),
            "original is not a positive number");
  REFUSE_IF(scaling == DEX_ROTARY_BANDS && (!(slow >= 0) || !(fast > slow) || !std::isfinite(fast)),
            "slow and fast are not 0 <= slow < fast");
  const double base = scaling == DEX_ROTARY_BASE ? theta * std::pow(factor, rot_dim / (rot_dim - 2.0)) : theta;
  const double two_pi = 6.283185307179586476925;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == DEX_ROTARY_LINEAR) f /= factor;
    if (scaling == DEX_ROTARY_BANDS) {
      const double n = original * f / two_pi;            // turns over the original context
      const double keep = std::fmin(1.0, std::fmax(0.0, (n - slow) / (fast - slow)));
      f = f * keep + f / factor * (1.0 - keep);
    }
    if (!std::isfinite(f)) return refuse(fn, "theta and factor give a frequency that is not finite");
    turns[i] = f / two_pi;
  }
  return DEX_OK;
}

dex_status dex_rope(int32_t dtype, int32_t head_dim, const dex_rotary *rotary, int32_t inverse, int32_t n_rows,
                    const int32_t *pos, const void *q, int64_t q_row, int64_t q_head, int32_t n_heads, void *q_out,
                    int64_t q_out_row, int64_t q_out_head, const void *k, int64_t k_row, int64_t k_head,
                    int32_t n_kv_heads, void *k_out, int64_t k_out_row, int64_t k_out_head, void *stream) {
  static const char fn[] = "dex_rope";
  REFUSE_IF(!known(dtype), "dtype is neither DEX_F32 nor DEX_BF16");
  REFUSE_IF(head_dim < 2 || head_dim > 1024 || head_dim % 2, "head_dim is not even, 2 to 1024");
  REFUSE_IF(!rotary, "rotary is NULL");
  if (const char *why = rotary_fault(rotary, head_dim)) return refuse(fn, why);
  if (const char *why = heads_fault(q, n_heads, "queries: heads without data, or the other way round")) return refuse(fn, why);
  if (const char *why = heads_fault(k, n_kv_heads, "keys: heads without data, or the other way round")) return refuse(fn, why);
  REFUSE_IF(n_heads + n_kv_heads == 0, "neither queries nor keys");
  REFUSE_IF((n_heads > 0 && !q_out) || (n_kv_heads > 0 && !k_out), "an output is NULL");
  REFUSE_IF(n_rows < 0 || (n_rows > 0 && !pos), "n_rows is below 0, or pos is NULL");
  REFUSE_IF(!words(pos) || !aligned(q, elem(dtype)) || !aligned(q_out, elem(dtype)) || !aligned(k, elem(dtype)) ||
                !aligned(k_out, elem(dtype)), kType);
  REFUSE_IF(overlaps(n_rows, q_out_row, n_heads, q_out_head, head_dim) ||
                overlaps(n_rows, k_out_row, n_kv_heads, k_out_head, head_dim), kOverlap);
  REFUSE_IF(too_many(n_rows, head_dim, n_heads + n_kv_heads), "too many rows for one call");
  if (n_rows == 0) return DEX_OK;
  RopeArgs a{};
  a.turns = rotary->turns; a.rot_dim = rotary->rot_dim; a.interleaved = rotary->interleaved; a.amplitude = rotary->amplitude;
  a.head_dim = head_dim; a.inverse = inverse; a.n_rows = n_rows; a.pos = pos;
  a.q = HeadsIn{q, q_row, q_head, n_heads};
  a.k = HeadsIn{k, k_row, k_head, n_kv_heads};
  a.q_out = HeadsOut{q_out, q_out_row, q_out_head};
  a.k_out = HeadsOut{k_out, k_out_row, k_out_head};
  return launched(fn, launch_rope(dtype, a, (hipStream_t)stream));
}

dex_status dex_pages_append(int32_t dtype, int32_t head_dim, const dex_rotary *rotary, int32_t n_rows,
                            const int32_t *row_seq, const int32_t *row_pos, const void *q, int64_t q_row, int64_t q_head,
                            int32_t n_heads, void *q_out, int64_t q_out_row, int64_t q_out_head, const void *k,
                            int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                            int32_t n_kv_heads, void *k_pages, void *v_pages, int32_t n_pages, int32_t page_size,
                            const int32_t *table, int32_t n_seqs, int32_t max_pages, void *stream) {
  static const char fn[] = "dex_pages_append";
  if (const char *why = cache_fault(dtype, head_dim, n_pages, n_kv_heads, page_size)) return refuse(fn, why);
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return refuse(fn, why);
  if (rotary)
    if (const char *why = rotary_fault(rotary, head_dim)) return refuse(fn, why);
  if (const char *why = heads_fault(q, n_heads, "queries: heads without data, or the other way round")) return refuse(fn, why);
  REFUSE_IF(n_heads > 0 && !q_out, "q_out is NULL");
  REFUSE_IF(!k || !v || !k_pages || !v_pages || !table, "keys, values, pages or table are NULL");
  REFUSE_IF(!aligned(k_pages, 16) || !aligned(v_pages, 16), "the pages are not 16-byte aligned");
  REFUSE_IF(n_rows < 0 || (n_rows > 0 && !row_pos), "n_rows is below 0, or row_pos is NULL");
  REFUSE_IF(!words(row_seq, row_pos, table) || !aligned(q, elem(dtype)) || !aligned(q_out, elem(dtype)) ||
                !aligned(k, elem(dtype)) || !aligned(v, elem(dtype)), kType);
  REFUSE_IF(overlaps(n_rows, q_out_row, n_heads, q_out_head, head_dim), kOverlap);
  REFUSE_IF(too_many(n_rows, head_dim, n_heads + 2 * n_kv_heads), "too many rows for one call");
  if (n_rows == 0) return DEX_OK;
  RopeArgs a{};
  if (rotary) {
    a.turns = rotary->turns; a.rot_dim = rotary->rot_dim; a.interleaved = rotary->interleaved;
    a.amplitude = rotary->amplitude;
  }
  a.head_dim = head_dim; a.n_rows = n_rows; a.pos = row_pos; a.seq = row_seq;
  a.q = HeadsIn{q, q_row, q_head, n_heads};
  a.k = HeadsIn{k, k_row, k_head, n_kv_heads};
  a.v = HeadsIn{v, v_row, v_head, n_kv_heads};
  a.q_out = HeadsOut{q_out, q_out_row, q_out_head};
  a.k_pages = k_pages; a.v_pages = v_pages;
  a.map = PageMap{table, n_seqs, max_pages, n_pages, n_kv_heads, page_shift(page_size)};
  return launched(fn, launch_rope(dtype, a, (hipStream_t)stream));
}

int64_t dex_pages_attention_work(int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len,
                                 int32_t group) {
  if (n_rows < 0 || n_heads < 1 || n_kv_heads < 1 || head_dim < 1 || max_len < 0 || group < 1) return 0;
  return (int64_t)paged_attention_work(n_rows, n_heads, head_dim, max_len, group);
}

dex_status dex_pages_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t n_rows,
                               const int32_t *row_seq, const int32_t *row_len, int32_t max_len, int32_t window,
                               int32_t group, float scale, const void *q, int64_t q_row, int64_t q_head,
                               const void *k_pages, const void *v_pages, int32_t n_pages, int32_t page_size,
                               const int32_t *table, int32_t n_seqs, int32_t max_pages, void *out, int64_t out_row,
                               int64_t out_head, float *lse, void *work, void *stream) {
  static const char fn[] = "dex_pages_attention";
  if (const char *why = cache_fault(dtype, head_dim, n_pages, n_kv_heads, page_size)) return refuse(fn, why);
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return refuse(fn, why);
  REFUSE_IF(head_dim != 32 && head_dim != 64 && head_dim != 128, "head_dim is not 32, 64 or 128");
  REFUSE_IF(n_heads < n_kv_heads || n_heads % n_kv_heads || n_heads / n_kv_heads > 64,
            "n_heads is not a multiple of n_kv_heads, up to 64 times it");
  REFUSE_IF(n_heads > 8192, "n_heads is over 8192");
  REFUSE_IF(n_rows < 0 || n_rows > (1 << 20), "n_rows is not 0 to 2^20");
  REFUSE_IF(max_len < 0 || window < 0 || group < 1, "max_len or window is below 0, or group below 1");
  REFUSE_IF(!std::isfinite(scale), "scale is not finite");
  if (n_rows == 0) return DEX_OK;
  REFUSE_IF(!q || !k_pages || !v_pages || !table || !row_len || !out, "queries, pages, table, lengths or out are NULL");
  REFUSE_IF(!aligned(k_pages, 16) || !aligned(v_pages, 16), "the pages are not 16-byte aligned");
  REFUSE_IF(!words(row_seq, row_len, table, lse) || !aligned(q, elem(dtype)) || !aligned(out, elem(dtype)), kType);
  REFUSE_IF(overlaps(n_rows, out_row, n_heads, out_head, head_dim), kOverlap);
  PagedAttnArgs a{};
  a.q = q; a.q_row = q_row; a.q_head = q_head; a.k = k_pages; a.v = v_pages;
  a.map = PageMap{table, n_seqs, max_pages, n_pages, n_kv_heads, page_shift(page_size)};
  a.seq = row_seq; a.len = row_len; a.n_rows = n_rows; a.n_heads = n_heads; a.head_dim = head_dim;
  a.group = group; a.max_len = max_len; a.window = window; a.scale = scale;
  a.out = out; a.out_row = out_row; a.out_head = out_head; a.lse = lse; a.work = work;
  REFUSE_IF(paged_attention_work(n_rows, n_heads, head_dim, max_len, group) > 0 && (!work || !aligned(work, 16)),
            "the work memory is NULL or not 16-byte aligned");
  return launched(fn, launch_paged_attention(dtype, a, (hipStream_t)stream));
}

dex_status dex_pages_fork(const int32_t *table, const int32_t *ref, const int32_t *length, const int32_t *parent,
                          int32_t n_seqs, int32_t max_pages, int32_t n_pages, int32_t *table_out, int32_t *ref_out,
                          int32_t *length_out, void *stream) {
  static const char fn[] = "dex_pages_fork";
  REFUSE_IF(!table || !ref || !length || !parent || !table_out || !ref_out || !length_out, "an array is NULL");
  REFUSE_IF(n_seqs < 1 || n_seqs > kMaxSeqs, "n_seqs is not 1 to 1024");
  REFUSE_IF(n_pages < 1 || n_pages > (1 << 30), "n_pages is not 1 to 2^30");
  if (const char *why = table_fault(n_seqs, max_pages, 1)) return refuse(fn, why);
  if (const char *why = entries_fault(n_seqs, max_pages)) return refuse(fn, why);
  REFUSE_IF(!words(table, ref, length, parent, table_out, ref_out, length_out), kType);
  const ForkArgs a{table, ref, length, parent, table_out, ref_out, length_out, n_seqs, max_pages, n_pages};
  return launched(fn, launch_fork(a, (hipStream_t)stream));
}

dex_status dex_pages_reserve(int32_t *table, int32_t *ref, int32_t *length, const int32_t *n_new, int32_t n_seqs,
                             int32_t max_pages, int32_t n_pages, int32_t page_size, int32_t *pos, int32_t *src,
                             int32_t *dst, int32_t *tokens, int32_t *state, void *stream) {
  static const char fn[] = "dex_pages_reserve";
  REFUSE_IF(!table || !ref || !length || !n_new || !pos || !src || !dst || !tokens || !state, "an array is NULL");
  REFUSE_IF(n_seqs < 1 || n_seqs > kMaxSeqs, "n_seqs is not 1 to 1024");
  REFUSE_IF(n_pages < 1 || n_pages > (1 << 30), "n_pages is not 1 to 2^30");
  REFUSE_IF(page_shift(page_size) < 0, "page_size is not a power of two up to 1024");
  if (const char *why = table_fault(n_seqs, max_pages, page_size)) return refuse(fn, why);
  if (const char *why = entries_fault(n_seqs, max_pages)) return refuse(fn, why);
  REFUSE_IF(!words(table, ref, length, n_new, pos, src, dst, tokens, state), kType);
  const ReserveArgs a{table, ref, length, n_new, n_seqs, max_pages, n_pages, page_shift(page_size),
                      pos, src, dst, tokens, state};
  return launched(fn, launch_reserve(a, (hipStream_t)stream));
}

dex_status dex_pages_compact(const int32_t *table, const int32_t *ref, int32_t n_seqs, int32_t max_pages,
                             int32_t n_pages, int32_t *table_out, int32_t *ref_out, int32_t *map, int32_t *src,
                             int32_t *dst, int32_t *state, void *stream) {
  static const char fn[] = "dex_pages_compact";
  REFUSE_IF(!table || !ref || !table_out || !ref_out || !map || !state, "an array is NULL");
  REFUSE_IF(n_pages < 1 || n_pages > (1 << 30), "n_pages is not 1 to 2^30");
  REFUSE_IF(n_pages > 1 && (!src || !dst), "src or dst is NULL");
  if (const char *why = table_fault(n_seqs, max_pages, 1)) return refuse(fn, why);
  REFUSE_IF(!words(table, ref, table_out, ref_out, map, src, dst, state), kType);
  const CompactArgs a{table, ref, table_out, ref_out, map, src, dst, state, n_seqs, max_pages, n_pages};
  return launched(fn, launch_compact(a, (hipStream_t)stream));
}

dex_status dex_pages_copy(int32_t dtype, int32_t head_dim, int32_t n_layers, int32_t n_pages, int32_t n_kv_heads,
                          int32_t page_size, void *k_pool, void *v_pool, const int32_t *src, const int32_t *dst,
                          const int32_t *tokens, const int32_t *count, int32_t capacity, void *stream) {
  static const char fn[] = "dex_pages_copy";
  if (const char *why = cache_fault(dtype, head_dim, n_pages, n_kv_heads, page_size)) return refuse(fn, why);
  REFUSE_IF(head_dim * elem(dtype) % 16, "a head's row is not a multiple of 16 bytes");
  REFUSE_IF(n_layers < 1 || (int64_t)n_layers * n_kv_heads > (1 << 20), "n_layers is not 1 to 2^20 / n_kv_heads");
  REFUSE_IF(capacity < 0, "capacity is below 0");
  REFUSE_IF(!k_pool || !v_pool, "a pool is NULL");
  REFUSE_IF(!aligned(k_pool, 16) || !aligned(v_pool, 16), "the pools are not 16-byte aligned");
  if (capacity == 0) return DEX_OK;
  REFUSE_IF(!src || !dst, "src or dst is NULL");
  REFUSE_IF(!words(src, dst, tokens, count), kType);
  const PageCopyArgs a{k_pool, v_pool, n_layers, n_pages, n_kv_heads, page_size, (int)(head_dim * elem(dtype)),
                       src, dst, tokens, count, capacity};
  return launched(fn, launch_page_copy(a, (hipStream_t)stream));
}

int64_t dex_beam_select_work(int32_t dtype, int32_t requests, int32_t beams, int32_t vocab, int32_t n_out) {
  if (!known(dtype) || requests < 0 || beams < 1 || vocab < 1 || n_out < 1 || n_out > kMaxBeams) return 0;
  if ((int64_t)requests * beams > (1 << 20)) return 0;
  return (int64_t)beam_work(requests * beams, vocab, n_out);
}

dex_status dex_beam_select(int32_t dtype, const void *logits, int64_t ld, int32_t requests, int32_t beams, int32_t vocab,
                           const float *score, const uint8_t *done, int32_t eos, int32_t n_out, int32_t *parent,
                           int32_t *token, float *score_out, uint8_t *done_out, void *work, void *stream) {
  static const char fn[] = "dex_beam_select";
  REFUSE_IF(!known(dtype), "dtype is neither DEX_F32 nor DEX_BF16");
  REFUSE_IF(requests < 0 || beams < 1 || beams > kMaxBeams, "requests is below 0, or beams not 1 to 64");
  REFUSE_IF((int64_t)requests * beams > (1 << 20), "requests * beams is over 2^20");
  REFUSE_IF(vocab < 1 || vocab > (1 << 30), "vocab is not 1 to 2^30");
  REFUSE_IF(n_out < 1 || n_out > kMaxBeams || n_out > (int64_t)beams * vocab, "n_out is not 1 to 64, at most beams * vocab");
  REFUSE_IF((int64_t)requests * beams * (vocab / 2048 + 2) > (1 << 25), "too many logits for one call");
  REFUSE_IF(eos < -1 || eos >= vocab, "eos is not in [-1, vocab)");
  REFUSE_IF(done && eos < 0, "finished beams need an eos");
  if (requests == 0) return DEX_OK;
  REFUSE_IF(ld < vocab && (int64_t)requests * beams > 1, "ld is below vocab");
  REFUSE_IF(!logits || !score || !parent || !token || !score_out || !work, "an array is NULL");
  REFUSE_IF(!aligned(work, 16), "the work memory is not 16-byte aligned");
  REFUSE_IF(!aligned(logits, elem(dtype)) || !words(score, parent, token, score_out), kType);
  BeamArgs a{};
  a.logits = logits; a.ld = ld; a.requests = requests; a.beams = beams; a.vocab = vocab; a.n_out = n_out;
  a.score = score; a.done = done; a.eos = eos; a.parent = parent; a.token = token; a.score_out = score_out;
  a.done_out = done_out; a.work = work;
  return launched(fn, launch_beam(dtype, a, (hipStream_t)stream));
}

}  // extern "C"
