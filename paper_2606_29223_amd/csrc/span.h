// Internal declarations of the operators for drafted trees, page selection and
// eviction over a paged key/value cache.
#pragma once

#include "paged.h"

namespace dex {

constexpr int kMaxDraft = 256;          // drafted tokens of a tree

// A launch has fewer than 2^32 threads in a dimension.  Whether the launches of
// a call have (*_fits) is asked before the first of them.
inline bool launch_fits(int64_t blocks, int threads) { return blocks <= (int64_t)0xffffffff / threads; }

// Attention of `draft` rows a sequence over its keys (span_attn.hip).
struct SpanArgs {
  const void *q;
  int64_t q_row, q_head;
  const void *k, *v;                    // [n_pages][n_kv_heads][page_size][head_dim]
  PageMap map;
  const int *seq;                       // [n], or null: sequence i
  const int *len;                       // [n] keys before the drafted ones
  int n, draft, n_heads, head_dim;
  int max_len, most;                    // a longer len counts as max_len; places looked at without the drafted ones
  float scale;
  // drafted keys, at the positions behind len (mask null: none, and draft is 1)
  const uint64_t *mask;                 // [n][draft][words]
  int words;
  const int *n_draft;                   // [n], or null: draft
  // the columns of the table to read, of each sequence and kv head (null: all)
  const int *columns;                   // [n][n_kv_heads][n_cols]
  int n_cols;
  // running totals of the softmax weights (null: not wanted)
  const float *weight;                  // [n][n_kv_heads], rows weight_ld apart
  float *weight_out;
  int64_t weight_ld, weight_out_ld;
  void *out;
  int64_t out_row, out_head;
  float *lse;                           // [n * draft][n_heads], or null
  void *work;
};
size_t span_work(int dtype, int n, int draft, int n_heads, int n_kv_heads, int head_dim, int most, bool trees, bool weigh);
bool span_fits(int dtype, const SpanArgs &a);
hipError_t launch_span(int dtype, const SpanArgs &a, hipStream_t s);

struct TreeMaskArgs {
  const int *parent;                    // [n][draft]
  int n, draft;
  uint64_t *mask;                       // [n][draft][words]
  int words;
  int *depth;                           // [n][draft], or null
};
hipError_t launch_tree_mask(const TreeMaskArgs &a, hipStream_t s);

struct TreeAcceptArgs {
  const int *parent, *token, *target;   // [n][draft]
  const int *n_draft, *root;            // [n], or null
  int n, draft;
  int *path, *count, *next;             // [n][draft], [n], [n]
};
hipError_t launch_tree_accept(const TreeAcceptArgs &a, hipStream_t s);

struct KeepArgs {
  void *k, *v;                          // [n_layers][n_pages][n_kv_heads][page_size][head_dim]
  int n_layers, row_bytes;
  PageMap map;                          // the table read
  const int *to;                        // the table written (null: the same)
  int to_pages;                         // its columns
  const int *first;                     // [n_seqs], or null: 0
  const int *index;                     // [.. layers][n_seqs][.. heads][capacity]
  int64_t index_layer, index_seq, index_head;   // strides, 0 for what it is the same for
  int capacity;
  const int *count;                     // [n_seqs]
};
bool keep_fits(const KeepArgs &a);
hipError_t launch_keep(const KeepArgs &a, hipStream_t s);

struct TrimArgs {
  const int *table, *ref, *len;
  int *table_out, *ref_out;             // each may be its input
  int n_seqs, max_pages, n_pages, shift;
};
hipError_t launch_trim(const TrimArgs &a, hipStream_t s);

struct BoundsArgs {
  const void *k;                        // [n_pages][n_kv_heads][page_size][head_dim]
  PageMap map;
  const int *len;                       // [n_seqs]
  int head_dim, n_new;
  void *bounds;                         // [n_pages][n_kv_heads][2][head_dim]
};
bool bounds_fits(const BoundsArgs &a);
hipError_t launch_bounds(int dtype, const BoundsArgs &a, hipStream_t s);

struct SelectArgs {
  const void *q;
  int64_t q_row, q_head;
  const void *bounds;
  PageMap map;
  const int *seq, *len;                 // [n_rows]
  int n_rows, n_heads, head_dim, max_len;
  int n_select, sinks, recent;
  int *columns;                         // [n_rows][n_kv_heads][n_select]
  void *work;
};
size_t select_work(int n_rows, int n_kv_heads, int page_shift, int max_len);
bool select_fits(int dtype, const SelectArgs &a);
hipError_t launch_select(int dtype, const SelectArgs &a, hipStream_t s);

struct EvictArgs {
  const float *weight;                  // [n][heads], rows weight_ld apart
  float *weight_out;
  int64_t weight_ld, weight_out_ld;
  int capacity;                         // columns of either
  const int *len;
  int n, heads, budget, sinks, recent;
  int *index;                           // [n][heads][budget]
  int *count;                           // [n]
};
bool evict_fits(const EvictArgs &a);
hipError_t launch_evict(const EvictArgs &a, hipStream_t s);

}  // namespace dex
