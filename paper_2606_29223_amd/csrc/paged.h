// Internal declarations of the operators over a paged key/value cache
// (rotary positions, page tables, attention over pages, beam selection).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dex {

// Message dex_last_error(NULL) gives on this thread.
void set_call_error(const char *msg) noexcept;

// The cache row (one key's or value's head_dim elements) of position p of a
// sequence: page table[p / page_size] of kv head h, slot p % page_size.  Rows
// are numbered over the whole layer; the host refuses a layer of 2^32 - 1 rows
// or more, so kNoRow is never a row.
constexpr uint32_t kNoRow = 0xffffffffu;
struct PageMap {
  const int *table;           // [n_seqs][max_pages]
  int n_seqs, max_pages;
  int n_pages, n_kv_heads;
  int shift;                  // log2 of the page size
};
// kNoRow where the table holds no page there: an entry outside [0, n_pages),
// or a position outside the table.
__host__ __device__ __forceinline__ uint32_t page_row(const PageMap &m, int seq, int pos, int kv_head) {
  const int c = pos >> m.shift;
  if (pos < 0 || c >= m.max_pages) return kNoRow;
  const int page = m.table[(size_t)seq * m.max_pages + c];
  if (page < 0 || page >= m.n_pages) return kNoRow;
  return (((uint32_t)page * (uint32_t)m.n_kv_heads + (uint32_t)kv_head) << m.shift) +
         (uint32_t)(pos & ((1 << m.shift) - 1));
}

// Heads of rows: element d of head h of row r at p + r * row + h * head + d.
struct HeadsIn {
  const void *p;
  int64_t row, head;
  int n;                      // heads
};
struct HeadsOut {
  void *p;
  int64_t row, head;
};

struct RopeArgs {
  const double *turns;        // [rot_dim / 2] turns a position (null: no rotation)
  int head_dim, rot_dim, interleaved, inverse;
  float amplitude;
  int n_rows;
  const int *pos;             // [n_rows]
  HeadsIn q, k, v;            // n 0: absent
  HeadsOut q_out, k_out;      // k_out unused with pages
  // pages (null: k goes to k_out and v is absent)
  void *k_pages, *v_pages;
  PageMap map;
  const int *seq;             // [n_rows], or null: row r is sequence r
};
// Pairs a lane turns at a time: the widest access that the call allows.
int rope_vec(int dtype, const RopeArgs &a);
hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t s);

struct ForkArgs {
  const int *table, *ref, *len, *parent;
  int *table_out, *ref_out, *len_out;   // each may be its input
  int n_seqs, max_pages, n_pages;
};
hipError_t launch_fork(const ForkArgs &a, hipStream_t s);

constexpr int kMaxSeqs = 1024;          // sequences of a page table that fork and reserve take
struct ReserveArgs {
  int *table, *ref, *len;
  const int *n_new;
  int n_seqs, max_pages, n_pages, shift;
  int *pos, *src, *dst, *tokens, *state;
};
hipError_t launch_reserve(const ReserveArgs &a, hipStream_t s);

struct CompactArgs {
  const int *table, *ref;
  int *table_out, *ref_out, *map, *src, *dst, *state;
  int n_seqs, max_pages, n_pages;
};
hipError_t launch_compact(const CompactArgs &a, hipStream_t s);

struct PageCopyArgs {
  void *k, *v;                // [n_layers][n_pages][n_kv_heads][page_size][head_dim]
  int n_layers, n_pages, n_kv_heads, page_size;
  int row_bytes;              // head_dim elements, a multiple of 16 bytes
  const int *src, *dst, *tokens, *count;
  int capacity;               // entries of src and dst
};
hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t s);

struct PagedAttnArgs {
  const void *q;
  int64_t q_row, q_head;
  const void *k, *v;          // [n_pages][n_kv_heads][page_size][head_dim]
  PageMap map;
  const int *seq;             // [n_rows], or null: row r is sequence r
  const int *len;             // [n_rows] keys
  int n_rows, n_heads, head_dim;
  int group;                  // consecutive rows whose common pages are read once
  int max_len, window;
  float scale;
  void *out;
  int64_t out_row, out_head;
  float *lse;                 // [n_rows][n_heads], or null
  void *work;                 // paged_attention_work bytes
};
size_t paged_attention_work(int n_rows, int n_heads, int head_dim, int max_len, int group);
hipError_t launch_paged_attention(int dtype, const PagedAttnArgs &a, hipStream_t s);

constexpr int kMaxBeams = 64;
struct BeamArgs {
  const void *logits;         // [requests * beams] rows, ld elements apart
  int64_t ld;
  int requests, beams, vocab, n_out;
  const float *score;         // [requests][beams]
  const uint8_t *done;        // [requests][beams], or null
  int eos;
  int *parent, *token;        // [requests][n_out]
  float *score_out;
  uint8_t *done_out;          // or null
  void *work;
};
size_t beam_work(int rows, int vocab, int n_out);
hipError_t launch_beam(int dtype, const BeamArgs &a, hipStream_t s);

}  // namespace dex
