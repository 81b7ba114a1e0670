// What the C ABI of the paged operators checks before it launches anything.
#pragma once

#include <cmath>
#include <cstdio>

#include "dex.h"
#include "paged.h"

namespace dex {
namespace {

[[maybe_unused]] dex_status refuse(const char *fn, const char *why) noexcept {
  char msg[256];
  snprintf(msg, sizeof msg, "%s: %s", fn, why);
  set_call_error(msg);
  return DEX_E_INVAL;
}

[[maybe_unused]] dex_status launched(const char *fn, hipError_t e) noexcept {
  if (e == hipSuccess) return DEX_OK;
  char msg[256];
  snprintf(msg, sizeof msg, "%s: %s", fn, hipGetErrorString(e));
  set_call_error(msg);
  return DEX_E_HIP;
}

#define REFUSE_IF(cond, why) \
  do {                       \
    if (cond) return refuse(fn, why); \
  } while (0)

[[maybe_unused]] bool known(int dtype) { return dtype == DEX_F32 || dtype == DEX_BF16; }
[[maybe_unused]] int64_t elem(int dtype) { return dtype == DEX_F32 ? 4 : 2; }
[[maybe_unused]] bool aligned(const void *p, uintptr_t to) { return (uintptr_t)p % to == 0; }

// Arrays of int32 (or float) at their type's alignment: counts change by atomics.
template <typename... P>
bool words(P... p) {
  return (aligned(p, 4) && ...);
}

// Whether elements of an output share memory.  A row's heads lie apart from each
// other and the rows apart from each other, or the other way round.
[[maybe_unused]] bool overlaps(int64_t n_rows, int64_t row, int64_t heads, int64_t head, int64_t head_dim) {
  typedef __int128 wide;
  const wide r = row < 0 ? -(wide)row : row, h = head < 0 ? -(wide)head : head;
  auto apart = [&](wide n0, wide s0, wide n1, wide s1) {      // n0 inside n1
    return (n0 == 1 || s0 >= head_dim) && (n1 == 1 || s1 >= (n0 - 1) * s0 + head_dim);
  };
  return n_rows > 0 && heads > 0 && !apart(heads, h, n_rows, r) && !apart(n_rows, r, heads, h);
}
[[maybe_unused]] const char kOverlap[] = "elements of an output overlap";
[[maybe_unused]] const char kType[] = "an array is not aligned to its type";

// log2 of a page size, -1 if it is none
[[maybe_unused]] int page_shift(int page_size) {
  if (page_size < 1 || page_size > 1024 || (page_size & (page_size - 1))) return -1;
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

[[maybe_unused]] const char *cache_fault(int dtype, int head_dim, int n_pages, int n_kv_heads, int page_size) {
  if (!known(dtype)) return "dtype is neither DEX_F32 nor DEX_BF16";
  if (head_dim < 2 || head_dim > 1024 || head_dim % 2) return "head_dim is not even, 2 to 1024";
  if (n_kv_heads < 1 || n_kv_heads > 4096) return "n_kv_heads is not 1 to 4096";
  if (page_shift(page_size) < 0) return "page_size is not a power of two up to 1024";
  if (n_pages < 1 || n_pages > (1 << 30)) return "n_pages is not 1 to 2^30";
  if ((int64_t)n_pages * n_kv_heads * page_size >= (int64_t)kNoRow) return "the layer has 2^32 - 1 cache rows or more";
  return nullptr;
}

[[maybe_unused]] const char *table_fault(int n_seqs, int max_pages, int page_size) {
  if (n_seqs < 1 || n_seqs > (1 << 24)) return "n_seqs is not 1 to 2^24";
  if (max_pages < 1 || (int64_t)max_pages * page_size > (1 << 30)) return "max_pages is below 1, or ends past position 2^30";
  return nullptr;
}

// What one workgroup numbers in 32 bits: all pages that a table can list.
[[maybe_unused]] const char *entries_fault(int n_seqs, int max_pages) {
  return (int64_t)n_seqs * max_pages > (1 << 30) ? "the table has over 2^30 entries" : nullptr;
}

[[maybe_unused]] const char *rotary_fault(const dex_rotary *r, int head_dim) {
  if (!r->turns) return "the plan has no turns";
  if (!aligned(r->turns, 8)) return "the plan's turns are not aligned to their type";
  if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_dim > head_dim) return "rot_dim is not even, 2 to head_dim";
  if (!std::isfinite(r->amplitude)) return "amplitude is not finite";
  return nullptr;
}

// Heads of an array: present with data, or absent with neither.
[[maybe_unused]] const char *heads_fault(const void *p, int n, const char *what) {
  if (n < 0 || n > 4096) return what;
  if ((n > 0) != (p != nullptr)) return what;
  return nullptr;
}

[[maybe_unused]] bool too_many(int n_rows, int head_dim, int heads) { return (int64_t)n_rows * head_dim * (heads + 8) >= (1ll << 35); }

}  // namespace
}  // namespace dex
