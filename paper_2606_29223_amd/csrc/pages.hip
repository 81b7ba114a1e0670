// Page tables of a paged cache: fork and free, reserve with copy on write,
// compaction, and the copies of pages they ask for.
//
// A table row holds a sequence's pages in order, then -1.  ref[p] counts the
// rows (and whoever else) that hold page p; a page nobody holds has count 0
// and may be taken.  Everything is decided on the device, in one fixed order
// (sequences by number, free pages by number), so a decoding step needs no
// word from the host between the choice of parents and the next attention,
// and two runs give the same page numbers.
#include "dex.h"
#include "dex_kernels.h"
#include "paged.h"

#include <algorithm>

namespace dex {

namespace {

constexpr int BIG = 1024;                 // lanes of the one-workgroup kernels
constexpr int SCAN = BIG * 16;            // pages that they look at in one turn
constexpr int kForkTile = 8192;           // table entries of a fork tile (32 KiB of LDS)

__device__ __forceinline__ bool is_page(int p, int n_pages) { return p >= 0 && p < n_pages; }

// Exclusive prefix sum over the workgroup's BIG lanes; *total is the sum.
// Ends with a barrier, so `part` (BIG / 64 ints) may be used again.
__device__ __forceinline__ int block_scan(int v, int *part, int *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < BIG / 64; ++w) {
    const int p = part[w];
    if (w < wave) before += p;
    all += p;
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

// The pages p0 .. p0 + SCAN - 1 that a predicate picks, in order: each wave
// takes 1024 of them, 64 neighbours a load, and keeps their ballots.
struct Picked {
  unsigned long long m[16];
  int base, total;                        // picked before this wave's, and in all
};
template <typename Pred>
__device__ __forceinline__ Picked pick(int p0, int n_pages, Pred pred, int *part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Picked k;
  int n = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const int p = p0 + wave * 1024 + j * 64 + lane;
    k.m[j] = __ballot(p < n_pages && pred(p));
    n += __popcll(k.m[j]);
  }
  if (lane == 0) part[wave] = n;
  __syncthreads();
  k.base = 0;
  k.total = 0;
#pragma unroll
  for (int w = 0; w < BIG / 64; ++w) {
    const int c = part[w];
    if (w < wave) k.base += c;
    k.total += c;
  }
  __syncthreads();
  return k;
}
// f(index among the picked, page) for each.
template <typename F>
__device__ __forceinline__ void each(const Picked &k, int p0, F f) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int at = k.base;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    if (k.m[j] >> lane & 1) f(at + __popcll(k.m[j] & ((1ull << lane) - 1)), p0 + wave * 1024 + j * 64 + lane);
    at += __popcll(k.m[j]);
  }
}

}  // namespace

// ------------------------------------------------------------------- fork
// Row s of the new table is row parent[s] of the old one (nothing, where
// parent[s] names no row); a page's count changes by (children - 1) for every
// old row that held it.  A workgroup takes a tile of columns of every row
// through LDS, so the table may be written over itself.
__global__ __launch_bounds__(BIG) void fork_kernel(ForkArgs a, int cols, int put_counts) {
  extern __shared__ int lds[];
  int *children = lds, *par = lds + a.n_seqs, *tile = par + a.n_seqs;
  const int S = a.n_seqs, C = a.max_pages;
  const int nt = blockDim.x;
  for (int s = threadIdx.x; s < S; s += nt) {
    const int p = a.parent[s];
    children[s] = 0;
    par[s] = p >= 0 && p < S ? p : -1;
    if (blockIdx.x == 0) tile[s] = a.len[s];
  }
  if (put_counts)                         // the only workgroup: counts first, then their changes
    for (int p = threadIdx.x; p < a.n_pages; p += nt) a.ref_out[p] = a.ref[p];
  __threadfence();
  __syncthreads();
  for (int s = threadIdx.x; s < S; s += nt) {
    const int p = par[s];
    if (p >= 0) atomicAdd(&children[p], 1);
    if (blockIdx.x == 0) a.len_out[s] = p >= 0 ? tile[p] : 0;
  }
  __syncthreads();
  for (int c0 = blockIdx.x * cols; c0 < C; c0 += gridDim.x * cols) {
    const int w = min(cols, C - c0);
    for (int i = threadIdx.x; i < S * w; i += nt) {
      const int s = i / w, c = i - s * w;
      const int p = a.table[(size_t)s * C + c0 + c];
      tile[i] = p;
      const int d = children[s] - 1;
      if (d != 0 && is_page(p, a.n_pages)) atomicAdd(&a.ref_out[p], d);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < S * w; i += nt) {
      const int s = i / w, c = i - s * w;
      const int p = par[s];
      a.table_out[(size_t)s * C + c0 + c] = p >= 0 ? tile[p * w + c] : -1;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void copy_ints_kernel(int *dst, const int *src, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) dst[i] = src[i];
}

hipError_t launch_fork(const ForkArgs &a, hipStream_t s) {
  // columns of a tile: as many as 32 KiB hold of every row, at most 64
  const int cols = std::min(std::min(64, kForkTile / a.n_seqs), a.max_pages);
  const int tiles = (a.max_pages + cols - 1) / cols;
  const size_t lds = (2 * (size_t)a.n_seqs + (size_t)a.n_seqs * cols) * sizeof(int);
  // counts written elsewhere: a small cache goes through one workgroup, which
  // puts them in place first; a larger one has a launch of its own for that
  const bool apart = a.ref_out != a.ref;
  const bool one = apart && (int64_t)a.n_seqs * a.max_pages + a.n_pages <= SCAN;
  if (apart && !one) {
    copy_ints_kernel<<<(a.n_pages + 255) / 256, 256, 0, s>>>(a.ref_out, a.ref, a.n_pages);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (one) fork_kernel<<<1, BIG, lds, s>>>(a, cols, 1);
  else fork_kernel<<<std::min(tiles, 1024), 256, lds, s>>>(a, cols, 0);
  return hipGetLastError();
}

// ---------------------------------------------------------------- reserve
// Room for n_new[s] more tokens of every sequence: pages past those it has,
// and a page of its own for a partly filled one that others hold too (the
// old one then goes on the copy list).  Of several sequences that write the
// same page, those counted first take a copy while anyone else is left, as if
// they came one after another.  All sequences get their pages or, where the
// cache or the table is too small, none does and only pos, the lists and
// state are written.
//
// One workgroup, a lane a sequence; the scan for free pages reads 64 KiB of
// counts a turn.
__global__ __launch_bounds__(BIG) void reserve_kernel(ReserveArgs a) {
  constexpr int KEEP = 4096;              // free pages that the counting scan keeps
  __shared__ int part[BIG / 64];
  __shared__ __align__(16) int pg[BIG];   // the partly filled page a sequence writes, or -1
  __shared__ int start[BIG];              // pages taken before the sequence's
  __shared__ int col0[BIG];               // the table column of its first
  __shared__ int mine[BIG];               // the first page it got
  __shared__ int freed[KEEP];
  __shared__ int bad;
  const int s = threadIdx.x, C = a.max_pages, ps = 1 << a.shift;
  const bool on = s < a.n_seqs;
  const int len0 = on ? a.len[s] : 0;
  const int add0 = on ? max(a.n_new[s], 0) : 0;
  if (s == 0) bad = 0;
  __syncthreads();
  // a length below zero, or one that grows past the table, fails the call
  const bool fits = len0 >= 0 && (int64_t)len0 + add0 <= ((int64_t)C << a.shift);
  if (add0 > 0 && !fits) bad = 1;
  const int len = fits ? len0 : 0, add = fits ? add0 : 0;
  const int have = (int)(((int64_t)len + ps - 1) >> a.shift);
  const int want = add > 0 ? (int)(((int64_t)len + add + ps - 1) >> a.shift) : have;
  const int slot = len & (ps - 1);
  const bool partly = add > 0 && slot != 0;
  int page = -1;
  if (partly) {
    page = a.table[(size_t)s * C + (len >> a.shift)];
    if (!is_page(page, a.n_pages)) page = -1;
  }
  const int others = page >= 0 ? a.ref[page] - 1 : 0;
  pg[s] = page;
  __syncthreads();
  int rank = 0;                           // writers of the page counted before this one
  if (others > 0) {
    for (int j = 0; j < (s & ~3); j += 4) {
      const int4 q = *(const int4 *)&pg[j];
      rank += (q.x == page) + (q.y == page) + (q.z == page) + (q.w == page);
    }
    for (int j = s & ~3; j < s; ++j) rank += pg[j] == page;
  }
  const bool copies = partly && (page < 0 || rank < others);
  const int need = (copies ? 1 : 0) + want - have;
  int total, n_moved;
  start[s] = block_scan(need, part, &total);
  col0[s] = copies ? len >> a.shift : have;
  const int moved = copies && page >= 0 ? 1 : 0;
  const int at = block_scan(moved, part, &n_moved);
  int found = 0;
  for (int p0 = 0; p0 < a.n_pages && found < total; p0 += SCAN) {
    const Picked k = pick(p0, a.n_pages, [&](int p) { return a.ref[p] == 0; }, part);
    each(k, p0, [&](int i, int p) { if (found + i < KEEP) freed[found + i] = p; });
    found += k.total;
  }
  __syncthreads();
  const bool go = found >= total && bad == 0;
  if (go && total > 0) {
    // page i of those taken goes to the last sequence whose run starts at or before i
    auto take = [&](int i, int p) {
      int lo = 0, hi = a.n_seqs - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (start[mid] <= i) lo = mid;
        else hi = mid - 1;
      }
      const int k = i - start[lo];
      a.table[(size_t)lo * C + col0[lo] + k] = p;
      a.ref[p] = 1;
      if (k == 0) mine[lo] = p;
    };
    if (total <= KEEP) {
      for (int i = s; i < total; i += BIG) take(i, freed[i]);
    } else {                              // a lane writes the counts of its own pages only
      int n = 0;
      for (int p0 = 0; p0 < a.n_pages && n < total; p0 += SCAN) {
        const Picked k = pick(p0, a.n_pages, [&](int p) { return a.ref[p] == 0; }, part);
        each(k, p0, [&](int i, int p) { if (n + i < total) take(n + i, p); });
        n += k.total;
      }
    }
  }
  __syncthreads();
  if (go && moved) atomicSub(&a.ref[page], 1);
  if (on) {
    // the list's entries, packed to its front, and nothing behind them
    const int n = go ? n_moved : 0;
    if (go && moved) {
      a.src[at] = page;
      a.dst[at] = mine[s];
      a.tokens[at] = slot;
    }
    if (s >= n) {
      a.src[s] = -1;
      a.dst[s] = -1;
      a.tokens[s] = 0;
    }
    a.pos[s] = go && add > 0 ? len : -1;
    if (go && add > 0) a.len[s] = len + add;
  }
  if (s == 0) {
    a.state[0] = go ? n_moved : 0;
    a.state[1] = go ? total : 0;
    a.state[2] = max(0, total - found);
    a.state[3] = bad;
  }
}

hipError_t launch_reserve(const ReserveArgs &a, hipStream_t s) {
  reserve_kernel<<<1, BIG, 0, s>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------- compact
// The n pages in use become pages 0 .. n - 1: the i-th page in use at or past
// n moves to the i-th free page before n.  Sources and destinations are
// disjoint, so the copies may run in any order.
__global__ __launch_bounds__(BIG) void compact_kernel(CompactArgs a) {
  __shared__ int part[BIG / 64];
  const int n = a.n_pages;
  auto live = [&](int p) { return a.ref[p] > 0; };
  int used = 0;
  for (int p0 = 0; p0 < n; p0 += SCAN) used += pick(p0, n, live, part).total;
  int movers = 0, holes = 0;
  for (int p0 = 0; p0 < n; p0 += SCAN) {
    const Picked m = pick(p0, n, [&](int p) { return p >= used && live(p); }, part);
    each(m, p0, [&](int i, int p) { a.src[movers + i] = p; });
    movers += m.total;
    const Picked h = pick(p0, n, [&](int p) { return p < used && !live(p); }, part);
    each(h, p0, [&](int i, int p) { a.dst[holes + i] = p; });
    holes += h.total;
  }
  for (int p = threadIdx.x; p < n; p += BIG) {
    const int r = a.ref[p];
    if (p < used || r <= 0) a.map[p] = r > 0 ? p : -1;
    if (a.ref_out != a.ref) a.ref_out[p] = r;
  }
  __threadfence();
  __syncthreads();
  for (int i = threadIdx.x; i < n / 2; i += BIG) {
    if (i < movers) {
      const int from = __hip_atomic_load(&a.src[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const int to = __hip_atomic_load(&a.dst[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      a.map[from] = to;
      const int r = a.ref[from];
      a.ref_out[to] = r;
      a.ref_out[from] = 0;
    } else {
      a.src[i] = -1;
      a.dst[i] = -1;
    }
  }
  if (threadIdx.x == 0) {
    a.state[0] = movers;
    a.state[1] = used;
    a.state[2] = 0;
    a.state[3] = 0;
  }
}

__global__ __launch_bounds__(256) void remap_kernel(int *out, const int *table, const int *map, int64_t n, int n_pages) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int p = table[i];
    out[i] = is_page(p, n_pages) ? map[p] : -1;
  }
}

hipError_t launch_compact(const CompactArgs &a, hipStream_t s) {
  compact_kernel<<<1, BIG, 0, s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t n = (int64_t)a.n_seqs * a.max_pages;
  remap_kernel<<<(unsigned)std::min<int64_t>((n + 255) / 256, 2048), 256, 0, s>>>(a.table_out, a.table, a.map, n,
                                                                                  a.n_pages);
  return hipGetLastError();
}

// ------------------------------------------------------------------- copy
// Entry i of the list: the first tokens[i] slots (all, without tokens) of
// page src[i] of every layer, key and value and head go to page dst[i].  A
// workgroup takes about 16 KiB of one page at a time: heads of one layer's
// keys or values.
__global__ __launch_bounds__(256) void page_copy_kernel(PageCopyArgs a, int heads, int parts) {
  const int per_entry = a.n_layers * 2 * parts;
  const int count = min(a.count != nullptr ? *a.count : a.capacity, a.capacity);
  const int64_t items = (int64_t)max(count, 0) * per_entry;
  const size_t head_bytes = (size_t)a.page_size * a.row_bytes, page_bytes = head_bytes * a.n_kv_heads;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int e = (int)(it / per_entry), r = (int)(it - (int64_t)e * per_entry);
    const int src = a.src[e], dst = a.dst[e];
    if (!is_page(src, a.n_pages) || !is_page(dst, a.n_pages)) continue;
    const int n = a.tokens != nullptr ? min(max(a.tokens[e], 0), a.page_size) : a.page_size;
    const int part = r % parts, kv = (r / parts) & 1, layer = r / (2 * parts);
    const int h0 = part * heads, hn = min(heads, a.n_kv_heads - h0);
    char *base = (char *)(kv ? a.v : a.k) + (size_t)layer * a.n_pages * page_bytes + h0 * head_bytes;
    const char *from = base + src * page_bytes;
    char *to = base + dst * page_bytes;
    const int vh = n * a.row_bytes / 16, all = vh * hn;
    for (int i0 = threadIdx.x; i0 < all; i0 += 4 * 256) {
      uint4 x[4];
      size_t off[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + k * 256;
        if (i < all) {
          const int h = i / vh;
          off[k] = h * head_bytes + (size_t)(i - h * vh) * 16;
          x[k] = *(const uint4 *)(from + off[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i0 + k * 256 < all) *(uint4 *)(to + off[k]) = x[k];
    }
  }
}

hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t s) {
  const int64_t head_bytes = (int64_t)a.page_size * a.row_bytes;
  const int heads = (int)std::min<int64_t>(a.n_kv_heads, std::max<int64_t>(1, (16 << 10) / head_bytes));
  const int parts = (a.n_kv_heads + heads - 1) / heads;
  const int64_t items = (int64_t)a.capacity * a.n_layers * 2 * parts;
  page_copy_kernel<<<(unsigned)std::min<int64_t>(items, 2048), 256, 0, s>>>(a, heads, parts);
  return hipGetLastError();
}

}  // namespace dex
