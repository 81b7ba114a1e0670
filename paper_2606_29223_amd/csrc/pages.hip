// Page tables of a paged cache: fork and free, reserve with copy on write,
// compaction, and the copies of pages they ask for.
//
// Tables are small: all of a step's kernels but the copy are bound by the
// latency of a few dependent loads, so they take few launches and ask for
// everything they can at once.  64 rows of 58 pages: fork 2.9 us, reserve 5.9;
// compaction of 4096 pages 7.5 and its table 4.6.
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

constexpr int BIG = 1024;                 // lanes of a one-workgroup kernel at most
constexpr int kForkTile = 8192;           // table entries of a fork tile (32 KiB of LDS)
constexpr int kForkSmall = 8192;          // table entries, and pages, that one workgroup forks

__device__ __forceinline__ bool is_page(int p, int n_pages) { return p >= 0 && p < n_pages; }

// Sums of two numbers a wave over the workgroup's W waves: before this wave's,
// and in all.  `part` is one of two, in turns: a call's barrier also ends the
// reads of the call before the last.
struct Sums {
  int before_a, all_a, before_b, all_b;
};
template <int W>
__device__ __forceinline__ Sums wave_sums(int a, int b, int (&part)[2][W]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) {
    part[0][wave] = a;
    part[1][wave] = b;
  }
  __syncthreads();
  Sums s = {0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int x = part[0][w], y = part[1][w];
    if (w < wave) {
      s.before_a += x;
      s.before_b += y;
    }
    s.all_a += x;
    s.all_b += y;
  }
  return s;
}
__device__ __forceinline__ int wave_scan(int v) {           // inclusive, over a wave
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  return v;
}

// Which of a turn's pages a predicate picks, as ballots.  A turn is W * 64 *
// GROUPS pages from p0 on; a wave takes `span` <= GROUPS groups of 64
// neighbours, so that few pages spread over all waves.
template <int GROUPS>
struct Picked {
  unsigned long long m[GROUPS];
  __device__ __forceinline__ int count() const {
    int n = 0;
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) n += __popcll(m[j]);
    return n;
  }
};
template <int W, int GROUPS>
struct Pages {
  static constexpr int kTurn = W * 64 * GROUPS;
  int n, span;
  __device__ __forceinline__ explicit Pages(int n_pages) : n(n_pages), span(min(GROUPS, (n_pages + W * 64 - 1) / (W * 64))) {}
  __device__ __forceinline__ int first(int p0, int j) const { return p0 + ((int)(threadIdx.x >> 6) * span + j) * 64; }
  __device__ __forceinline__ bool here(int p0, int j, int *p) const {
    *p = first(p0, j) + (int)(threadIdx.x & 63);
    return j < span && *p < n;
  }
  template <typename Pred>
  __device__ __forceinline__ Picked<GROUPS> pick(int p0, Pred pred) const {
    Picked<GROUPS> k;
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      int p;
      k.m[j] = __ballot(here(p0, j, &p) && pred(p));
    }
    return k;
  }
  // f(index among the picked, page) for each, `base` of them before this wave's
  template <typename F>
  __device__ __forceinline__ void each(const Picked<GROUPS> &k, int p0, int base, F f) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      if (k.m[j] == 0) continue;
      if (k.m[j] >> lane & 1) f(base + __popcll(k.m[j] & ((1ull << lane) - 1)), first(p0, j) + lane);
      base += __popcll(k.m[j]);
    }
  }
};

}  // namespace

// ------------------------------------------------------------------- fork
// Row s of the new table is row parent[s] of the old one (nothing, where
// parent[s] names no row); a page's count changes by (children - 1) for every
// old row that held it.  A workgroup takes a tile of columns of every row
// through LDS, so the table may be written over itself.
__global__ __launch_bounds__(256) void fork_kernel(ForkArgs a, int cols) {
  extern __shared__ int lds[];
  int *children = lds, *par = lds + a.n_seqs, *tile = par + a.n_seqs;
  const int S = a.n_seqs, C = a.max_pages, nt = 256;
  for (int s = threadIdx.x; s < S; s += nt) {
    const int p = a.parent[s];
    children[s] = 0;
    par[s] = p >= 0 && p < S ? p : -1;
    if (blockIdx.x == 0) tile[s] = a.len[s];
  }
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

// The same for a cache whose table and counts fit one workgroup's LDS (a
// decoding step of a hundred beams): everything is requested at once, and the
// counts change in LDS, where a page that many rows hold costs no round trips.
__global__ __launch_bounds__(BIG) void fork_small_kernel(ForkArgs a) {
  constexpr int PER = kForkSmall / BIG;
  __shared__ int children[BIG], par[BIG], lens[BIG];
  __shared__ int tile[kForkSmall], delta[kForkSmall];
  const int t = threadIdx.x, S = a.n_seqs, C = a.max_pages, n = S * C;
  int page[PER], ref[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = t + k * BIG;
    page[k] = i < n ? a.table[i] : -1;
    ref[k] = i < a.n_pages ? a.ref[i] : 0;
  }
  if (t < S) {
    const int p = a.parent[t];
    par[t] = p >= 0 && p < S ? p : -1;
    lens[t] = a.len[t];
    children[t] = 0;
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    tile[t + k * BIG] = page[k];
    delta[t + k * BIG] = 0;
  }
  __syncthreads();
  if (t < S) {
    const int p = par[t];
    if (p >= 0) atomicAdd(&children[p], 1);
    a.len_out[t] = p >= 0 ? lens[p] : 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = t + k * BIG;
    if (i >= n) break;
    const int s = i / C, d = children[s] - 1, p = par[s];
    if (d != 0 && is_page(page[k], a.n_pages)) atomicAdd(&delta[page[k]], d);
    a.table_out[i] = p >= 0 ? tile[p * C + (i - s * C)] : -1;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = t + k * BIG;
    if (i < a.n_pages) a.ref_out[i] = ref[k] + delta[i];
  }
}

__global__ __launch_bounds__(256) void copy_ints_kernel(int *dst, const int *src, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) dst[i] = src[i];
}

hipError_t launch_fork(const ForkArgs &a, hipStream_t s) {
  if ((int64_t)a.n_seqs * a.max_pages <= kForkSmall && a.n_pages <= kForkSmall) {
    fork_small_kernel<<<1, BIG, 0, s>>>(a);
    return hipGetLastError();
  }
  if (a.ref_out != a.ref) {               // the counts in place before their changes
    copy_ints_kernel<<<(a.n_pages + 255) / 256, 256, 0, s>>>(a.ref_out, a.ref, a.n_pages);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // columns of a tile: as many as 32 KiB hold of every row, at most 64
  const int cols = std::min(std::min(64, kForkTile / a.n_seqs), a.max_pages);
  const int tiles = (a.max_pages + cols - 1) / cols;
  const size_t lds = (2 * (size_t)a.n_seqs + (size_t)a.n_seqs * cols) * sizeof(int);
  fork_kernel<<<std::min(tiles, 1024), 256, lds, s>>>(a, cols);
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
template <int W>
__global__ __launch_bounds__(W * 64) void reserve_kernel(ReserveArgs a) {
  constexpr int KEEP = 4096;              // free pages that the counting scan keeps
  constexpr int BIG = W * 64;
  __shared__ int part[2][2][W];
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
  const Pages<W, 16> pages(a.n_pages);
  auto is_free = [&](int p) { return a.ref[p] == 0; };
  // a length below zero, or one that grows past the table, fails the call
  const bool fits = len0 >= 0 && (int64_t)len0 + add0 <= ((int64_t)C << a.shift);
  const int len = fits ? len0 : 0, add = fits ? add0 : 0;
  const int have = (int)(((int64_t)len + ps - 1) >> a.shift);
  const int want = add > 0 ? (int)(((int64_t)len + add + ps - 1) >> a.shift) : have;
  const int slot = len & (ps - 1);
  const bool partly = add > 0 && slot != 0;
  int page = -1;
  if (partly) page = a.table[(size_t)s * C + (len >> a.shift)];
  const Picked<16> k0 = pages.pick(0, is_free);             // meanwhile
  if (!is_page(page, a.n_pages)) page = -1;
  const int others = page >= 0 ? a.ref[page] - 1 : 0;
  if (s == 0) bad = 0;
  pg[s] = page;
  __syncthreads();
  if (add0 > 0 && !fits) bad = 1;
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
  const bool moved = copies && page >= 0;
  const unsigned long long movers = __ballot(moved);
  const int needed = wave_scan(need);
  const Sums sum = wave_sums(__shfl(needed, 63, 64), __popcll(movers), part[0]);
  const int total = sum.all_a, n_moved = sum.all_b;
  const int at = sum.before_b + __popcll(movers & ((1ull << (s & 63)) - 1));
  start[s] = sum.before_a + needed - need;
  col0[s] = copies ? len >> a.shift : have;
  int found = 0, turn = 1;
  for (int p0 = 0; p0 < a.n_pages && found < total; p0 += pages.kTurn) {
    const Picked<16> k = p0 == 0 ? k0 : pages.pick(p0, is_free);
    const Sums f = wave_sums(k.count(), 0, part[turn]);
    turn ^= 1;
    pages.each(k, p0, found + f.before_a, [&](int i, int p) { if (i < KEEP) freed[i] = p; });
    found += f.all_a;
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
      for (int p0 = 0; p0 < a.n_pages && n < total; p0 += pages.kTurn) {
        const Picked<16> k = pages.pick(p0, is_free);
        const Sums f = wave_sums(k.count(), 0, part[turn]);
        turn ^= 1;
        pages.each(k, p0, n + f.before_a, [&](int i, int p) { if (i < total) take(i, p); });
        n += f.all_a;
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
  // four waves where they suffice: barriers among sixteen take longer
  if (a.n_seqs <= 256 && a.n_pages <= (Pages<4, 16>::kTurn)) reserve_kernel<4><<<1, 256, 0, s>>>(a);
  else reserve_kernel<16><<<1, BIG, 0, s>>>(a);
  return hipGetLastError();
}

// ---------------------------------------------------------------- compact
// The n pages in use become pages 0 .. n - 1: the i-th page in use at or past
// n moves to the i-th free page before n.  Sources and destinations are
// disjoint, so the copies may run in any order.
__global__ __launch_bounds__(BIG) void compact_kernel(CompactArgs a) {
  constexpr int W = BIG / 64, GROUPS = 4;      // more groups a lane and their addresses fill the registers
  __shared__ int part[2][2][W];
  const int n = a.n_pages, lane = threadIdx.x & 63;
  const Pages<W, GROUPS> pages(n);
  auto live = [&](int p) { return a.ref[p] > 0; };
  const Picked<GROUPS> k0 = pages.pick(0, live);
  int used = 0, turn = 0;
  for (int p0 = 0; p0 < n; p0 += pages.kTurn) {
    used += wave_sums<W>((p0 == 0 ? k0 : pages.pick(p0, live)).count(), 0, part[turn]).all_a;
    turn ^= 1;
  }
  int movers = 0, holes = 0;
  for (int p0 = 0; p0 < n; p0 += pages.kTurn) {
    const Picked<GROUPS> k = p0 == 0 ? k0 : pages.pick(p0, live);
    if (a.ref_out != a.ref) {
      int r[GROUPS];
#pragma unroll
      for (int j = 0; j < GROUPS; ++j) {
        int p;
        r[j] = pages.here(p0, j, &p) ? a.ref[p] : 0;
      }
#pragma unroll
      for (int j = 0; j < GROUPS; ++j) {
        int p;
        if (pages.here(p0, j, &p)) a.ref_out[p] = r[j];
      }
    }
    Picked<GROUPS> m, h;                          // in use at or past `used`, free before it
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const int before = j < pages.span ? min(max(used - pages.first(p0, j), 0), 64) : 0;
      const unsigned long long low = before == 64 ? ~0ull : (1ull << before) - 1;
      m.m[j] = k.m[j] & ~low;
      h.m[j] = ~k.m[j] & low;
      int p;
      if (pages.here(p0, j, &p) && !(m.m[j] >> lane & 1)) a.map[p] = k.m[j] >> lane & 1 ? p : -1;
    }
    const Sums f = wave_sums<W>(m.count(), h.count(), part[turn]);
    turn ^= 1;
    pages.each(m, p0, movers + f.before_a, [&](int i, int p) { a.src[i] = p; });
    pages.each(h, p0, holes + f.before_b, [&](int i, int p) { a.dst[i] = p; });
    movers += f.all_a;
    holes += f.all_b;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n / 2; i += BIG) {
    if (i < movers) {
      const int from = a.src[i], to = a.dst[i];
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
// keys or values, four 16-byte loads a lane on their way.  Bound by memory: 40
// part pages of 32 layers (70 MB read and written) 14 us, 5.0 TB/s; 1000 pages
// of 12 layers (1.18 GB) 246 us, 4.8 TB/s, as a large copy.
__global__ __launch_bounds__(256) void page_copy_kernel(PageCopyArgs a, int heads, int parts) {
  const int count = min(a.count != nullptr ? *a.count : a.capacity, a.capacity);
  const int part = blockIdx.x % parts, kv = blockIdx.x / parts & 1, layer = blockIdx.x / parts >> 1;
  const size_t head_bytes = (size_t)a.page_size * a.row_bytes, page_bytes = head_bytes * a.n_kv_heads;
  const int h0 = part * heads, hn = min(heads, a.n_kv_heads - h0);
  char *base = (char *)(kv ? a.v : a.k) + (size_t)layer * a.n_pages * page_bytes + h0 * head_bytes;
  for (int e = blockIdx.y; e < count; e += gridDim.y) {
    const int src = a.src[e], dst = a.dst[e];
    const int n = a.tokens != nullptr ? min(max(a.tokens[e], 0), a.page_size) : a.page_size;
    if (!is_page(src, a.n_pages) || !is_page(dst, a.n_pages)) continue;
    const char *from = base + src * page_bytes;
    char *to = base + dst * page_bytes;
    const int vh = n * a.row_bytes / 16, all = vh * hn;
    for (int i0 = threadIdx.x; i0 < all; i0 += 4 * 256) {
      // four loads on their way before the first store; those past the end
      // repeat the last and are not stored
      auto off = [&](int k) {
        const int i = min(i0 + k * 256, all - 1), h = i / vh;
        return h * head_bytes + (size_t)(i - h * vh) * 16;
      };
      const size_t o0 = off(0), o1 = off(1), o2 = off(2), o3 = off(3);
      const uint4 x0 = *(const uint4 *)(from + o0), x1 = *(const uint4 *)(from + o1);
      const uint4 x2 = *(const uint4 *)(from + o2), x3 = *(const uint4 *)(from + o3);
      *(uint4 *)(to + o0) = x0;
      if (i0 + 256 < all) *(uint4 *)(to + o1) = x1;
      if (i0 + 512 < all) *(uint4 *)(to + o2) = x2;
      if (i0 + 768 < all) *(uint4 *)(to + o3) = x3;
    }
  }
}

hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t s) {
  const int64_t head_bytes = (int64_t)a.page_size * a.row_bytes;
  const int heads = (int)std::min<int64_t>(a.n_kv_heads, std::max<int64_t>(1, (16 << 10) / head_bytes));
  const int parts = (a.n_kv_heads + heads - 1) / heads;
  // a column of workgroups a piece of a page, its entries dealt to about 8192
  // workgroups in all (the list's length is known on the device only)
  const int64_t pieces = (int64_t)a.n_layers * 2 * parts;
  const int64_t rows = std::min<int64_t>(a.capacity, std::max<int64_t>(1, 8192 / pieces));
  page_copy_kernel<<<dim3((unsigned)pieces, (unsigned)rows), 256, 0, s>>>(a, heads, parts);
  return hipGetLastError();
}

}  // namespace dex
