// Trees of drafted tokens: masks, the accepted path, its keys and values moved
// behind the sequence, and pages given back.
//
// But for the moved rows these are a few hundred integers and bounded by the
// latency of a launch and of their loads one after the other: 16 trees of 64,
// masks 2.5 us, paths 3.4, rows of 32 layers x 8 heads 6.2 (4.7 MB read and written),
// pages 5.2.  Moved rows of a long list are a copy, bounded by memory: 192 lists of up
// to 1999 fp32 rows of 64 into new pages 70 us, 300 MB, 4.3 TB/s.
#include "dex.h"
#include "dex_kernels.h"
#include "span.h"

#include <algorithm>

namespace dex {

namespace {

// A node's parent, or -1: parents come before their children, so that no chain
// has a cycle.
__device__ __forceinline__ int parent_of(int p, int i) { return p >= 0 && p < i ? p : -1; }

// A lane a node walks to its root: mask[i] = bits of the nodes on the way.  The
// parents are in LDS, so a step is one LDS read: 256 nodes 2.7 us as a binary tree,
// 18.6 as one chain.
__global__ __launch_bounds__(kMaxDraft) void tree_mask_kernel(TreeMaskArgs a) {
  __shared__ int parent[kMaxDraft];
  const int i = threadIdx.x;
  const size_t at = (size_t)blockIdx.x * a.draft + i;
  if (i < a.draft) parent[i] = parent_of(a.parent[at], i);
  __syncthreads();
  if (i >= a.draft) return;
  uint64_t bits[kMaxDraft / 64] = {};
  int depth = -1;
  for (int j = i; j >= 0; j = parent[j]) {
    ++depth;
#pragma unroll
    for (int w = 0; w < kMaxDraft / 64; ++w)
      if (j >> 6 == w) bits[w] |= 1ull << (j & 63);
  }
#pragma unroll
  for (int w = 0; w < kMaxDraft / 64; ++w)
    if (w < a.words) a.mask[at * a.words + w] = bits[w];
  if (a.depth != nullptr) a.depth[at] = depth;
}

// A lane a node walks to its root and sees whether every token on the way is
// the one wanted; the deepest such node wins, the lowest number among equals.  A
// node's own token is looked at first, so that a step of the way is one LDS read:
// 256 nodes 2.8 us as a binary tree, 30 as one chain that is accepted.
__global__ __launch_bounds__(kMaxDraft) void tree_accept_kernel(TreeAcceptArgs a) {
  constexpr int kUnwanted = -2;
  __shared__ int up[kMaxDraft], target[kMaxDraft], path[kMaxDraft], best;
  const int i = threadIdx.x, b = blockIdx.x;
  const size_t at = (size_t)b * a.draft + i;
  const int n = a.n_draft != nullptr ? max(0, min(a.n_draft[b], a.draft)) : a.draft;
  const int root = a.root != nullptr ? a.root[b] : -1;
  int parent = -1, token = 0;
  if (i < a.draft) {
    parent = parent_of(a.parent[at], i);
    token = a.token[at];
    target[i] = a.target[at];
  }
  path[i] = -1;
  if (i == 0) best = 0;
  __syncthreads();
  // its parent, if its token is the one wanted
  const bool own = i < n && (parent >= 0 ? token == target[parent] : a.root == nullptr || token == root);
  up[i] = own ? parent : kUnwanted;
  __syncthreads();
  if (own) {
    int depth = 1, j = parent;
    for (; j >= 0; j = up[j]) ++depth;
    if (j != kUnwanted) atomicMax(&best, depth << 16 | (0xffff - i));
  }
  __syncthreads();
  const int depth = best >> 16, last = 0xffff - (best & 0xffff);
  if (i == 0) {
    int at_depth = depth;
    if (depth > 0)
      for (int j = last; j >= 0; j = up[j]) path[--at_depth] = j;
    a.count[b] = depth;
    a.next[b] = depth > 0 ? target[last] : root;
  }
  __syncthreads();
  if (i < a.draft) a.path[at] = path[i];
}

// Entries of `pairs` neighbouring (layer, kv head)s of a sequence, a slice of
// their rows' 16-byte chunks.  In place the entries go in turns: a turn's loads
// are all done before its first store, and a source is never before its own
// destination, so it is behind all earlier ones and no store overtakes a load.
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void keep_kernel(KeepArgs a, int lanes, int slices, int pairs, int groups, int turns) {
  typedef __attribute__((ext_vector_type(4))) uint32_t chunk_t;
  const int kv = a.map.n_kv_heads;
  int x = blockIdx.x;
  const int slice = x % slices;
  x /= slices;
  const int pair0 = x % groups * pairs, s = x / groups, n_pairs = min(pairs, a.n_layers * kv - pair0);
  const int n = min(a.count[s], a.capacity);
  const int first = a.first != nullptr ? a.first[s] : 0;
  if (first < 0 || n <= 0) return;
  const bool in_place = a.to == nullptr;
  PageMap to = a.map;
  if (!in_place) to.table = a.to, to.max_pages = a.to_pages;
  const size_t layer_rows = (size_t)a.map.n_pages * kv << a.map.shift;
  // entries of the pairs one after the other, `per` of them a turn (a list of more
  // than 256 has one pair)
  const int per = THREADS * EACH / lanes, entries = n_pairs * n;
  const int e_first = blockIdx.y * turns * per, e_end = min((int64_t)entries, (int64_t)e_first + (int64_t)turns * per);
  for (int e0 = e_first; e0 < e_end; e0 += per) {
    chunk_t k[EACH], v[EACH];
    size_t dst[EACH];
    bool go[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int item = e * THREADS + threadIdx.x, in_turn = item / lanes, chunk = slice * lanes + item - in_turn * lanes;
      const int entry = e0 + in_turn, in_pairs = pairs > 1 ? entry / n : 0, j = entry - in_pairs * n;
      const int pair = pair0 + in_pairs, layer = pair / kv, head = pair - layer * kv;
      go[e] = in_turn < per && entry < e_end && chunk * 16 < a.row_bytes;
      uint32_t from = kNoRow, into = kNoRow;
      if (go[e]) {
        const int i = a.index[layer * a.index_layer + s * a.index_seq + head * a.index_head + j];
        if (i >= 0 && i <= (1 << 30) && first <= (1 << 30) && !(in_place && i <= j)) {
          from = page_row(a.map, s, first + i, head);
          into = page_row(to, s, first + j, head);
        }
      }
      go[e] = from != kNoRow && into != kNoRow;
      // (one that copies nothing reads the pools' first row)
      const size_t at = layer * layer_rows, src = go[e] ? (at + from) * a.row_bytes + chunk * 16 : 0;
      dst[e] = go[e] ? (at + into) * a.row_bytes + chunk * 16 : 0;
      k[e] = *(const chunk_t *)((const char *)a.k + src);
      v[e] = *(const chunk_t *)((const char *)a.v + src);
    }
    if (in_place) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (go[e]) {
        *(chunk_t *)((char *)a.k + dst[e]) = k[e];
        *(chunk_t *)((char *)a.v + dst[e]) = v[e];
      }
  }
}

// Pages behind a sequence's last token leave its row of the table.  Small tables
// go through one workgroup, which copies the counts first.
constexpr int kTrimSmall = 16384, kTrimThreads = 1024;
__device__ __forceinline__ void trim_entry(const TrimArgs &a, int64_t e) {
  const int s = (int)(e / a.max_pages), c = (int)(e - (int64_t)s * a.max_pages);
  int p = a.table[e];
  if ((int64_t)c << a.shift >= max(0, a.len[s])) {
    if (p >= 0 && p < a.n_pages) atomicSub(&a.ref_out[p], 1);
    p = -1;
  }
  a.table_out[e] = p;
}
__global__ __launch_bounds__(kTrimThreads) void trim_small_kernel(TrimArgs a) {
  if (a.ref_out != a.ref) {
    for (int p = threadIdx.x; p < a.n_pages; p += kTrimThreads) a.ref_out[p] = a.ref[p];
    __threadfence();                      // the counts are where the atomics see them
    __syncthreads();
  }
  for (int e = threadIdx.x; e < a.n_seqs * a.max_pages; e += kTrimThreads) trim_entry(a, e);
}
__global__ __launch_bounds__(256) void trim_copy_kernel(TrimArgs a) {
  for (int p = blockIdx.x * 256 + threadIdx.x; p < a.n_pages; p += gridDim.x * 256) a.ref_out[p] = a.ref[p];
}
__global__ __launch_bounds__(256) void trim_kernel(TrimArgs a) {
  const int64_t entries = (int64_t)a.n_seqs * a.max_pages;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += (int64_t)gridDim.x * 256) trim_entry(a, e);
}

// How a call's lists are cut.  Short lists (a tree's path) take several pairs a
// workgroup, as long as there are 512 workgroups: 4 lists of 200 in 8 heads 67 us
// with eight pairs, 10 with one.  Long ones in place go in turns of as much as
// 1024 threads hold, in slices of 128 bytes, or of 64 where those are fewer than
// 256 workgroups: 128 lists of 2000 of bf16 rows of 128 53 us (4.9 TB/s; 76 with
// the narrow ones), 16 of 4000 32 (51 with the wide ones).  What does not wait for
// itself has few loads a thread and many workgroups: 192 lists of up to 1999 fp32
// rows of 64 into new pages 70 us with two of 16 bytes, 79 with eight.
struct KeepGrid {
  bool turn;
  int lanes, slices, pairs, split, turns;
  int64_t groups, blocks;
};
KeepGrid keep_grid(const KeepArgs &a) {
  KeepGrid g;
  const int chunks = a.row_bytes / 16;
  const int64_t all = (int64_t)a.n_layers * a.map.n_kv_heads, rows = all * a.map.n_seqs;
  const bool in_place = a.to == nullptr, brief = a.capacity <= 256;
  g.turn = in_place && !brief;
  const int wide = std::min(chunks, 8), narrow = std::min(chunks, 4);
  g.lanes = !g.turn ? chunks : rows * ((chunks + wide - 1) / wide) >= 256 ? wide : narrow;
  g.slices = (chunks + g.lanes - 1) / g.lanes;
  g.pairs = brief ? (int)std::max<int64_t>(1, std::min<int64_t>(8, rows / 512)) : 1;
  g.groups = (all + g.pairs - 1) / g.pairs;
  g.blocks = (int64_t)a.map.n_seqs * g.groups * g.slices;
  const int per = (g.turn ? 1024 * 4 : 512 * 2) / g.lanes, most = (int)(((int64_t)g.pairs * a.capacity + per - 1) / per);
  g.split = in_place ? 1 : std::min(most, 65535);
  g.turns = (most + g.split - 1) / g.split;
  return g;
}

}  // namespace

bool keep_fits(const KeepArgs &a) {
  const KeepGrid g = keep_grid(a);
  return launch_fits(g.blocks, g.turn ? 1024 : 512);
}

hipError_t launch_tree_mask(const TreeMaskArgs &a, hipStream_t s) {
  tree_mask_kernel<<<a.n, (a.draft + 63) / 64 * 64, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_tree_accept(const TreeAcceptArgs &a, hipStream_t s) {
  tree_accept_kernel<<<a.n, kMaxDraft, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_keep(const KeepArgs &a, hipStream_t s) {
  const KeepGrid g = keep_grid(a);
  const dim3 grid((unsigned)g.blocks, g.split);
  if (g.turn) keep_kernel<1024, 4><<<grid, 1024, 0, s>>>(a, g.lanes, g.slices, g.pairs, (int)g.groups, g.turns);
  else keep_kernel<512, 2><<<grid, 512, 0, s>>>(a, g.lanes, g.slices, g.pairs, (int)g.groups, g.turns);
  return hipGetLastError();
}

hipError_t launch_trim(const TrimArgs &a, hipStream_t s) {
  if (a.n_pages <= kTrimSmall && (int64_t)a.n_seqs * a.max_pages <= kTrimSmall) {
    trim_small_kernel<<<1, kTrimThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  hipError_t e = hipSuccess;
  if (a.ref_out != a.ref) {
    trim_copy_kernel<<<std::min((a.n_pages + 255) / 256, 1024), 256, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t entries = (int64_t)a.n_seqs * a.max_pages;
  trim_kernel<<<(unsigned)std::min<int64_t>((entries + 255) / 256, 2048), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dex
