// Pages that a cheap score selects, and keys that accumulated weights keep.
//
// Bounds of a page are the least and the largest of its keys in every
// dimension; a query's product with a key of the page is at most
//   sum_d max(q_d min_d, q_d max_d) = sum_d q+_d max_d + q-_d min_d,
// q+ and q- its positive and negative parts, and the sum of that over the query
// heads of a kv head is the page's score: one vector a (row, kv head), its
// heads' parts summed.  Scores decide whole numbers, so they are in double.
//
// On one MI355X: the bounds of 32 rows' last pages 5.0 us and of a whole step's
// pages a stream over their keys; the scores of 32 ragged rows up to 16000 keys in
// pages of 32, 8 kv heads of 128, 18 us for 20 MB: 696 of 2048 workgroups have pages,
// and as a row has eight parts, part p of every row is on one XCD, 256 of the 696
// on the first and 8 on the last.  The choice of 64 of up to 500 pages 9.8 us and of
// 1999 of up to 9000 keys 27 (192 lists), by the latency of the passes: range, one or
// two digits, places, with barriers between.
#include "dex.h"
#include "dex_kernels.h"
#include "span.h"

#include <algorithm>

namespace dex {

namespace {

constexpr int THREADS = 256;

template <typename T>
struct Chunk {                            // 16 bytes of T
  static constexpr int N = 16 / sizeof(T);
  uint4 raw;
  __device__ __forceinline__ float get(int i) const {
    T t[N];
    __builtin_memcpy(t, &raw, 16);
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)t[i] << 16);
    else return t[i];
  }
};

// ------------------------------------------------------------------ bounds
// A wave a (page, kv head): HD sizeof(T) / 16 lanes a key.
template <typename T, int HD>
__global__ __launch_bounds__(THREADS) void bounds_kernel(BoundsArgs a, int items) {
  constexpr int N = 16 / sizeof(T), LPR = HD / N, ROWS = 64 / LPR;
  const int lane = threadIdx.x & 63, kv = a.map.n_kv_heads, ps = 1 << a.map.shift;
  const int64_t id = (int64_t)blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
  const int s = (int)(id / items), item = (int)(id - (int64_t)s * items), head = item % kv;
  if (s >= a.map.n_seqs) return;
  const int64_t cap = (int64_t)a.map.max_pages << a.map.shift;
  const int len = (int)min((int64_t)max(a.len[s], 0), cap);
  const int c = (len > a.n_new ? len - a.n_new : 0) / ps + item / kv;
  if ((int64_t)c * ps >= len) return;
  const int page = a.map.table[(size_t)s * a.map.max_pages + c];
  if (page < 0 || page >= a.map.n_pages) return;
  const int n = min(ps, len - c * ps), d = lane % LPR;
  const size_t at = ((size_t)page * kv + head) << a.map.shift;
  const T *keys = (const T *)a.k + at * HD + d * N;
  float lo[N], hi[N];
#pragma unroll
  for (int i = 0; i < N; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
#pragma unroll 4
  for (int j = lane / LPR; j < n; j += ROWS) {
    Chunk<T> x;
    x.raw = *(const uint4 *)(keys + (size_t)j * HD);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      lo[i] = fminf(lo[i], x.get(i));
      hi[i] = fmaxf(hi[i], x.get(i));
    }
  }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      lo[i] = fminf(lo[i], __shfl_xor(lo[i], o, 64));
      hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], o, 64));
    }
  if (lane >= 2 * LPR) return;
  // lanes of the first row write the least, those of the second the largest
  T out[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = lane < LPR ? lo[i] : hi[i], x = lo[i] > hi[i] ? NAN : y;     // (inverted: all were NaN)
    if constexpr (sizeof(T) == 2) out[i] = (uint16_t)(__float_as_uint(x) >> 16);
    else out[i] = x;
  }
  uint4 raw;
  __builtin_memcpy(&raw, out, 16);
  *(uint4 *)((T *)a.bounds + (((size_t)page * kv + head) * 2 + lane / LPR) * HD + d * N) = raw;
}

// ------------------------------------------------------------------- scores
// A key that orders scores: larger is better, 0 is no page, the largest is kept
// whatever its score.  A NaN counts as infinity.
__device__ __forceinline__ uint64_t order_of(double x) {
  if (x != x) x = INFINITY;
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ uint32_t order_of(float x) {
  if (x != x) x = INFINITY;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? ~u : u | 1u << 31;
}

struct Row {
  int seq, len, columns;
};
__device__ __forceinline__ Row row_of(const SelectArgs &a, int r) {
  Row x;
  x.seq = a.seq != nullptr ? a.seq[r] : r;
  const bool is = x.seq >= 0 && x.seq < a.map.n_seqs;
  x.len = is ? max(0, min(min(a.len[r], a.max_len), a.map.max_pages << a.map.shift)) : 0;
  x.columns = (x.len + (1 << a.map.shift) - 1) >> a.map.shift;
  return x;
}

// LPR lanes a page, a lane N dimensions of its least and largest keys.  A
// workgroup asks for all its pages' bounds at once: the kernel is the latency of
// the chain length, table, bounds, and their stream.
constexpr int SCORE_EACH = 4;             // pages a lane
template <typename T, int HD>
__global__ __launch_bounds__(THREADS) void score_kernel(SelectArgs a, int stride, int parts, bool whole) {
  constexpr int N = 16 / sizeof(T), LPR = HD / N, PAGES = THREADS / LPR;
  const int kv = a.map.n_kv_heads, G = a.n_heads / kv, row = blockIdx.x / parts, head = row % kv, r = row / kv;
  const Row x = row_of(a, r);
  const int first = (blockIdx.x - row * parts) * PAGES * SCORE_EACH + threadIdx.x / LPR;
  if (first - (int)threadIdx.x / LPR >= x.columns) return;
  const int d = threadIdx.x % LPR;
  Chunk<T> lo[SCORE_EACH], hi[SCORE_EACH];
  bool there[SCORE_EACH];
  int page[SCORE_EACH];
#pragma unroll
  for (int e = 0; e < SCORE_EACH; ++e) {
    const int c = first + e * PAGES;
    page[e] = a.map.table[(size_t)x.seq * a.map.max_pages + min(c, x.columns - 1)];
    there[e] = c < x.columns && page[e] >= 0 && page[e] < a.map.n_pages;
  }
  const T *src = (const T *)a.q + (int64_t)r * a.q_row + (int64_t)head * G * a.q_head + d * N;
  auto query = [&](int g) {
    const T *from = src + min(g, G - 1) * a.q_head;
    Chunk<T> q;
    if (whole) {
      q.raw = *(const uint4 *)from;
    } else {
      T t[N];
#pragma unroll
      for (int i = 0; i < N; ++i) t[i] = from[i];
      __builtin_memcpy(&q.raw, t, 16);
    }
    return q;
  };
  // (four heads' queries are asked for before the first is looked at)
  constexpr int HEADS = 4;
  Chunk<T> q[HEADS];
#pragma unroll
  for (int j = 0; j < HEADS; ++j) q[j] = query(j);
#pragma unroll
  for (int e = 0; e < SCORE_EACH; ++e) {
    const T *b = (const T *)a.bounds + ((size_t)(there[e] ? page[e] : 0) * kv + head) * 2 * HD + d * N;
    lo[e].raw = *(const uint4 *)b;
    hi[e].raw = *(const uint4 *)(b + HD);
  }
  double up[N], down[N];                  // q+ and q-, of all the kv head's heads
#pragma unroll
  for (int i = 0; i < N; ++i) up[i] = down[i] = 0.0;
  for (int g = 0; g < G; g += HEADS) {
#pragma unroll
    for (int j = 0; j < HEADS; ++j) {
      if (g + j >= G) break;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float v = q[j].get(i);
        up[i] += v < 0.f ? 0.f : v;       // (a NaN goes on in both)
        down[i] += v > 0.f ? 0.f : v;
      }
    }
    if (g + HEADS < G) {
#pragma unroll
      for (int j = 0; j < HEADS; ++j) q[j] = query(g + HEADS + j);
    }
  }
  // a part of 0 adds nothing, whatever the bound (0 times infinity is not 0)
  uint32_t some_up[N], some_down[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    some_up[i] = up[i] == 0.0 ? 0u : ~0u;
    some_down[i] = down[i] == 0.0 ? 0u : ~0u;
  }
  uint64_t *keys = (uint64_t *)a.work + (size_t)row * stride;
#pragma unroll
  for (int e = 0; e < SCORE_EACH; ++e) {
    const int c = first + e * PAGES;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float l = lo[e].get(i), h = hi[e].get(i);
      const uint32_t least = __float_as_uint(l > h ? h : l), most = __float_as_uint(l > h ? l : h);
      sum = __builtin_fma(up[i], (double)__uint_as_float(most & some_up[i]), sum);
      sum = __builtin_fma(down[i], (double)__uint_as_float(least & some_down[i]), sum);
    }
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (d == 0 && c < x.columns) {
      const bool fixed = c < a.sinks || c >= x.columns - a.recent;
      keys[c] = !there[e] ? 0 : fixed ? ~0ull : order_of(sum);
    }
  }
}

// ----------------------------------------------------------- the n largest
// The n largest of `count` keys, of equal ones those of the lowest places, in
// ascending places.  A key of 0 is none, the largest one (all bits) is always
// taken: the caller sees to it that no more than n have it.
//
// A workgroup keeps EACH neighbouring keys a lane, all of them where they are few
// enough, and otherwise reads them again each time.  Keys of a row are alike in
// their upper bits: the digits by which they are told apart begin at the first
// bit in which the least and the largest differ.  Digit by digit, 8 bits a pass,
// the bucket that holds the n-th largest narrows until it is taken whole.
template <typename K, int TH>
struct Pick {
  int hist[TH / 64][256];                 // a wave's own: lanes of one wave alone meet in a bucket
  K lo[TH / 64], hi[TH / 64];
  int sum[TH / 64];
  K prefix;
  int left;
};

__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int o) { return (uint32_t)__shfl_xor((int)v, o, 64); }
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int o) { return (uint64_t)__shfl_xor((long long)v, o, 64); }
__device__ __forceinline__ int high_bits(uint32_t v) { return v == 0 ? 0 : 32 - __builtin_clz(v); }
__device__ __forceinline__ int high_bits(uint64_t v) { return v == 0 ? 0 : 64 - __builtin_clzll(v); }

// raw(place) is read for each place, key(raw, place) made of it; take(place, rank,
// raw) is called for each that is taken, after all of its turn's raw were read.
template <typename K, int TH, int EACH, typename Raw, typename Read, typename Key, typename Take>
__device__ __forceinline__ int pick_largest(Pick<K, TH> &s, int count, int n, Read read, Key key, Take take) {
  constexpr int TURN = TH * EACH, WAVES = TH / 64;
  constexpr K kAlways = ~(K)0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool once = count <= TURN;
  Raw raw[EACH];
  auto load = [&](int j0) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int j = j0 + tid * EACH + e;
      raw[e] = read(j < count ? j : 0);
    }
  };
  auto key_at = [&](int j0, int e) -> K {
    const int j = j0 + tid * EACH + e;
    return j < count ? key(raw[e], j) : 0;
  };
  auto turns = [&](auto f) {
    for (int j0 = 0; j0 < count; j0 += TURN) {
      if (!once) load(j0);
      f(j0);
    }
  };
  if (once && count > 0) load(0);
  // how many are always taken, how many others there are, and their range
  K lo = kAlways, hi = 0;
  int fixed = 0, others = 0;
  turns([&](int j0) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const K k = key_at(j0, e);
      if (k == kAlways) ++fixed;
      else if (k != 0) {
        ++others;
        lo = min(lo, k);
        hi = max(hi, k);
      }
    }
  });
  auto all = [&](int v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if (lane == 0) s.sum[wave] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t += s.sum[w];
    return t;
  };
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, lane_xor(lo, o));
    hi = max(hi, lane_xor(hi, o));
  }
  if (lane == 0) {
    s.lo[wave] = lo;
    s.hi[wave] = hi;
  }
  fixed = all(fixed);
  others = all(others);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    lo = min(lo, s.lo[w]);
    hi = max(hi, s.hi[w]);
  }
  int left = min(n - fixed, others);      // to take of the others
  // those above `floor` are taken, and of those that equal it above `shift` the
  // first `left` (all, if `every`)
  int shift = others > 0 ? high_bits((K)(lo ^ hi)) : 0;
  K prefix = shift < (int)(8 * sizeof(K)) ? hi >> shift : 0;
  bool every = left == others;
  while (!every && left > 0 && shift > 0) {
    const int bits = min(8, shift), next = shift - bits;
    for (int i = tid; i < 256 * WAVES; i += TH) s.hist[i / 256][i % 256] = 0;
    __syncthreads();
    turns([&](int j0) {
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const K k = key_at(j0, e);
        if (k != 0 && k != kAlways && (shift == (int)(8 * sizeof(K)) || k >> shift == prefix))
          atomicAdd(&s.hist[wave][(int)(k >> next) & ((1 << bits) - 1)], 1);
      }
    });
    __syncthreads();
    if (tid < 256) {
      int sum = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += s.hist[w][tid];
      s.hist[0][tid] = sum;
    }
    __syncthreads();
    // a lane four digits, the largest first: those with larger digits
    if (wave == 0) {
      int h[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = s.hist[0][255 - 4 * lane - i];
        sum += h[i];
      }
      int upto = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      int above = upto - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (above < left && above + h[i] >= left) {
          s.prefix = (shift == (int)(8 * sizeof(K)) ? 0 : prefix << bits) | (K)(255 - 4 * lane - i);
          s.left = above + h[i] == left ? -1 : left - above;
        }
        above += h[i];
      }
    }
    __syncthreads();
    prefix = s.prefix;
    shift = next;
    every = s.left < 0;
    left = s.left;
    __syncthreads();
  }
  // (no digit left to tell them apart: equal keys)
  const bool whole_range = shift == (int)(8 * sizeof(K));    // every one of all is taken
  int done = 0, tied = 0;
  turns([&](int j0) {
    uint32_t same = 0, above = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const K k = key_at(j0, e), top = whole_range ? 0 : k >> shift;
      if (k == kAlways) above |= 1u << e;
      else if (k != 0) {
        if (top == prefix) same |= 1u << e;
        else if (top > prefix) above |= 1u << e;
      }
    }
    // both counts in one number, 16 bits each
    const int mine = __popc(same) << 16 | __popc(above);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == 63) s.sum[wave] = upto;
    __syncthreads();
    int before = upto - mine, total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) before += s.sum[w];
      total += s.sum[w];
    }
    int a = done + (before & 0xffff), t = tied + (before >> 16);
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const bool is_same = same >> e & 1, is_above = above >> e & 1;
      if (is_above || (is_same && (every || t < left))) take(j0 + tid * EACH + e, a + (every ? t : min(t, left)), raw[e]);
      a += is_above;
      t += is_same;
    }
    done += total & 0xffff;
    tied += total >> 16;
  });
  return done + (every ? tied : min(tied, left));
}

template <int TH, int EACH>
__global__ __launch_bounds__(TH) void select_kernel(SelectArgs a, int stride) {
  __shared__ Pick<uint64_t, TH> s;
  const Row x = row_of(a, blockIdx.x / a.map.n_kv_heads);
  const uint64_t *keys = (const uint64_t *)a.work + (size_t)blockIdx.x * stride;
  int *out = a.columns + (size_t)blockIdx.x * a.n_select;
  const int n = pick_largest<uint64_t, TH, EACH, uint64_t>(
      s, x.columns, a.n_select, [&](int j) { return keys[j]; }, [](uint64_t k, int) { return k; },
      [&](int j, int rank, uint64_t) { out[rank] = j; });
  for (int i = n + threadIdx.x; i < a.n_select; i += TH) out[i] = -1;
}

// The weights follow their keys, in place too: a turn's are all read before the
// first is written, and a place is never behind its source.
template <int TH, int EACH>
__global__ __launch_bounds__(TH) void evict_kernel(EvictArgs a) {
  __shared__ Pick<uint32_t, TH> s;
  const int b = blockIdx.x / a.heads;
  const int len = max(0, min(a.len[b], a.capacity));
  const float *in = a.weight + (size_t)blockIdx.x * a.weight_ld;
  float *out = a.weight_out + (size_t)blockIdx.x * a.weight_out_ld;
  int *index = a.index + (size_t)blockIdx.x * a.budget;
  const int n = pick_largest<uint32_t, TH, EACH, float>(
      s, len, a.budget, [&](int j) { return in[j]; },
      [&](float w, int j) { return j < a.sinks || j >= len - a.recent ? ~0u : order_of(w); },
      [&](int j, int rank, float w) {
        index[rank] = j;
        out[rank] = w;
      });
  __syncthreads();
  for (int j = n + threadIdx.x; j < a.capacity; j += TH) out[j] = 0.f;
  for (int i = n + threadIdx.x; i < a.budget; i += TH) index[i] = -1;
  if (blockIdx.x % a.heads == 0 && threadIdx.x == 0) a.count[b] = n;
}

int columns_of(int page_shift, int max_len) { return (int)(((int64_t)max_len + (1 << page_shift) - 1) >> page_shift); }

// The (page, kv head) pairs of a sequence, and the workgroups of all.
struct BoundsGrid {
  int64_t items, blocks;
};
BoundsGrid bounds_grid(const BoundsArgs &a) {
  const int64_t pages = (((int64_t)a.n_new + (1 << a.map.shift) - 2) >> a.map.shift) + 1, items = pages * a.map.n_kv_heads;
  return {items, (items * a.map.n_seqs + THREADS / 64 - 1) / (THREADS / 64)};
}

// The workgroups that score a (row, kv head)'s columns, and the threads that
// choose among them: as many as keep all in registers, which few threads pass
// faster: 8 rows of 500 14 us with 256, 18 with 1024, of 6000 24 and 20.
struct SelectGrid {
  int columns, parts, threads;
  int64_t heads;
};
SelectGrid select_grid(int dtype, const SelectArgs &a) {
  const int chunk = 16 / (dtype == DEX_F32 ? 4 : 2), per = THREADS / (a.head_dim / chunk) * SCORE_EACH;
  const int columns = columns_of(a.map.shift, a.max_len);
  return {columns, (columns + per - 1) / per, columns <= 2048 ? 256 : 1024, (int64_t)a.n_rows * a.map.n_kv_heads};
}

// As many threads and keys a thread as keep them all in registers: 256 rows of 700
// 7.7 us so, 12 and 17 in the wider two; 8 of 4100 15.4, 18.7 in the narrow one
// and 18.8 in the widest; 32 of 16000 36, 55 and 42 in the others.
int evict_threads(int capacity) { return capacity <= 1024 ? 256 : 1024; }

}  // namespace

bool bounds_fits(const BoundsArgs &a) {
  const BoundsGrid g = bounds_grid(a);
  return g.items <= 0x7fffffff && launch_fits(g.blocks, THREADS);
}
bool select_fits(int dtype, const SelectArgs &a) {
  const SelectGrid g = select_grid(dtype, a);
  return launch_fits(g.heads * g.parts, THREADS) && launch_fits(g.heads, g.threads);
}
bool evict_fits(const EvictArgs &a) { return launch_fits((int64_t)a.n * a.heads, evict_threads(a.capacity)); }

hipError_t launch_bounds(int dtype, const BoundsArgs &a, hipStream_t s) {
  const BoundsGrid g = bounds_grid(a);
#define DEX_BOUNDS(T, HD) bounds_kernel<T, HD><<<(unsigned)g.blocks, THREADS, 0, s>>>(a, (int)g.items)
  if (dtype == DEX_F32) {
    if (a.head_dim == 32) DEX_BOUNDS(float, 32);
    else if (a.head_dim == 64) DEX_BOUNDS(float, 64);
    else DEX_BOUNDS(float, 128);
  } else {
    if (a.head_dim == 32) DEX_BOUNDS(uint16_t, 32);
    else if (a.head_dim == 64) DEX_BOUNDS(uint16_t, 64);
    else DEX_BOUNDS(uint16_t, 128);
  }
#undef DEX_BOUNDS
  return hipGetLastError();
}

size_t select_work(int n_rows, int n_kv_heads, int page_shift, int max_len) {
  return (size_t)n_rows * n_kv_heads * columns_of(page_shift, max_len) * sizeof(uint64_t);
}

hipError_t launch_select(int dtype, const SelectArgs &a, hipStream_t s) {
  const SelectGrid g = select_grid(dtype, a);
  if (g.columns > 0) {
    const int64_t elem = dtype == DEX_F32 ? 4 : 2;
    const bool whole = (uintptr_t)a.q % 16 == 0 && a.q_row * elem % 16 == 0 && a.q_head * elem % 16 == 0;
#define DEX_SCORE(T, HD) score_kernel<T, HD><<<(unsigned)(g.heads * g.parts), THREADS, 0, s>>>(a, g.columns, g.parts, whole)
    if (dtype == DEX_F32) {
      if (a.head_dim == 32) DEX_SCORE(float, 32);
      else if (a.head_dim == 64) DEX_SCORE(float, 64);
      else DEX_SCORE(float, 128);
    } else {
      if (a.head_dim == 32) DEX_SCORE(uint16_t, 32);
      else if (a.head_dim == 64) DEX_SCORE(uint16_t, 64);
      else DEX_SCORE(uint16_t, 128);
    }
#undef DEX_SCORE
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (g.threads == 256) select_kernel<256, 8><<<(unsigned)g.heads, 256, 0, s>>>(a, g.columns);
  else select_kernel<1024, 8><<<(unsigned)g.heads, 1024, 0, s>>>(a, g.columns);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictArgs &a, hipStream_t s) {
  const int rows = a.n * a.heads;
  if (evict_threads(a.capacity) == 256) evict_kernel<256, 4><<<rows, 256, 0, s>>>(a);
  else if (a.capacity <= 8192) evict_kernel<1024, 8><<<rows, 1024, 0, s>>>(a);
  else evict_kernel<1024, 16><<<rows, 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dex
