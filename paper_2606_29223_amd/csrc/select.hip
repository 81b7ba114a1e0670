// Pages that a cheap score selects, and keys that accumulated weights keep.
//
// Bounds of a page are the least and the largest of its keys in every
// dimension; a query's product with a key of the page is at most
//   sum_d max(q_d min_d, q_d max_d) = sum_d q+_d max_d + q-_d min_d,
// q+ and q- its positive and negative parts, and the sum of that over the query
// heads of a kv head is the page's score: one vector a (row, kv head), its
// heads' parts summed.  Scores decide whole numbers, so they are in double.
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

// LPR lanes a page, a lane N dimensions of its least and largest keys.
template <typename T, int HD>
__global__ __launch_bounds__(THREADS) void score_kernel(SelectArgs a, int stride, int per, int parts) {
  constexpr int N = 16 / sizeof(T), LPR = HD / N, PAGES = THREADS / LPR;
  const int kv = a.map.n_kv_heads, G = a.n_heads / kv, row = blockIdx.x / parts, head = row % kv, r = row / kv;
  const Row x = row_of(a, r);
  const int first = (blockIdx.x - row * parts) * per, end = min(first + per, x.columns);
  if (first >= end) return;
  const int d = threadIdx.x % LPR;
  double up[N], down[N];                  // q+ and q-, of all the kv head's heads
#pragma unroll
  for (int i = 0; i < N; ++i) up[i] = down[i] = 0.0;
  const T *src = (const T *)a.q + (int64_t)r * a.q_row + (int64_t)head * G * a.q_head + d * N;
  for (int g = 0; g < G; ++g, src += a.q_head)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float v;
      if constexpr (sizeof(T) == 2) v = __uint_as_float((uint32_t)src[i] << 16);
      else v = src[i];
      up[i] += v < 0.f ? 0.f : v;         // (a NaN goes on in both)
      down[i] += v > 0.f ? 0.f : v;
    }
  // a part of 0 adds nothing, whatever the bound (0 times infinity is not 0)
  uint32_t some_up[N], some_down[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    some_up[i] = up[i] == 0.0 ? 0u : ~0u;
    some_down[i] = down[i] == 0.0 ? 0u : ~0u;
  }
  uint64_t *keys = (uint64_t *)a.work + (size_t)row * stride;
  for (int c0 = first; c0 < end; c0 += PAGES) {
    const int c = c0 + threadIdx.x / LPR;
    int page = -1;
    if (c < end) page = a.map.table[(size_t)x.seq * a.map.max_pages + c];
    const bool there = page >= 0 && page < a.map.n_pages;
    Chunk<T> lo, hi;
    lo.raw = hi.raw = make_uint4(0, 0, 0, 0);
    if (there) {
      const T *b = (const T *)a.bounds + ((size_t)page * kv + head) * 2 * HD + d * N;
      lo.raw = *(const uint4 *)b;
      hi.raw = *(const uint4 *)(b + HD);
    }
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float l = lo.get(i), h = hi.get(i);
      const uint32_t least = __float_as_uint(l > h ? h : l), most = __float_as_uint(l > h ? l : h);
      sum = __builtin_fma(up[i], (double)__uint_as_float(most & some_up[i]), sum);
      sum = __builtin_fma(down[i], (double)__uint_as_float(least & some_down[i]), sum);
    }
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (d == 0 && c < end) {
      const bool fixed = c < a.sinks || c >= x.columns - a.recent;
      keys[c] = !there ? 0 : fixed ? ~0ull : order_of(sum);
    }
  }
}

// ----------------------------------------------------------- the n largest
// The n largest of the keys 1 .. of places 0 .. count - 1, in ascending places;
// the lowest places among equals.  take(place, rank, key) is called for each,
// once all keys of its turn have been read.
template <typename K>
struct Pick {
  int hist[256];
  int before[THREADS / 64], ties[THREADS / 64];
  K prefix;
  int left, shift;
};

template <typename K, typename Key, typename Take>
__device__ __forceinline__ int pick_largest(Pick<K> &s, int count, int n, Key key, Take take) {
  constexpr int BITS = 8 * sizeof(K);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // digit by digit: of those that agree with the n-th largest so far, which
  // digit it has next
  K prefix = 0;
  int left = n, shift = BITS;
  while (shift > 0) {
    s.hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < count; j += THREADS) {
      const K k = key(j);
      if (k != 0 && (shift == BITS || k >> (shift % BITS) == prefix)) atomicAdd(&s.hist[(int)(k >> (shift - 8)) & 255], 1);
    }
    __syncthreads();
    // a lane a digit, the largest first: those with larger digits
    if (wave == 0) {
      int h[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = s.hist[255 - 4 * lane - i];
        sum += h[i];
      }
      int upto = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(upto, o, 64);
        if (lane >= o) upto += y;
      }
      int above = upto - sum;
      const int all = __shfl(upto, 63, 64);
      if (all <= left) {                  // all of them
        if (lane == 0) s.left = -1;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < left && above + h[i] >= left) {
            s.prefix = prefix << 8 | (K)(255 - 4 * lane - i);
            s.left = above + h[i] == left ? 0 : left - above;
          }
          above += h[i];
        }
      }
    }
    __syncthreads();
    const int now = s.left;
    if (now < 0) break;
    prefix = s.prefix;
    shift -= 8;
    left = now;
    __syncthreads();
    if (now == 0) break;
  }
  // keys above the prefix, and of those that agree with it all (left 0, or no
  // digit looked at) or the first `left`
  const bool every = left == 0 || shift == BITS || s.left < 0;
  int done = 0, tied = 0;
  for (int j0 = 0; j0 < count; j0 += THREADS) {
    const int j = j0 + tid;
    const K k = j < count ? key(j) : 0;
    const K top = shift == BITS ? 0 : k >> (shift % BITS);
    const bool same = k != 0 && top == prefix, above = k != 0 && top > prefix;
    const unsigned long long ts = __ballot(same), as = __ballot(above);
    if (lane == 0) {
      s.ties[wave] = __popcll(ts);
      s.before[wave] = __popcll(as);
    }
    __syncthreads();
    int t = tied, a = done, all_t = tied, all_a = done;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) {
        t += s.ties[w];
        a += s.before[w];
      }
      all_t += s.ties[w];
      all_a += s.before[w];
    }
    const unsigned long long under = (1ull << lane) - 1;
    t += __popcll(ts & under);
    a += __popcll(as & under);
    // places before this one that are taken: a above, and of the ties
    const bool mine = above || (same && (every || t < left));
    if (mine) take(j, a + (every ? t : min(t, left)), k);
    done = all_a;
    tied = all_t;
    __syncthreads();
  }
  return done + (every ? tied : min(tied, left));
}

__global__ __launch_bounds__(THREADS) void select_kernel(SelectArgs a, int stride) {
  __shared__ Pick<uint64_t> s;
  const Row x = row_of(a, blockIdx.x / a.map.n_kv_heads);
  const uint64_t *keys = (const uint64_t *)a.work + (size_t)blockIdx.x * stride;
  int *out = a.columns + (size_t)blockIdx.x * a.n_select;
  const int n = pick_largest<uint64_t>(s, x.columns, a.n_select, [&](int j) { return keys[j]; },
                                       [&](int j, int rank, uint64_t) { out[rank] = j; });
  for (int i = n + threadIdx.x; i < a.n_select; i += THREADS) out[i] = -1;
}

__global__ __launch_bounds__(THREADS) void evict_kernel(EvictArgs a) {
  __shared__ Pick<uint32_t> s;
  const int b = blockIdx.x / a.heads;
  const int len = max(0, min(a.len[b], a.capacity));
  const float *in = a.weight + (size_t)blockIdx.x * a.weight_ld;
  float *out = a.weight_out + (size_t)blockIdx.x * a.weight_out_ld;
  int *index = a.index + (size_t)blockIdx.x * a.budget;
  const int n = pick_largest<uint32_t>(
      s, len, a.budget,
      [&](int j) { return j < a.sinks || j >= len - a.recent ? 0xffffffffu : order_of(in[j]); },
      [&](int j, int rank, uint32_t) {
        index[rank] = j;
      });
  __syncthreads();
  // the weights follow, turn by turn: a turn's are read before any is written,
  // and a place is never behind its source
  for (int j0 = 0; j0 < n; j0 += THREADS) {
    const int j = j0 + threadIdx.x;
    float w = 0.f;
    if (j < n) w = in[index[j]];
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (j < n) out[j] = w;
  }
  for (int j = n + threadIdx.x; j < a.capacity; j += THREADS) out[j] = 0.f;
  for (int i = n + threadIdx.x; i < a.budget; i += THREADS) index[i] = -1;
  if (blockIdx.x % a.heads == 0 && threadIdx.x == 0) a.count[b] = n;
}

int columns_of(int page_shift, int max_len) { return (int)(((int64_t)max_len + (1 << page_shift) - 1) >> page_shift); }

}  // namespace

hipError_t launch_bounds(int dtype, const BoundsArgs &a, hipStream_t s) {
  const int64_t pages = (((int64_t)a.n_new + (1 << a.map.shift) - 2) >> a.map.shift) + 1;
  const int64_t items = pages * a.map.n_kv_heads, grid = (items * a.map.n_seqs + THREADS / 64 - 1) / (THREADS / 64);
  if (items > 0x7fffffff || grid > 0x7fffffff) return hipErrorInvalidValue;
#define DEX_BOUNDS(T, HD) bounds_kernel<T, HD><<<(unsigned)grid, THREADS, 0, s>>>(a, (int)items)
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
  const int columns = columns_of(a.map.shift, a.max_len), heads = a.n_rows * a.map.n_kv_heads;
  if (columns > 0) {
    const int per = 128;
    const int parts = (columns + per - 1) / per;
    const int64_t grid = (int64_t)parts * heads;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
#define DEX_SCORE(T, HD) score_kernel<T, HD><<<(unsigned)grid, THREADS, 0, s>>>(a, columns, per, parts)
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
  select_kernel<<<heads, THREADS, 0, s>>>(a, columns);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictArgs &a, hipStream_t s) {
  evict_kernel<<<a.n * a.heads, THREADS, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dex
