// Beam search's selection: the n best continuations of a request's beams.
//
// Candidate (beam, token) has score[beam] + logit - lse(beam's logits), a
// finished beam only (eos) with its score as it is.  Within a beam the order
// is the logits', so only each beam's n best tokens can be among the n best
// of all: the first kernel reads every logit once, gives the n best of each
// 2048-logit segment and the segment's maximum and sum of exponentials; the
// second joins a beam's segments and then the request's beams, with the
// scores in double (logits are ordered as they are; two beams' candidates are
// told apart to 2^-52 of their score plus what the float exponentials leave
// in lse, about 2^-25).
#include "dex.h"
#include "dex_kernels.h"
#include "paged.h"

namespace dex {

namespace {

constexpr int SEG = 2048;                 // logits of a segment: one wave, 32 a lane
constexpr int PER_LANE = SEG / 64;
constexpr int WAVES = 4;
constexpr int LIST = 256;                 // candidates a wave sorts

struct Cand {
  uint32_t key;                           // order-preserving bits of the logit; 0: none
  int idx;                                // token
};

// Unsigned order of the keys is the order of the floats; -0 and +0 are one.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

__device__ __forceinline__ float max64(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ float sum64(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ double sum64(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ void wave_sync() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// The largest t such that at least n of the wave's lanes hold a key >= t: the
// n-th largest of them, found bit by bit.
__device__ __forceinline__ uint32_t nth_of_lanes(uint32_t key, int n) {
  uint32_t t = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = t | 1u << b;
    if (__popcll(__ballot(key >= c)) >= n) t = c;
  }
  return t;
}

// The n best (key down, index up) of `list[0 .. cnt)` to out[0 .. n), by their
// ranks; (0, -1) behind the last.  One wave; cnt <= LIST.
__device__ __forceinline__ void rank_out(const Cand *list, int cnt, int n, Cand *out) {
  const int lane = threadIdx.x & 63;
  for (int i = lane; i < cnt; i += 64) {
    const Cand c = list[i];
    int r = 0;
    for (int j = 0; j < cnt; ++j) {
      const Cand o = list[j];
      r += o.key > c.key || (o.key == c.key && o.idx < c.idx) ? 1 : 0;
    }
    if (r < n) out[r] = c;
  }
  for (int i = cnt + lane; i < n; i += 64) out[i] = Cand{0u, -1};
}

struct SegStat {
  float top, sum;
};

template <typename T>
constexpr int kGrain = 16 / (int)sizeof(T);       // logits of a 16-byte load

// Segments of a row: its logits may begin anywhere in their first 16 bytes.
__host__ __device__ inline int segments(int vocab, int grain) { return (vocab + grain - 1 + SEG - 1) / SEG; }

template <typename T>
__global__ __launch_bounds__(WAVES * 64) void beam_segment_kernel(BeamArgs a, int n_seg, Cand *cand, SegStat *stat) {
  constexpr int GR = kGrain<T>, IT = PER_LANE / GR;
  __shared__ Cand lists[WAVES][LIST];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (n_seg + WAVES - 1) / WAVES;          // of a row
  const int row = blockIdx.x / blocks;
  const int seg = (blockIdx.x - row * blocks) * WAVES + wave;
  if (seg >= n_seg) return;
  if (a.done != nullptr && a.done[row]) return;   // the second kernel asks nothing of it
  const T *x = (const T *)a.logits + (int64_t)row * a.ld;
  // index 0 of the grains is the 16-byte boundary at or before the row
  const int shift = (int)(((uintptr_t)x & 15) / sizeof(T));
  float v[PER_LANE];
  int bad = 0;
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int e0 = seg * SEG + (i * 64 + lane) * GR - shift;
    if (e0 >= 0 && e0 + GR <= a.vocab) {
      const uint4 raw = *(const uint4 *)(x + e0);
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        if constexpr (sizeof(T) == 2) v[i * GR + j] = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        else v[i * GR + j] = __uint_as_float(w[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        const int e = e0 + j;
        float f = -INFINITY;
        if (e >= 0 && e < a.vocab) {
          if constexpr (sizeof(T) == 2) f = __uint_as_float((uint32_t)((const uint16_t *)x)[e] << 16);
          else f = x[e];
        }
        v[i * GR + j] = f;
      }
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < PER_LANE; ++k) {
    bad |= !(v[k] < INFINITY);                    // NaN or +inf
    top = fmaxf(top, v[k]);
  }
  const uint32_t lane_key = key_of(top);
  const float m = max64(top);
  // exp(v - m) as a power of two; log2(e) in two parts, so that a distance of
  // tens keeps its last bits
  float s0 = 0.f, s1 = 0.f;
  const float m0 = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int k = 0; k < PER_LANE; k += 2) {
    const float d0 = v[k] - m0, d1 = v[k + 1] - m0;
    s0 += __builtin_amdgcn_exp2f(fmaf(d0, 1.44269502f, d0 * 1.92596303e-8f));
    s1 += __builtin_amdgcn_exp2f(fmaf(d1, 1.44269502f, d1 * 1.92596303e-8f));
  }
  const float sum = sum64(s0 + s1);
  if (__ballot(bad) != 0) bad = 1;
  if (lane == 0) stat[(size_t)row * n_seg + seg] = SegStat{m, bad ? NAN : sum};

  // candidates: at least n logits reach the n-th largest of the lanes' maxima
  const int n = a.n_out;
  Cand *list = lists[wave], *out = cand + ((size_t)row * n_seg + seg) * n;
  uint32_t t = nth_of_lanes(lane_key, n);
  auto exists = [&](int k) {
    const int e = seg * SEG + (k / GR * 64 + lane) * GR + k % GR - shift;
    return e >= 0 && e < a.vocab;
  };
  auto index = [&](int k) { return seg * SEG + (k / GR * 64 + lane) * GR + k % GR - shift; };
  const unsigned long long lt = (1ull << lane) - 1;
  int cnt = 0;
#pragma unroll
  for (int k = 0; k < PER_LANE; ++k) {
    const bool in = key_of(v[k]) >= t && exists(k);
    const unsigned long long b = __ballot(in);
    const int at = cnt + __popcll(b & lt);
    if (in && at < LIST) list[at] = Cand{key_of(v[k]), index(k)};
    cnt += __popcll(b);
  }
  if (cnt > LIST) {
    // many equal logits: the exact n-th largest key t of the segment, those
    // above it (fewer than n) and the first of those equal to it
    t = 0;
    for (int b = 31; b >= 0; --b) {
      const uint32_t c = t | 1u << b;
      int here = 0;
#pragma unroll
      for (int k = 0; k < PER_LANE; ++k) here += __popcll(__ballot(key_of(v[k]) >= c && exists(k)));
      if (here >= n) t = c;
    }
    cnt = 0;
#pragma unroll
    for (int k = 0; k < PER_LANE; ++k) {
      const bool in = key_of(v[k]) > t && exists(k);
      const unsigned long long b = __ballot(in);
      if (in) list[cnt + __popcll(b & lt)] = Cand{key_of(v[k]), index(k)};
      cnt += __popcll(b);
    }
    const int room = n - cnt;
    int seen = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {                // tokens go up by grain, lane, place in the grain
      unsigned long long eq[GR];
      int before = 0, all = 0;
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        eq[j] = __ballot(key_of(v[i * GR + j]) == t && exists(i * GR + j));
        before += __popcll(eq[j] & lt);
        all += __popcll(eq[j]);
      }
#pragma unroll
      for (int j = 0; j < GR; ++j)
        if (eq[j] >> lane & 1) {
          const int r = seen + before++;
          if (r < room) list[cnt + r] = Cand{t, index(i * GR + j)};
        }
      seen += all;
    }
    cnt += min(seen, room);
  }
  wave_sync();
  rank_out(list, cnt, n, out);
}

// One workgroup a request, a wave a beam at a time, then all beams together.
__global__ __launch_bounds__(WAVES * 64) void beam_join_kernel(BeamArgs a, int n_seg, const Cand *cand,
                                                              const SegStat *stat) {
  extern __shared__ double shared[];
  const int K = a.beams, n = a.n_out, per = n < a.vocab ? n : a.vocab;   // candidates of a beam
  double *total = shared;                                                // [K][n]
  int *token = (int *)(total + (size_t)K * n);                           // [K][n]
  Cand *lists = (Cand *)(token + (size_t)K * n + ((size_t)K * n & 1));   // [WAVES][LIST]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = blockIdx.x;
  Cand *list = lists + wave * LIST;
  for (int b = wave; b < K; b += WAVES) {
    const int row = r * K + b;
    const double score = (double)a.score[row];
    const bool done = a.done != nullptr && a.done[row];
    double lse = 0.0;
    bool dead = !(score > -INFINITY && score < INFINITY);
    if (!done) {
      const SegStat *st = stat + (size_t)row * n_seg;
      float m = -INFINITY;
      bool nan = false;
      for (int i = lane; i < n_seg; i += 64) {
        m = fmaxf(m, st[i].top);
        nan |= st[i].sum != st[i].sum;
      }
      m = max64(m);
      dead |= m == -INFINITY || __ballot(nan) != 0;
      double sum = 0.0;
      if (!dead)
        for (int i = lane; i < n_seg; i += 64)
          if (st[i].top > -INFINITY) sum += (double)st[i].sum * exp((double)st[i].top - (double)m);
      lse = (double)m + log(sum64(sum));
    }
    if (done || dead) {
      // tokens in order without a chance, after the finished beam's one candidate
      const bool stays = done && !dead;
      for (int i = lane; i < per; i += 64) {
        const int k = i - (stays ? 1 : 0);        // the k-th token other than eos
        token[b * n + i] = !stays ? i : i == 0 ? a.eos : k < a.eos ? k : k + 1;
        total[b * n + i] = stays && i == 0 ? score : -INFINITY;
      }
    } else {
      const Cand *c = cand + (size_t)row * n_seg * n;
      const int all = n_seg * n;
      uint32_t best = 0;
      for (int i = lane; i < all; i += 64) best = max(best, c[i].key);
      // keys of absent candidates are 0 and never among the `per` there are
      const uint32_t t = max(nth_of_lanes(best, per), 1u);
      int cnt = 0;
      for (int i0 = 0; i0 < all; i0 += 64) {
        const Cand x = i0 + lane < all ? c[i0 + lane] : Cand{0u, -1};
        const bool in = x.key >= t;
        const unsigned long long bal = __ballot(in);
        const int at = cnt + __popcll(bal & ((1ull << lane) - 1));
        if (in && at < LIST) list[at] = x;
        cnt += __popcll(bal);
      }
      wave_sync();
      if (cnt <= LIST) {
        for (int i = lane; i < cnt; i += 64) {
          const Cand x = list[i];
          int rank = 0;
          for (int j = 0; j < cnt; ++j) {
            const Cand o = list[j];
            rank += o.key > x.key || (o.key == x.key && o.idx < x.idx) ? 1 : 0;
          }
          if (rank < per) {
            token[b * n + rank] = x.idx;
            total[b * n + rank] = score + ((double)of_key(x.key) - lse);
          }
        }
      } else {
        // many equal logits: the segments' lists are sorted, so take the best
        // of all again and again
        uint32_t last_key = 0xffffffffu;
        int last_idx = -1;
        for (int k = 0; k < per; ++k) {
          uint32_t bk = 0;
          int bi = INT32_MAX;
          for (int i = lane; i < all; i += 64) {
            const Cand x = c[i];
            if (x.key == 0) continue;
            if (x.key > last_key || (x.key == last_key && x.idx <= last_idx)) continue;   // taken already
            if (x.key > bk || (x.key == bk && x.idx < bi)) { bk = x.key; bi = x.idx; }
          }
#pragma unroll
          for (int o = 32; o >= 1; o >>= 1) {
            const uint32_t ok = __shfl_xor(bk, o, 64);
            const int oi = __shfl_xor(bi, o, 64);
            if (ok > bk || (ok == bk && oi < bi)) { bk = ok; bi = oi; }
          }
          last_key = bk;
          last_idx = bi;
          if (lane == 0) {
            token[b * n + k] = bi;
            total[b * n + k] = score + ((double)of_key(bk) - lse);
          }
        }
      }
      wave_sync();
    }
  }
  __syncthreads();
  // A candidate's rank: those before it in its own beam, and in every other
  // beam those with a larger total, or an equal one where that beam comes
  // first.  Each beam's totals go down, so those are found by bisection.
  for (int i = threadIdx.x; i < K * per; i += WAVES * 64) {
    const int b = i / per, k = i - b * per;
    const double t = total[b * n + k];
    int rank = k;
    for (int o = 0; o < K && rank < n; ++o) {
      if (o == b) continue;
      int lo = 0, hi = per;                       // candidates of beam o that go before this one
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const double v = total[o * n + mid];
        if (v > t || (v == t && o < b)) lo = mid + 1;
        else hi = mid;
      }
      rank += lo;
    }
    if (rank < n) {
      const int row = r * K + b, w = r * n + rank, tok = token[b * n + k];
      a.parent[w] = row;
      a.token[w] = tok;
      a.score_out[w] = (float)t;
      if (a.done_out != nullptr) a.done_out[w] = (a.done != nullptr && a.done[row]) || tok == a.eos ? 1 : 0;
    }
  }
}

}  // namespace

size_t beam_work(int dtype, int rows, int vocab, int n_out) {
  const size_t n_seg = segments(vocab, dtype == DEX_F32 ? kGrain<float> : kGrain<uint16_t>);
  return (size_t)rows * n_seg * (n_out * sizeof(Cand) + sizeof(SegStat));
}

hipError_t launch_beam(int dtype, const BeamArgs &a, hipStream_t s) {
  const int rows = a.requests * a.beams;
  const int n_seg = segments(a.vocab, dtype == DEX_F32 ? kGrain<float> : kGrain<uint16_t>);
  Cand *cand = (Cand *)a.work;
  SegStat *stat = (SegStat *)(cand + (size_t)rows * n_seg * a.n_out);
  const unsigned grid = (unsigned)((n_seg + WAVES - 1) / WAVES) * rows;
  if (dtype == DEX_F32) beam_segment_kernel<float><<<grid, WAVES * 64, 0, s>>>(a, n_seg, cand, stat);
  else beam_segment_kernel<uint16_t><<<grid, WAVES * 64, 0, s>>>(a, n_seg, cand, stat);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t kn = (size_t)a.beams * a.n_out;
  const size_t lds = kn * 8 + (kn + (kn & 1)) * 4 + WAVES * LIST * sizeof(Cand);
  beam_join_kernel<<<a.requests, WAVES * 64, lds, s>>>(a, n_seg, cand, stat);
  return hipGetLastError();
}

}  // namespace dex
