// Beam search's selection: the n best continuations of a request's beams.
//
// Candidate (beam, token) has score[beam] + logit - lse(beam's logits), a
// finished beam only (eos) with its score as it is.  Within a beam the order
// is the logits', so only each beam's n best tokens can be among the n best
// of all: the first kernel reads every logit once, gives the n best of each
// segment and the segment's maximum and sum of exponentials; the
// second joins a beam's segments and then the request's beams, with the
// scores in double.  Logits are ordered as they are; two beams' candidates are
// told apart to 2^-52 of their score and what the float exponentials and a
// lane's float sums of them, at most eight in a sum, leave in the two lse: each
// is off by at most (9 + 2 E) 2^-24, E the mean of maximum - logit under the
// softmax.  Measured on normal logits of deviation 1 to 10, 8000 to 65537 of
// them, 256 rows each: 2^-26 on the average, 2^-23 in the worst row.
#include "dex.h"
#include "dex_kernels.h"
#include "paged.h"

namespace dex {

namespace {

constexpr int WAVES = 4;                  // of a segment workgroup
constexpr int LIST = 252;                 // candidates a wave sorts
constexpr int LIST_ROOM = LIST + 4;
constexpr int JOIN_WAVES = 8;
constexpr int HOLD = 32;                  // lanes whose logits go through LDS
constexpr int HELD = 8;                   // candidates a lane of the join keeps; further ones are read twice

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

// Reductions over a wave, the same value in every lane: by rotations within
// the rows of 16 lanes (no LDS round trip each), then over the four rows.
template <int CTRL>
__device__ __forceinline__ float rotated(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_of(float x, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}
constexpr int kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;
__device__ __forceinline__ float max64(float v) {
  v = fmaxf(v, rotated<kRor8>(v));
  v = fmaxf(v, rotated<kRor4>(v));
  v = fmaxf(v, rotated<kRor2>(v));
  v = fmaxf(v, rotated<kRor1>(v));
  return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
template <int CTRL>
__device__ __forceinline__ double rotated(double x) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, 0xf, 0xf, false),
                          __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ double lane_of(double x, int lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane),
                          __builtin_amdgcn_readlane(__double2loint(x), lane));
}
__device__ __forceinline__ double sum64(double v) {
  v += rotated<kRor8>(v);
  v += rotated<kRor4>(v);
  v += rotated<kRor2>(v);
  v += rotated<kRor1>(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ void wave_sync() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// A key t that at least n of the wave's lanes reach: the n-th largest of them,
// cut to its leading 20 bits (a bfloat16 has 16), found bit by bit.
__device__ __forceinline__ uint32_t nth_of_lanes(uint32_t key, int n) {
  uint32_t t = 0;
#pragma unroll
  for (int b = 31; b >= 12; --b) {
    const uint32_t c = t | 1u << b;
    if (__popcll(__ballot(key >= c)) >= n) t = c;
  }
  return t;
}

// f(rank, candidate) for each of list[0 .. cnt), ranked by key down, index up.
// One wave; cnt <= LIST, and the list has room for three more.
template <typename F>
__device__ __forceinline__ void rank_list(Cand *list, int cnt, F f) {
  const int lane = threadIdx.x & 63;
  if (cnt <= 64) {                        // one a lane: no more round trips to LDS
    wave_sync();
    const Cand c = lane < cnt ? list[lane] : Cand{0u, -1};
    const uint64_t mine = (uint64_t)c.key << 32 | ~(uint32_t)c.idx;
    int r = 0;
    for (int j = 0; j < cnt; ++j) {
      const uint64_t o = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)c.key, j) << 32 |
                         ~(uint32_t)__builtin_amdgcn_readlane(c.idx, j);
      r += o > mine ? 1 : 0;
    }
    if (lane < cnt) f(r, c);
    return;
  }
  if (lane < 3) list[cnt + lane] = Cand{0u, -1};  // ranks before nothing
  wave_sync();
  for (int i = lane; i < cnt; i += 64) {
    const Cand c = list[i];
    int r = 0;
    for (int j = 0; j < cnt; j += 4) {
      Cand o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = list[j + k];
#pragma unroll
      for (int k = 0; k < 4; ++k) r += o[k].key > c.key || (o[k].key == c.key && o[k].idx < c.idx) ? 1 : 0;
    }
    f(r, c);
  }
}

struct SegStat {
  double sum;                             // of e^(logit - top); NaN where the logits are no distribution
  float top;
};
// log2 e to 2^-50: 2^(d kLog2eHi + d kLog2eLo) rounds d log2 e once, where the
// first part alone is off by 2^-26 of it for all logits alike.
constexpr float kLog2eHi = 1.44269502f, kLog2eLo = 1.92596299e-8f;
__device__ __forceinline__ float exp_of(float d) {
  return __builtin_amdgcn_exp2f(fmaf(d, kLog2eHi, d * kLog2eLo));
}

template <typename T>
constexpr int kGrain = 16 / (int)sizeof(T);       // logits of a 16-byte load

inline int segments(int vocab, int seg) { return (vocab + seg - 1) / seg; }

// 16 bytes from any element on: segments are cut at tokens, not at boundaries of
// memory, so that rows of the same logits have the same sums to the last bit,
// wherever they begin (an odd vocabulary has them begin everywhere), and tie.
template <typename T>
__device__ __forceinline__ uint4 load_grain(const T *p) {
  uint4 g;
  __builtin_memcpy(&g, p, sizeof g);
  return g;
}

// A wave takes a segment of 64 LANE logits, LANE a lane, all in registers.
// What bounds it is the instructions: a logit takes a conversion, the maximum,
// the exponential's five and one comparison with the threshold below, a wave
// about 200 more.  320 rows of 65537 bf16 logits (42 MB, 8 us at a copy's rate)
// take 18 us; 4 rows of 32000 floats 3.8 us, the latency of one wave.
template <typename T, int LANE>
__global__ __launch_bounds__(WAVES * 64, 5) void beam_segment_kernel(BeamArgs a, int n_seg, Cand *cand, SegStat *stat) {
  constexpr int GR = kGrain<T>, IT = LANE / GR, SEG = 64 * LANE;
  __shared__ Cand lists[WAVES][LIST_ROOM];
  __shared__ __align__(16) float holds[WAVES][HOLD][LANE + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x * WAVES + wave, row = item / n_seg, seg = item - row * n_seg;
  if (row >= a.requests * a.beams) return;
  if (a.done != nullptr && a.done[row]) return;   // the second kernel asks nothing of it
  const T *x = (const T *)a.logits + (int64_t)row * a.ld;
  const int at = seg * SEG + lane * GR;           // a lane's k-th logit is token at + k / GR * 64 * GR + k % GR
  const bool whole = (seg + 1) * SEG <= a.vocab;  // every place is a token
  auto token = [&](int k) { return at + k / GR * 64 * GR + k % GR; };
  auto exists = [&](int k) { return token(k) < a.vocab; };
  float v[LANE];
  if (whole) {
    uint4 raw[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) raw[i] = load_grain(x + token(i * GR));
#pragma unroll
    for (int k = 0; k < LANE; ++k) {
      const uint4 g = raw[k / GR];
      const uint32_t w = k % GR * sizeof(T) / 4 == 0 ? g.x : k % GR * sizeof(T) / 4 == 1 ? g.y
                       : k % GR * sizeof(T) / 4 == 2 ? g.z : g.w;
      if constexpr (sizeof(T) == 2) v[k] = __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
      else v[k] = __uint_as_float(w);
    }
  } else {                                        // a row's end: by elements, the same places
    T e[LANE];
#pragma unroll
    for (int k = 0; k < LANE; ++k) e[k] = x[min(token(k), a.vocab - 1)];
#pragma unroll
    for (int k = 0; k < LANE; ++k) {
      float f;
      if constexpr (sizeof(T) == 2) f = __uint_as_float((uint32_t)e[k] << 16);
      else f = e[k];
      v[k] = exists(k) ? f : -INFINITY;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < LANE; ++k) top = fmaxf(top, v[k]);
  const float m = max64(top);
  // A NaN or +inf makes the sum a NaN by itself.
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  const float m0 = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int k = 0; k < LANE; ++k) s[k % 4] += exp_of(v[k] - m0);
  const double sum = sum64(((double)s[0] + (double)s[1]) + ((double)s[2] + (double)s[3]));
  if (lane == 0) stat[(size_t)row * n_seg + seg] = SegStat{sum, m};

  // At least n logits reach t, a key that n lanes' maxima reach.
  const int n = a.n_out;
  Cand *list = lists[wave], *out = cand + ((size_t)row * n_seg + seg) * n;
  const uint32_t none = key_of(-INFINITY);
  const uint32_t t = nth_of_lanes(key_of(top), n);
  const unsigned long long lt = (1ull << lane) - 1;
  int cnt = 0;
  // the tokens whose key is u, in order, as long as there is room for n
  auto add_equal = [&](uint32_t u) {
    const int room = n - cnt;
    int seen = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {                // tokens go up by grain, lane, place in the grain
      unsigned long long eq[GR];
      int before = 0, all = 0;
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        eq[j] = __ballot(key_of(v[i * GR + j]) == u && exists(i * GR + j));
        before += __popcll(eq[j] & lt);
        all += __popcll(eq[j]);
      }
#pragma unroll
      for (int j = 0; j < GR; ++j)
        if (eq[j] >> lane & 1) {
          const int r = seen + before++;
          if (r < room) list[cnt + r] = Cand{u, token(i * GR + j)};
        }
      seen += all;
    }
    cnt += min(seen, room);
  };
  // absent places hold -inf: only what is above that goes by its value alone
  const float tf = of_key(max(t, none + 1));
  const unsigned long long have = __ballot(top >= tf);
  const int n_have = __popcll(have);
  if (n_have <= HOLD) {
    // few lanes reach t: theirs go through LDS and are spread over the wave (a
    // ballot for each of the LANE places takes 3 to 5 % longer)
    float(*hold)[LANE + 4] = holds[wave];
    if (top >= tf) {
      float *to = hold[__popcll(have & lt)];
#pragma unroll
      for (int k = 0; k < LANE; k += 4) *(float4 *)(to + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
      to[LANE] = __int_as_float(token(0));
    }
    wave_sync();
    for (int f0 = 0; f0 < n_have * LANE; f0 += 64) {
      const int f = f0 + lane, r = f / LANE, k = f % LANE;
      const float x1 = f < n_have * LANE ? hold[r][k] : -INFINITY;
      const bool in = x1 >= tf;
      const unsigned long long b = __ballot(in);
      if (b == 0) continue;
      const int p = cnt + __popcll(b & lt);
      if (in && p < LIST) list[p] = Cand{key_of(x1), __float_as_int(hold[r][LANE]) + k / GR * 64 * GR + k % GR};
      cnt += __popcll(b);
    }
  } else {
#pragma unroll
    for (int k = 0; k < LANE; ++k) {
      const bool in = v[k] >= tf;
      const unsigned long long b = __ballot(in);
      if (b != 0) {
        const int p = cnt + __popcll(b & lt);
        if (in && p < LIST) list[p] = Cand{key_of(v[k]), token(k)};
        cnt += __popcll(b);
      }
    }
  }
  if (cnt > LIST) {
    // many equal logits: the exact n-th largest key u of the segment, those
    // above it (fewer than n) and the first of those equal to it
    uint32_t u = 0;
    for (int b = 31; b >= 0; --b) {
      const uint32_t c = u | 1u << b;
      int here = 0;
#pragma unroll
      for (int k = 0; k < LANE; ++k) here += __popcll(__ballot(key_of(v[k]) >= c && exists(k)));
      if (here >= n) u = c;
    }
    cnt = 0;
#pragma unroll
    for (int k = 0; k < LANE; ++k) {
      const bool in = key_of(v[k]) > u && exists(k);
      const unsigned long long b = __ballot(in);
      if (in) list[cnt + __popcll(b & lt)] = Cand{key_of(v[k]), token(k)};
      cnt += __popcll(b);
    }
    add_equal(u);
  } else if (cnt < n) {
    add_equal(none);                              // nothing but -inf is left
  }
  rank_list(list, cnt, [&](int r, const Cand &c) { if (r < n) out[r] = c; });
  for (int i = cnt + lane; i < n; i += 64) out[i] = Cand{0u, -1};
}

// One workgroup a request, a wave a beam at a time, then all beams together:
// the latency of a few dependent loads and of the double logarithm (5.3 us for
// one request, 8.3 for 64 of eight beams) while few candidates reach the
// threshold.  Where most do they are ranked in LDS, and more than LIST are taken
// one by one in n passes over all: where fewer than n tokens of a large vocabulary
// are allowed, the rest being equal at -inf (one token, the whole call: 64 x 8 x
// 65537 51 us for 31, 4 x 32000 fp32 50 for 8.8), and with many beams (16 of 32000
// 24 us, 64 of 4000 490).
__global__ __launch_bounds__(JOIN_WAVES * 64) void beam_join_kernel(BeamArgs a, int n_seg, const Cand *cand,
                                                                   const SegStat *stat) {
  extern __shared__ double shared[];
  const int K = a.beams, n = a.n_out, per = n < a.vocab ? n : a.vocab;   // candidates of a beam
  const int waves = blockDim.x / 64;
  double *total = shared;                                                // [K][n]
  int *token = (int *)(total + (size_t)K * n);                           // [K][n]
  Cand *lists = (Cand *)(token + (size_t)K * n + ((size_t)K * n & 1));   // [waves][LIST_ROOM]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = blockIdx.x;
  Cand *list = lists + wave * LIST_ROOM;
  for (int b = wave; b < K; b += waves) {
    const int row = r * K + b;
    const double score = (double)a.score[row];
    const bool done = a.done != nullptr && a.done[row];
    bool dead = !(score > -INFINITY && score < INFINITY);
    const Cand *c = cand + (size_t)row * n_seg * n;
    const int all = n_seg * n;
    Cand held[HELD];
    uint32_t best = 0;
    double lse = 0.0;
    if (!done) {
#pragma unroll
      for (int k = 0; k < HELD; ++k) held[k] = lane + 64 * k < all ? c[lane + 64 * k] : Cand{0u, -1};
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
          sum += st[i].sum * exp((double)st[i].top - (double)m);
      lse = (double)m + log(sum64(sum));
#pragma unroll
      for (int k = 0; k < HELD; ++k) best = max(best, held[k].key);
      for (int i = lane + 64 * HELD; i < all; i += 64) best = max(best, c[i].key);
    }
    if (done || dead) {
      // tokens in order without a chance, after the finished beam's one candidate
      const bool stays = done && !dead;
      for (int i = lane; i < per; i += 64) {
        const int k = i - (stays ? 1 : 0);        // the k-th token other than eos
        token[b * n + i] = !stays ? i : i == 0 ? a.eos : k < a.eos ? k : k + 1;
        total[b * n + i] = stays && i == 0 ? score : -INFINITY;
      }
      continue;
    }
    // keys of absent candidates are 0 and never among the `per` there are
    const uint32_t t = max(nth_of_lanes(best, per), 1u);
    int cnt = 0;
    auto collect = [&](const Cand &x) {
      const bool in = x.key >= t;
      const unsigned long long bal = __ballot(in);
      if (bal == 0) return;
      const int at = cnt + __popcll(bal & ((1ull << lane) - 1));
      if (in && at < LIST) list[at] = x;
      cnt += __popcll(bal);
    };
#pragma unroll
    for (int k = 0; k < HELD; ++k) collect(held[k]);
    for (int i0 = 64 * HELD; i0 < all; i0 += 64) collect(i0 + lane < all ? c[i0 + lane] : Cand{0u, -1});
    if (cnt <= LIST) {
      rank_list(list, cnt, [&](int rank, const Cand &x) {
        if (rank < per) {
          token[b * n + rank] = x.idx;
          total[b * n + rank] = score + ((double)of_key(x.key) - lse);
        }
      });
    } else {
      // many equal logits: the best of all again and again
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
  __syncthreads();
  // A candidate's rank: those before it in its own beam, and in every other
  // beam those with a larger total, or an equal one where that beam comes
  // first.  Each beam's totals go down, so those are found by bisection.
  for (int i = threadIdx.x; i < K * per; i += blockDim.x) {
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

// Logits of a lane: 32, or 8 where that leaves the join of a row one segment a
// lane and no more candidates than its lanes hold, and the GPU's 1024 SIMDs at
// most a wave each, so that a call is one wave's time.  8 against 32, bf16, us: 4
// rows of 8000 logits 8.7 / 9.7, of 32000 8.9 / 9.6, 16 rows of 32000 in requests
// of eight 12.4 / 12.7; past a limit 8 rows of 65000 16.6 / 13.0, 64 rows of 32000
// 13.9 / 13.1, 512 rows 28.9 / 22.0; more candidates: 12 beams of 32000 20.6 /
// 16.9, 16 44.8 / 23.9, 4 beams and 64 candidates 874 / 290.
static int lane_logits(int rows, int vocab, int n_out) {
  const int n_seg = segments(vocab, 64 * 8);
  return n_seg <= 64 && n_out <= HELD && (int64_t)rows * n_seg <= 1024 ? 8 : 32;
}

size_t beam_work(int rows, int vocab, int n_out) {
  const size_t n_seg = segments(vocab, 64 * lane_logits(rows, vocab, n_out));
  return (size_t)rows * n_seg * (n_out * sizeof(Cand) + sizeof(SegStat));
}

hipError_t launch_beam(int dtype, const BeamArgs &a, hipStream_t s) {
  const int rows = a.requests * a.beams, lane = lane_logits(rows, a.vocab, a.n_out);
  const int n_seg = segments(a.vocab, 64 * lane);
  Cand *cand = (Cand *)a.work;
  SegStat *stat = (SegStat *)(cand + (size_t)rows * n_seg * a.n_out);
  const unsigned grid = (unsigned)((rows * n_seg + WAVES - 1) / WAVES);
  if (dtype == DEX_F32) {
    if (lane == 8) beam_segment_kernel<float, 8><<<grid, WAVES * 64, 0, s>>>(a, n_seg, cand, stat);
    else beam_segment_kernel<float, 32><<<grid, WAVES * 64, 0, s>>>(a, n_seg, cand, stat);
  } else {
    if (lane == 8) beam_segment_kernel<uint16_t, 8><<<grid, WAVES * 64, 0, s>>>(a, n_seg, cand, stat);
    else beam_segment_kernel<uint16_t, 32><<<grid, WAVES * 64, 0, s>>>(a, n_seg, cand, stat);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t kn = (size_t)a.beams * a.n_out;
  const int waves = a.beams < JOIN_WAVES ? a.beams : JOIN_WAVES;
  // at most 48 KiB of totals and tokens (64 beams of 64) and 16 KiB of lists: within 64 KiB
  const size_t lds = kn * 8 + (kn + (kn & 1)) * 4 + waves * LIST_ROOM * sizeof(Cand);
  beam_join_kernel<<<a.requests, waves * 64, lds, s>>>(a, n_seg, cand, stat);
  return hipGetLastError();
}

}  // namespace dex
