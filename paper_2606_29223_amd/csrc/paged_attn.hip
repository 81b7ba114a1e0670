// Attention of one new token a row over a paged cache, split over the keys
// and joined.
//
// Row r with query heads h sees the keys lo <= j < len of its sequence whose
// page is there: s_j = scale q.k_j, out = sum e^{s_j - m} v_j / sum e^{s_j - m},
// lse = m + ln sum e^{s_j - m}.
//
// A row's keys are cut into units of 64 at fixed places of the sequence, its
// units into at most 96 runs of 2^n units, and four runs are a split (RowPlan).
// A workgroup takes a split, a wave each run with a running maximum and sum;
// the four meet in LDS, and the join adds a row's splits in a fixed order.  All
// of that follows from the row's own length and window, so its bits do not
// depend on the call's other rows.
//
// A unit is S^T = K Q^T and O^T = V^T P^T on the matrix cores, the kv head's
// query heads as columns, so that each lane holds the scores and outputs of
// one query head.  Keys and values are read once from HBM, which bounds the
// kernel; the products are 5 % of what the matrix cores could do meanwhile.
// That is why P goes through them in three bf16 parts, which are all of its 24
// bits, so that weights are as exact as in fp32: against two parts (2^-17) it
// costs 0 to 3 % (16 x 2000 keys 37.5 and 38.2 us, 8 x 8300 62.6 and 62.5).
//
// Measured (32 / 8 heads of 128, bf16): 8 rows of 8300 keys 58.8 us and the join
// 4.8 for 272 MB, 4.6 TB/s in the kernel; 64 rows of 1 to 16000 keys 100 + 5.1
// (461 MB); the loads alone, without products, take as long (392 of 395 us at 64
// x 8000).  Items go to the workgroups in turn whatever their size, and the most
// loaded one has 1.5 and 1.4 to 1.7 times the mean's keys there.  A single short
// row is the latency of the chain length, table, keys, products, join: 9.3 + 3.5
// us at 700 keys.  Splits: with 32 a row the records cost 64 x 8000 keys 5 %,
// with 16 one long row lost 8 %.
#include "attn_decode.h"
#include "dex.h"
#include "paged.h"

#include <algorithm>

namespace dex {

namespace {

constexpr int PA_WAVES = 4;
constexpr int PA_THREADS = PA_WAVES * 64;
constexpr int PA_UNIT = 64;               // keys of a unit
constexpr int PA_SPLITS = 24;             // splits of a row at most
constexpr int PA_ROWS = 512;              // rows of a launch
constexpr int PA_COLS = 32;               // query heads of an item
constexpr int kAlone = 256;               // in share_of: the row is one split (of PA_SPLITS at most)
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// How a row of `len` keys is cut: units [unit0, unit0 + units), 2^shift a run.
struct RowPlan {
  int lo, unit0, units, shift, n;         // lo: first key; n: splits
};
__host__ __device__ __forceinline__ RowPlan row_plan(int len, int window) {
  RowPlan p;
  p.lo = window > 0 && len > window ? len - window : 0;
  p.unit0 = p.lo / PA_UNIT;
  p.units = len > 0 ? (len - 1) / PA_UNIT - p.unit0 + 1 : 0;
  p.shift = 0;
  while ((p.units - 1) >> p.shift >= PA_SPLITS * PA_WAVES) ++p.shift;
  p.n = len > 0 ? ((p.units - 1) >> p.shift) / PA_WAVES + 1 : 1;   // an empty row has one, to say so
  return p;
}
constexpr int kSplitKeys = PA_UNIT * PA_WAVES;              // keys of a split, times 2^shift

// A wave's: the values (or keys) of a unit, then its part of a split's sums.
template <typename T, int HD, int NB>
union Lds {
  uint16_t v[sizeof(T) == 2 ? PA_UNIT : 1][HD + 16];
  float o[16 * NB][HD + 4];
};
// Barrier for what the workgroup's waves leave each other in LDS; loads from
// memory stay on their way across it.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Scores of NT 16-key tiles to powers of two under the new reference m; l is
// this lane's part of their sum.  Keys outside `mask` get 0.  Returns by what
// earlier sums shrink.
template <int NT>
__device__ __forceinline__ float soften(pf_f32x4 (&sc)[NT], unsigned long long mask, bool full, float scale2, float &m,
                                        float &l) {
  const unsigned long long mine = mask >> (4 * ((threadIdx.x & 63) >> 4));   // bit 16 nt + i: the lane's keys
  float mx = -INFINITY;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = sc[nt][i] * scale2;
      if (!full && !(mine >> (nt * 16 + i) & 1)) v = -INFINITY;
      sc[nt][i] = v;
      mx = fmaxf(mx, v);
    }
  const float m1 = fmaxf(m, quad_max(mx));
  const float ref = m1 == -INFINITY ? 0.f : m1;              // nothing seen yet: every power is 0
  const float shrink = __builtin_amdgcn_exp2f(m - ref);
  float sum = 0.f;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sc[nt][i] = __builtin_amdgcn_exp2f(sc[nt][i] - ref);
      sum += sc[nt][i];
    }
  l = fmaf(l, shrink, sum);
  m = m1;
  return shrink;
}

// One wave's work on tiles of TK keys, for 16 NB columns (column r16 of block
// nb).  `rows` of a tile: lane j holds the cache row of key j, or 0 where its
// page is none (row 0 is there; what is read for a key that is not attended to
// is put out).  RUN neighbouring keys lie in one page, so their address is one
// scalar and a lane's offset from it never changes: the 4, 8 or 16 keys of a
// 1 KB load in bf16, 16 in fp32.  RUN 1, for smaller pages and for queries or
// outputs off a 16-byte boundary, has an address a lane and accesses by
// elements (16 x 2000 keys of 128 bf16: 50 us against 36).
template <typename T, int HD, int NB, int RUN>
struct Wave;

// The cache rows that begin with key j of a tile, the same j for all lanes.
template <typename T, int HD>
__device__ __forceinline__ const char *run_at(const void *base, uint32_t rows, int j) {
  const uint32_t r = (uint32_t)__builtin_amdgcn_readlane((int)rows, j);
  return (const char *)base + (uint64_t)r * (HD * sizeof(T));
}
// The cache row of key j (any lane's choice of j).
template <typename T, int HD>
__device__ __forceinline__ const char *row_at(const void *base, uint32_t rows, int j) {
  return (const char *)base + (uint64_t)(uint32_t)__shfl((int)rows, j, 64) * (HD * sizeof(T));
}

// A float's upper half is a bf16, and what is left of its 24 bits after that two
// more: three parts that are the float, with no rounding.  Where nothing is left
// a part is the least bf16, 2^-133 (the products keep it), not 0, so that an
// infinite value times its weight, the sum over the parts, is infinite (0 would
// make it NaN).  The two add at most 2^-132 to a weight, which goes to 0 below
// 2^-126 in the power already.
__device__ __forceinline__ uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float after_upper(float a) {
  return fmaxf(a - __uint_as_float(__float_as_uint(a) & 0xffff0000u), 0x1p-133f);
}

// bf16: a tile is a unit.  Keys and values come as whole rows, 1 KB a load
// (keys in fragment order are sixteen 64-byte pieces, 4 % slower), and go
// through LDS: keys are read back as fragments, values transposed.
template <int HD, int NB, int RUN>
struct Wave<uint16_t, HD, NB, RUN> {
  static constexpr int TK = 64, NT = 4, KS = HD / 32, DT = HD / 16, V4 = HD / 8, RPI = 64 / V4;
  pf_bf16x8 q[NB][KS];
  // Two column blocks of 128 dimensions leave room for a tile's keys or its
  // values on their way, not both: then both use k, in turns.
  static constexpr bool kTurns = HD * NB > 128;
  uint4 k[V4], v[kTurns ? 1 : V4];
  // Values of a product read from LDS ahead of their use: the next tile is in
  // registers, and with more the compiler spills (two column blocks with four:
  // 105 us for 99 at 16 x 8 beams; an address a lane with four: 52 for 44 at 16 x
  // 2000 keys).
  static constexpr int kReads = NB > 1 ? 2 : RUN > 1 ? 4 : 1;
  pf_f32x4 o[NB][DT];

  // a column's query, from `src` (null: none)
  __device__ __forceinline__ void load_q(int nb, const uint16_t *src) {
    const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (src != nullptr) {
        if constexpr (RUN > 1) {
          x = *(const uint4 *)(src + st * 32 + grp * 8);
        } else {
          uint16_t e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = src[st * 32 + grp * 8 + i];
          __builtin_memcpy(&x, e, 16);
        }
      }
      q[nb][st] = __builtin_bit_cast(pf_bf16x8, x);
    }
  }
  __device__ __forceinline__ static void load(const void *base, uint32_t rows, uint4 (&x)[V4]) {
    const int lane = threadIdx.x & 63;
    const uint32_t off = RUN == 1 ? (lane % V4) * 16 : (lane / V4) * (HD * 2) + (lane % V4) * 16;
#pragma unroll
    for (int c = 0; c < V4; ++c) {
      if constexpr (RUN == 1) {
        x[c] = *(const uint4 *)(row_at<uint16_t, HD>(base, rows, c * RPI + lane / V4) + off);
      } else {
        static_assert(RUN % RPI == 0, "a load's rows lie in one run");
        const int key = c * RPI;
        x[c] = *(const uint4 *)(run_at<uint16_t, HD>(base, rows, key / RUN * RUN) + off + (key % RUN) * (HD * 2));
      }
    }
  }
  __device__ __forceinline__ static void stage(const uint4 (&x)[V4], Lds<uint16_t, HD, NB> &lds) {
    const int lane = threadIdx.x & 63;
    uint16_t *to = &lds.v[lane / V4][(lane % V4) * 8];       // the rest are constants of the instructions
#pragma unroll
    for (int c = 0; c < V4; ++c) *(uint4 *)(to + c * RPI * (HD + 16)) = x[c];
    wave_lds_sync();
  }
  __device__ __forceinline__ void load_k(const void *base, uint32_t rows) { load(base, rows, k); }
  __device__ __forceinline__ void load_v(const void *base, uint32_t rows) {
    if constexpr (kTurns) load(base, rows, k);
    else load(base, rows, v);
  }
  __device__ __forceinline__ void stage_k(Lds<uint16_t, HD, NB> &lds) const { stage(k, lds); }
  __device__ __forceinline__ void scores(int nb_used, pf_f32x4 (&sc)[NB][NT], const Lds<uint16_t, HD, NB> &lds) const {
    const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
    const uint16_t *from = &lds.v[r16][grp * 8];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      pf_bf16x8 kf[KS];
#pragma unroll
      for (int st = 0; st < KS; ++st) kf[st] = *(const pf_bf16x8 *)(from + nt * 16 * (HD + 16) + st * 32);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        if (nb < nb_used) {
          sc[nb][nt] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int st = 0; st < KS; ++st)
            sc[nb][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[st], q[nb][st], sc[nb][nt], 0, 0, 0);
        }
    }
  }
  // values to LDS, those of absent keys as zeros (0 times NaN is not 0)
  __device__ __forceinline__ void stage_v(unsigned long long mask, bool full, Lds<uint16_t, HD, NB> &lds) {
    if constexpr (kTurns) stage_masked(k, mask, full, lds);
    else stage_masked(v, mask, full, lds);
  }
  __device__ __forceinline__ static void stage_masked(uint4 (&x)[V4], unsigned long long mask, bool full,
                                                      Lds<uint16_t, HD, NB> &lds) {
    if (!full) {
      const unsigned long long mine = mask >> ((threadIdx.x & 63) / V4);
#pragma unroll
      for (int c = 0; c < V4; ++c)
        if (!(mine >> (c * RPI) & 1)) x[c] = make_uint4(0, 0, 0, 0);
    }
    stage(x, lds);
  }
  __device__ __forceinline__ void outputs(int nb, const pf_f32x4 (&p)[NT], const Lds<uint16_t, HD, NB> &lds) {
    const int lane = threadIdx.x & 63, tq = lane >> 4, ti = (lane & 15) >> 2, tg = lane & 3;
    const uint16_t *from = &lds.v[4 * tq + ti][4 * tg];
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      if constexpr (NB > 1) __builtin_amdgcn_sched_barrier(0);
      uint32_t part[3][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a = p[2 * st + i / 2][2 * (i % 2)], b = p[2 * st + i / 2][2 * (i % 2) + 1];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          part[k][i] = upper_halves(a, b);
          a = after_upper(a);
          b = after_upper(b);
        }
      }
      pf_bf16x8 pp[3];
#pragma unroll
      for (int k = 0; k < 3; ++k)
        pp[k] = __builtin_bit_cast(pf_bf16x8, make_uint4(part[k][0], part[k][1], part[k][2], part[k][3]));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const pf_bf16x8 vf = tr_frag(from + 32 * st * (HD + 16) + 16 * dt, from + (32 * st + 16) * (HD + 16) + 16 * dt);
#pragma unroll
        for (int k = 0; k < 3; ++k) o[nb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pp[k], o[nb][dt], 0, 0, 0);
        if (dt % kReads == kReads - 1) __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // dimension of o[.][dt][i]: four neighbours in a register
  static constexpr int kRun = 4;
  __device__ __forceinline__ static int dim(int dt, int i) { return 16 * dt + 4 * ((threadIdx.x & 63) >> 4) + i; }
};

// fp32, on the fp32 matrix instructions: a tile is half a unit.  A key lane
// holds dimensions 4 grp .. + 3 of each 16, so one 16-byte load feeds four
// k-steps; a value lane holds W neighbouring dimensions of one key, each the
// row of another 16-dimension tile, so values need no transposition: tile
// (b, e) holds the dimensions 16 W b + W i + e.
template <int HD, int NB, int RUN>
struct Wave<float, HD, NB, RUN> {
  static constexpr int TK = 32, NT = 2, DT = HD / 16, W = HD >= 64 ? 4 : 2, VB = HD / (16 * W);
  typedef __attribute__((ext_vector_type(W))) float vecw;
  static constexpr bool kTurns = false;
  pf_f32x4 q[NB][DT], k[NT][DT];
  vecw v[NT][4][VB];
  pf_f32x4 o[NB][DT];

  __device__ __forceinline__ void load_q(int nb, const float *src) {
    const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      pf_f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (src != nullptr) {
        if constexpr (RUN > 1) {
          x = *(const pf_f32x4 *)(src + t * 16 + grp * 4);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = src[t * 16 + grp * 4 + i];
        }
      }
      q[nb][t] = x;
    }
  }
  __device__ __forceinline__ void load_k(const void *base, uint32_t rows) {
    const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
    const uint32_t off = RUN == 1 ? grp * 16 : r16 * (HD * 4) + grp * 16;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const char *p = RUN == 1 ? row_at<float, HD>(base, rows, nt * 16 + r16) : run_at<float, HD>(base, rows, nt * 16);
#pragma unroll
      for (int t = 0; t < DT; ++t) k[nt][t] = *(const pf_f32x4 *)(p + off + t * 64);
    }
  }
  __device__ __forceinline__ void load_v(const void *base, uint32_t rows) {
    const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
    const uint32_t off = RUN == 1 ? r16 * (W * 4) : 4 * grp * (HD * 4) + r16 * (W * 4);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char *p = RUN == 1 ? row_at<float, HD>(base, rows, nt * 16 + 4 * grp + i)
                               : run_at<float, HD>(base, rows, nt * 16) + i * (HD * 4);
#pragma unroll
        for (int b = 0; b < VB; ++b) v[nt][i][b] = *(const vecw *)(p + off + b * (64 * W));
      }
  }
  __device__ __forceinline__ void stage_k(Lds<float, HD, NB> &) const {}
  __device__ __forceinline__ void scores(int nb_used, pf_f32x4 (&sc)[NB][NT], const Lds<float, HD, NB> &) const {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      if (nb < nb_used) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // four sums of a quarter of the dimensions each: one sum of all rounds more
          // (outputs over 700 keys of 128 are 1.1e-6 off for 4e-7, times are equal)
          pf_f32x4 part[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            part[e] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < DT; ++t)
              part[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[nt][t][e], q[nb][t][e], part[e], 0, 0, 0);
          }
          sc[nb][nt] = (part[0] + part[1]) + (part[2] + part[3]);
        }
      }
  }
  __device__ __forceinline__ void stage_v(unsigned long long mask, bool full, Lds<float, HD, NB> &) {
    if (!full) {
      const unsigned long long mine = mask >> (4 * ((threadIdx.x & 63) >> 4));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int b = 0; b < VB; ++b)
            if (!(mine >> (nt * 16 + i) & 1)) v[nt][i][b] = (vecw)0.f;
    }
  }
  __device__ __forceinline__ void outputs(int nb, const pf_f32x4 (&p)[NT], const Lds<float, HD, NB> &) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < VB; ++b)
#pragma unroll
          for (int e = 0; e < W; ++e)
            o[nb][b * W + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[nt][i][b][e], p[nt][i], o[nb][b * W + e], 0, 0, 0);
  }
  static constexpr int kRun = 1;
  __device__ __forceinline__ static int dim(int dt, int i) {
    return 16 * W * (dt / W) + W * (4 * ((threadIdx.x & 63) >> 4) + i) + dt % W;
  }
};

template <typename T>
__device__ __forceinline__ void put(T *p, float v) {
  if constexpr (sizeof(T) == 2) *p = __builtin_bit_cast(uint16_t, (__bf16)v);
  else *p = v;
}
// What a sum over l is multiplied by: a NaN as it is, nothing as 0.
__device__ __forceinline__ float inverse(float l) { return l > 0.f ? 1.f / l : l != l ? l : 0.f; }
__device__ __forceinline__ float log_sum(float m, float l) { return (m + __builtin_amdgcn_logf(l)) * kLn2; }

// Records: [rows][heads][smax] of HD floats, then (m, l) of each.
__device__ __forceinline__ size_t rec_index(const PagedAttnArgs &a, int row, int head, int split, int smax) {
  return ((size_t)row * a.n_heads + head) * smax + split;
}

// The keys row r attends to: 0 where its sequence is none.
__device__ __forceinline__ int row_keys(const PagedAttnArgs &a, int r) {
  const int s = a.seq != nullptr ? a.seq[r] : r;
  const int n = min(min(a.len[r], a.max_len), a.map.max_pages << a.map.shift);
  return s >= 0 && s < a.map.n_seqs && n > 0 ? n : 0;
}

// Four neighbouring dimensions of a row's output, and its lse.
template <typename T, int RUN>
__device__ __forceinline__ void finish(const PagedAttnArgs &a, int row, int head, int d, const pf_f32x4 &o, float m,
                                       float l) {
  const float inv = inverse(l);
  T *out = (T *)a.out + (int64_t)row * a.out_row + (int64_t)head * a.out_head + d;
  if constexpr (RUN > 1) {
    rec_store4(out, o * inv);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) put(out + i, o[i] * inv);
  }
  if (d == 0 && a.lse != nullptr) a.lse[(size_t)row * a.n_heads + head] = log_sum(m, l);
}
// Rows of a group (group_rows of them, from a leader on) that share leading
// splits: share[r] is how many the leader takes for all of them.
struct Sharing {
  int group, rows;                        // the caller's group; rows a leader takes along
  const int *share;                       // null: none
};
__device__ __forceinline__ int place_in_group(const Sharing &g, int r) { return r % g.group % g.rows; }
__device__ __forceinline__ int group_rows(const Sharing &g, int r, int n_rows) {   // r a leader
  return min(min(g.rows, g.group - r % g.group), n_rows - r);
}

// The leading splits that are the same keys for every row of a group: one
// workgroup compares their table rows (6 us; 16 x 8 rows that share 4000 of 4090
// keys then take 99 us in all, alone 249).  They are the same work only where all
// rows are cut alike and see all of the split, or all have one length; one row
// that is not (an empty one, one of another shift) leaves each to itself.
__global__ __launch_bounds__(PA_THREADS) void paged_share_kernel(PagedAttnArgs a, Sharing g, int *share) {
  __shared__ int lens[PA_COLS], seqs[PA_COLS], first;
  const int tid = threadIdx.x, parts = (g.group + g.rows - 1) / g.rows;
  const int r0 = blockIdx.x / parts * g.group + blockIdx.x % parts * g.rows;
  if (r0 >= a.n_rows) return;
  const int nr = group_rows(g, r0, a.n_rows);
  if (tid < nr) {
    lens[tid] = row_keys(a, r0 + tid);
    seqs[tid] = a.seq != nullptr ? a.seq[r0 + tid] : r0 + tid;
  }
  __syncthreads();
  const int len = lens[0];
  const RowPlan pl = row_plan(len, a.window);
  int least = len;
  bool alike = nr > 1 && len > 0, equal = true;
  for (int i = 1; i < nr; ++i) {
    const int n = lens[i];
    const RowPlan p = row_plan(n, a.window);
    least = min(least, n);
    equal = equal && n == len;
    alike = alike && n > 0 && p.shift == pl.shift && p.lo == pl.lo;
  }
  int n_share = 0;
  if (alike) {
    // the first column of the table where a row differs
    const int c0 = (pl.unit0 * PA_UNIT) >> a.map.shift, c1 = (least + (1 << a.map.shift) - 1) >> a.map.shift;
    if (tid == 0) first = c1;
    __syncthreads();
    int mine = c1;
    for (int c = c0 + tid; c < mine; c += PA_THREADS) {
      const int p = a.map.table[(size_t)seqs[0] * a.map.max_pages + c];
      bool differs = false;
#pragma unroll 4
      for (int i = 1; i < nr; ++i) differs |= a.map.table[(size_t)seqs[i] * a.map.max_pages + c] != p;
      if (differs) mine = c;
    }
    if (mine < c1) atomicMin(&first, mine);
    __syncthreads();
    // the keys before `until` lie on the same pages
    const int until = first == c1 ? least : first << a.map.shift;
    n_share = equal && until == len ? pl.n : max(0, until - pl.unit0 * PA_UNIT) / (kSplitKeys << pl.shift);
  }
  if (tid < nr) share[r0 + tid] = n_share;
}

// Where a workgroup is in its work: a tile of its waves' runs of an item.
struct Place {
  int item;                               // >= the number of items: nowhere
  int row, rows, head, head0, cols, split, seq, lo, len;   // kv head; first query head; heads a row
  int tile, tiles, key, end;              // of the run; this wave's first key of the tile; the row's end
};

template <typename T, int HD, int NB, int RUN>
__global__ __launch_bounds__(PA_THREADS, sizeof(T) == 4 && HD * NB > 128 ? 1 : 2) void paged_attn_kernel(PagedAttnArgs a, Sharing g, int smax, float *rec,
                                                                 float2 *stat) {
  using W = Wave<T, HD, NB, RUN>;
  constexpr int UNIT_TILES = PA_UNIT / W::TK;
  // (the LDS below is at most half of a compute unit's 160 KiB, 80.9 KB at
  // head_dim 128 in bf16; with 82.5 KB one workgroup a unit was left and 8 x
  // 8300 keys took 77 us for 62)
  __shared__ Lds<T, HD, NB> lds_all[PA_WAVES];
  __shared__ int first_item[PA_ROWS], keys_of[PA_ROWS], share_of[PA_ROWS];   // items before a row's; its keys
  __shared__ int part[PA_WAVES];
  __shared__ float wm[PA_WAVES][16 * NB], wl[PA_WAVES][16 * NB];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Lds<T, HD, NB> &lds = lds_all[wave];
  const int kv = a.map.n_kv_heads, G = a.n_heads / kv;
  const int chunks = (G + PA_COLS - 1) / PA_COLS, per_split = kv * chunks;   // items of a split
  const float scale2 = a.scale * kLog2e;
  // number the items: every row's splits, the kv heads of a split together
  int items;
  {
    constexpr int PER = PA_ROWS / PA_THREADS;
    int n[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int r = tid * PER + k;
      const int len = r < a.n_rows ? row_keys(a, r) : 0;
      const int sh = g.share != nullptr && r < a.n_rows ? g.share[r] : 0;
      keys_of[r] = len;
      int c = row_plan(len, a.window).n;
      share_of[r] = c == 1 ? sh | kAlone : sh;
      if (sh > 0 && place_in_group(g, r) > 0) c -= sh;
      n[k] = r < a.n_rows ? c * per_split : 0;
      sum += n[k];
    }
    int x = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int before = x - sum;
    items = 0;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) {
      if (w < wave) before += part[w];
      items += part[w];
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      first_item[tid * PER + k] = before;
      before += n[k];
    }
    __syncthreads();
  }
  items = __builtin_amdgcn_readfirstlane(items);
  auto begin = [&](Place &p) {            // the item's first tile
    int lo = 0, hi = a.n_rows - 1;
    while (lo < hi) {                     // the last row with items at or before this one
      const int mid = (lo + hi + 1) >> 1;
      if (__builtin_amdgcn_readfirstlane(first_item[mid]) <= p.item) lo = mid;
      else hi = mid - 1;
    }
    p.row = lo;
    const int rem = p.item - __builtin_amdgcn_readfirstlane(first_item[lo]);
    p.len = __builtin_amdgcn_readfirstlane(keys_of[lo]);
    p.split = rem / per_split;
    const int hc = rem - p.split * per_split, chunk = hc / kv;
    p.head = hc - chunk * kv;
    p.head0 = p.head * G + chunk * PA_COLS;
    p.cols = min(PA_COLS, G - chunk * PA_COLS);
    p.rows = 1;
    const int sh = __builtin_amdgcn_readfirstlane(share_of[lo]) & (kAlone - 1);
    if (sh > 0) {
      if (place_in_group(g, lo) > 0) p.split += sh;
      else if (p.split < sh) p.rows = group_rows(g, lo, a.n_rows);
    }
    p.seq = a.seq != nullptr ? __builtin_amdgcn_readfirstlane(a.seq[lo]) : lo;
    const RowPlan pl = row_plan(p.len, a.window);
    p.lo = pl.lo;
    p.tile = 0;
    p.tiles = UNIT_TILES << pl.shift;
    p.key = (pl.unit0 + ((p.split * PA_WAVES + wave) << pl.shift)) * PA_UNIT;
    p.end = (pl.unit0 + pl.units) * PA_UNIT;
  };
  auto next = [&](Place &p) {             // the tile after p
    p.key += W::TK;
    if (++p.tile < p.tiles) return;
    p.item += gridDim.x;
    if (p.item < items) begin(p);
  };
  // the cache rows of a tile's keys; which of them the row attends to
  auto look = [&](const Place &p) -> uint32_t {
    if (p.item >= items || p.len == 0 || p.key >= p.end) return kNoRow;
    return page_row(a.map, p.seq, p.key + (lane & (W::TK - 1)), p.head);
  };
  auto seen = [&](const Place &p, uint32_t r) -> unsigned long long {
    const int key = p.key + lane;
    return __ballot(lane < W::TK && key >= p.lo && key < p.len && r != kNoRow);
  };
  auto there = [](uint32_t r) { return r == kNoRow ? 0u : r; };
  Place cur;
  cur.item = blockIdx.x;
  if (cur.item >= items) return;
  W w;
  float m[NB], l[NB];
  // column c of an item: query head head0 + c % cols of row row + c / cols
  auto query = [&](const Place &p) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int c = nb * 16 + r16, i = c / p.cols;
      const T *src = (const T *)a.q + (int64_t)(p.row + i) * a.q_row + (int64_t)(p.head0 + c - i * p.cols) * a.q_head;
      w.load_q(nb, i < p.rows ? src : nullptr);
    }
  };
  auto clear = [&] {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb] = -INFINITY;
      l[nb] = 0.f;
#pragma unroll
      for (int dt = 0; dt < W::DT; ++dt) w.o[nb][dt] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  begin(cur);
  uint32_t rows = look(cur);
  w.load_k(a.k, there(rows));
  if constexpr (!W::kTurns) w.load_v(a.v, there(rows));
  query(cur);
  clear();
  Place nxt = cur;
  next(nxt);
  uint32_t rows1 = look(nxt);
  for (;;) {
    // the tile after next is looked up while this one is worked on, and the
    // next one's keys and values are on their way as soon as registers allow
    Place far = nxt;
    if (far.item < items) next(far);
    const uint32_t rows2 = look(far);
    const unsigned long long mask = seen(cur, rows);
    const bool full = mask == (W::TK == 64 ? ~0ull : 0xffffffffull);
    const int nb_used = (cur.rows * cur.cols + 15) / 16;
    pf_f32x4 sc[NB][W::NT];
    const bool last = nxt.item != cur.item;                  // cur is its item's last tile
    w.stage_k(lds);
    if constexpr (W::kTurns) w.load_v(a.v, there(rows));
    w.scores(nb_used, sc, lds);
    // (without these the scheduler moves loads over the products that free
    // their registers, and spills)
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!W::kTurns) w.load_k(a.k, there(rows1));
    if (last && nxt.item < items) query(nxt);
    if constexpr (sizeof(T) == 2) wave_lds_sync();           // the keys are read before values take their place
    w.stage_v(mask, full, lds);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (W::kTurns) w.load_k(a.k, there(rows1));
    else if constexpr (sizeof(T) == 2) w.load_v(a.v, there(rows1));
    if (mask != 0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        if (nb < nb_used) {
          const float shrink = soften<W::NT>(sc[nb], mask, full, scale2, m[nb], l[nb]);
#pragma unroll
          for (int dt = 0; dt < W::DT; ++dt) w.o[nb][dt] *= shrink;
          w.outputs(nb, sc[nb], lds);
        }
    }
    if constexpr (sizeof(T) == 4) w.load_v(a.v, there(rows1));
    else wave_lds_sync();                 // the values are read before anything takes their place
    if (last) {
      // the four waves' sums under one reference
      const int cols = cur.rows * cur.cols;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int c = nb * 16 + r16;
        const float sum = quad_sum(l[nb]);
        if (c < cols) {
          if (grp == 0) {
            wm[wave][c] = m[nb];
            wl[wave][c] = sum;
          }
#pragma unroll
          for (int dt = 0; dt < W::DT; ++dt) {
            if constexpr (W::kRun == 4) {
              *(pf_f32x4 *)&lds.o[c][W::dim(dt, 0)] = w.o[nb][dt];
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) lds.o[c][W::dim(dt, i)] = w.o[nb][dt][i];
            }
          }
        }
      }
      // The item's rows that are this split alone: output or record goes by the
      // row's own number of splits, as its join does, for of rows that share a
      // split one may end with it (256 keys) where others go on.  (Worked out
      // from each row's length below it spills six registers, 69 us for 62 at 8
      // x 8300 keys.)
      const unsigned long long alone = __ballot(lane < cur.rows && share_of[cur.row + lane] >= kAlone);
      lds_barrier();
      for (int e = tid; e < cols * (HD / 4); e += PA_THREADS) {
        const int c = e / (HD / 4), d = e % (HD / 4) * 4;
        float mm = wm[0][c];
#pragma unroll
        for (int v = 1; v < PA_WAVES; ++v) mm = fmaxf(mm, wm[v][c]);
        const float ref = mm == -INFINITY ? 0.f : mm;
        pf_f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float ll = 0.f;
#pragma unroll
        for (int v = 0; v < PA_WAVES; ++v) {
          const float f = __builtin_amdgcn_exp2f(wm[v][c] - ref);
          const pf_f32x4 x = *(const pf_f32x4 *)&lds_all[v].o[c][d];
          ll = fmaf(f, wl[v][c], ll);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = fmaf(f, x[i], o[i]);
        }
        const int i = c / cur.cols, row = cur.row + i, head = cur.head0 + c - i * cur.cols;
        if (alone >> i & 1) {
          finish<T, RUN>(a, row, head, d, o, mm, ll);
        } else {
          const size_t at = rec_index(a, row, head, cur.split, smax);
          *(pf_f32x4 *)(rec + at * HD + d) = o;
          if (d == 0) stat[at] = make_float2(mm, ll);
        }
      }
      lds_barrier();
      if (nxt.item >= items) break;
      clear();
    }
    cur = nxt;
    nxt = far;
    rows = rows1;
    rows1 = rows2;
  }
}

// A row's records together: HD / 4 lanes a record, AT records at a time (record
// j with the others j % AT), then the AT sums in order.  A workgroup is a
// (row, query head); every record is requested before the statistics are in.
template <typename T, int HD, int RUN>
__global__ __launch_bounds__(PA_THREADS) void paged_join_kernel(PagedAttnArgs a, int smax, const float *rec,
                                                              const float2 *stat) {
  constexpr int LPR = HD / 4, AT = PA_THREADS / LPR, PER = (PA_SPLITS + AT - 1) / AT;
  __shared__ pf_f32x4 sums[AT][LPR];
  __shared__ float lsum[AT];
  const int row = blockIdx.x / a.n_heads, head = blockIdx.x - row * a.n_heads;
  const int n = row_plan(row_keys(a, row), a.window).n;
  if (n == 1) return;
  const int tid = threadIdx.x, lane = tid & 63, j0 = tid / LPR, d = tid % LPR;
  const size_t base = rec_index(a, row, head, 0, smax);
  const float2 mine = lane < n ? stat[base + lane] : make_float2(-INFINITY, 0.f);
  pf_f32x4 x[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = j0 + k * AT;
    x[k] = j < n ? *(const pf_f32x4 *)(rec + (base + j) * HD + 4 * d) : pf_f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float m = wave_max(mine.x);
  const float factor = __builtin_amdgcn_exp2f(mine.x - (m == -INFINITY ? 0.f : m));
  pf_f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const float f = __shfl(factor, j0 + k * AT, 64), lj = __shfl(mine.y, j0 + k * AT, 64);
    if (j0 + k * AT < n) {
      l = fmaf(f, lj, l);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = fmaf(f, x[k][i], o[i]);
    }
  }
  sums[j0][d] = o;
  if (d == 0) lsum[j0] = l;
  __syncthreads();
  if (j0 != 0) return;
#pragma unroll
  for (int k = 1; k < AT; ++k) {
    o += sums[k][d];
    l += lsum[k];
  }
  finish<T, RUN>(a, row, head, 4 * d, o, m, l);
}

int max_splits(int max_len) { return max_len > 0 ? std::min(PA_SPLITS, (max_len - 1) / kSplitKeys + 1) : 1; }

// The call's rows in launches of at most PA_ROWS.
template <typename T, int HD, int NB, int RUN>
hipError_t go(const PagedAttnArgs &a, int rows_along, hipStream_t s) {
  const int smax = max_splits(a.max_len);
  const int group = std::min(a.group, PA_ROWS), at_once = PA_ROWS / group * group;
  for (int r0 = 0; r0 < a.n_rows; r0 += at_once) {
    PagedAttnArgs b = a;
    b.n_rows = std::min(at_once, a.n_rows - r0);
    b.q = (const T *)a.q + r0 * a.q_row;
    b.out = (T *)a.out + r0 * a.out_row;
    b.len = a.len + r0;
    if (a.lse != nullptr) b.lse = a.lse + (size_t)r0 * a.n_heads;
    if (a.seq != nullptr) b.seq = a.seq + r0;
    else b.map.table = a.map.table + (size_t)r0 * a.map.max_pages, b.map.n_seqs = std::max(0, a.map.n_seqs - r0);
    float *rec = (float *)a.work;
    float2 *stat = (float2 *)(rec + (size_t)std::min(a.n_rows, PA_ROWS) * a.n_heads * smax * HD);
    Sharing g{group, rows_along, nullptr};
    hipError_t e;
    const int chunks = (a.n_heads / a.map.n_kv_heads + PA_COLS - 1) / PA_COLS;
    const int64_t row_items = (int64_t)b.n_rows * a.map.n_kv_heads * chunks;
    if (rows_along > 1) {
      int *share = (int *)(stat + (size_t)std::min(a.n_rows, PA_ROWS) * a.n_heads * smax);
      const int parts = (group + rows_along - 1) / rows_along;
      paged_share_kernel<<<(b.n_rows + group - 1) / group * parts, PA_THREADS, 0, s>>>(b, g, share);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      g.share = share;
    }
    // the workgroups that fit a compute unit, by their registers; further items
    // wait their turn in them (two a unit everywhere: 2 to 6 % slower below 128)
    constexpr int kPerUnit = HD * NB > 64 ? 2 : HD * NB == 64 ? 3 : 4;
    paged_attn_kernel<T, HD, NB, RUN>
        <<<(unsigned)std::min<int64_t>(row_items * smax, 256 * kPerUnit), PA_THREADS, 0, s>>>(b, g, smax, rec, stat);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (smax > 1) {
      paged_join_kernel<T, HD, RUN><<<b.n_rows * a.n_heads, PA_THREADS, 0, s>>>(b, smax, rec, stat);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

template <typename T, int HD>
hipError_t go_hd(const PagedAttnArgs &a, hipStream_t s) {
  auto whole = [](const void *p, int64_t row, int64_t head) {
    return (uintptr_t)p % 16 == 0 && row * sizeof(T) % 16 == 0 && head * sizeof(T) % 16 == 0;
  };
  const bool vectors = whole(a.q, a.q_row, a.q_head) && whole(a.out, a.out_row, a.out_head);
  const int G = a.n_heads / a.map.n_kv_heads;
  // rows whose query heads fill the columns of an item together
  const int along = std::max(1, std::min(std::min(a.group, a.n_rows), PA_COLS / G));
  const bool one = std::min(G, PA_COLS) * along <= 16;
  constexpr int RUN = sizeof(T) == 2 ? 512 / HD : 16;
  if (vectors && 1 << a.map.shift >= RUN) return one ? go<T, HD, 1, RUN>(a, along, s) : go<T, HD, 2, RUN>(a, along, s);
  return one ? go<T, HD, 1, 1>(a, along, s) : go<T, HD, 2, 1>(a, along, s);
}

}  // namespace

size_t paged_attention_work(int n_rows, int n_heads, int head_dim, int max_len, int group) {
  const int smax = max_splits(max_len);
  if (smax == 1 && group == 1) return 0;
  const size_t rows = std::min(n_rows, PA_ROWS);
  return rows * n_heads * smax * (head_dim + 2) * sizeof(float) + rows * sizeof(int);
}

hipError_t launch_paged_attention(int dtype, const PagedAttnArgs &a, hipStream_t s) {
  if (dtype == DEX_F32)
    return a.head_dim == 32 ? go_hd<float, 32>(a, s) : a.head_dim == 64 ? go_hd<float, 64>(a, s) : go_hd<float, 128>(a, s);
  return a.head_dim == 32 ? go_hd<uint16_t, 32>(a, s)
                          : a.head_dim == 64 ? go_hd<uint16_t, 64>(a, s) : go_hd<uint16_t, 128>(a, s);
}

}  // namespace dex
