// Attention of the rows of a sequence that share its keys: a tree of drafted
// tokens, or one row over chosen pages, or one row whose softmax weights are
// kept.
//
// Row i of a sequence with L keys sees the keys j < L whose page is there and,
// of the drafted keys L + t, those with bit t of its mask: s_j = scale q.k_j,
// out = sum e^{s_j - m} v_j / sum e^{s_j - m}, lse = m + ln sum e^{s_j - m}.
//
// One pass over the keys, with a running reference in place of the maximum.  The
// rows of a sequence and the query heads of a kv head are the columns of the
// products S^T = K Q^T and O^T = V^T P^T, so a tile of keys and values in LDS is
// read for all of them, and a score lies in the lane that needs it as a weight.
//
// What bounds it, bf16 heads of 128, 8 kv heads of 4 query heads, on one MI355X:
// * 8 sequences of 8200 keys, trees of 64 (256 columns): 163 to 172 us a call with
//   its join; in a kernel trace 161 in the first three calls and 189 in the middle
//   of 24, as the clock falls, and the join 15.  The weights go to the matrix cores
//   in three bf16 parts that hold all 24 bits, four products a key and column for
//   the two of the formula: 138 GFLOP, 0.73 to 0.86 PFLOP/s for the 1.2 of a large
//   library product here.  A step of a wave has 2048 cycles of products and as much
//   vector work as fits between them (2.4 us for two waves a SIMD).  Two parts
//   would take 12 % less and round to 17 bits.
// * 24 ragged trees of 25 up to 12000 keys: 79 us, of which the CUs' mean is 43 and
//   the rest the difference between them.  Columns of rows behind n_draft, half of
//   all here, are computed like the others.
// * 32 single rows of 4000 keys: 5.3 TB/s in the kernel, memory's.
// Not better: tiles of 64 keys (they spill, or are equal), three waves a SIMD
// (spills), eight waves a workgroup (equal), the ring four tiles deep (181 us for
// 175: the transfers are not what a step waits for), the next tile's scores
// between the weights of this one (equal).
#include "attn_decode.h"
#include "dex.h"
#include "span.h"

#include <algorithm>
#include <type_traits>

namespace dex {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// What keys that no row sees are read from: a row of zeros.
__device__ uint4 zero_row[32];

// How the keys of a sequence are cut: `n` splits of `steps` steps, a step being
// a tile for each of a workgroup's key groups, at most a quarter longer than
// `least` steps while there are fewer than `smax`.
struct SpanPlan {
  int steps, n;
};
__host__ __device__ __forceinline__ int splits_of(int steps, int least) {
  return max(1, (steps + least - 1 - least / 4) / least);
}
__host__ __device__ __forceinline__ SpanPlan span_plan(int keys, int step_keys, int smax, int least) {
  const int all = (keys + step_keys - 1) / step_keys, n = min(smax, splits_of(all, least));
  SpanPlan p;
  p.steps = max(1, (all + n - 1) / n);
  p.n = max(1, (all + p.steps - 1) / p.steps);
  return p;
}

// What a launch of a case is told beside its arguments.
struct SpanGrid {
  int blocks;                             // column blocks of a (sequence, kv head)
  int smax, least;                        // splits at most, steps of a split at least
  float *rec;                             // [n * draft][n_heads][smax][head_dim]
  float2 *stat;                           // [n * draft][n_heads][smax]: maximum, sum
  float *score;                           // [n][n_heads][score_ld], or null
  int64_t score_ld;
  bool whole;                             // queries and outputs lie on 16-byte boundaries
};

// The sequence's own numbers: keys before the drafted ones, drafted ones, and
// the places that are looked at (all keys, or those of the listed columns).
struct Span {
  int seq, len, drafted, keys;
};
__device__ __forceinline__ Span span_of(const SpanArgs &a, int i) {
  Span s;
  s.seq = a.seq != nullptr ? a.seq[i] : i;
  const bool is = s.seq >= 0 && s.seq < a.map.n_seqs;
  s.len = is ? max(0, min(min(a.len[i], a.max_len), a.map.max_pages << a.map.shift)) : 0;
  s.drafted = 0;
  if (a.mask != nullptr && is) s.drafted = a.n_draft != nullptr ? max(0, min(a.n_draft[i], a.draft)) : a.draft;
  s.keys = s.len + s.drafted;
  if (a.columns != nullptr) s.keys = min(a.n_cols, (s.len + (1 << a.map.shift) - 1) >> a.map.shift) << a.map.shift;
  return s;
}

// Max over the four lanes r16, r16 + 16, + 32, + 48.
__device__ __forceinline__ float quarters_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float quarters_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// A float's upper half is a bf16, and what is left of its 24 bits after that two
// more: three parts that are the float, with no rounding.  Where nothing is left
// a part is the least bf16, 2^-133 (the products keep it), not 0, so that an
// infinite value times its weight, the sum over the parts, is infinite (0 would
// make it NaN).  The two add at most 2^-132 to a weight, which goes to 0 below
// 2^-126 in the power already; only of a weight of 0 would that be too much where
// the key is hidden, so in steps with drafted keys, where values that are no
// finite numbers go by themselves, the parts are what they are.  (To make them 0 for
// a weight of 0 in all steps is one instruction more for two weights: 8 trees of 64
// over 8200 keys 167 us for 164, 24 ragged ones of 25 85 for 81.)
__device__ __forceinline__ uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ float after_upper(float a) { return a - __uint_as_float(__float_as_uint(a) & 0xffff0000u); }
// (positive bf16 compare as integers: one instruction for two)
__device__ __forceinline__ uint32_t some_halves(uint32_t x) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), (u16x2)(uint16_t)1));
}

// A tile of keys or values in LDS: TK rows of HD elements, whose 16-byte chunks
// are swapped within a row (chunk c lies at c ^ swizzle) so that the 16 rows of
// a key fragment, and the rows that half a wave reads of the values, lie in
// different banks.  Filled by direct transfers of 1 KB, RPT rows each.
template <typename T, int HD, int KEYS>
struct Tile {
  static constexpr int TK = KEYS;
  static constexpr int NT = TK / 16, DT = HD / 16;
  static constexpr int RB = HD * sizeof(T), CPR = RB / 16, RPT = 64 / CPR, NTR = TK / RPT;
  static constexpr int BYTES = TK * RB;
  __device__ __forceinline__ static int kswz(int row) {
    return CPR >= 16 ? (row & 15) : CPR == 8 ? ((row >> 1) & 7) : ((row >> 2) & 3);
  }
  __device__ __forceinline__ static int vswz(int row) {
    if (sizeof(T) == 4) return 0;
    return CPR == 16 ? 2 * (row & 7) : CPR == 8 ? 2 * ((row >> 1) & 3) : 2 * ((row >> 2) & 1);
  }
};

// One wave's columns: 16 NB of them, column r16 of block nb; its scores and
// outputs of them on the matrix cores.
template <typename L, typename T, int HD, int NB>
struct Cols;

template <typename L, int HD, int NB>
struct Cols<L, uint16_t, HD, NB> {
  static constexpr int KS = HD / 32, NT = L::NT, DT = L::DT, CPR = L::CPR;
  static_assert(NT == 2, "the keys of one product of the values");
  pf_bf16x8 q[NB][KS];
  pf_f32x4 o[NB][DT];

  __device__ __forceinline__ void load_q(int nb, const uint16_t *src, bool whole, float scale) {
    const int grp = (threadIdx.x & 63) >> 4;
    const uint32_t sign = scale < 0.f ? 0x80008000u : 0u, some = scale != 0.f ? ~0u : 0u;
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (src != nullptr) {
        if (whole) {
          x = *(const uint4 *)(src + st * 32 + grp * 8);
        } else {
          uint16_t e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = src[st * 32 + grp * 8 + i];
          __builtin_memcpy(&x, e, 16);
        }
      }
      x = make_uint4((x.x ^ sign) & some, (x.y ^ sign) & some, (x.z ^ sign) & some, (x.w ^ sign) & some);
      q[nb][st] = __builtin_bit_cast(pf_bf16x8, x);
    }
  }
  // The values' fragments: of 16 dimensions dt, the rows 4 tq .. + 3 and those 16
  // on (tr_frag).  In assembly with its own wait, since the builtin waits for the
  // transfers of the next tile first.
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  struct Values {
    u32x2 lo[DT], hi[DT];
  };
  __device__ __forceinline__ static void read_values(const uint4 *v, Values &f) {
    const int lane = threadIdx.x & 63, ti = (lane & 15) >> 2, tg = lane & 3;
    const int row = 4 * (lane >> 4) + ti;     // and the row 16 on, with the same swizzle
    const uint32_t from = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)v + row * L::RB + (tg & 1) * 8;
    uint32_t at[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) at[dt] = from + ((2 * dt + (tg >> 1)) ^ L::vswz(row)) * 16;
    static_assert(DT % 2 == 0, "two at a time");
    if constexpr (DT % 4 == 0) {
#pragma unroll
      for (int dt = 0; dt < DT; dt += 4)
        asm volatile(
            "ds_read_b64_tr_b16 %0, %8\n ds_read_b64_tr_b16 %1, %8 offset:%12\n"
            "ds_read_b64_tr_b16 %2, %9\n ds_read_b64_tr_b16 %3, %9 offset:%12\n"
            "ds_read_b64_tr_b16 %4, %10\n ds_read_b64_tr_b16 %5, %10 offset:%12\n"
            "ds_read_b64_tr_b16 %6, %11\n ds_read_b64_tr_b16 %7, %11 offset:%12\n"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(f.lo[dt]), "=&v"(f.hi[dt]), "=&v"(f.lo[dt + 1]), "=&v"(f.hi[dt + 1]), "=&v"(f.lo[dt + 2]),
              "=&v"(f.hi[dt + 2]), "=&v"(f.lo[dt + 3]), "=&v"(f.hi[dt + 3])
            : "v"(at[dt]), "v"(at[dt + 1]), "v"(at[dt + 2]), "v"(at[dt + 3]), "i"(16 * L::RB)
            : "memory");
    } else {
      asm volatile(
          "ds_read_b64_tr_b16 %0, %4\n ds_read_b64_tr_b16 %1, %4 offset:%6\n"
          "ds_read_b64_tr_b16 %2, %5\n ds_read_b64_tr_b16 %3, %5 offset:%6\n"
          "s_waitcnt lgkmcnt(0)"
          : "=&v"(f.lo[0]), "=&v"(f.hi[0]), "=&v"(f.lo[1]), "=&v"(f.hi[1])
          : "v"(at[0]), "v"(at[1]), "i"(16 * L::RB)
          : "memory");
    }
  }
  // (also asks for the values, to wait once)
  __device__ __forceinline__ void scores(const uint4 *k, const uint4 *v, Values &f, pf_f32x4 (&sc)[NB][NT]) const {
    const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
    const uint4 *from = k + r16 * CPR;
    // all fragments are asked for before the first product
    pf_bf16x8 kf[KS][2];
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)        // (the swizzle is the same 16 rows on, so one address a k-step)
        kf[st][nt] = __builtin_bit_cast(pf_bf16x8, from[nt * 16 * CPR + ((st * 4 + grp) ^ L::kswz(r16))]);
    __builtin_amdgcn_sched_barrier(0);
    read_values(v, f);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sc[nb][0] = sc[nb][1] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          sc[nb][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[st][nt], q[nb][st], sc[nb][nt], 0, 0, 0);
  }
  // Scores to weights e^(s - reference), in powers of two, whose sum joins l, and
  // o += V^T P^T.  A column block at a time: the vector work on one is laid
  // between the products of the one before.
  template <bool DRAFT>
  __device__ __forceinline__ void outputs(const uint4 *, Values &f, pf_f32x4 (&sc)[NB][NT], float scale2, const float (&m)[NB],
                                          float (&l)[NB]) {
    pf_bf16x8 pp[2][3];
    auto weights = [&](int nb, pf_bf16x8 (&to)[3]) {
      const float ref = m[nb] == -INFINITY ? 0.f : -m[nb];
      float sum = 0.f;
      uint32_t part[3][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float e[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          pf_f32x4 &x = sc[nb][i / 2];
          x[2 * (i % 2) + j] = e[j] = __builtin_amdgcn_exp2f(fmaf(x[2 * (i % 2) + j], scale2, ref));
        }
        sum += e[0] + e[1];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          part[k][i] = upper_halves(e[0], e[1]);
          if (!DRAFT && k > 0) part[k][i] = some_halves(part[k][i]);
          e[0] = after_upper(e[0]);
          e[1] = after_upper(e[1]);
        }
      }
      l[nb] += sum;
#pragma unroll
      for (int k = 0; k < 3; ++k)
        to[k] = __builtin_bit_cast(pf_bf16x8, make_uint4(part[k][0], part[k][1], part[k][2], part[k][3]));
    };
    weights(0, pp[0]);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      __builtin_amdgcn_sched_barrier(0);
      if (nb + 1 < NB) weights(nb + 1, pp[(nb + 1) % 2]);
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const pf_bf16x8 vf = __builtin_bit_cast(pf_bf16x8, make_uint4(f.lo[dt].x, f.lo[dt].y, f.hi[dt].x, f.hi[dt].y));
          o[nb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pp[nb % 2][k], o[nb][dt], 0, 0, 0);
        }
      if (nb + 1 < NB) {
#pragma unroll
        for (int i = 0; i < 3 * DT; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, DT == 8 ? 4 : DT == 4 ? 8 : 16, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ static float value(const void *row, int d) {
    return __uint_as_float((uint32_t)((const uint16_t *)row)[d] << 16);
  }
  // Whether a chunk of values holds one that is no finite number; it without those.
  __device__ __forceinline__ static bool odd_chunk(const uint4 &x) {
    auto odd = [](uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; };
    return odd(x.x) || odd(x.y) || odd(x.z) || odd(x.w);
  }
  __device__ __forceinline__ static uint4 even_chunk(const uint4 &x) {
    auto even = [](uint32_t w) {
      if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
      return (w & 0x7f800000u) == 0x7f800000u ? w & 0xffffu : w;
    };
    return make_uint4(even(x.x), even(x.y), even(x.z), even(x.w));
  }
  // four neighbouring dimensions of an output: which, and their values
  static constexpr int QUADS = DT;
  __device__ __forceinline__ static int dim(int j) { return 16 * j + 4 * ((threadIdx.x & 63) >> 4); }
  __device__ __forceinline__ pf_f32x4 quad(int nb, int j) const { return o[nb][j]; }
  // dimension of o[.][dt][i]
  __device__ __forceinline__ static int dim_of(int dt, int i) { return 16 * dt + 4 * ((threadIdx.x & 63) >> 4) + i; }
};

// fp32: a key lane holds dimensions 4 grp .. + 3 of each 16, so one 16-byte read
// feeds four k-steps; a value lane holds W neighbouring dimensions of one key,
// each the row of another 16-dimension tile.
template <typename L, int HD, int NB>
struct Cols<L, float, HD, NB> {
  static constexpr int NT = L::NT, DT = L::DT, CPR = L::CPR, W = HD >= 64 ? 4 : 2, VB = HD / (16 * W);
  typedef __attribute__((ext_vector_type(W))) float vecw;
  pf_f32x4 q[NB][DT], o[NB][DT];
  struct Values {};

  __device__ __forceinline__ void load_q(int nb, const float *src, bool whole, float scale) {
    const int grp = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      pf_f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (src != nullptr) {
        if (whole) {
          x = *(const pf_f32x4 *)(src + t * 16 + grp * 4);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = src[t * 16 + grp * 4 + i];
        }
      }
      q[nb][t] = scale < 0.f ? -x : scale != 0.f ? x : (pf_f32x4)0.f;
    }
  }
  __device__ __forceinline__ void scores(const uint4 *k, const uint4 *, Values &, pf_f32x4 (&sc)[NB][NT]) const {
    const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
    // four sums of a quarter of the dimensions each: one sum of all rounds more
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      pf_f32x4 part[NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[nb][e] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const pf_f32x4 kf = __builtin_bit_cast(pf_f32x4, k[(16 * nt + r16) * CPR + ((4 * t + grp) ^ L::kswz(r16))]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            part[nb][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], q[nb][t][e], part[nb][e], 0, 0, 0);
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) sc[nb][nt] = (part[nb][0] + part[nb][1]) + (part[nb][2] + part[nb][3]);
    }
  }
  template <bool>
  __device__ __forceinline__ void outputs(const uint4 *v, Values &, pf_f32x4 (&sc)[NB][NT], float scale2, const float (&m)[NB],
                                          float (&l)[NB]) {
    const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float ref = m[nb] == -INFINITY ? 0.f : -m[nb];
      float sum = 0.f;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[nb][nt][i] = __builtin_amdgcn_exp2f(fmaf(sc[nb][nt][i], scale2, ref));
          sum += sc[nb][nt][i];
        }
      l[nb] += sum;
    }
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) {
      const int nt = j / 4, i = j % 4;
      const float *row = (const float *)(v + (16 * nt + 4 * grp + i) * CPR) + r16 * W;
#pragma unroll
      for (int b = 0; b < VB; ++b) {
        const vecw x = *(const vecw *)(row + b * 16 * W);
#pragma unroll
        for (int e = 0; e < W; ++e)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            o[nb][b * W + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], sc[nb][nt][i], o[nb][b * W + e], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ static float value(const void *row, int d) { return ((const float *)row)[d]; }
  __device__ __forceinline__ static bool odd_chunk(const uint4 &x) {
    auto odd = [](uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; };
    return odd(x.x) || odd(x.y) || odd(x.z) || odd(x.w);
  }
  __device__ __forceinline__ static uint4 even_chunk(const uint4 &x) {
    auto even = [](uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u ? 0u : w; };
    return make_uint4(even(x.x), even(x.y), even(x.z), even(x.w));
  }
  static constexpr int QUADS = HD / 16;
  __device__ __forceinline__ static int dim(int j) {
    const int grp = (threadIdx.x & 63) >> 4;
    return W == 4 ? 64 * (j / 4) + 16 * grp + 4 * (j % 4) : 8 * grp + 4 * j;
  }
  __device__ __forceinline__ pf_f32x4 quad(int nb, int j) const {
    if constexpr (W == 4) {
      const int b = 4 * (j / 4), i = j % 4;
      return pf_f32x4{o[nb][b][i], o[nb][b + 1][i], o[nb][b + 2][i], o[nb][b + 3][i]};
    } else {
      return pf_f32x4{o[nb][0][2 * j], o[nb][1][2 * j], o[nb][0][2 * j + 1], o[nb][1][2 * j + 1]};
    }
  }
  __device__ __forceinline__ static int dim_of(int dt, int i) {
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

// Four neighbouring dimensions of a row's output, and with the first its lse.
template <typename T>
__device__ __forceinline__ void finish(const SpanArgs &a, bool whole, int row, int head, int d, const pf_f32x4 &o, float m,
                                       float l) {
  const float inv = inverse(l);
  T *out = (T *)a.out + (int64_t)row * a.out_row + (int64_t)head * a.out_head + d;
  if (whole) {
    rec_store4(out, o * inv);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) put(out + i, o[i] * inv);
  }
  if (d == 0 && a.lse != nullptr) a.lse[(size_t)row * a.n_heads + head] = log_sum(m, l);
}
__device__ __forceinline__ size_t rec_index(const SpanArgs &a, int row, int head, int split, int smax) {
  return ((size_t)row * a.n_heads + head) * smax + split;
}

// A wave's transfers are in LDS, but for the youngest N.
template <int N>
__device__ __forceinline__ void landed() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// The waves of a workgroup: WC neighbouring column blocks over the same keys,
// WK = NW / WC groups of keys.  Waves alone whose tiles would be 128 KB for four
// go by two, since one workgroup on a CU waits for its first tiles: 32 ragged
// rows' weights 78 us with four, 74 with two.
template <typename T, int HD, int NB, int WC>
struct Shape {
  static constexpr int TK = sizeof(T) == 2 ? 32 : 16;
  using L = Tile<T, HD, TK>;
  static constexpr int RING = 4 * L::BYTES;                  // a key group's two tiles of keys and values
  static constexpr int NW = WC > 1 || 4 * RING <= 65536 ? 4 : 2, WK = NW / WC, COLS = 16 * NB * WC;
  static constexpr int STEP = L::TK * WK;                    // keys of a step
  static constexpr int MEET = WK > 1 ? NW * 16 * NB * (HD + 4) * 4 : 0;
  static constexpr int LDS = RING * WK > MEET ? RING * WK : MEET;
};

template <bool TREE, typename T, int HD, int NB, int WC>
__global__ __launch_bounds__((64 * Shape<T, HD, NB, WC>::NW))
    __attribute__((amdgpu_waves_per_eu(WC == 1 && HD * sizeof(T) > 128 ? 1 : 2))) void span_attn_kernel(SpanArgs a, SpanGrid g) {
  using S = Shape<T, HD, NB, WC>;
  using L = typename S::L;
  using C = Cols<L, T, HD, NB>;
  constexpr int TK = L::TK, NT = L::NT, NW = S::NW, WK = S::WK;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  __shared__ float wm[NW][16 * NB], wl[NW][16 * NB];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wc = wave % WC, wk = wave / WC;
  const int kv = a.map.n_kv_heads, G = a.n_heads / kv, cols = a.draft * G;
  // kv heads innermost: with a multiple of eight of them the column blocks and
  // neighbours of a head stay on one XCD
  int x = blockIdx.x;
  const int head = x % kv;
  x /= kv;
  const int block = x % g.blocks;
  x /= g.blocks;
  // (turned on by one each split: workgroups go to the parts of an XCD in turn, and
  // the splits of a long sequence would all go to one of them: 24 ragged trees 102
  // us for 90)
  const int split = x / a.n, b = (x + split) % a.n;
  const Span sp = span_of(a, b);
  const SpanPlan plan = span_plan(sp.keys, S::STEP, g.smax, g.least);
  if (split >= plan.n) return;
  const int first = split * plan.steps * S::STEP;
  const int steps = min(plan.steps, (sp.keys - first + S::STEP - 1) / S::STEP);
  const int c0 = (block * WC + wc) * 16 * NB;                // the wave's first column
  uint4 *ring = (uint4 *)(lds + wk * S::RING);

  // The cache rows of a step's keys, lane j key j's.  The pages of 64 columns are
  // held, lane j the j-th's, so that between the transfers there is hardly ever a
  // load to wait for: a wait is for all that was asked for before.
  auto key_of = [&](int step) { return first + step * S::STEP + wk * TK; };
  int held = 0, page = -1, column = 0;    // column of lane 0; this lane's page and column
  auto hold = [&](int step) {
    held = key_of(step) >> a.map.shift;
    column = held + lane;
    bool is = column <= (sp.keys - 1) >> a.map.shift;        // (no keys, nothing is read: the sequence may be none)
    if (!TREE && a.columns != nullptr) column = a.columns[((size_t)b * kv + head) * a.n_cols + (is ? column : 0)];
    is = is && column >= 0 && column < a.map.max_pages;
    page = a.map.table[is ? (size_t)sp.seq * a.map.max_pages + column : 0];
    if (!is || page >= a.map.n_pages) page = -1;
  };
  auto row = [&](int step) -> uint32_t {
    if (step >= steps) return kNoRow;
    const int key0 = key_of(step);
    if (((key0 + TK - 1) >> a.map.shift) - held >= 64) hold(step);
    const int key = key0 + (lane & (TK - 1)), at = key & ((1 << a.map.shift) - 1), j = (key >> a.map.shift) - held;
    const int p = __shfl(page, j, 64), c = TREE || a.columns == nullptr ? 0 : __shfl(column, j, 64);    // (of all lanes)
    const bool is = key < sp.keys && p >= 0 && (TREE || a.columns == nullptr || (c << a.map.shift) + at < sp.len);
    return is ? (((uint32_t)p * (uint32_t)kv + (uint32_t)head) << a.map.shift) + (uint32_t)at : kNoRow;
  };
  // A step's keys and values into the ring: transfer c moves rows RPT c ..; lane l
  // fills chunk l % CPR of row RPT c + l / CPR with the swizzled one.  Where all
  // keys are there and a transfer's rows lie in one page, its address is one
  // scalar; otherwise a lane's, of zeros for keys that no row sees.
  const bool runs = 1 << a.map.shift >= L::RPT;
  const int l_row = lane / L::CPR, l_chunk = lane % L::CPR;
  auto issue = [&](int step, uint32_t rows) {
    uint4 *to = ring + (step & 1) * (2 * L::BYTES / 16);
    auto move = [&](int c, const char *kp, const char *vp) {
      __builtin_amdgcn_global_load_lds((const void *)kp, (__attribute__((address_space(3))) void *)(to + c * 64), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const void *)vp,
                                       (__attribute__((address_space(3))) void *)(to + L::BYTES / 16 + c * 64), 16, 0, 0);
    };
    auto each = [&](auto address) {
#pragma unroll
      for (int t = 0; t < (L::NTR + WC - 1) / WC; ++t) {
        const int c = t * WC + wc, row = c * L::RPT + l_row;
        if (L::NTR % WC != 0 && c >= L::NTR) break;
        address(c, row, (uint32_t)(l_chunk ^ L::kswz(row)) * 16, (uint32_t)(l_chunk ^ L::vswz(row)) * 16);
      }
    };
    if (runs && __ballot(lane >= TK || rows != kNoRow) == ~0ull) {
      each([&](int c, int, uint32_t kc, uint32_t vc) {
        const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)rows, c * L::RPT) * L::RB;
        const uint32_t in = l_row * L::RB;
        move(c, (const char *)a.k + off + (in + kc), (const char *)a.v + off + (in + vc));
      });
    } else {
      each([&](int c, int row, uint32_t kc, uint32_t vc) {
        const uint32_t at = (uint32_t)__shfl((int)rows, row, 64);
        const uint64_t off = (uint64_t)at * L::RB;
        move(c, (at == kNoRow ? (const char *)zero_row : (const char *)a.k + off) + kc,
             (at == kNoRow ? (const char *)zero_row : (const char *)a.v + off) + vc);
      });
    }
  };

  hold(0);
  uint32_t rows = row(0);
  if (steps > 0) issue(0, rows);
  C w;
  float m[NB], l[NB];                     // reference (powers of two) and this lane's part of the sum
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int c = c0 + nb * 16 + r16;
    const T *src = (const T *)a.q + ((int64_t)b * a.draft + c / G) * a.q_row + (int64_t)(head * G + c % G) * a.q_head;
    w.load_q(nb, c < cols ? src : nullptr, g.whole, a.scale);
    m[nb] = -INFINITY;
    l[nb] = 0.f;
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt) w.o[nb][dt] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale2 = a.scale != 0.f ? fabsf(a.scale) * kLog2e : 1.f;   // the query has the sign, or is 0

  auto work = [&](int step, auto drafted) {
    constexpr bool DRAFT = decltype(drafted)::value;         // the step may have drafted keys
    const uint32_t next = row(step + 1);
    if constexpr (WC > 1) {
      // the step has landed for every wave, and every wave is past the last one,
      // whose place the next takes
      lds_ring_step<0>();
      if (step + 1 < steps) issue(step + 1, next);
      __builtin_amdgcn_sched_barrier(0);
    } else if (step + 1 < steps) {
      issue(step + 1, next);
      landed<2 * L::NTR>();
    } else {
      landed<0>();
    }
    uint4 *k = ring + (step & 1) * (2 * L::BYTES / 16), *v = k + L::BYTES / 16;
    const int key0 = key_of(step);
    const uint32_t there = (uint32_t)__ballot(lane < TK && rows != kNoRow);    // keys that some row may see
    constexpr uint32_t kAll = ~0u >> (32 - TK);
    const bool trees = DRAFT && key0 + TK > sp.len;
    uint32_t odd = 0;
    if (DRAFT) {
      // Drafted values that some rows see and others do not: 0 times an infinity
      // or NaN is not 0, so those leave the tile and go by themselves.  (The same
      // steps for all waves: they share tiles.)
      for (int e = lane; e < TK * L::CPR; e += 64)
        if (C::odd_chunk(v[e])) odd |= (uint32_t)1 << (e / L::CPR);
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) odd |= (uint32_t)__shfl_xor((int)odd, s, 64);
      if constexpr (WC > 1) __syncthreads();
      if (odd != 0) {
        for (int e = lane; e < TK * L::CPR; e += 64) v[e] = C::even_chunk(v[e]);
        wave_lds_sync();
      }
      if constexpr (WC > 1) __syncthreads();
    }
    if (c0 < cols && there != 0) {
      pf_f32x4 sc[NB][NT];
      typename C::Values f;
      w.scores(k, v, f, sc);
      uint32_t sees[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) sees[nb] = there;
      if (trees) {
        // bit t of the row's mask is key len + t; keys before len are seen
        const int d0 = key0 - sp.len, from = max(d0, 0);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int c = min(c0 + nb * 16 + r16, cols - 1);
          const uint64_t *bits = a.mask + ((size_t)b * a.draft + c / G) * a.words;
          const int at = from >> 6, sh = from & 63;
          uint64_t x = at < a.words ? bits[at] >> sh : 0;
          if (sh > 0 && at + 1 < a.words) x |= bits[at + 1] << (64 - sh);
          if (d0 < 0) x = x << -d0 | ((1ull << -d0) - 1);    // (-d0 < TK)
          sees[nb] &= (uint32_t)x;
        }
      }
      if (trees || there != kAll) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const uint32_t mine = sees[nb] >> (4 * grp);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!(mine >> (nt * 16 + i) & 1)) sc[nb][nt][i] = -INFINITY;
        }
      }
      if (!TREE && g.score != nullptr) {
        // (one row: a column is a head, and lies in block 0 .. NB - 1)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int c = c0 + nb * 16 + r16;
          if (c < cols) {
            float *to = g.score + ((size_t)b * a.n_heads + head * G + c) * g.score_ld + key0 + 4 * grp;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) *(pf_f32x4 *)(to + 16 * nt) = sc[nb][nt] * scale2;
          }
        }
      }
      // A column's reference is raised, and its sums rescaled, only once a score
      // exceeds it by 2^8, which leaves every rounding relative.  Each lane looks at
      // its own scores; the four of a column meet where one of them calls for it.
      float mx[NB];
      bool up = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        mx[nb] = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) mx[nb] = fmaxf(mx[nb], sc[nb][nt][i]);
        mx[nb] *= scale2;
        up |= mx[nb] > m[nb] + 8.f;
      }
      if (__any(up)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float top = quarters_max(mx[nb]);
          const float now = top > m[nb] + 8.f ? top : m[nb];
          const float shrink = now == m[nb] ? 1.f : __builtin_amdgcn_exp2f(m[nb] - now);
          m[nb] = now;
          l[nb] *= shrink;
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt) w.o[nb][dt] *= shrink;
        }
      }
      w.template outputs<DRAFT>(v, f, sc, scale2, m, l);
      for (uint32_t left = odd; left != 0; left &= left - 1) {
        const int key = __builtin_amdgcn_readfirstlane(__builtin_ctz(left));
        const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)rows, key);
        const char *from = (const char *)a.v + (uint64_t)at * L::RB;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float p = 0.f;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key / 16 == nt && key % 4 == i) p = sc[nb][nt][i];
          p = fmaxf(__shfl(p, (key >> 2 & 3) * 16 + r16, 64), 0x1p-100f);
          if (sees[nb] >> key & 1) {
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float y = C::value(from, C::dim_of(dt, i));
                if ((__float_as_uint(y) & 0x7f800000u) == 0x7f800000u) w.o[nb][dt][i] += p * y;
              }
          }
        }
      }
    }
    wave_lds_sync();                      // the tile is read before anything takes its place
    rows = next;
  };
  // (a loop without what only drafted keys need: with it the registers do not
  // suffice, and a spilled one's reload waits for the next tile's transfers)
  int step = 0;
  if constexpr (TREE) {
    const int before = max(0, min(steps, (sp.len - first) / S::STEP));
    for (; step < before; ++step) work(step, std::false_type());
    for (; step < steps; ++step) work(step, std::true_type());
  } else {
    for (; step < steps; ++step) work(step, std::false_type());
  }

  // rows behind the drafted ones see nothing
  auto give = [&](int c, int d, const pf_f32x4 &o, float mm, float ll) {
    const int i = c / G, row = b * a.draft + i, hd = head * G + c - i * G;
    const bool none = a.mask != nullptr && i >= sp.drafted;
    const pf_f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    if (plan.n == 1) {
      finish<T>(a, g.whole, row, hd, d, none ? zero : o, none ? -INFINITY : mm, none ? 0.f : ll);
      if (g.score == nullptr) return;
    } else {
      *(pf_f32x4 *)(g.rec + rec_index(a, row, hd, split, g.smax) * HD + d) = none ? zero : o;
    }
    if (d == 0) g.stat[rec_index(a, row, hd, split, g.smax)] = none ? make_float2(-INFINITY, 0.f) : make_float2(mm, ll);
  };
  if constexpr (WK == 1) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int c = c0 + nb * 16 + r16;
      const float sum = quarters_sum(l[nb]);
      if (c < cols) {
#pragma unroll
        for (int j = 0; j < C::QUADS; ++j) give(c, C::dim(j), w.quad(nb, j), m[nb], sum);
      }
    }
  } else {
    // the key groups' sums under one reference
    typedef float Row[HD + 4];
    __syncthreads();
    Row *mine = (Row *)lds + wave * 16 * NB;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float sum = quarters_sum(l[nb]);
      if (grp == 0) {
        wm[wave][nb * 16 + r16] = m[nb];
        wl[wave][nb * 16 + r16] = sum;
      }
#pragma unroll
      for (int j = 0; j < C::QUADS; ++j) *(pf_f32x4 *)&mine[nb * 16 + r16][C::dim(j)] = w.quad(nb, j);
    }
    __syncthreads();
    const int base = block * S::COLS, n = min(S::COLS, cols - base);
    for (int e = tid; e < n * (HD / 4); e += 64 * NW) {
      const int c = e / (HD / 4), d = e % (HD / 4) * 4, u = c / (16 * NB), at = c % (16 * NB);
      float mm = wm[u][at];
#pragma unroll
      for (int s = 1; s < WK; ++s) mm = fmaxf(mm, wm[s * WC + u][at]);
      const float ref = mm == -INFINITY ? 0.f : mm;
      pf_f32x4 o = {0.f, 0.f, 0.f, 0.f};
      float ll = 0.f;
#pragma unroll
      for (int s = 0; s < WK; ++s) {
        const float f = __builtin_amdgcn_exp2f(wm[s * WC + u][at] - ref);
        const pf_f32x4 y = *(const pf_f32x4 *)&((const Row *)lds)[(s * WC + u) * 16 * NB + at][d];
        ll = fmaf(f, wl[s * WC + u][at], ll);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(f, y[i], o[i]);
      }
      give(base + c, d, o, mm, ll);
    }
  }
}

// A row's records together, HD / 4 lanes a (row, query head).
template <typename T, int HD>
__global__ __launch_bounds__(256) void span_join_kernel(SpanArgs a, SpanGrid g, int step_keys) {
  constexpr int LPR = HD / 4, PER = 256 / LPR;
  const int64_t id = (int64_t)blockIdx.x * PER + threadIdx.x / LPR;
  if (id >= (int64_t)a.n * a.draft * a.n_heads) return;
  const int row = (int)(id / a.n_heads), head = (int)(id - (int64_t)row * a.n_heads), d = threadIdx.x % LPR * 4;
  const Span sp = span_of(a, row / a.draft);
  const int n = span_plan(sp.keys, step_keys, g.smax, g.least).n;
  if (n == 1) return;
  const size_t base = rec_index(a, row, head, 0, g.smax);
  float m = -INFINITY;
  for (int s = 0; s < n; ++s) m = fmaxf(m, g.stat[base + s].x);
  const float ref = m == -INFINITY ? 0.f : m;
  pf_f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
#pragma unroll 4
  for (int s = 0; s < n; ++s) {
    const float2 st = g.stat[base + s];
    const float f = __builtin_amdgcn_exp2f(st.x - ref);
    const pf_f32x4 x = *(const pf_f32x4 *)(g.rec + (base + s) * HD + d);
    l = fmaf(f, st.y, l);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(f, x[i], o[i]);
  }
  finish<T>(a, g.whole, row, head, d, o, m, l);
}

// The reference and the sum of a row's n splits, eight of them asked for at once.
__device__ __forceinline__ float2 stats_of(const float2 *stat, int n) {
  auto each = [&](auto f) {
    for (int s0 = 0; s0 < n; s0 += 8) {
      float2 st[8];
#pragma unroll
      for (int s = 0; s < 8; ++s) st[s] = stat[min(s0 + s, n - 1)];
#pragma unroll
      for (int s = 0; s < 8; ++s)
        if (s0 + s < n) f(st[s]);
    }
  };
  float m = -INFINITY, l = 0.f;
  each([&](float2 st) { m = fmaxf(m, st.x); });
  const float ref = m == -INFINITY ? 0.f : m;
  each([&](float2 st) { l = fmaf(__builtin_amdgcn_exp2f(st.x - ref), st.y, l); });
  return make_float2(m, l);
}

// The weights of a row's keys, from its scores and sums, added to its totals.  A
// lane has four neighbouring keys, whose loads are all on their way at once: the
// kernel is the latency of lengths, sums and scores, one after the other.
constexpr int WEIGH_KEYS = 4 * 256;
__global__ __launch_bounds__(256) void span_weigh_kernel(SpanArgs a, SpanGrid g, int step_keys, int parts) {
  __shared__ float2 norm[64];             // of a query head: reference, 1 / sum
  const int kv = a.map.n_kv_heads, G = a.n_heads / kv;
  const int id = blockIdx.x / parts, head = id % kv, b = id / kv, first = (blockIdx.x - id * parts) * WEIGH_KEYS;
  const Span sp = span_of(a, b);
  if (first >= sp.len) return;
  const size_t row = (size_t)b * kv + head;
  const float *in = a.weight + row * a.weight_ld;
  float *out = a.weight_out + row * a.weight_out_ld;
  const float *score = g.score + ((size_t)b * a.n_heads + head * G) * g.score_ld;
  const int j0 = first + 4 * threadIdx.x, last = sp.len - 1;
  float total[4];
  bool there[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    total[i] = in[min(j0 + i, last)];
    there[i] = page_row(a.map, sp.seq, min(j0 + i, last), head) != kNoRow;
  }
  if (threadIdx.x < G) {
    const int n = span_plan(sp.keys, step_keys, g.smax, g.least).n;
    const float2 all = stats_of(g.stat + rec_index(a, b, head * G + threadIdx.x, 0, g.smax), n);
    norm[threadIdx.x] = make_float2(all.x == -INFINITY ? 0.f : all.x, inverse(all.y));
  }
  __syncthreads();
  if (j0 > last) return;
  pf_f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int h = 0; h < G; ++h) {
    const pf_f32x4 x = *(const pf_f32x4 *)(score + (size_t)h * g.score_ld + j0);     // (rows of whole steps)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] += __builtin_amdgcn_exp2f(x[i] - norm[h].x) * norm[h].y;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (j0 + i <= last) out[j0 + i] = total[i] + (there[i] ? sum[i] : 0.f);
}

struct SpanSizes {
  int blocks, smax, least, step;
  size_t records, stats, scores;          // bytes
  int64_t score_ld;
  int64_t grid, join, parts, weights;     // workgroups of the kernels (0: not launched); of a row's weights
  bool fits;
};
template <typename T, int HD, int NB, int WC>
SpanSizes sizes_of(int n, int draft, int n_heads, int n_kv_heads, int keys, bool trees, bool weigh) {
  using S = Shape<T, HD, NB, WC>;
  SpanSizes z;
  const int cols = draft * (n_heads / n_kv_heads);
  z.blocks = (cols + S::COLS - 1) / S::COLS;
  z.step = S::STEP;
  const int64_t most = (int64_t)keys + (trees ? draft : 0), items = (int64_t)std::max(n, 1) * n_kv_heads * z.blocks;
  // Splits of about 1024 keys, shorter only where they would be fewer than 512
  // workgroups.  With 512, 768, 1024 and 2048: 24 ragged trees of 25 91, 81, 84 and
  // 131 us; 8 x 64 x 8200 191, 184, 169 and 163; 8 x 8 x 8200 72, 77, 63 and 63 (512
  // workgroups are one turn of the chip); the weights of 32 ragged rows 81, 83, 76
  // and 88.  128 keys at least: four rows of 700 19 us, with 256 21.  At most 4096
  // workgroups, 64 splits a sequence.
  const int64_t least = std::min<int64_t>(1024, std::max<int64_t>(128, most * items / 512));
  z.least = std::max<int>(1, (int)(least / S::STEP));
  z.smax = (int)std::min<int64_t>(64, std::max<int64_t>(1, 4096 / items));
  z.smax = (int)std::min(z.smax, splits_of((int)((most + S::STEP - 1) / S::STEP), z.least));
  const size_t heads = (size_t)n * draft * n_heads;
  z.records = z.smax > 1 ? heads * z.smax * HD * sizeof(float) : 0;
  z.stats = z.smax > 1 || weigh ? heads * z.smax * sizeof(float2) : 0;
  z.stats = (z.stats + 15) / 16 * 16;
  z.score_ld = weigh ? (most + S::STEP - 1) / S::STEP * S::STEP : 0;
  z.scores = weigh ? (size_t)n * n_heads * z.score_ld * sizeof(float) : 0;
  constexpr int PER = 256 / (HD / 4);
  z.grid = items * z.smax;
  z.join = z.smax > 1 ? ((int64_t)heads + PER - 1) / PER : 0;
  z.parts = weigh ? (most + WEIGH_KEYS - 1) / WEIGH_KEYS : 0;
  z.weights = z.parts * n * n_kv_heads;
  z.fits = launch_fits(z.grid, 64 * S::NW) && launch_fits(z.join, 256) && launch_fits(z.weights, 256);
  return z;
}

template <bool TREE, typename T, int HD, int NB, int WC>
hipError_t go(const SpanArgs &a, hipStream_t s) {
  using S = Shape<T, HD, NB, WC>;
  const bool weigh = a.weight_out != nullptr;
  const SpanSizes z = sizes_of<T, HD, NB, WC>(a.n, a.draft, a.n_heads, a.map.n_kv_heads, a.most, TREE, weigh);
  SpanGrid g{};
  g.blocks = z.blocks;
  g.smax = z.smax;
  g.least = z.least;
  g.rec = (float *)a.work;
  g.stat = (float2 *)((char *)a.work + z.records);
  g.score = weigh ? (float *)((char *)a.work + z.records + z.stats) : nullptr;
  g.score_ld = z.score_ld;
  auto whole = [](const void *p, int64_t row, int64_t head) {
    return (uintptr_t)p % 16 == 0 && row * sizeof(T) % 16 == 0 && head * sizeof(T) % 16 == 0;
  };
  g.whole = whole(a.q, a.q_row, a.q_head) && whole(a.out, a.out_row, a.out_head);
  span_attn_kernel<TREE, T, HD, NB, WC><<<(unsigned)z.grid, 64 * S::NW, 0, s>>>(a, g);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (z.join > 0) {
    span_join_kernel<T, HD><<<(unsigned)z.join, 256, 0, s>>>(a, g, z.step);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (z.weights > 0) {
    span_weigh_kernel<<<(unsigned)z.weights, 256, 0, s>>>(a, g, z.step, (int)z.parts);
    e = hipGetLastError();
  }
  return e;
}

// Column blocks a wave, and neighbouring waves over the same keys.  Few columns
// have a wave each, with keys of its own: 32 rows of 4000 keys and their weights
// 131 us, 147 with four waves that share tiles (8 trees of 16 columns and 8200 keys
// 64 and 60).  More share their tiles, in one block a wave up to 64 columns (24
// columns 60 us, 63 with two waves and two groups of keys) and in two behind
// that: 128 columns 115 us with one, 96 with two.  A few workgroups alone take the
// smaller blocks: one tree of 64 x 8200 39 us for 58.
template <typename F>
auto by_columns(int cols, int64_t pairs, F f) {
  if (cols <= 16) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  if (cols <= 64 || pairs * ((cols + 127) / 128) <= 32)
    return f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
  return f(std::integral_constant<int, 2>(), std::integral_constant<int, 4>());
}
template <typename F>
auto by_type(int dtype, int head_dim, F f) {
  if (dtype == DEX_F32)
    return head_dim == 32   ? f(float(), std::integral_constant<int, 32>())
           : head_dim == 64 ? f(float(), std::integral_constant<int, 64>())
                            : f(float(), std::integral_constant<int, 128>());
  return head_dim == 32   ? f(uint16_t(), std::integral_constant<int, 32>())
         : head_dim == 64 ? f(uint16_t(), std::integral_constant<int, 64>())
                          : f(uint16_t(), std::integral_constant<int, 128>());
}

}  // namespace

namespace {
SpanSizes span_sizes(int dtype, int n, int draft, int n_heads, int n_kv_heads, int head_dim, int most, bool trees, bool weigh) {
  return by_type(dtype, head_dim, [&](auto t, auto hd) {
    return by_columns(draft * (n_heads / n_kv_heads), (int64_t)n * n_kv_heads, [&](auto nb, auto wc) {
      return sizes_of<decltype(t), hd.value, nb.value, wc.value>(n, draft, n_heads, n_kv_heads, most, trees, weigh);
    });
  });
}
}  // namespace

size_t span_work(int dtype, int n, int draft, int n_heads, int n_kv_heads, int head_dim, int most, bool trees, bool weigh) {
  const SpanSizes z = span_sizes(dtype, n, draft, n_heads, n_kv_heads, head_dim, most, trees, weigh);
  return z.records + z.stats + z.scores;
}

bool span_fits(int dtype, const SpanArgs &a) {
  return span_sizes(dtype, a.n, a.draft, a.n_heads, a.map.n_kv_heads, a.head_dim, a.most, a.mask != nullptr,
                    a.weight_out != nullptr).fits;
}

hipError_t launch_span(int dtype, const SpanArgs &a, hipStream_t s) {
  return by_type(dtype, a.head_dim, [&](auto t, auto hd) {
    return by_columns(a.draft * (a.n_heads / a.map.n_kv_heads), (int64_t)a.n * a.map.n_kv_heads, [&](auto nb, auto wc) {
      // one row has at most 64 columns, in blocks of 16 a wave
      if constexpr (nb.value == 1)
        if (a.mask == nullptr) return go<false, decltype(t), hd.value, nb.value, wc.value>(a, s);
      return a.mask == nullptr ? hipErrorInvalidValue : go<true, decltype(t), hd.value, nb.value, wc.value>(a, s);
    });
  });
}

}  // namespace dex
