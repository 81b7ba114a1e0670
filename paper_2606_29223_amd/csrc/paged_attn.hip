// Attention of one new token a row over a paged cache, split over the keys
// and joined.
//
// Row r with query heads h sees the keys lo <= j < len of its sequence whose
// page is there: s_j = scale q.k_j, out = sum e^{s_j - m} v_j / sum e^{s_j - m},
// lse = m + ln sum e^{s_j - m}.  A split is 256 keys at a fixed place of the
// sequence; its record (sum of v, m, sum) goes to the join, which adds a
// row's records in order, so a row's bits depend on its own keys alone.
//
// A workgroup takes (row, kv head, split) items, 64 keys (32 in fp32) of a
// split a wave:  S^T = K Q^T and O^T = V^T P^T on the matrix cores, the kv
// head's query heads as the 16 columns, so each lane holds the scores and
// outputs of one query head.  The kernel reads each key and value once from
// HBM and is bound by that: the products are 4 % of what the matrix cores
// could do meanwhile, which is why P goes through them in two bf16 parts
// (p = hi + lo to 2^-17) and costs the output no accuracy.
#include "attn_decode.h"
#include "dex.h"
#include "paged.h"

#include <algorithm>
#include <climits>

namespace dex {

namespace {

constexpr int PA_WAVES = 4;
constexpr int PA_THREADS = PA_WAVES * 64;
constexpr int PA_SPLIT = 256;             // keys of a split
constexpr int PA_ROWS = 1024;             // rows of a launch
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Splits of a row, and the first of them.
__device__ __forceinline__ int row_splits(int len, int window, int *first) {
  const int lo = window > 0 ? max(0, len - window) : 0;
  *first = lo / PA_SPLIT;
  return len > 0 ? (len - 1) / PA_SPLIT - *first + 1 : 1;      // an empty row has one item, to say so
}

// What one wave makes of its keys of a split, for 16 NB columns: column r16
// of block nb is query head nb * 16 + r16 of the kv head.
template <int HD, int NB>
struct WaveState {
  float m[NB], l[NB];                     // in powers of two; m of the reference, l the lane's own keys' sum
  pf_f32x4 o[NB][HD / 16];
};

template <typename T, int HD>
struct Lds;
template <int HD>
struct Lds<uint16_t, HD> {                // V tile rows, then the wave's part of the sum
  union {
    uint16_t v[64][HD + 16];
    float o[16][HD + 4];
  };
};
template <int HD>
struct Lds<float, HD> {
  float o[16][HD + 4];
};

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Scores of NT 16-key tiles to probabilities under the new reference; returns
// by what the wave's earlier sums shrink.  Keys outside `mask` get 0.
template <int NT>
__device__ __forceinline__ float soften(pf_f32x4 (&sc)[NT], unsigned long long mask, bool full, float scale2, float &m,
                                        float &l) {
  const int grp = (threadIdx.x & 63) >> 4;
  float mx = -INFINITY;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = sc[nt][i] * scale2;
      if (!full && !(mask >> (nt * 16 + grp * 4 + i) & 1)) v = -INFINITY;
      sc[nt][i] = v;
      mx = fmaxf(mx, v);
    }
  const float m1 = fmaxf(m, quad_max(mx));
  const float ref = m1 == -INFINITY ? 0.f : m1;       // nothing seen yet: every power is 0
  const float shrink = __builtin_amdgcn_exp2f(m - ref);
  float sum = 0.f;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sc[nt][i] = __builtin_amdgcn_exp2f(sc[nt][i] - ref);
      sum += sc[nt][i];
    }
  l = l * shrink + quad_sum(sum);
  m = m1;
  return shrink;
}

// bf16: 64 keys at cache rows `mine` (lane j: key j; kNoRow: none).
template <int HD, int NB>
__device__ __forceinline__ void keys_bf16(const PagedAttnArgs &a, uint32_t mine, int nb_used,
                                          const pf_bf16x8 (&qf)[NB][HD / 32], float scale2, Lds<uint16_t, HD> &lds,
                                          WaveState<HD, NB> &w) {
  constexpr int KS = HD / 32, DT = HD / 16, V4 = HD / 8, RPI = 64 / V4;
  const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
  const unsigned long long mask = __ballot(mine != kNoRow);
  if (mask == 0) return;
  const bool full = mask == ~0ull;
  // an absent key reads row 0, which is there; its score and value are put out below
  const uint32_t at = mine == kNoRow ? 0u : mine;
  const uint16_t *kp = (const uint16_t *)a.k + grp * 8, *vp = (const uint16_t *)a.v + (lane % V4) * 8;
  uint4 kf[4][KS], vv[V4];
#pragma unroll
  for (int nt = 0; nt < 4; ++nt) {
    const uint16_t *row = kp + (size_t)(uint32_t)__shfl((int)at, nt * 16 + r16, 64) * HD;
#pragma unroll
    for (int st = 0; st < KS; ++st) kf[nt][st] = *(const uint4 *)(row + st * 32);
  }
#pragma unroll
  for (int c = 0; c < V4; ++c)
    vv[c] = *(const uint4 *)(vp + (size_t)(uint32_t)__shfl((int)at, c * RPI + lane / V4, 64) * HD);
  pf_f32x4 sc[NB][4];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (nb < nb_used) {
#pragma unroll
      for (int nt = 0; nt < 4; ++nt) {
        sc[nb][nt] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; ++st)
          sc[nb][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pf_bf16x8, kf[nt][st]), qf[nb][st],
                                                               sc[nb][nt], 0, 0, 0);
      }
    }
  }
  if (!full) {
#pragma unroll
    for (int c = 0; c < V4; ++c)
      if (!(mask >> (c * RPI + lane / V4) & 1)) vv[c] = make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int c = 0; c < V4; ++c) *(uint4 *)&lds.v[c * RPI + lane / V4][(lane % V4) * 8] = vv[c];
  wave_lds_sync();
  const int tq = grp, ti = r16 >> 2, tg = lane & 3;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (nb < nb_used) {
      const float shrink = soften<4>(sc[nb], mask, full, scale2, w.m[nb], w.l[nb]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) w.o[nb][dt] *= shrink;
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        float p[8], r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = sc[nb][2 * st + i / 4][i % 4];
        const uint4 hi = make_uint4(pf_pack_bf16(p[0], p[1]), pf_pack_bf16(p[2], p[3]), pf_pack_bf16(p[4], p[5]),
                                    pf_pack_bf16(p[6], p[7]));
        const uint32_t hw[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = p[i] - __uint_as_float(i & 1 ? hw[i / 2] & 0xffff0000u : hw[i / 2] << 16);
        const uint4 lo = make_uint4(pf_pack_bf16(r[0], r[1]), pf_pack_bf16(r[2], r[3]), pf_pack_bf16(r[4], r[5]),
                                    pf_pack_bf16(r[6], r[7]));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const pf_bf16x8 vf = tr_frag(&lds.v[32 * st + 4 * tq + ti][16 * dt + 4 * tg],
                                       &lds.v[32 * st + 16 + 4 * tq + ti][16 * dt + 4 * tg]);
          w.o[nb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(pf_bf16x8, hi), w.o[nb][dt], 0, 0, 0);
          w.o[nb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(pf_bf16x8, lo), w.o[nb][dt], 0, 0, 0);
        }
      }
    }
  }
  wave_lds_sync();                        // the tile is read before the next one is written
}

// fp32: 32 keys at cache rows `mine` (lanes 0 .. 31), on the fp32 matrix
// instructions.  A key lane holds dimensions 4 grp .. + 3 of each 16, so one
// 16-byte load feeds four k-steps; a value lane holds W neighbouring
// dimensions of one key, each the row of another 16-dimension tile, so values
// need no transposition: tile (b, e) holds the dimensions 16 W b + W i + e.
template <int HD, int NB>
__device__ __forceinline__ void keys_f32(const PagedAttnArgs &a, uint32_t mine, int nb_used,
                                         const pf_f32x4 (&qf)[NB][HD / 16], float scale2, WaveState<HD, NB> &w) {
  constexpr int DT = HD / 16, W = HD >= 64 ? 4 : 2, VB = HD / (16 * W);
  typedef __attribute__((ext_vector_type(W))) float vecw;
  const int lane = threadIdx.x & 63, r16 = lane & 15, grp = lane >> 4;
  const unsigned long long mask = __ballot(lane < 32 && mine != kNoRow);
  if (mask == 0) return;
  const bool full = mask == 0xffffffffull;
  const uint32_t at = mine == kNoRow ? 0u : mine;
  const float *kp = (const float *)a.k + 4 * grp, *vp = (const float *)a.v + W * r16;
  pf_f32x4 kf[2][DT];
  vecw vv[2][4][VB];
#pragma unroll
  for (int nt = 0; nt < 2; ++nt) {
    const float *row = kp + (size_t)(uint32_t)__shfl((int)at, nt * 16 + r16, 64) * HD;
#pragma unroll
    for (int t = 0; t < DT; ++t) kf[nt][t] = *(const pf_f32x4 *)(row + 16 * t);
  }
#pragma unroll
  for (int nt = 0; nt < 2; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float *row = vp + (size_t)(uint32_t)__shfl((int)at, nt * 16 + 4 * grp + i, 64) * HD;
#pragma unroll
      for (int b = 0; b < VB; ++b) vv[nt][i][b] = *(const vecw *)(row + 16 * W * b);
    }
  if (!full) {
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < VB; ++b)
          if (!(mask >> (nt * 16 + 4 * grp + i) & 1)) vv[nt][i][b] = (vecw)0.f;
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    if (nb < nb_used) {
      pf_f32x4 sc[2];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
        sc[nt] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sc[nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[nt][t][e], qf[nb][t][e], sc[nt], 0, 0, 0);
      }
      const float shrink = soften<2>(sc, mask, full, scale2, w.m[nb], w.l[nb]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) w.o[nb][dt] *= shrink;
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int b = 0; b < VB; ++b)
#pragma unroll
            for (int e = 0; e < W; ++e)
              w.o[nb][b * W + e] =
                  __builtin_amdgcn_mfma_f32_16x16x4f32(vv[nt][i][b][e], sc[nt][i], w.o[nb][b * W + e], 0, 0, 0);
    }
  }
}

// Where a row's records lie: [rows][heads][splits] of head_dim floats, then
// the statistics of (m, l).
__device__ __forceinline__ size_t rec_index(const PagedAttnArgs &a, int row, int head, int split, int smax) {
  return ((size_t)row * a.n_heads + head) * smax + split;
}

template <typename T, int HD, int NB>
__global__ __launch_bounds__(PA_THREADS) void paged_attn_kernel(PagedAttnArgs a, int smax, float *rec, float2 *stat) {
  constexpr int TK = sizeof(T) == 2 ? 64 : 32;          // keys of a wave's tile
  constexpr int TILES = PA_SPLIT / (PA_WAVES * TK);
  __shared__ Lds<T, HD> lds[PA_WAVES];
  __shared__ int first_item[PA_ROWS];                   // items before a row's
  __shared__ int part[PA_WAVES];
  __shared__ float wm[PA_WAVES][16], wl[PA_WAVES][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, grp = lane >> 4;
  const int kv = a.map.n_kv_heads, G = a.n_heads / kv, cap = a.max_len;
  const float scale2 = a.scale * kLog2e;
  auto row_len = [&](int r) {
    const int s = a.seq != nullptr ? a.seq[r] : r;
    const int n = min(a.len[r], cap);
    return s >= 0 && s < a.map.n_seqs && n > 0 ? n : 0;
  };
  // number the items: every row's splits, the kv heads of a split together
  int items;
  {
    constexpr int PER = PA_ROWS / PA_THREADS;
    int n[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int r = tid * PER + k;
      int f;
      n[k] = r < a.n_rows ? row_splits(row_len(r), a.window, &f) * kv : 0;
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
  for (int it = blockIdx.x; it < items; it += gridDim.x) {
    int lo_r = 0, hi_r = a.n_rows - 1;
    while (lo_r < hi_r) {
      const int mid = (lo_r + hi_r + 1) >> 1;
      if (first_item[mid] <= it) lo_r = mid;
      else hi_r = mid - 1;
    }
    const int row = lo_r, rem = it - first_item[row];
    const int h = rem % kv;
    const int len = row_len(row);
    const int seq = a.seq != nullptr ? a.seq[row] : row;
    int split0;
    const int n_splits = row_splits(len, a.window, &split0), sp = rem / kv;
    const int lo = a.window > 0 ? max(0, len - a.window) : 0;
    const int k0 = (split0 + sp) * PA_SPLIT + wave * (PA_SPLIT / PA_WAVES);
    const int nb_used = (G + 15) / 16;
    WaveState<HD, NB> w;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      w.m[nb] = -INFINITY;
      w.l[nb] = 0.f;
#pragma unroll
      for (int dt = 0; dt < HD / 16; ++dt) w.o[nb][dt] = pf_f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const T *qrow = (const T *)a.q + (int64_t)row * a.q_row + (int64_t)(h * G) * a.q_head;
    auto cache_row = [&](int key) {
      return key >= lo && key < len ? page_row(a.map, seq, key, h) : kNoRow;
    };
    if constexpr (sizeof(T) == 2) {
      pf_bf16x8 qf[NB][HD / 32];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int p = nb * 16 + r16;
#pragma unroll
        for (int st = 0; st < HD / 32; ++st) {
          uint16_t x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = p < G ? qrow[(int64_t)p * a.q_head + st * 32 + grp * 8 + i] : 0;
          __builtin_memcpy(&qf[nb][st], x, 16);
        }
      }
#pragma unroll
      for (int t = 0; t < TILES; ++t) keys_bf16<HD, NB>(a, cache_row(k0 + t * TK + lane), nb_used, qf, scale2, lds[wave], w);
    } else {
      pf_f32x4 qf[NB][HD / 16];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int p = nb * 16 + r16;
#pragma unroll
        for (int t = 0; t < HD / 16; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) qf[nb][t][i] = p < G ? qrow[(int64_t)p * a.q_head + t * 16 + grp * 4 + i] : 0.f;
      }
#pragma unroll
      for (int t = 0; t < TILES; ++t)
        keys_f32<HD, NB>(a, lane < TK ? cache_row(k0 + t * TK + lane) : kNoRow, nb_used, qf, scale2, w);
    }
    // the four waves' sums under one reference, 16 columns at a time
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb < nb_used) {
        if (grp == 0) {
          wm[wave][r16] = w.m[nb];
          wl[wave][r16] = w.l[nb];
        }
#pragma unroll
        for (int dt = 0; dt < HD / 16; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            constexpr int W = HD >= 64 ? 4 : 2;
            const int d = sizeof(T) == 2 ? 16 * dt + 4 * grp + i : 16 * W * (dt / W) + W * (4 * grp + i) + dt % W;
            lds[wave].o[r16][d] = w.o[nb][dt][i];
          }
        __syncthreads();
        const int cols = min(16, G - nb * 16);
        for (int e = tid; e < cols * HD; e += PA_THREADS) {
          const int c = e / HD, d = e % HD;
          float m = wm[0][c];
#pragma unroll
          for (int v = 1; v < PA_WAVES; ++v) m = fmaxf(m, wm[v][c]);
          const float ref = m == -INFINITY ? 0.f : m;
          float o = 0.f, l = 0.f;
#pragma unroll
          for (int v = 0; v < PA_WAVES; ++v) {
            const float f = __builtin_amdgcn_exp2f(wm[v][c] - ref);
            o += f * lds[v].o[c][d];
            l += f * wl[v][c];
          }
          const int head = h * G + nb * 16 + c;
          if (n_splits == 1) {
            T *out = (T *)a.out + (int64_t)row * a.out_row + (int64_t)head * a.out_head;
            const float y = l > 0.f ? o / l : l != l ? l : 0.f;
            if constexpr (sizeof(T) == 2) out[d] = __builtin_bit_cast(uint16_t, (__bf16)y);
            else out[d] = y;
            if (d == 0 && a.lse != nullptr) a.lse[(size_t)row * a.n_heads + head] = (m + __builtin_amdgcn_logf(l)) * kLn2;
          } else {
            const size_t at = rec_index(a, row, head, sp, smax);
            rec[at * HD + d] = o;
            if (d == 0) stat[at] = make_float2(m, l);
          }
        }
        __syncthreads();
      }
    }
  }
}

// A row's records, added in order: a workgroup a (row, query head), HD / 4
// lanes a record.
template <typename T, int HD>
__global__ __launch_bounds__(PA_THREADS) void paged_join_kernel(PagedAttnArgs a, int smax, const float *rec,
                                                              const float2 *stat) {
  constexpr int LPR = HD / 4, AT = PA_THREADS / LPR;    // records at a time
  __shared__ float4 sum[AT][LPR];
  __shared__ float lsum[AT];
  const int row = blockIdx.x / a.n_heads, head = blockIdx.x - row * a.n_heads;
  const int s = a.seq != nullptr ? a.seq[row] : row;
  const int n0 = min(a.len[row], a.max_len);
  if (s < 0 || s >= a.map.n_seqs || n0 <= 0) return;
  int split0;
  const int n = row_splits(n0, a.window, &split0);
  if (n == 1) return;
  const int tid = threadIdx.x, j0 = tid / LPR, d = tid % LPR;
  const size_t base = rec_index(a, row, head, 0, smax);
  float m = -INFINITY;
  for (int j = 0; j < n; ++j) m = fmaxf(m, stat[base + j].x);
  const float ref = m == -INFINITY ? 0.f : m;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
  for (int j = j0; j < n; j += AT) {
    const float2 st = stat[base + j];
    const float4 x = *(const float4 *)(rec + (base + j) * HD + 4 * d);
    const float f = __builtin_amdgcn_exp2f(st.x - ref);
    l += f * st.y;
    o.x += f * x.x;
    o.y += f * x.y;
    o.z += f * x.z;
    o.w += f * x.w;
  }
  sum[j0][d] = o;
  if (d == 0) lsum[j0] = l;
  __syncthreads();
  if (j0 != 0) return;
#pragma unroll
  for (int k = 1; k < AT; ++k) {
    const float4 x = sum[k][d];
    o.x += x.x;
    o.y += x.y;
    o.z += x.z;
    o.w += x.w;
    l += lsum[k];
  }
  const float y[4] = {o.x, o.y, o.z, o.w};
  T *out = (T *)a.out + (int64_t)row * a.out_row + (int64_t)head * a.out_head + 4 * d;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float v = l > 0.f ? y[i] / l : l != l ? l : 0.f;
    if constexpr (sizeof(T) == 2) out[i] = __builtin_bit_cast(uint16_t, (__bf16)v);
    else out[i] = v;
  }
  if (d == 0 && a.lse != nullptr) a.lse[(size_t)row * a.n_heads + head] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

int max_splits(int max_len) { return std::max(1, (max_len + PA_SPLIT - 1) / PA_SPLIT); }

template <typename T, int HD, int NB>
hipError_t go(const PagedAttnArgs &a, hipStream_t s) {
  const int smax = max_splits(a.max_len);
  for (int r0 = 0; r0 < a.n_rows; r0 += PA_ROWS) {
    PagedAttnArgs b = a;
    b.n_rows = std::min(PA_ROWS, a.n_rows - r0);
    b.q = (const T *)a.q + r0 * a.q_row;
    b.out = (T *)a.out + r0 * a.out_row;
    b.len = a.len + r0;
    if (a.lse != nullptr) b.lse = a.lse + (size_t)r0 * a.n_heads;
    if (a.seq != nullptr) b.seq = a.seq + r0;
    else b.map.table = a.map.table + (size_t)r0 * a.map.max_pages, b.map.n_seqs = std::max(0, a.map.n_seqs - r0);
    float *rec = (float *)a.work;
    float2 *stat = (float2 *)(rec + (size_t)std::min(a.n_rows, PA_ROWS) * a.n_heads * smax * HD);
    const int64_t most = (int64_t)b.n_rows * a.map.n_kv_heads * smax;
    paged_attn_kernel<T, HD, NB><<<(unsigned)std::min<int64_t>(most, 1024), PA_THREADS, 0, s>>>(b, smax, rec, stat);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (smax > 1) {
      paged_join_kernel<T, HD><<<b.n_rows * a.n_heads, PA_THREADS, 0, s>>>(b, smax, rec, stat);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

template <typename T, int HD>
hipError_t go_nb(const PagedAttnArgs &a, hipStream_t s) {
  const int g = a.n_heads / a.map.n_kv_heads;
  return g <= 16 ? go<T, HD, 1>(a, s) : g <= 32 ? go<T, HD, 2>(a, s) : go<T, HD, 4>(a, s);
}

}  // namespace

size_t paged_attention_work(int n_rows, int n_heads, int head_dim, int max_len) {
  const int smax = max_splits(max_len);
  if (smax == 1) return 0;
  return (size_t)std::min(n_rows, PA_ROWS) * n_heads * smax * (head_dim + 2) * sizeof(float);
}

hipError_t launch_paged_attention(int dtype, const PagedAttnArgs &a, hipStream_t s) {
  if (dtype == DEX_F32)
    return a.head_dim == 32 ? go_nb<float, 32>(a, s) : a.head_dim == 64 ? go_nb<float, 64>(a, s) : go_nb<float, 128>(a, s);
  return a.head_dim == 32 ? go_nb<uint16_t, 32>(a, s)
                          : a.head_dim == 64 ? go_nb<uint16_t, 64>(a, s) : go_nb<uint16_t, 128>(a, s);
}

}  // namespace dex
