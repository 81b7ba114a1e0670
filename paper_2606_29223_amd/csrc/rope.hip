// Rotary positions of queries and keys, alone or with the keys and values
// written into a cache's pages.
//
// Pair i of a head turns by pos * f_i: (x, y) -> (x cos - y sin, y cos + x
// sin), times the plan's amplitude.  The plan holds f_i / 2 pi in double, so
// pos * turns_i is exact to 2^-53 of the number of turns; its fraction, less
// the nearest quarter, lies in [-1/8, 1/8] and goes on in float.  An angle of
// a far position is as good as one near zero (a float angle at position 10^6
// is off by 0.06 radian).  Sine and cosine of the remaining |x| <= pi / 4 are
// their Taylor series to x^9 and x^10: the next terms are below 2^-29.
#include "dex.h"
#include "dex_kernels.h"
#include "paged.h"

namespace dex {

namespace {

constexpr int ROPE_THREADS = 256;

// Every multiply-add is spelled out, so that all forms of the kernel round
// alike and a row's bits do not depend on its alignment.
__device__ __forceinline__ void turn_sincos(double pos, double turn, float &s, float &c) {
  const double r0 = __builtin_fma(pos, turn, -rint(pos * turn));   // [-1/2, 1/2]
  const double q = rint(4.0 * r0);                                 // -2 .. 2
  const float x = (float)(__builtin_fma(-0.25, q, r0) * 6.283185307179586476925);
  const float x2 = x * x;
  const float sp = fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6);
  const float cp = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f);
  const float sx = fmaf(x * x2, sp, x), cx = fmaf(x2, cp, 1.f);
  const int k = (int)q & 3;
  const float a = (k & 1) ? cx : sx, b = (k & 1) ? sx : cx;
  s = (k & 2) ? -a : a;
  c = (k == 1 || k == 2) ? -b : b;
}
// (x, y) turned by cosine c and sine s.
__device__ __forceinline__ float turn_x(float x, float y, float c, float s) { return fmaf(x, c, -(y * s)); }
__device__ __forceinline__ float turn_y(float x, float y, float c, float s) { return fmaf(y, c, x * s); }

// N elements in one access (N elements of T are 2, 4, 8 or 16 bytes).
template <typename T, int N>
struct Raw;
template <> struct Raw<uint16_t, 1> { typedef uint16_t type; };
template <> struct Raw<uint16_t, 4> { typedef uint2 type; };
template <> struct Raw<uint16_t, 8> { typedef uint4 type; };
template <> struct Raw<float, 1> { typedef float type; };
template <> struct Raw<float, 4> { typedef uint4 type; };

template <typename T, int N>
struct Vec {
  typename Raw<T, N>::type raw;
  __device__ __forceinline__ void load(const T *p) { raw = *(const typename Raw<T, N>::type *)p; }
  __device__ __forceinline__ void store(T *p) const { *(typename Raw<T, N>::type *)p = raw; }
  __device__ __forceinline__ float get(int i) const {
    T t[N];
    __builtin_memcpy(t, &raw, sizeof raw);
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)t[i] << 16);
    else return t[i];
  }
  __device__ __forceinline__ void set(const float *f) {
    T t[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 2) t[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
      else t[i] = f[i];
    }
    __builtin_memcpy(&raw, t, sizeof raw);
  }
};

// A lane owns one unit of a row -- VEC pairs, or 2 VEC elements past rot_dim --
// works out its VEC angles once and takes the unit through the heads
// slot, slot + slots, ... of queries, keys and values.  With the angles shared
// memory bounds the kernel: 8192 rows of 32 and 8 heads of 128 in
// bf16 (168 MB) take 33 us, with the values written to pages too (201 MB) 41 us,
// 5.0 TB/s, where a copy of that size runs at 5.3.  A few rows take 3.5 to 4.5
// us, the launch and two dependent loads.
template <typename T, int VEC, bool INTER>
__global__ __launch_bounds__(ROPE_THREADS) void rope_kernel(RopeArgs a, int units, int slots) {
  const int tid = blockIdx.x * ROPE_THREADS + threadIdx.x;
  const int row = tid / (units * slots);
  if (row >= a.n_rows) return;
  const int rem = tid - row * (units * slots);
  const int slot = rem / units, u = rem - slot * units;
  const int pos = a.pos[row];
  T *kd = nullptr, *vd = nullptr;
  int64_t kstep = 0;
  if (a.k_pages != nullptr) {
    const int seq = a.seq != nullptr ? a.seq[row] : row;
    if (seq < 0 || seq >= a.map.n_seqs) return;
    const uint32_t r = page_row(a.map, seq, pos, 0);
    if (r == kNoRow) return;
    kd = (T *)a.k_pages + (size_t)r * a.head_dim;
    vd = (T *)a.v_pages + (size_t)r * a.head_dim;
    kstep = (int64_t)a.head_dim << a.map.shift;
  } else if (a.k.n > 0) {
    kd = (T *)a.k_out.p + (int64_t)row * a.k_out.row;
    kstep = a.k_out.head;
  }
  const bool turn = a.turns != nullptr && u * 2 * VEC < a.rot_dim;
  const int e0 = (turn && !INTER) ? u * VEC : u * 2 * VEC;
  const int e1 = (turn && !INTER) ? a.rot_dim / 2 + u * VEC : u * 2 * VEC + VEC;
  float cs[VEC], sn[VEC];
  if (turn) {
    const double p = (double)(a.inverse ? -(int64_t)pos : (int64_t)pos);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      turn_sincos(p, a.turns[u * VEC + i], sn[i], cs[i]);
      sn[i] *= a.amplitude;
      cs[i] *= a.amplitude;
    }
  }
  const int jobs = a.q.n + a.k.n + a.v.n;
  for (int j = slot; j < jobs; j += slots) {
    const T *src;
    T *dst;
    bool rotate = turn;
    if (j < a.q.n) {
      src = (const T *)a.q.p + (int64_t)row * a.q.row + (int64_t)j * a.q.head;
      dst = (T *)a.q_out.p + (int64_t)row * a.q_out.row + (int64_t)j * a.q_out.head;
    } else if (j < a.q.n + a.k.n) {
      const int h = j - a.q.n;
      src = (const T *)a.k.p + (int64_t)row * a.k.row + (int64_t)h * a.k.head;
      dst = kd + h * kstep;
    } else {
      const int h = j - a.q.n - a.k.n;
      src = (const T *)a.v.p + (int64_t)row * a.v.row + (int64_t)h * a.v.head;
      dst = vd + h * kstep;
      rotate = false;
    }
    Vec<T, VEC> x, y;
    x.load(src + e0);
    y.load(src + e1);
    if (rotate) {
      float f[2 * VEC];
      if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float xe = 2 * i < VEC ? x.get((2 * i) % VEC) : y.get((2 * i) % VEC);
          const float yo = 2 * i + 1 < VEC ? x.get((2 * i + 1) % VEC) : y.get((2 * i + 1) % VEC);
          f[2 * i] = turn_x(xe, yo, cs[i], sn[i]);
          f[2 * i + 1] = turn_y(xe, yo, cs[i], sn[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          f[i] = turn_x(x.get(i), y.get(i), cs[i], sn[i]);
          f[VEC + i] = turn_y(x.get(i), y.get(i), cs[i], sn[i]);
        }
      }
      x.set(f);
      y.set(f + VEC);
    }
    x.store(dst + e0);
    y.store(dst + e1);
  }
}

}  // namespace

// The widest access that every row, head and half of the call allows.
int rope_vec(int dtype, const RopeArgs &a) {
  const int es = dtype == DEX_F32 ? 4 : 2;
  const int top = 16 / es;
  for (int v = top; v > 1; v /= 2) {
    if (v != 8 && v != 4) continue;
    auto fits = [&](const void *p, int64_t row, int64_t head) {
      return (uintptr_t)p % (v * es) == 0 && row % v == 0 && head % v == 0;
    };
    bool ok = a.head_dim % (2 * v) == 0 && a.rot_dim % (2 * v) == 0;
    if (a.q.n > 0) ok = ok && fits(a.q.p, a.q.row, a.q.head) && fits(a.q_out.p, a.q_out.row, a.q_out.head);
    if (a.k.n > 0) ok = ok && fits(a.k.p, a.k.row, a.k.head);
    if (a.k.n > 0 && a.k_pages == nullptr) ok = ok && fits(a.k_out.p, a.k_out.row, a.k_out.head);
    if (a.v.n > 0) ok = ok && fits(a.v.p, a.v.row, a.v.head);
    if (ok) return v;
  }
  return 1;
}

template <typename T, int VEC>
static hipError_t rope_go(const RopeArgs &a, hipStream_t s) {
  const int units = a.head_dim / (2 * VEC), jobs = a.q.n + a.k.n + a.v.n;
  // Heads a lane: one while that leaves fewer than 2^18 lanes (500 rows of 40
  // heads of 128 in bf16: 5.5 us with one, 8.7 with eight), then more, which
  // share one set of angles, up to eight in bf16 (8192 rows written to pages: 55
  // us with one, 40 with eight) and four in fp32, where the angles weigh half as
  // much (8192 rows: 62 with one, 64 with four, 67 with eight).  The limit on a
  // call's elements is for eight: fewer may leave more lanes than an int counts.
  const int most = sizeof(T) == 2 ? 8 : 4;
  int heads = 1;
  auto lanes_of = [&](int h) { return (int64_t)a.n_rows * units * ((jobs + h - 1) / h); };
  while (heads < 8 && lanes_of(heads) > (heads < most ? 1 << 18 : 1 << 30)) heads *= 2;
  const int slots = (jobs + heads - 1) / heads;
  const int64_t lanes = lanes_of(heads);
  const dim3 grid((unsigned)((lanes + ROPE_THREADS - 1) / ROPE_THREADS));
  if (a.interleaved) rope_kernel<T, VEC, true><<<grid, ROPE_THREADS, 0, s>>>(a, units, slots);
  else rope_kernel<T, VEC, false><<<grid, ROPE_THREADS, 0, s>>>(a, units, slots);
  return hipGetLastError();
}

hipError_t launch_rope(int dtype, const RopeArgs &a, hipStream_t s) {
  const int v = rope_vec(dtype, a);
  if (dtype == DEX_F32) return v == 4 ? rope_go<float, 4>(a, s) : rope_go<float, 1>(a, s);
  return v == 8 ? rope_go<uint16_t, 8>(a, s) : v == 4 ? rope_go<uint16_t, 4>(a, s) : rope_go<uint16_t, 1>(a, s);
}

}  // namespace dex
