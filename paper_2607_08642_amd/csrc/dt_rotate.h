// Heads normed and rotated by position (dt_rotary), on the device.
//
// A head's D elements are dealt to lanes in units of two runs of eight, so that both elements of a pair are with one
// lane and neighbouring lanes have neighbouring runs: unit u of the pairs [8 u, 8 u + 8) is the runs at 8 u and at
// pairs + 8 u; where pairs are interleaved, or none, the runs u and u + n of the 2 n.  (Units of 16 neighbours, whose lanes
// are 64 bytes apart in fp32, took 80 us where these take 65: 8000 rows of 40 heads of 128.)
#pragma once

#include "dt_cache.h"

namespace dt {

struct RotaryView {
  const int32_t *pos;
  const float *freq;
  int pairs, interleaved;   // (kernels know the second when they are compiled: kNear below)
  float eps;
};

// cos and sin of pos * freq.  Quarter turns in 64 bits, less the nearest whole number; what is left, within an
// eighth of a turn, in fp32 by the Taylor series (the terms left out: below 2e-9 and 2e-10).
__device__ inline float2 angle_of(int pos, float freq) {
  const double t = (double)pos * (double)freq * 0.63661977236758134308;  // 2 / pi
  const double n = rint(t);
  const float y = (float)(t - n) * 1.57079632679489662f;
  const int quarter = (int)((long long)n & 3);
  const float z = y * y;
  float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(z, s, 8.33333333e-3f);
  s = fmaf(z, s, -1.66666667e-1f);
  s = fmaf(z * s, y, y);
  float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  c = fmaf(z, c, -1.38888889e-3f);
  c = fmaf(z, c, 4.16666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.0f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter & 2 ? -b : b);
}

// the first element of run h of unit u of a head of D elements; kNear: pairs are neighbours
template <bool kNear>
__device__ inline int unit_at(const RotaryView &r, int D, int u, int h) {
  const int n = kNear ? 0 : r.pairs / 8;   // units of pairs across runs
  return u < n ? 8 * u + h * r.pairs : 16 * n + 8 * (u - n + h * (D / 16 - n));
}

// cos and sin for a unit's pairs: eight across its runs (from element e0), or four in each (from e0 and e1)
struct Turn {
  float2 a[8];
  bool on0, on1;   // whether a run is turned
};
template <bool kNear, typename F>
__device__ __forceinline__ Turn turn_of(const RotaryView &r, int e0, int e1, F angle) {
  Turn t;
  t.on0 = e0 < 2 * r.pairs;
  t.on1 = kNear ? e1 < 2 * r.pairs : t.on0;
#pragma unroll
  for (int j = 0; j < 8; ++j) t.a[j] = make_float2(1.0f, 0.0f);
  if (t.on0)
#pragma unroll
    for (int j = 0; j < (kNear ? 4 : 8); ++j) t.a[j] = angle(kNear ? e0 / 2 + j : e0 + j);
  if (kNear && t.on1)
#pragma unroll
    for (int j = 0; j < 4; ++j) t.a[4 + j] = angle(e1 / 2 + j);
  return t;
}

// the unit turned (x: its runs one after the other); the products' order is fixed, so that the
// kernels that share this agree in every bit
template <bool kNear>
__device__ __forceinline__ void turn(float (&x)[16], const Turn &t) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (!(h ? t.on1 : t.on0)) continue;
#pragma unroll
    for (int j = 4 * h; j < 4 * h + 4; ++j) {
      const int a = kNear ? 2 * j : j, b = kNear ? 2 * j + 1 : 8 + j;
      const float p = x[a], q = x[b];
      x[a] = fmaf(p, t.a[j].x, -(q * t.a[j].y));
      x[b] = fmaf(q, t.a[j].x, p * t.a[j].y);
    }
  }
}

// eight elements of a row of the caller's tensor, as 32-bit words (bf16: two a word)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <bool vec>
__device__ __forceinline__ void load8(const float *p, uint32_t (&w)[8]) {
  if (vec) {
    const u32x4 a = reinterpret_cast<const u32x4 *>(p)[0], b = reinterpret_cast<const u32x4 *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a[i], w[4 + i] = b[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(p[i]);
  }
}
template <bool vec>
__device__ __forceinline__ void load8(const uint16_t *p, uint32_t (&w)[4]) {
  if (vec) {
    const u32x4 a = reinterpret_cast<const u32x4 *>(p)[0];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  }
}
template <bool vec>
__device__ __forceinline__ void store8(float *p, const uint32_t (&w)[8]) {
  if (vec) {
    reinterpret_cast<u32x4 *>(p)[0] = u32x4{w[0], w[1], w[2], w[3]};
    reinterpret_cast<u32x4 *>(p)[1] = u32x4{w[4], w[5], w[6], w[7]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __uint_as_float(w[i]);
  }
}
template <bool vec>
__device__ __forceinline__ void store8(uint16_t *p, const uint32_t (&w)[4]) {
  if (vec) {
    *reinterpret_cast<u32x4 *>(p) = u32x4{w[0], w[1], w[2], w[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
  }
}

__device__ inline uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}
// eight words' values, and back (rounded to nearest even)
__device__ inline void widen8(const uint32_t (&w)[8], float *x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
}
__device__ inline void widen8(const uint32_t (&w)[4], float *x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
__device__ inline void round8(const float *x, uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[i]);
}
__device__ inline void round8(const float *x, uint32_t (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
}

constexpr int kMaxPairs = 256;  // of dt_rotate (D <= 512)
constexpr int kRotWaves = 4;    // waves of a workgroup

// What a wave does of a row's heads: passes [first, last) of the heads that its lanes hold side by side, the
// queries' first, then the keys'.
struct HeadsView {
  RowsView in, out;
  const void *weight;
  int heads;
};

// One row by a wave.  `lanes` lanes a head (a power of two, 16 elements each); cs: the wave's own LDS.
template <typename T, bool vec, bool kNear>
__device__ __forceinline__ void rotate_row(const RotaryView &r, const HeadsView &q, const HeadsView &k, int D,
                                           int lanes, int64_t row, int first, int last, float2 *cs) {
  constexpr int kWords = sizeof(T) == 4 ? 8 : 4;
  const int lane = threadIdx.x & 63, u = lane & (lanes - 1), wide = 64 / lanes;
  const int q_passes = (q.heads + wide - 1) / wide;
  const bool here = 16 * u < D;
  const int at[2] = {unit_at<kNear>(r, D, u, 0), unit_at<kNear>(r, D, u, 1)};
  // a pass's head of this lane, and its elements (asked for a pass ahead: the first before the angles are computed)
  const auto head_of = [&](int pass) { return (pass < q_passes ? pass : pass - q_passes) * wide + lane / lanes; };
  uint32_t next[2][kWords];
  const auto ask = [&](int pass) {
    const bool of_q = pass < q_passes;
    const int head = head_of(pass);
    const T *p = reinterpret_cast<const T *>(of_q ? q.in.p : k.in.p) + row * (of_q ? q.in.row : k.in.row) +
                 head * (of_q ? q.in.head : k.in.head);
    if (here && head < (of_q ? q.heads : k.heads))
#pragma unroll
      for (int h = 0; h < 2; ++h) load8<vec>(p + at[h], next[h]);
  };
  ask(first);
  const int pos = r.pos[row];
  for (int j = lane; j < r.pairs; j += 64) cs[j] = angle_of(pos, r.freq[j]);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // (a wave's LDS accesses keep their order)
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const Turn a = turn_of<kNear>(r, at[0], at[1], [&](int j) { return cs[j]; });
  const float inv_d = 1.0f / (float)D;
  float w[16] = {};
  for (int pass = first; pass < last; ++pass) {
    const bool of_q = pass < q_passes;
    const T *weight = static_cast<const T *>(of_q ? q.weight : k.weight);
    if (weight && here && (pass == first || pass == q_passes)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t b[kWords];
        load8<true>(weight + at[h], b);
        widen8(b, w + 8 * h);
      }
    }
    const int head = head_of(pass);
    const bool on = here && head < (of_q ? q.heads : k.heads);
    float y[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t b[kWords];
#pragma unroll
      for (int j = 0; j < kWords; ++j) b[j] = on ? next[h][j] : 0u;
      widen8(b, y + 8 * h);
    }
    if (pass + 1 < last) ask(pass + 1);
    if (weight) {
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 16; ++j) sum = fmaf(y[j], y[j], sum);
      for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor(sum, o);
      const float f = rsqrtf(fmaf(sum, inv_d, r.eps));
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] *= f * w[j];
    }
    turn<kNear>(y, a);
    T *p = reinterpret_cast<T *>(of_q ? q.out.p : k.out.p) + row * (of_q ? q.out.row : k.out.row) +
           head * (of_q ? q.out.head : k.out.head);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t b[kWords];
      round8(y + 8 * h, b);
      if (on) store8<vec>(p + at[h], b);
    }
  }
}

// How rows are dealt: `lanes` lanes a head, `passes` passes a row, `splits` waves a row.
struct RotatePlan {
  int lanes, passes, splits, per;
};
RotatePlan rotate_plan(int64_t rows, int heads, int kv_heads, int D);

hipError_t launch_rotate(const RotaryView &r, const HeadsView &q, const HeadsView &k, int rows, int D, int dtype,
                         hipStream_t s);
hipError_t launch_append_rotated(const CacheView &c, int dtype, const ChunkView &k, const RotaryView &r,
                                 const HeadsView &q, const RowsView &kr, const void *k_weight, const RowsView &vr,
                                 hipStream_t s);

}  // namespace dt
