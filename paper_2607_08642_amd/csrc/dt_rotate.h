// Heads normed and rotated by position (dt_rotary), on the device.
//
// A head's D elements are dealt to lanes in units of 16, so that both elements of a pair are with one lane
// and every access is 16 bytes: unit u of pairs [8 u, 8 u + 8) is the runs of eight at 8 u and at
// pairs + 8 u, or the 16 neighbours where pairs are interleaved; past the pairs, 16 neighbours.
#pragma once

#include "dt_cache.h"

namespace dt {

struct RotaryView {
  const int32_t *pos;
  const float *freq;
  int pairs, interleaved;
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

// the first element of half h (eight elements) of unit u
__device__ inline int unit_at(const RotaryView &r, int u, int h) {
  return u < r.pairs / 8 && !r.interleaved ? 8 * u + h * r.pairs : 16 * u + 8 * h;
}

// the unit's pairs turned (x: its halves one after the other); the products' order is fixed, so that the
// kernels that share this agree in every bit
__device__ inline void turn(float (&x)[16], const float2 (&a)[8], int interleaved) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (interleaved) {
      const float p = x[2 * j], q = x[2 * j + 1];
      x[2 * j] = fmaf(p, a[j].x, -(q * a[j].y));
      x[2 * j + 1] = fmaf(q, a[j].x, p * a[j].y);
    } else {
      const float p = x[j], q = x[8 + j];
      x[j] = fmaf(p, a[j].x, -(q * a[j].y));
      x[8 + j] = fmaf(q, a[j].x, p * a[j].y);
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
template <typename T, bool vec>
__device__ __forceinline__ void rotate_row(const RotaryView &r, const HeadsView &q, const HeadsView &k, int D,
                                           int lanes, int64_t row, int first, int last, float2 *cs) {
  constexpr int kWords = sizeof(T) == 4 ? 8 : 4;
  const int lane = threadIdx.x & 63, u = lane & (lanes - 1), wide = 64 / lanes;
  const int pos = r.pos[row];
  for (int j = lane; j < r.pairs; j += 64) cs[j] = angle_of(pos, r.freq[j]);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // (a wave's LDS accesses keep their order)
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const bool turns = u < r.pairs / 8, here = 16 * u < D;
  float2 a[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) a[j] = turns ? cs[8 * u + j] : make_float2(1.0f, 0.0f);
  const int at[2] = {unit_at(r, u, 0), unit_at(r, u, 1)};
  const float inv_d = 1.0f / (float)D;
  const int q_passes = (q.heads + wide - 1) / wide;
  for (int part = 0; part < 2; ++part) {
    const HeadsView &x = part ? k : q;
    const int p0 = part ? max(first - q_passes, 0) : first, p1 = part ? last - q_passes : min(last, q_passes);
    if (p0 >= p1) continue;
    const T *weight = static_cast<const T *>(x.weight);
    float w[16] = {};
    if (weight && here) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t b[kWords];
        load8<true>(weight + at[h], b);
        widen8(b, w + 8 * h);
      }
    }
    for (int p = p0; p < p1; ++p) {
      const int head = p * wide + lane / lanes;
      const bool on = here && head < x.heads;
      float y[16];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t b[kWords] = {};
        if (on) load8<vec>(reinterpret_cast<const T *>(x.in.p) + row * x.in.row + head * x.in.head + at[h], b);
        widen8(b, y + 8 * h);
      }
      if (weight) {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) sum = fmaf(y[j], y[j], sum);
        for (int o = 1; o < lanes; o <<= 1) sum += __shfl_xor(sum, o);
        const float f = rsqrtf(fmaf(sum, inv_d, r.eps));
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] *= f * w[j];
      }
      if (turns) turn(y, a, r.interleaved);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t b[kWords];
        round8(y + 8 * h, b);
        if (on) store8<vec>(reinterpret_cast<T *>(x.out.p) + row * x.out.row + head * x.out.head + at[h], b);
      }
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
