// Attention over the paged cache: what the two kernels share (geometry of a tile, masks,
// one block's softmax, the step that keeps unseen non-finite values out).
//
// Rows of a tile are (query i, head) pairs of one kv head, i-major: r = i * group + h.
// A wave holds 32 rows as the columns of the 32x32 matrix products
//   S^T [32 keys x 32 rows] = K Q^T,   O^T [D x 32 rows] += V^T P^T,
// so a lane owns one row: its running maximum, its sum and its rescaling are plain
// registers, and a row's 32 scores lie in two lanes (lane and lane ^ 32).
#pragma once

#include "dt_cache.h"

namespace dt {
namespace att {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The running maximum (of scores in units of log 2) of a row that has seen nothing.
// Finite, so that exp2(-inf - kFloor) = 0 needs no special case.
constexpr float kFloor = -1e30f;
constexpr int kTreeWords = (kMaxB + 2 * kBlk - 2) / kBlk;  // blocks that a tree's nodes touch
constexpr int kMaxSplits = 64;                              // (one lane each where they are joined)

__device__ inline float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }  // (NaN stays)
__device__ inline float max3(float a, float b, float c) { return max2(max2(a, b), c); }
// x of this lane and of lane ^ 32
__device__ inline float2 halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline bf16x8 as_bf16x8(u32x4 v) {
  bf16x8 r;
  __builtin_memcpy(&r, &v, 16);
  return r;
}
__device__ inline uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : ~(~0u << n); }

// A workgroup's rows and the key blocks that they see.
struct Tile {
  Seq q;
  int rows, r0;          // (query, head) rows of the sequence, first of the tile
  int i0, i1;            // its first and last query
  int tree0;             // position of the first node (no tree: INT_MAX)
  int nsb, wb, n_iter;   // iterations [0, nsb) are blocks 0.., the others blocks wb..
  __device__ int block(int it) const { return it < nsb ? it : wb + it - nsb; }
};
// false: the tile has no rows
__device__ inline bool tile_of(const AttendArgs &a, int b, int r0, int tile_rows, Tile *t) {
  t->q = seq_of(a.chunk, a.cache.page_shift, b);
  t->rows = t->q.n * a.group;
  t->r0 = r0;
  if (r0 >= t->rows) return false;
  t->i0 = r0 / a.group;
  t->i1 = (min(r0 + tile_rows, t->rows) - 1) / a.group;
  const int base = t->q.base, lead = t->q.n - a.nodes;
  const bool nodes = a.nodes > 0 && t->i1 >= lead;
  t->tree0 = a.nodes > 0 ? base + lead : 0x7fffffff;
  const int end = min(nodes ? base + t->q.n : base + t->i1 + 1, t->q.len);  // keys before it
  const int blocks = (max(end, 0) + kBlk - 1) / kBlk;
  // (a node's position is the root's or after it: depths are taken as >= 0)
  const int low = nodes ? min(base + t->i0, t->tree0 - 1) : base + t->i0;
  const int wb = a.window > 0 ? min(max(low - a.window + 1, 0) / kBlk, blocks) : 0;
  const int nsb = a.window > 0 ? min((a.sinks + kBlk - 1) / kBlk, blocks) : 0;
  const bool gap = nsb < wb;
  t->nsb = gap ? nsb : 0;
  t->wb = gap ? wb : 0;
  t->n_iter = t->nsb + blocks - t->wb;
  return true;
}
// workgroups that share the tile's blocks (those after them have none; the last takes
// what the host's bound left out)
__device__ inline int active_splits(const AttendArgs &a, const Tile &t) {
  return min(a.splits, max(1, (t.n_iter + a.split_blocks - 1) / a.split_blocks));
}

// The rows' nodes as bits: word w of query i0 + t holds its mask over block
// tree0 / 32 + w, into words[t * kTreeWords + w].  Every thread of the workgroup.
__device__ inline void tree_words(const AttendArgs &a, const Tile &t, int b, uint32_t *words, int threads) {
  const int lead = t.q.n - a.nodes, tb0 = max(t.tree0, 0) / kBlk, n = (t.i1 - t.i0 + 1) * kTreeWords;
  for (int x = threadIdx.x; x < n; x += threads) {
    const int m = t.i0 + x / kTreeWords - lead, j0 = (tb0 + x % kTreeWords) * kBlk - t.tree0;
    uint32_t w = 0;
    if (m >= 0 && j0 < a.nodes) {
      const uint8_t *row = a.mask + ((int64_t)b * a.nodes + m) * a.nodes;
#pragma unroll 8
      for (int j = 0; j < kBlk; ++j)
        if (j0 + j >= 0 && j0 + j < a.nodes && row[j0 + j]) w |= 1u << j;
    }
    words[x] = w;
  }
}

// A lane's row and what it sees.
struct Row {
  int r, i;            // (rows past the last repeat it)
  int hi, lo;          // keys before the nodes: lo < key <= hi, or key < sinks
  const uint32_t *words;  // the nodes it sees (null: none)
  // over the wave: bounds that settle most blocks without looking at a lane
  int min_hi, max_lo, min_lo, reach, tree_from;
};
__device__ inline int wave_min(int x) {
  for (int o = 1; o < 64; o <<= 1) x = min(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ inline Row row_of(const AttendArgs &a, const Tile &t, int b, int r, const uint32_t *words) {
  Row w;
  w.r = min(r, t.rows - 1);
  w.i = w.r / a.group;
  const int lead = t.q.n - a.nodes, last = t.q.len - 1;
  const bool node = a.nodes > 0 && w.i >= lead;
  int pos = t.q.base + w.i;
  if (node) {
    pos = t.tree0 - 1;
    if (a.window > 0) pos += min(max(a.depth[(int64_t)b * a.nodes + w.i - lead], 0), 1 << 20);
  }
  w.hi = min(node ? t.tree0 - 1 : t.q.base + w.i, last);
  w.lo = a.window > 0 ? pos - a.window : -1;
  w.words = node ? words + (w.i - t.i0) * kTreeWords : nullptr;
  const bool nodes = __ballot(node) != 0;
  w.min_hi = wave_min(w.hi);
  w.max_lo = -wave_min(-w.lo);
  w.min_lo = wave_min(w.lo);
  w.reach = nodes ? last : -wave_min(-w.hi);
  w.tree_from = nodes ? t.tree0 : 0x7fffffff;
  return w;
}
__device__ inline bool sees_all(const AttendArgs &a, const Row &w, int k0) {
  return k0 + kBlk - 1 <= w.min_hi && (k0 > w.max_lo || (a.window > 0 && k0 + kBlk <= a.sinks));
}
__device__ inline bool sees_none(const AttendArgs &a, const Row &w, int k0) {
  return k0 > w.reach || (k0 + kBlk - 1 <= w.min_lo && k0 >= a.sinks && k0 + kBlk <= w.tree_from);
}
// bit j: the lane's row sees token j of block k0
__device__ inline uint32_t seen_word(const AttendArgs &a, const Tile &t, const Row &w, int k0) {
  uint32_t v = low_bits(w.hi - k0 + 1);
  if (a.window > 0) v &= ~low_bits(w.lo + 1 - k0) | low_bits(a.sinks - k0);
  if (w.words) {
    const int x = k0 / kBlk - max(t.tree0, 0) / kBlk;
    if (x >= 0 && x < kTreeWords) v |= w.words[x] & low_bits(t.q.len - k0);
  }
  return v;
}

// token of a block in register i of a lane's half of S^T
__device__ constexpr int reg_token(int i) { return 8 * (i / 4) + i % 4; }  // + 4 h

// One block's scores into probabilities (masked: bits of `seen`, already shifted by 4 h).
// m: running maximum, l: this lane's part of the sum.  Returns the factor of what was
// summed before, and whether any row of the wave needs it.
template <bool MASKED>
__device__ inline float softmax_block(const f32x16 &s, uint32_t seen, float c, float &m, float &l, float (&p)[16]) {
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = MASKED && !(seen >> reg_token(i) & 1) ? -__builtin_huge_valf() : s[i];
  float top = max3(x[0], x[1], x[2]);
#pragma unroll
  for (int i = 3; i < 15; i += 2) top = max3(top, x[i], x[i + 1]);
  const float2 th = halves(max3(top, x[15], x[15]));
  const float now = max3(m, max3(th.x, th.y, th.y) * c, kFloor);
  const float f = __builtin_amdgcn_exp2f(m - now);
  m = now;
  float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -now));
    if (MASKED) p[i] = seen >> reg_token(i) & 1 ? p[i] : 0.0f;
    if (i & 1)
      sum1 += p[i];
    else
      sum0 += p[i];
  }
  l = l * f + (sum0 + sum1);
  return f;
}

// eight probabilities (registers 8 s .. 8 s + 7) as the second operand of step s
__device__ inline bf16x8 pack_p(const float (&p)[16], int s) {
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = p[8 * s + i];
  return __builtin_convertvector(v, bf16x8);
}
__device__ inline bf16x8 pack_seen(uint32_t seen, int s) {  // 1 where a token is seen
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = seen >> reg_token(8 * s + i) & 1 ? 1.0f : 0.0f;
  return __builtin_convertvector(v, bf16x8);
}
// values with their NaN and infinities as 0, and 1 in their places
__device__ inline void split_bad(u32x4 v, u32x4 &clean, u32x4 &bad) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (v[i] & 0x7f80u) == 0x7f80u, hi = (v[i] & 0x7f800000u) == 0x7f800000u;
    clean[i] = v[i] & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
    bad[i] = (lo ? 0x3f80u : 0u) | (hi ? 0x3f800000u : 0u);
  }
}
__device__ inline bool has_bad(u32x4 v) {
  bool r = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) r |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
  return r;
}

__device__ inline f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}

// a lane's row of q as operands: register piece n of a 16-byte piece layout (E elements a
// piece, this lane's half h takes pieces 2 n + h); bf16: eight elements an operand
template <int DT, int D>
struct QRegs {
  static constexpr int N = DT == DT_F32 ? D / 8 : D / 16;  // 16-byte registers
  u32x4 v[N];
};
// (scale < 0: the sign goes into q)
template <int DT, int D>
__device__ inline void load_q(const AttendArgs &a, const Tile &t, const Row &w, int head, int h, bool interleave8,
                              QRegs<DT, D> &q) {
  const int64_t at = (int64_t)(t.q.row0 + w.i) * a.q.row + (int64_t)(head * a.group + w.r % a.group) * a.q.head;
  const uint32_t flip = a.scale_log2e < 0.0f ? (DT == DT_F32 ? 0x80000000u : 0x80008000u) : 0u;
#pragma unroll
  for (int n = 0; n < QRegs<DT, D>::N; ++n) {
    // first element of piece n: f32 pieces of 4, bf16 of 8; an 8-bit cache's pieces of 16
    // elements are two operands
    const int d = DT == DT_F32 ? (2 * n + h) * 4 : interleave8 ? (2 * (n >> 1) + h) * 16 + 8 * (n & 1) : (2 * n + h) * 8;
    u32x4 v;
    if (DT == DT_F32) {
      const float *p = reinterpret_cast<const float *>(a.q.p) + at + d;
      if (a.q.vec)
        v = *reinterpret_cast<const u32x4 *>(p);
      else
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(p[j]);
    } else {
      const uint16_t *p = reinterpret_cast<const uint16_t *>(a.q.p) + at + d;
      if (a.q.vec)
        v = *reinterpret_cast<const u32x4 *>(p);
      else
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) q.v[n][j] = v[j] ^ flip;
  }
}

// A wave's 32 finished rows: the result, or one split's part of it.
template <int DT, int D>
__device__ inline void write_rows(const AttendArgs &a, const Tile &t, const Row &w, int head, int split, bool direct,
                                  bool valid, int h, const f32x16 (&o)[D / 32], float m, float l) {
  if (!valid) return;
  const int hq = head * a.group + w.r % a.group;
  const int64_t row = t.q.row0 + w.i;
  if (!direct) {
    const int64_t at = (row * a.heads + hq) * a.splits + split;
    if (h == 0) a.part_ml[at] = make_float2(m, l);
    float *p = a.part + at * D;
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *reinterpret_cast<f32x4 *>(p + 32 * n + 8 * x + 4 * h) =
            f32x4{o[n][4 * x], o[n][4 * x + 1], o[n][4 * x + 2], o[n][4 * x + 3]};
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // (l = 0: the row saw nothing, o is 0)
  const int64_t at = row * a.out.row + (int64_t)hq * a.out.head;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int d = 32 * n + 8 * x + 4 * h;
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = o[n][4 * x + j] * inv;
      if (DT == DT_F32) {
        float *p = reinterpret_cast<float *>(a.out.p) + at + d;
        if (a.out.vec)
          *reinterpret_cast<f32x4 *>(p) = f32x4{y[0], y[1], y[2], y[3]};
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) p[j] = y[j];
      } else {
        __bf16 *p = reinterpret_cast<__bf16 *>(a.out.p) + at + d;
        const bf16x2 u = {(__bf16)y[0], (__bf16)y[1]}, v = {(__bf16)y[2], (__bf16)y[3]};
        if (a.out.vec) {
          uint2 z;
          __builtin_memcpy(&z.x, &u, 4);
          __builtin_memcpy(&z.y, &v, 4);
          *reinterpret_cast<uint2 *>(p) = z;
        } else {
          p[0] = u[0];
          p[1] = u[1];
          p[2] = v[0];
          p[3] = v[1];
        }
      }
    }
}

}  // namespace att
hipError_t launch_attend_tile(const AttendArgs &a, const AttendPlan &p, hipStream_t s);
}  // namespace dt
