// Attention over the paged cache: what the two kernels share (geometry of a tile, masks,
// one block's softmax, the step that keeps unseen non-finite values out).
//
// Rows of a tile are (query i, head) pairs of one kv head, i-major: r = i * group + h.
// A wave holds 32 rows as the columns of the 32x32 matrix products
//   S^T [32 keys x 32 rows] = K Q^T,   O^T [D x 32 rows] += V^T P^T,
// so a lane owns one row: its running maximum, its sum and its rescaling are plain
// registers, and a row's 32 scores lie in two lanes (lane and lane ^ 32).
#pragma once

#include <type_traits>

#include "dt_cache.h"

namespace dt {
namespace att {

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

__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }  // (NaN stays)
__device__ __forceinline__ float max3(float a, float b, float c) { return max2(max2(a, b), c); }
// x of this lane and of lane ^ 32
__device__ __forceinline__ float2 halves(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
  bf16x8 r;
  __builtin_memcpy(&r, &v, 16);
  return r;
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : ~(~0u << n); }

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
__device__ __forceinline__ bool tile_of(const AttendArgs &a, int b, int r0, int tile_rows, Tile *t) {
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
__device__ __forceinline__ int active_splits(const AttendArgs &a, const Tile &t) {
  return min(a.splits, max(1, (t.n_iter + a.split_blocks - 1) / a.split_blocks));
}

// The rows' nodes as bits: word w of query i0 + t holds its mask over block
// tree0 / 32 + w, into words[t * kTreeWords + w].  Every thread of the workgroup.
__device__ __forceinline__ void tree_words(const AttendArgs &a, const Tile &t, int b, uint32_t *words, int threads) {
  const int lead = t.q.n - a.nodes, tb0 = max(t.tree0, 0) / kBlk, n = (t.i1 - t.i0 + 1) * kTreeWords;
  for (int x = threadIdx.x; x < n; x += threads) {
    const int m = t.i0 + x / kTreeWords - lead, j0 = (tb0 + x % kTreeWords) * kBlk - t.tree0;
    uint32_t w = 0;
    if (m >= 0 && j0 < a.nodes) {
      const uint8_t *row = a.mask + ((int64_t)b * a.nodes + m) * a.nodes;
      uint32_t v[kBlk];  // (bytes outside the row are read as its ends and not taken)
#pragma unroll
      for (int j = 0; j < kBlk; ++j) v[j] = row[min(max(j0 + j, 0), a.nodes - 1)];
      __builtin_amdgcn_sched_barrier(0);  // (all on their way before the first is looked at)
#pragma unroll
      for (int j = 0; j < kBlk; ++j) w |= (v[j] != 0 ? 1u : 0u) << j;
      w &= ~low_bits(-j0) & low_bits(a.nodes - j0);
    }
    words[x] = w;
  }
}

// A walk over a tile's blocks from iteration `it` on, in steps of STEP: where the present one lies.
// Blocks of one page follow each other, so the table is looked at once a page, and a page ahead
// (the scalar load takes its time).
template <int STEP>
struct Walk {
  const char *base;  // of the kv head in page 0
  const int32_t *table;
  int64_t page_bytes;
  int pages, shift, it, end;
  int left;         // blocks of the walk left in the page
  int next_page;    // of the first block after those, as the table has it
  bool there;       // the page is in range (else: page 0, whose tokens then count as unseen)
  const char *keys;  // the block's keys (its values v_off behind them)
  const char *exps;  // DT_F8: its keys' exponents
  __device__ __forceinline__ Walk(const AttendArgs &a, const Tile &t, int b, int head, int from, int to)
      : base(a.cache.base + head * a.cache.head_bytes), table(a.chunk.table + (int64_t)b * a.chunk.width),
        page_bytes(a.cache.page_bytes), pages(a.cache.pages), shift(a.cache.page_shift), it(from), end(to), left(0),
        next_page(0), there(false), keys(base), exps(base) {
    look(t, it);
  }
  __device__ __forceinline__ void look(const Tile &t, int at) {
    if (at < end) next_page = scalar_at(table, t.block(at) * kBlk >> shift);
  }
  __device__ __forceinline__ bool done() const { return it >= end; }
  // the present block (not done): keys, exps and there hold for it
  __device__ __forceinline__ void open(const AttendArgs &a, const Tile &t, int block_bytes) {
    if (left > 0) return;
    const int block = t.block(it), n = block * kBlk & ((1 << shift) - 1);
    there = (uint32_t)next_page < (uint32_t)pages;
    const char *page = base + (int64_t)(there ? next_page : 0) * page_bytes;
    keys = page + (int64_t)(n / kBlk) * block_bytes;
    exps = page + a.cache.s_off + n;
    const int in_page = ((1 << shift) - n) / kBlk, run = it < t.nsb ? min(in_page, t.nsb - it) : in_page;
    left = (run + STEP - 1) / STEP;
    look(t, it + left * STEP);
  }
  __device__ __forceinline__ void step(int block_bytes) {
    keys += STEP * block_bytes;
    exps += STEP * kBlk;
    --left;
    it += STEP;
  }
};

// A lane's row and what it sees.
struct Row {
  int r, i;            // (rows past the last repeat it)
  int hi, lo;          // keys before the nodes: lo < key <= hi, or key < sinks
  const uint32_t *words;  // the nodes it sees (null: none)
  // over the wave: bounds that settle most blocks without looking at a lane
  int min_hi, max_lo, min_lo, reach, tree_from;
};
__device__ __forceinline__ int wave_min(int x) {
  for (int o = 1; o < 64; o <<= 1) x = min(x, __shfl_xor(x, o));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ Row row_of(const AttendArgs &a, const Tile &t, int b, int r, const uint32_t *words) {
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
  // the bounds, from the wave's first and last query where they follow from them
  const int ia = __builtin_amdgcn_readfirstlane(w.i), ib = __builtin_amdgcn_readlane(w.i, 63);
  const bool nodes = a.nodes > 0 && ib >= lead;
  const int hi_a = min(nodes && ia >= lead ? t.tree0 - 1 : t.q.base + ia, last);
  w.min_hi = hi_a;
  w.reach = nodes ? last : min(t.q.base + ib, last);
  w.tree_from = nodes ? t.tree0 : 0x7fffffff;
  w.min_lo = w.max_lo = -1;
  if (a.window > 0) {
    if (nodes) {
      w.max_lo = -wave_min(-w.lo);
      w.min_lo = wave_min(w.lo);
    } else {
      w.min_lo = t.q.base + ia - a.window;
      w.max_lo = t.q.base + ib - a.window;
    }
  }
  return w;
}
__device__ __forceinline__ bool sees_none(const AttendArgs &a, const Row &w, int k0) {
  return k0 > w.reach || (k0 + kBlk - 1 <= w.min_lo && k0 >= a.sinks && k0 + kBlk <= w.tree_from);
}
// The end of the run of blocks from iteration `it` on that all rows see whole (`it`: none).
__device__ __forceinline__ int full_end(const AttendArgs &a, const Tile &t, const Row &w, int it) {
  const int blocks = max(w.min_hi + 1, 0) / kBlk;  // (those before it lie below every row's bound)
  const int block = t.block(it);
  int end;
  if (block * kBlk > w.max_lo)
    end = blocks;
  else if (a.window > 0 && block * kBlk + kBlk <= a.sinks)
    end = min(blocks, a.sinks / kBlk);
  else
    return it;
  if (it < t.nsb) end = min(end, t.nsb);  // (then a gap follows)
  return max(it, it + end - block);
}
// bit j: the lane's row sees token j of block k0
__device__ __forceinline__ uint32_t seen_word(const AttendArgs &a, const Tile &t, const Row &w, int k0) {
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

template <int T>
__device__ __forceinline__ void rescale(f32x16 (&o)[T], float f) {
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] *= f;
}

// One block's scores into probabilities (masked: bits of `seen`, already shifted by 4 h).
// m: the reference that exponents are taken against, l: this lane's part of the sum (which the
// probabilities join as they become an operand: POperand).  m is never below a maximum, so no
// probability is above one and sums of p v stay within what the values themselves sum to.  It is raised, and
// what was summed scaled, to kSlack above the maximum that passed it: the lesser probabilities do no harm in
// fp32, nor rounded to bf16 (both have their bits down to 2^-126), and after a tile's first blocks the
// scaling (as many products as there are sums) hardly ever runs.
constexpr float kSlack = 8.0f;
template <bool MASKED, int T>
__device__ __forceinline__ void softmax_block(const f32x16 &s, uint32_t seen, float c, float &m, float &l,
                                              f32x16 (&o)[T], float (&p)[16]) {
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = MASKED && !(seen >> reg_token(i) & 1) ? -__builtin_huge_valf() : s[i];
  float top = max3(x[0], x[1], x[2]);
#pragma unroll
  for (int i = 3; i < 15; i += 2) top = max3(top, x[i], x[i + 1]);
  const float2 th = halves(max2(top, x[15]));
  const float now = max2(th.x, th.y) * c;
  if (__builtin_expect(__ballot(now > m) != 0, 0)) {
    const float to = now > m ? now + kSlack : m, f = __builtin_amdgcn_exp2f(m - to);
    m = to;
    l *= f;
    rescale(o, f);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -m));
    if (MASKED) p[i] = seen >> reg_token(i) & 1 ? p[i] : 0.0f;
  }
}

// eight probabilities (registers 8 s .. 8 s + 7) as the second operand of step s
__device__ __forceinline__ bf16x8 pack_p(const float (&p)[16], int s) {
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = p[8 * s + i];
  return __builtin_convertvector(v, bf16x8);
}
// A word of values: all bits of its non-finite elements (`one` masked by them: 1 in their places).
template <int DT>
constexpr uint32_t kOnes = DT == DT_F32 ? 0x3f800000u : DT == DT_BF16 ? 0x3f803f80u : 0x38383838u;
template <int DT>
__device__ __forceinline__ uint32_t bad_bits(uint32_t v) {
  if (DT == DT_F32) return (v & 0x7f800000u) == 0x7f800000u ? ~0u : 0u;
  if (DT == DT_BF16)
    return ((v & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((v & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
  // a code of seven ones; a carry out of them is bit 7
  const uint32_t t = ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (t >> 7) * 0xffu;
}
// Whether any of many words has a non-finite element: two or three instructions a word.
template <int DT>
struct AnyBad {
  uint32_t acc = 0;
  __device__ __forceinline__ void look(uint32_t v) {
    if constexpr (DT == DT_F32) {
      acc = max(acc, v & 0x7f800000u);
    } else if constexpr (DT == DT_BF16) {  // (the largest exponent of either half)
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      u16x2 x, y;
      const uint32_t e = v & 0x7f807f80u;
      __builtin_memcpy(&x, &acc, 4);
      __builtin_memcpy(&y, &e, 4);
      x = __builtin_elementwise_max(x, y);
      __builtin_memcpy(&acc, &x, 4);
    } else {
      acc |= (v & 0x7f7f7f7fu) + 0x01010101u;
    }
  }
  __device__ __forceinline__ bool any() const {
    if (DT == DT_F32) return acc == 0x7f800000u;
    if (DT == DT_BF16) return (acc & 0xffffu) == 0x7f80u || acc >> 16 == 0x7f80u;
    return (acc & 0x80808080u) != 0;
  }
};
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
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
// (scale < 0: the sign goes into q; elements d0 on)
template <int DT, int D>
__device__ __forceinline__ void load_q(const AttendArgs &a, const Tile &t, const Row &w, int head, int h, int d0,
                              QRegs<DT, D> &q) {
  const int64_t at = (int64_t)(t.q.row0 + w.i) * a.q.row + (int64_t)(head * a.group + w.r % a.group) * a.q.head + d0;
  // first element of piece n: f32 pieces of 4, bf16 of 8; an 8-bit cache's pieces of 16
  // elements are two operands
  auto first = [&](int n) {
    return DT == DT_F32 ? (2 * n + h) * 4 : DT == DT_F8 ? (2 * (n >> 1) + h) * 16 + 8 * (n & 1) : (2 * n + h) * 8;
  };
  if (a.q.vec) {
#pragma unroll
    for (int n = 0; n < QRegs<DT, D>::N; ++n)
      q.v[n] = *reinterpret_cast<const u32x4 *>(a.q.p + (at + first(n)) * (DT == DT_F32 ? 4 : 2));
  } else {
#pragma unroll
    for (int n = 0; n < QRegs<DT, D>::N; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (DT == DT_F32) {
          q.v[n][j] = reinterpret_cast<const uint32_t *>(a.q.p)[at + first(n) + j];
        } else {
          const uint16_t *p = reinterpret_cast<const uint16_t *>(a.q.p) + at + first(n) + 2 * j;
          q.v[n][j] = p[0] | (uint32_t)p[1] << 16;
        }
  }
  const uint32_t flip = a.scale_log2e < 0.0f ? (DT == DT_F32 ? 0x80000000u : 0x80008000u) : 0u;
#pragma unroll
  for (int n = 0; n < QRegs<DT, D>::N; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) q.v[n][j] ^= flip;
}

// Waits of a wave for its copies from memory to LDS: at most N of them on their way, its LDS
// reads done.  (Copies are not in the compiler's sight: no read moves over a wait.)
template <int N>
__device__ __forceinline__ void wait_copies() {
  static_assert(N < 64, "");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | (N >> 4) << 14);  // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
}
// 64 lanes' 16 bytes (or 4) at src + lane_off to LDS, lane after lane
__device__ __forceinline__ void copy16(const char *src, uint32_t lane_off, char *dst) {
  __builtin_amdgcn_global_load_lds(src + lane_off, (__attribute__((address_space(3))) char *)dst, 16, 0, 0);
}
__device__ __forceinline__ void copy4(const char *src, uint32_t lane_off, char *dst) {
  __builtin_amdgcn_global_load_lds(src + lane_off, (__attribute__((address_space(3))) char *)dst, 4, 0, 0);
}

// eight 8-bit elements (words a, b) times a power of two
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b, float scale) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false),
               y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
               z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false),
               w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

__device__ __forceinline__ u32x4 lds16(const char *p) { return *reinterpret_cast<const u32x4 *>(p); }

// Results of matrix products that are read behind a branch.  The products take cycles that the
// hardware does not wait for and the compiler has to fill; it has been seen to leave out the
// wait behind a branch (four of sixteen scores were read too early), so it stands here, in front of it:
// 20 states, which suffice for the longest product here (fp32: 16 passes).  Every result that is read behind a
// branch has one, or needs none because a later product's result has been waited for (products of a wave end in
// the order in which they are issued): the sums `o` that softmax_block scales and masked_block overwrites were
// issued before the block's scores, which softmax_block's maximum has read by then.  A new read of `o` or of scores
// behind a branch has to have either.
__device__ __forceinline__ void settle(f32x16 &s) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s)); }
struct Nothing {  // (no branch)
  __device__ __forceinline__ void operator()(f32x16 &) const {}
};

// S^T of a block: `keys` in LDS in the cache's order (DT_F8: `exps` their 32 exponents).
template <int DT, int D>
__device__ __forceinline__ f32x16 scores(const char *keys, const char *exps, const QRegs<DT, D> &q, int lane) {
  f32x16 s = zero16();
  const char *kp = keys + lane * 16;
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int n = 0; n < D / 8; ++n) {
      const u32x4 k = lds16(kp + n * 1024);
#pragma unroll
      for (int j = 0; j < 4; ++j) s = mfma(__uint_as_float(k[j]), __uint_as_float(q.v[n][j]), s);
    }
  } else if constexpr (DT == DT_BF16) {
#pragma unroll
    for (int n = 0; n < D / 16; ++n) s = mfma(as_bf16x8(lds16(kp + n * 1024)), as_bf16x8(q.v[n]), s);
  } else {
    const float e = exp_of(reinterpret_cast<const uint8_t *>(exps)[lane & 31]);
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
      const u32x4 k = lds16(kp + n * 1024);
#pragma unroll
      for (int u = 0; u < 2; ++u) s = mfma(widen8(k[2 * u], k[2 * u + 1], e), as_bf16x8(q.v[2 * n + u]), s);
    }
  }
  return s;
}

// A block's values in a lane's registers, in the cache's order: piece (s, t) holds element
// 32 t + (lane & 31) of 4, 8 or 16 tokens.
template <int DT, int D>
struct VRegs {
  static constexpr int S = DT == DT_F32 ? 4 : DT == DT_BF16 ? 2 : 1, T = D / 32;
  u32x4 v[T][S];
};
template <int DT, int D>
__device__ __forceinline__ const char *v_at(const char *vals, int s, int t, int lane) {
  return vals + ((lane >> 5) * D + (lane & 31)) * 16 + (2 * s * D + 32 * t) * 16;
}
// 2^(byte j of w - 127): byte j to the exponent's place (one instruction, where a shift and a mask would do)
__device__ __forceinline__ float power_of(uint32_t w, int j) {
  float e;
#define DT_SHIFT(n)                                                                                               \
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_" #n \
      : "=v"(e)                                                                                                   \
      : "v"(23), "v"(w))
  if (j == 0)
    DT_SHIFT(0);
  else if (j == 1)
    DT_SHIFT(1);
  else if (j == 2)
    DT_SHIFT(2);
  else
    DT_SHIFT(3);
#undef DT_SHIFT
  return e;
}
// An operand's elements added to a sum, two an instruction (products with 1 are exact).
__device__ __forceinline__ float sum_p(bf16x8 v, float sum) {
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{v[i], v[i + 1]}, one, sum, false);
  return sum;
}
__device__ __forceinline__ float sum_p(const float (&p)[16]) {
  float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; i += 2) sum0 += p[i], sum1 += p[i + 1];
  return sum0 + sum1;
}
// The probabilities as the operand of those products (DT_F8: times the tokens' powers of two, `exps`
// in LDS: exact), and in the row's sum l.  bf16 and 8-bit values are multiplied by probabilities rounded to
// bf16: error against 64 bits 2.2e-3, of which the rounding of the result is 1.66e-3.  A second product with what the
// rounding leaves makes that 1.66e-3, and was measured and not taken: half as many matrix instructions again where those
// count, and for single tokens in bf16 0.4 to 7% longer (32 of up to 8,192: 133.7 -> 134.3 us, eight of 2,048: 18.1 ->
// 19.4), in 8 bits 4 to 13% (87.6 -> 96.4).  With bf16 values the sum takes them as rounded, so that a row's weights
// add up to one as they are used (equal values give that value; a chunk of 4,096 rows 2.27e-3 with a sum of
// the unrounded and 2.24e-3, one of 2,047 under a window 2.27e-3 and 2.16e-3).  In 8 bits the product wants them
// times a power of two, and rounding them once more for the sum took 5% longer (1,024 rows over 8,192 tokens: 177 and
// 185 us) for values that are themselves off by up to 2^-4: there the sum takes them unrounded.
template <int DT, bool MASKED>
struct POperand {
  bf16x8 f[2];
  __device__ __forceinline__ POperand(float (&p)[16], const char *exps, uint32_t seen, int h, float &l) {
    if constexpr (DT == DT_F8) {
      l += sum_p(p);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(exps + 8 * t + 4 * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = power_of(w, j);
          p[4 * t + j] = MASKED && !(seen >> reg_token(4 * t + j) & 1) ? 0.0f : p[4 * t + j] * e;
        }
      }
    }
    f[0] = pack_p(p, 0);
    f[1] = pack_p(p, 1);
    if constexpr (DT != DT_F8) l = sum_p(f[0], l) + sum_p(f[1], 0.0f);
  }
};
template <bool MASKED>
struct POperand<DT_F32, MASKED> {
  float f[16];
  __device__ __forceinline__ POperand(float (&p)[16], const char *, uint32_t, int, float &l) {
    l += sum_p(p);
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = p[i];
  }
};
// one d tile's pieces times 32 probabilities
template <int DT, int S, class P>
__device__ __forceinline__ f32x16 products(const u32x4 (&v)[S], const P &p, f32x16 acc) {
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc = mfma(__uint_as_float(v[s][j]), p.f[4 * s + j], acc);
  } else if constexpr (DT == DT_BF16) {
    acc = mfma(as_bf16x8(v[0]), p.f[0], acc);
    acc = mfma(as_bf16x8(v[1]), p.f[1], acc);
  } else {
    acc = mfma(widen8(v[0][0], v[0][1], 1.0f), p.f[0], acc);
    acc = mfma(widen8(v[0][2], v[0][3], 1.0f), p.f[1], acc);
  }
  return acc;
}

// A block that all rows see whole: keys and values in LDS (DT_F8: with their exponents).
// between(scores): before the values are needed.
template <int DT, int D, class F>
__device__ __forceinline__ void full_block(const char *keys, const char *vals, const char *exps, const QRegs<DT, D> &q,
                                           float c, int lane, float &m, float &l, f32x16 (&o)[D / 32],
                                           const F &between) {
  constexpr int T = D / 32, S = VRegs<DT, D>::S;
  f32x16 s = scores<DT, D>(keys, exps, q, lane);
  if (!std::is_same<F, Nothing>::value) settle(s);
  between(s);
  // the values are asked for before the softmax where registers allow
  constexpr bool kEarly = S * T <= 8;
  VRegs<DT, D> r;
  if (kEarly)
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int x = 0; x < S; ++x) r.v[t][x] = lds16(v_at<DT, D>(vals, x, t, lane));
  float p[16];
  softmax_block<false>(s, 0, c, m, l, o, p);
  const POperand<DT, false> pf(p, exps + 32, 0, lane >> 5, l);
#pragma unroll
  for (int t = 0; t < T; ++t) {
    if (!kEarly)
#pragma unroll
      for (int x = 0; x < S; ++x) r.v[t][x] = lds16(v_at<DT, D>(vals, x, t, lane));
    o[t] = products<DT>(r.v[t], pf, o[t]);
  }
}

// Any other block.  Non-finite values that not all rows see make NaN (of those components)
// of the rows that do and are 0 for the others.
template <int DT, int D, class F>
__device__ __forceinline__ void masked_block(const char *keys, const char *vals, const char *exps,
                                             const QRegs<DT, D> &q, uint32_t seen, float c, int lane, float &m,
                                             float &l, f32x16 (&o)[D / 32], const F &between) {
  constexpr int T = D / 32, S = VRegs<DT, D>::S;
  f32x16 sc = scores<DT, D>(keys, exps, q, lane);
  settle(sc);
  between(sc);
  float p[16];
  softmax_block<true>(sc, seen, c, m, l, o, p);
  const POperand<DT, true> pf(p, exps + 32, seen, lane >> 5, l);
  AnyBad<DT> bad;
#pragma unroll
  for (int n = 0; n < S * T; ++n) {
    const u32x4 v = lds16(v_at<DT, D>(vals, n / T, n % T, lane));
#pragma unroll
    for (int i = 0; i < 4; ++i) bad.look(v[i]);
    if (n % 8 == 7) __builtin_amdgcn_sched_barrier(0);  // (eight pieces at a time: registers)
  }
  const bool any = __ballot(bad.any()) != 0;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    u32x4 v[S];
#pragma unroll
    for (int s = 0; s < S; ++s) v[s] = lds16(v_at<DT, D>(vals, s, t, lane));
    if (__builtin_expect(any, 0)) {
      float sf[16], none = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sf[i] = seen >> reg_token(i) & 1 ? 1.0f : 0.0f;
      u32x4 one[S];
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = bad_bits<DT>(v[s][i]);
          one[s][i] = x & kOnes<DT>;
          v[s][i] &= ~x;
        }
      const POperand<DT == DT_F8 ? DT_BF16 : DT, false> seen_op(sf, nullptr, 0, 0, none);
      const f32x16 hit = products<DT>(one, seen_op, zero16());
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = hit[i] > 0.0f ? __builtin_nanf("") : o[t][i];
    }
    o[t] = products<DT>(v, pf, o[t]);
    __builtin_amdgcn_sched_barrier(0);  // (one d tile at a time: registers)
  }
}

// Four elements of the result at element offset `at`.
template <int DT>
__device__ __forceinline__ void store4(const AttendArgs &a, int64_t at, float x, float y, float z, float w) {
  if (DT == DT_F32) {
    float *p = reinterpret_cast<float *>(a.out.p) + at;
    if (a.out.vec)
      *reinterpret_cast<f32x4 *>(p) = f32x4{x, y, z, w};
    else
      p[0] = x, p[1] = y, p[2] = z, p[3] = w;
  } else {
    __bf16 *p = reinterpret_cast<__bf16 *>(a.out.p) + at;
    const bf16x2 u = {(__bf16)x, (__bf16)y}, v = {(__bf16)z, (__bf16)w};
    if (a.out.vec) {
      uint2 q;
      __builtin_memcpy(&q.x, &u, 4);
      __builtin_memcpy(&q.y, &v, 4);
      *reinterpret_cast<uint2 *>(p) = q;
    } else {
      p[0] = u[0], p[1] = u[1], p[2] = v[0], p[3] = v[1];
    }
  }
}

// Four elements from d on of a finished row, maximum m and sum l: of the result, or of one split's part
// of it (the first split notes how many there are; one alone writes the result).
template <int DT>
__device__ __forceinline__ void write4(const AttendArgs &a, int64_t row, int hq, int d, int split, int active, f32x4 y,
                                       float m, float l) {
  if (a.splits > 1) {
    const int64_t x = row * a.heads + hq;
    float2 *ml = a.part_ml + x * (a.splits + 1);
    if (split == 0 && d == 0) ml[a.splits] = make_float2((float)active, 0.0f);
    if (active > 1) {
      if (d == 0) ml[split] = make_float2(m, l);
      *reinterpret_cast<f32x4 *>(a.part + (x * a.splits + split) * a.cache.D + d) = y;
      return;
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // (l = 0: the row saw nothing, y is 0)
  store4<DT>(a, row * a.out.row + (int64_t)hq * a.out.head + d, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
}

}  // namespace att
hipError_t launch_attend_tile(const AttendArgs &a, const AttendPlan &p, hipStream_t s);
}  // namespace dt
