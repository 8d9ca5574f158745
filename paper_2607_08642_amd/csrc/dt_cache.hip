// The paged cache: writing rows (quantising them for DT_F8), reading them back, and the
// two kernels that end a verification round (the accepted path, the move of its rows).
//
// All are copies: bound by memory traffic for prompts (append and read of four prompts of 11,437 to 16,384,
// 8 kv heads of 128: 85 and 58 us for 342 MB each in 8 bits, 4.0 and 5.9 TB/s; bf16 and fp32 together
// 5.0 to 5.2 TB/s; a copy: 4.7), by latency for the few rows of a decoding step (3.5 to 5 us a launch).
// A workgroup of append and read takes one block of 32
// tokens of one kv head, keys and values (layout: dt_cache.h), through two LDS tiles of
// 32 rows: rows of the caller's tensors are touched in runs of 128 bytes (eight lanes a
// row), pieces of the cache in runs of 512 bytes and more.  Values change sides in LDS two
// elements at a time.
#include <type_traits>

#include "dt_rotate.h"

namespace dt {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
static_assert(kThreads == 64 * kRotWaves, "a wave for each part of a row");
constexpr int kPad = 16;  // bytes after each row of the LDS tile: an odd number of 16-byte columns

template <int DT>
struct Elem;  // what a cache holds
template <>
struct Elem<DT_F32> {
  static constexpr int bytes = 4, E = 4;
  typedef float data;
};
template <>
struct Elem<DT_BF16> {
  static constexpr int bytes = 2, E = 8;
  typedef uint16_t data;
};
template <>
struct Elem<DT_F8> {
  static constexpr int bytes = 1, E = 16;
  typedef uint16_t data;
};

// The block of this workgroup: blocks of a chunk follow the cache's, so the first and the
// last may be partial.  False where it has no token.
struct Block {
  Seq q;
  int pos0;     // position of the block's token 0
  int lo, hi;   // tokens [lo, hi) of the block belong to the chunk
  int page;     // -1: out of range
  int in_page;  // token of the page that is the block's token 0
};
__device__ inline bool block_of(const CacheView &c, const ChunkView &k, int b, int blk, Block *o) {
  o->q = seq_of(k, c.page_shift, b);
  const int first = max(o->q.base, 0);
  o->pos0 = (first / kBlk + blk) * kBlk;
  o->lo = max(first - o->pos0, 0);
  o->hi = min(min(o->q.base + o->q.n, k.width << c.page_shift) - o->pos0, kBlk);
  if (o->lo >= o->hi) return false;
  const int page = scalar_at(k.table, (int64_t)b * k.width + (o->pos0 >> c.page_shift));
  o->page = page >= 0 && page < c.pages ? page : -1;
  o->in_page = o->pos0 & ((1 << c.page_shift) - 1);
  return true;
}

// Two rows' words side by side (bytes or halves of one token each): the low halves, the high halves.
__device__ inline uint32_t low16(uint32_t a, uint32_t b) { return (a & 0xffffu) | b << 16; }
__device__ inline uint32_t high16(uint32_t a, uint32_t b) { return a >> 16 | (b & 0xffff0000u); }

// A workgroup's block: kv head and block of the chunk (blockIdx.x), sequence (blockIdx.y).  kRotate: keys are normed
// and rotated between their load and the tile; a lane then holds both runs of a unit (dt_rotate.h).
template <int DT, int D, bool kRotate, bool kNear>
__device__ __forceinline__ void append_block(const CacheView &c, const ChunkView &k, const RowsView &kr,
                                             const RowsView &vr, const RotaryView &rot, const void *k_weight) {
  using El = Elem<DT>;
  using T = typename El::data;
  constexpr int E = El::E, kWords = sizeof(T) == 4 ? 8 : 4;  // words of eight elements
  constexpr int kRow = D * El::bytes + kPad, kRuns = kRotate ? (D / 16 + 7) / 8 * 2 : (D / 8 + 7) / 8;
  __shared__ __align__(16) char tiles[2][kBlk * kRow];
  const int head = blockIdx.x % c.kv;
  Block bl;
  if (!block_of(c, k, blockIdx.y, blockIdx.x / c.kv, &bl) || bl.page < 0) return;
  const int tid = threadIdx.x;
  char *page = c.base + bl.page * c.page_bytes + head * c.head_bytes;
  const int r = tid >> 3, sub = tid & 7;  // eight lanes a row
  const bool mine = r >= bl.lo && r < bl.hi;
  uint32_t w[2][kRuns][kWords];
  // the run's first element (of keys in units), and whether there is such a run
  auto at = [&](int v, int i) __attribute__((always_inline)) {
    return kRotate && !v ? unit_at<kNear>(rot, D, sub + 8 * (i / 2), i & 1) : 8 * (sub + 8 * i);
  };
  auto there = [&](int v, int i) __attribute__((always_inline)) {
    return kRotate && !v ? D % 128 == 0 || sub + 8 * (i / 2) < D / 16
                         : D % 64 == 0 ? i < D / 64 : sub + 8 * i < D / 8;  // (values may have fewer runs than units)
  };
  auto load = [&](auto vec) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const RowsView &src = v ? vr : kr;
      const T *p = reinterpret_cast<const T *>(src.p) + (int64_t)(bl.q.row0 + bl.pos0 + r - bl.q.base) * src.row +
                   (int64_t)head * src.head;
#pragma unroll
      for (int i = 0; i < kRuns; ++i)
        if (there(v, i)) load8<decltype(vec)::value>(p + at(v, i), w[v][i]);
    }
  };
  if (mine) {
    if (kr.vec && vr.vec)
      load(std::true_type());
    else
      load(std::false_type());
  }
  if constexpr (kRotate) {
    // (the eight lanes of a row are all `mine`, or none is)
    const int pos = mine ? rot.pos[bl.q.row0 + bl.pos0 + r - bl.q.base] : 0;
    const T *weight = static_cast<const T *>(k_weight);
    float x[kRuns / 2][16], sums[kRuns / 2], sum = 0.0f;  // (summed unit by unit, as rotate_row's lanes do)
#pragma unroll
    for (int n = 0; n < kRuns / 2; ++n) {
      sums[n] = 0.0f;
      if (mine && there(0, 2 * n)) {
        widen8(w[0][2 * n], x[n]);
        widen8(w[0][2 * n + 1], x[n] + 8);
#pragma unroll
        for (int j = 0; j < 16; ++j) sums[n] = fmaf(x[n][j], x[n][j], sums[n]);
      }
      for (int o = 1; o < 8; o <<= 1) sums[n] += __shfl_xor(sums[n], o);
      sum += sums[n];
    }
    const float f = rsqrtf(fmaf(sum, 1.0f / D, rot.eps));
#pragma unroll
    for (int n = 0; n < kRuns / 2; ++n)
      if (mine && there(0, 2 * n)) {
        const int runs[2] = {at(0, 2 * n), at(0, 2 * n + 1)};
        if (weight) {
          float g[16];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t b[kWords];
            load8<true>(weight + runs[h], b);
            widen8(b, g + 8 * h);
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) x[n][j] *= f * g[j];
        }
        turn<kNear>(x[n], turn_of<kNear>(rot, runs[0], runs[1], [&](int j) { return angle_of(pos, rot.freq[j]); }));
        round8(x[n], w[0][2 * n]);
        round8(x[n] + 8, w[0][2 * n + 1]);
      }
  }
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    char *row = tiles[v] + r * kRow;
    if constexpr (DT == DT_F8) {
      // the row's largest magnitude (bf16 bits order like the values), two at a time, over its
      // eight lanes; only where one is not finite, again without those
      u16x2 top2 = {0, 0};
      auto halves_of = [&](auto f) __attribute__((always_inline)) {
        if (mine)
#pragma unroll
          for (int i = 0; i < kRuns; ++i)
            if (there(v, i))
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                u16x2 x;
                const uint32_t m = w[v][i][j] & 0x7fff7fffu;
                __builtin_memcpy(&x, &m, 4);
                top2 = __builtin_elementwise_max(top2, f(x));
              }
      };
      halves_of([](u16x2 x) { return x; });
      const bool bad = top2[0] >= 0x7f80 || top2[1] >= 0x7f80;
      if (__ballot(bad)) {
        top2 = u16x2{0, 0};
        halves_of([](u16x2 x) { return u16x2{(uint16_t)(x[0] < 0x7f80 ? x[0] : 0), (uint16_t)(x[1] < 0x7f80 ? x[1] : 0)}; });
      }
      uint32_t top = max((uint32_t)top2[0], (uint32_t)top2[1]);
      for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
      // top = 1.m 2^(x - 127) <= 448 2^e = 1.75 2^(8 + e): e = x - 135, one more where 1.m > 1.75
      const int byte = min(max((int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), 7), 247);  // e + 127
      const float scale = exp_of((uint32_t)byte);
      if (mine) {
        if (sub == 0) page[c.s_off + (v ? (1 << c.page_shift) : 0) + bl.in_page + r] = (char)byte;
#pragma unroll
        for (int i = 0; i < kRuns; ++i)
          if (there(v, i)) {
            uint32_t code[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              // (x 2^-e, exact, rounded to nearest even)
              bf16x2 a, b;
              __builtin_memcpy(&a, &w[v][i][2 * u], 4);
              __builtin_memcpy(&b, &w[v][i][2 * u + 1], 4);
              i16x2 x = {0, 0};
              x = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(x, a, scale, false);
              x = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(x, b, scale, true);
              __builtin_memcpy(&code[u], &x, 4);
            }
            if (bad) {  // (0x7f and 0xff are the codes of NaN)
#pragma unroll
              for (int u = 0; u < 8; ++u) {
                const uint32_t x = w[v][i][u / 2] >> (16 * (u & 1)) & 0x7fffu;
                if (x >= 0x7f80u) code[u / 4] |= 0x7fu << (8 * (u & 3));
              }
            }
            *reinterpret_cast<uint2 *>(row + at(v, i)) = make_uint2(code[0], code[1]);
          }
      }
    } else if (mine) {
#pragma unroll
      for (int i = 0; i < kRuns; ++i)
        if (there(v, i)) {
          u32x4 *d = reinterpret_cast<u32x4 *>(row + El::bytes * at(v, i));
#pragma unroll
          for (int j = 0; j < kWords / 4; ++j)
            d[j] = u32x4{w[v][i][4 * j], w[v][i][4 * j + 1], w[v][i][4 * j + 2], w[v][i][4 * j + 3]};
        }
    }
  }
  __syncthreads();
  char *keys = page + (int64_t)bl.in_page * D * El::bytes, *vals = keys + c.v_off;
#pragma unroll
  for (int i = tid; i < kBlk * D / E; i += kThreads) {
    const int rr = i % kBlk;
    if (rr >= bl.lo && rr < bl.hi)
      reinterpret_cast<u32x4 *>(keys)[i] = *reinterpret_cast<const u32x4 *>(tiles[0] + rr * kRow + (i / kBlk) * 16);
  }
  if (bl.lo == 0 && bl.hi == kBlk) {
    // pieces (g, d) and (g, d + 1) from the rows of g's tokens
    for (int i = tid; i < kBlk / E * D / 2; i += kThreads) {
      const int g = i / (D / 2), d = i % (D / 2) * 2;
      u32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < E; j += El::bytes == 4 ? 1 : 2) {
        const char *s = tiles[1] + v_token<E>(g, j) * kRow + d * El::bytes;  // (tokens j and j + 1 are neighbours)
        if constexpr (El::bytes == 4) {
          const uint2 a = *reinterpret_cast<const uint2 *>(s);
          x[j] = a.x;
          y[j] = a.y;
        } else if constexpr (El::bytes == 2) {
          const uint32_t a = *reinterpret_cast<const uint32_t *>(s), b = *reinterpret_cast<const uint32_t *>(s + kRow);
          x[j / 2] = low16(a, b);
          y[j / 2] = high16(a, b);
        } else {
          const uint32_t a = *reinterpret_cast<const uint16_t *>(s), b = *reinterpret_cast<const uint16_t *>(s + kRow);
          x[j / 4] |= ((a & 0xffu) | (b & 0xffu) << 8) << (8 * (j & 3));
          y[j / 4] |= (a >> 8 | (b & 0xff00u)) << (8 * (j & 3));
        }
      }
      u32x4 *o = reinterpret_cast<u32x4 *>(vals) + g * D + d;
      o[0] = x;
      o[1] = y;
    }
    return;
  }
  // (a part of a block: the pieces' other tokens keep their elements)
  for (int i = tid; i < (bl.hi - bl.lo) * D; i += kThreads) {
    const int rr = bl.lo + i / D, d = i % D;
    const char *s = tiles[1] + rr * kRow + d * El::bytes;
    char *o = vals + (v_group<E>(rr) * D + d) * 16 + v_elem<E>(rr) * El::bytes;
    if constexpr (El::bytes == 4)
      *reinterpret_cast<uint32_t *>(o) = *reinterpret_cast<const uint32_t *>(s);
    else if constexpr (El::bytes == 2)
      *reinterpret_cast<uint16_t *>(o) = *reinterpret_cast<const uint16_t *>(s);
    else
      *o = *s;
  }
}

// grid: (kv head, block of the chunk), sequence
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(CacheView c, ChunkView k, RowsView kr, RowsView vr) {
  append_block<DT, D, false, false>(c, k, kr, vr, RotaryView{}, nullptr);
}

// The same blocks, keys rotated, and after them (blockIdx.x from kv * blocks on) the chunk's queries, a wave for a
// part of a row.  One pass over queries, keys and values where rotation and append would take two over the keys, and
// one launch: four prompts of 4,915 to 8,192 tokens (32 heads, 8 kv heads of 128 in bf16) 141 us, 4.6 TB/s; 32 tokens 5 us.
// Graph-captured, fp32 / bf16 / 8-bit pages: 32 tokens 5.7 / 5.6 / 6.0 us, 32 trees of 17 rows 10.1 / 8.5 / 9.1, the prompts
// 249 / 129 / 122 (5.2 / 5.0 / 4.8 TB/s).  Trees are bound by the chain of a block, not by memory: in bf16 7.5 us with one head (the
// keys' blocks, each of which computes its angles for its own kv head), 6.7 with one kv head, 5.7 with one of each.
template <int DT, int D, bool kNear>
__global__ __launch_bounds__(kThreads) void append_rotated_kernel(CacheView c, ChunkView k, RotaryView rot, HeadsView q,
                                                                  RotatePlan plan, RowsView kr, const void *k_weight,
                                                                  RowsView vr, int blocks) {
  const int group = (int)blockIdx.x - c.kv * blocks;
  if (group < 0) {
    append_block<DT, D, true, kNear>(c, k, kr, vr, rot, k_weight);
    return;
  }
  using T = typename Elem<DT>::data;
  __shared__ float2 cs[kRotWaves][D / 2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = group * kRotWaves + wave;
  const Seq s = seq_of(k, c.page_shift, blockIdx.y);
  const int row = at / plan.splits, first = at % plan.splits * plan.per;
  if (row >= s.n) return;
  const int last = min(first + plan.per, plan.passes);
  const HeadsView none{};
  if (q.in.vec && q.out.vec)
    rotate_row<T, true, kNear>(rot, q, none, D, plan.lanes, s.row0 + row, first, last, cs[wave]);
  else
    rotate_row<T, false, kNear>(rot, q, none, D, plan.lanes, s.row0 + row, first, last, cs[wave]);
}

// grid as append_kernel's; the tiles hold the data type
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheView c, ChunkView k, RowsView kr, RowsView vr) {
  using El = Elem<DT>;
  using T = typename El::data;
  constexpr int E = El::E, kRow = D * (int)sizeof(T) + kPad, kPieces = kBlk * D / E;
  __shared__ __align__(16) char tiles[2][kBlk * kRow];
  const int head = blockIdx.x % c.kv;
  Block bl;
  if (!block_of(c, k, blockIdx.y, blockIdx.x / c.kv, &bl)) return;
  const int tid = threadIdx.x;
  const bool there = bl.page >= 0;  // (else zeros)
  const char *page = c.base + (there ? bl.page : 0) * c.page_bytes + head * c.head_bytes;
  const char *keys = page + (int64_t)bl.in_page * D * El::bytes, *vals = keys + c.v_off;
  const uint8_t *ke = reinterpret_cast<const uint8_t *>(page + c.s_off) + bl.in_page, *ve = ke + (1 << c.page_shift);
  // all loads first
  constexpr int kK = (kPieces + kThreads - 1) / kThreads, kV = (kPieces / 2 + kThreads - 1) / kThreads;
  u32x4 kv[kK], vv[kV][2];
#pragma unroll
  for (int n = 0; n < kK; ++n) {
    kv[n] = u32x4{0, 0, 0, 0};
    if (there && (kPieces % kThreads == 0 || tid + n * kThreads < kPieces))
      kv[n] = reinterpret_cast<const u32x4 *>(keys)[tid + n * kThreads];
  }
#pragma unroll
  for (int n = 0; n < kV; ++n) {
    vv[n][0] = vv[n][1] = u32x4{0, 0, 0, 0};
    if (there && (kPieces / 2 % kThreads == 0 || tid + n * kThreads < kPieces / 2)) {
      vv[n][0] = reinterpret_cast<const u32x4 *>(vals)[2 * (tid + n * kThreads)];
      vv[n][1] = reinterpret_cast<const u32x4 *>(vals)[2 * (tid + n * kThreads) + 1];
    }
  }
#pragma unroll
  for (int n = 0; n < kK; ++n) {
    const int i = tid + n * kThreads, rr = i % kBlk, d = i / kBlk * E;
    if (kPieces % kThreads && i >= kPieces) break;
    char *o = tiles[0] + rr * kRow + d * (int)sizeof(T);
    if constexpr (DT == DT_F8) {
      const float s = there ? exp_of(ke[rr]) : 0.0f;
      u32x4 z[2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(kv[n][u], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(kv[n][u], true);
        z[u >> 1][2 * (u & 1)] = pack_bf16(a[0] * s, a[1] * s);
        z[u >> 1][2 * (u & 1) + 1] = pack_bf16(b[0] * s, b[1] * s);
      }
      reinterpret_cast<u32x4 *>(o)[0] = z[0];
      reinterpret_cast<u32x4 *>(o)[1] = z[1];
    } else {
      *reinterpret_cast<u32x4 *>(o) = kv[n];
    }
  }
#pragma unroll
  for (int n = 0; n < kV; ++n) {
    // pieces (g, d) and (g, d + 1) into the rows of g's tokens
    const int i = tid + n * kThreads, g = i / (D / 2), d = i % (D / 2) * 2;
    if (kPieces / 2 % kThreads && i >= kPieces / 2) break;
#pragma unroll
    for (int j = 0; j < E; j += El::bytes == 4 ? 1 : 2) {
      const int t = v_token<E>(g, j);  // (tokens j and j + 1 are neighbours)
      char *o = tiles[1] + t * kRow + d * (int)sizeof(T);
      if constexpr (DT == DT_F32) {
        *reinterpret_cast<uint2 *>(o) = make_uint2(vv[n][0][j], vv[n][1][j]);
      } else if constexpr (DT == DT_BF16) {
        *reinterpret_cast<uint32_t *>(o) = low16(vv[n][0][j / 2], vv[n][1][j / 2]);
        *reinterpret_cast<uint32_t *>(o + kRow) = high16(vv[n][0][j / 2], vv[n][1][j / 2]);
      } else {
        const bool hi = j & 2;
        const f32x2 a = hi ? __builtin_amdgcn_cvt_pk_f32_fp8(vv[n][0][j / 4], true)
                           : __builtin_amdgcn_cvt_pk_f32_fp8(vv[n][0][j / 4], false),
                    b = hi ? __builtin_amdgcn_cvt_pk_f32_fp8(vv[n][1][j / 4], true)
                           : __builtin_amdgcn_cvt_pk_f32_fp8(vv[n][1][j / 4], false);
        const uint32_t e2 = there ? *reinterpret_cast<const uint16_t *>(ve + t) : 0u;  // (t is even)
        const float s0 = exp_of(e2 & 0xffu), s1 = exp_of(e2 >> 8);
        *reinterpret_cast<uint32_t *>(o) = pack_bf16(a[0] * s0, b[0] * s0);
        *reinterpret_cast<uint32_t *>(o + kRow) = pack_bf16(a[1] * s1, b[1] * s1);
      }
    }
  }
  __syncthreads();
  const int r = tid >> 3, sub = tid & 7;
  if (r < bl.lo || r >= bl.hi) return;
  constexpr int n = 16 / (int)sizeof(T);  // elements of a 16-byte store
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const RowsView &dst = v ? vr : kr;
    T *p = reinterpret_cast<T *>(dst.p) + (int64_t)(bl.q.row0 + bl.pos0 + r - bl.q.base) * dst.row +
           (int64_t)head * dst.head;
#pragma unroll
    for (int i = sub; i < D / n; i += 8) {
      const u32x4 x = *reinterpret_cast<const u32x4 *>(tiles[v] + r * kRow + i * 16);
      if (dst.vec) {
        *reinterpret_cast<u32x4 *>(p + n * i) = x;
      } else {
#pragma unroll
        for (int j = 0; j < n; ++j) {
          if constexpr (sizeof(T) == 4)
            p[n * i + j] = __uint_as_float(x[j]);
          else
            p[n * i + j] = (uint16_t)(x[j >> 1] >> (16 * (j & 1)));
        }
      }
    }
  }
}

// Bound by latency (2.3 us at one tree of 64 nodes, 3.8 at 32 trees of 16).  One wave per tree: at every
// step the lanes look for the child among their nodes (four each at most); the lowest index counts.
__global__ __launch_bounds__(64) void accept_kernel(const int32_t *tokens, const int32_t *parents,
                                                    const int32_t *n_nodes, int B, const int32_t *target,
                                                    int32_t *path, int32_t *n_accepted, int32_t *next_token) {
  const int b = blockIdx.x, lane = threadIdx.x;
  __shared__ int32_t tgt[kMaxB + 1];
  const int n = min(max(n_nodes[b], 0), B);
  for (int i = lane; i <= B; i += 64) tgt[i] = target[(int64_t)b * (B + 1) + i];
  int tok[kMaxB / 64], par[kMaxB / 64];
#pragma unroll
  for (int i = 0; i < kMaxB / 64; ++i) {
    const int m = lane + 64 * i;
    tok[i] = m < n ? tokens[(int64_t)b * B + m] : 0;
    par[i] = m < n ? parents[(int64_t)b * B + m] : -2;  // (no node's index)
  }
  __syncthreads();
  int cur = -1, count = 0;
  while (count < B) {  // (a node's index is above its parent's: at most B steps)
    const int want = tgt[cur + 1];
    int found = -1;
#pragma unroll
    for (int i = 0; i < kMaxB / 64; ++i) {
      const uint64_t hit = __ballot(par[i] == cur && tok[i] == want && lane + 64 * i > cur);
      if (found < 0 && hit) found = 64 * i + __builtin_ctzll(hit);
    }
    if (found < 0) break;
    if (lane == 0) path[(int64_t)b * B + count] = found;
    cur = found;
    ++count;
  }
  for (int i = count + lane; i < B; i += 64) path[(int64_t)b * B + i] = -1;
  if (lane == 0) {
    n_accepted[b] = count;
    next_token[b] = tgt[cur + 1];
  }
}

// Workgroup: one kv head of one layer of one sequence.  A thread owns places of a head page's
// rows (a 16-byte piece of the keys, an element of the values, an exponent) and moves
// them for one accepted node after the other, so no two threads share an address and
// none has to wait for another: within a group of kMove rows all loads come before the
// stores, and a row is read (path[i] >= i) before or when it is written.  Bound by latency: the
// paths of 32 trees of 16 in two layers of 8 kv heads of 128 in bf16 take 5.8 us, of one tree of 64 in fp32 4.3.
constexpr int kMove = 8;
template <int DT>
__global__ __launch_bounds__(kThreads) void commit_kernel(CacheView c, int64_t layer_bytes, ChunkView k, int nodes,
                                                          const int32_t *path, const int32_t *n_accepted) {
  using El = Elem<DT>;
  constexpr int E = El::E;
  const int head = blockIdx.x % c.kv, layer = blockIdx.x / c.kv, b = blockIdx.y, tid = threadIdx.x;
  __shared__ int64_t from[kMaxB], to[kMaxB];  // page offsets of the rows that move, -1: none
  __shared__ int from_r[kMaxB], to_r[kMaxB];  // their tokens in the page
  const Seq q = seq_of(k, c.page_shift, b);
  const int n = min(max(n_accepted[b], 0), nodes), first = q.base + q.n - nodes, room = k.width << c.page_shift;
  for (int i = tid; i < n; i += kThreads) {
    const int p = path[(int64_t)b * nodes + i], s = first + p, t = first + i;
    int64_t fo = -1, tp = -1;
    if (p > i && p < nodes && t >= 0 && s < room) {
      const int sp = k.table[(int64_t)b * k.width + (s >> c.page_shift)];
      const int dp = k.table[(int64_t)b * k.width + (t >> c.page_shift)];
      if (sp >= 0 && sp < c.pages && dp >= 0 && dp < c.pages) {
        fo = sp * c.page_bytes;
        tp = dp * c.page_bytes;
      }
    }
    from[i] = fo;
    to[i] = tp;
    from_r[i] = s & ((1 << c.page_shift) - 1);
    to_r[i] = t & ((1 << c.page_shift) - 1);
  }
  __syncthreads();
  char *base = c.base + layer * layer_bytes + head * c.head_bytes;
  const int D = c.D, kp = D / E, places = kp + D + (DT == DT_F8 ? 2 : 0);
  for (int pl = tid; pl < places; pl += kThreads) {
    // a place's address in a head page for token r
    auto key_at = [&](int r) { return (int64_t)(r & ~(kBlk - 1)) * D * El::bytes + (pl * kBlk + (r & (kBlk - 1))) * 16; };
    auto val_at = [&](int r) {
      const int t = r & (kBlk - 1);
      return c.v_off + (int64_t)(r & ~(kBlk - 1)) * D * El::bytes + (v_group<E>(t) * D + pl - kp) * 16 +
             v_elem<E>(t) * El::bytes;
    };
    auto exp_at = [&](int r) { return c.s_off + (pl - kp - D) * (1 << c.page_shift) + r; };
    for (int i0 = 0; i0 < n; i0 += kMove) {
      u32x4 v[kMove];
#pragma unroll
      for (int j = 0; j < kMove; ++j) {
        const int i = i0 + j;
        if (i >= n || from[i] < 0) continue;
        const char *s = base + from[i];
        if (pl < kp)
          v[j] = *reinterpret_cast<const u32x4 *>(s + key_at(from_r[i]));
        else if (pl < kp + D) {
          s += val_at(from_r[i]);
          v[j][0] = El::bytes == 4   ? *reinterpret_cast<const uint32_t *>(s)
                    : El::bytes == 2 ? *reinterpret_cast<const uint16_t *>(s)
                                     : *reinterpret_cast<const uint8_t *>(s);
        } else
          v[j][0] = *reinterpret_cast<const uint8_t *>(s + exp_at(from_r[i]));
      }
#pragma unroll
      for (int j = 0; j < kMove; ++j) {
        const int i = i0 + j;
        if (i >= n || from[i] < 0) continue;
        char *d = base + to[i];
        if (pl < kp)
          *reinterpret_cast<u32x4 *>(d + key_at(to_r[i])) = v[j];
        else if (pl < kp + D) {
          d += val_at(to_r[i]);
          if (El::bytes == 4)
            *reinterpret_cast<uint32_t *>(d) = v[j][0];
          else if (El::bytes == 2)
            *reinterpret_cast<uint16_t *>(d) = (uint16_t)v[j][0];
          else
            *d = (char)v[j][0];
        } else
          d[exp_at(to_r[i])] = (char)v[j][0];
      }
    }
  }
}

// blocks of 32 tokens that a chunk of max_chunk tokens touches at most
int chunk_blocks(const ChunkView &k) { return (k.max_chunk + 2 * kBlk - 2) / kBlk; }

}  // namespace

template <int DT>
static hipError_t launch_store(bool read, const CacheView &c, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                               hipStream_t s) {
  const dim3 grid(c.kv * chunk_blocks(k), k.batch);
  auto f = c.D == 64    ? read ? read_kernel<DT, 64> : append_kernel<DT, 64>
           : c.D == 96  ? read ? read_kernel<DT, 96> : append_kernel<DT, 96>
           : c.D == 128 ? read ? read_kernel<DT, 128> : append_kernel<DT, 128>
                        : read ? read_kernel<DT, 256> : append_kernel<DT, 256>;
  f<<<grid, kThreads, 0, s>>>(c, k, kr, vr);
  return hipGetLastError();
}

hipError_t launch_append(const CacheView &c, int dtype, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                         hipStream_t s) {
  return dtype == DT_F32    ? launch_store<DT_F32>(false, c, k, kr, vr, s)
         : dtype == DT_BF16 ? launch_store<DT_BF16>(false, c, k, kr, vr, s)
                            : launch_store<DT_F8>(false, c, k, kr, vr, s);
}

hipError_t launch_read(const CacheView &c, int dtype, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                       hipStream_t s) {
  return dtype == DT_F32    ? launch_store<DT_F32>(true, c, k, kr, vr, s)
         : dtype == DT_BF16 ? launch_store<DT_BF16>(true, c, k, kr, vr, s)
                            : launch_store<DT_F8>(true, c, k, kr, vr, s);
}

hipError_t launch_append_rotated(const CacheView &c, int dtype, const ChunkView &k, const RotaryView &r,
                                 const HeadsView &q, const RowsView &kr, const void *k_weight, const RowsView &vr,
                                 hipStream_t s) {
  const int blocks = chunk_blocks(k);
  const RotatePlan plan = rotate_plan((int64_t)k.batch * k.max_chunk, q.heads, 0, c.D);
  const int64_t groups = ((int64_t)k.max_chunk * plan.splits + kRotWaves - 1) / kRotWaves;
  const dim3 grid((unsigned)(c.kv * blocks + groups), k.batch);
  auto pick = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    auto f = c.D == 64    ? r.interleaved ? append_rotated_kernel<DT, 64, true> : append_rotated_kernel<DT, 64, false>
             : c.D == 96  ? r.interleaved ? append_rotated_kernel<DT, 96, true> : append_rotated_kernel<DT, 96, false>
             : c.D == 128 ? r.interleaved ? append_rotated_kernel<DT, 128, true> : append_rotated_kernel<DT, 128, false>
             : r.interleaved ? append_rotated_kernel<DT, 256, true> : append_rotated_kernel<DT, 256, false>;
    f<<<grid, kThreads, 0, s>>>(c, k, r, q, plan, kr, k_weight, vr, blocks);
  };
  if (dtype == DT_F32)
    pick(std::integral_constant<int, DT_F32>());
  else if (dtype == DT_BF16)
    pick(std::integral_constant<int, DT_BF16>());
  else
    pick(std::integral_constant<int, DT_F8>());
  return hipGetLastError();
}

hipError_t launch_accept(const dt_tree &t, int batch, int B, const int32_t *target, int32_t *path, int32_t *n,
                         int32_t *next, hipStream_t s) {
  accept_kernel<<<batch, 64, 0, s>>>(t.tokens, t.parents, t.n_nodes, B, target, path, n, next);
  return hipGetLastError();
}

hipError_t launch_commit(const CacheView &c, int dtype, int layers, const ChunkView &k, int nodes,
                         const int32_t *path, const int32_t *n, hipStream_t s) {
  const dim3 grid(c.kv * layers, k.batch);
  auto f = dtype == DT_F32 ? commit_kernel<DT_F32> : dtype == DT_BF16 ? commit_kernel<DT_BF16> : commit_kernel<DT_F8>;
  f<<<grid, kThreads, 0, s>>>(c, c.page_bytes * c.pages, k, nodes, path, n);
  return hipGetLastError();
}

}  // namespace dt
