// The paged cache: writing rows (quantising them for DT_F8), reading them back, and the
// two kernels that end a verification round (the accepted path, the move of its rows).
//
// All are copies: bound by memory traffic for prompts, by latency for the few
// rows of a decoding step.  A workgroup of append and read takes one block of 32
// tokens of one kv head, keys or values (layout: dt_cache.h), through an LDS tile of
// 32 rows: rows of the caller's tensors are touched in runs of 128 bytes (eight lanes a
// row), pieces of the cache in runs of 512 bytes and more.
#include "dt_cache.h"

namespace dt {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
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

__device__ inline uint32_t pack_bf16(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}

// eight elements of a row of the caller's tensor, as 32-bit words (bf16: two a word)
__device__ inline void load8(const float *p, bool vec, uint32_t (&w)[8]) {
  if (vec) {
    const u32x4 a = reinterpret_cast<const u32x4 *>(p)[0], b = reinterpret_cast<const u32x4 *>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a[i], w[4 + i] = b[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(p[i]);
  }
}
__device__ inline void load8(const uint16_t *p, bool vec, uint32_t (&w)[4]) {
  if (vec) {
    const u32x4 a = reinterpret_cast<const u32x4 *>(p)[0];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = a[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
  }
}

__device__ inline bool finite_bits(uint32_t f32) { return (f32 & 0x7f800000u) != 0x7f800000u; }

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
  const int page = k.table[(int64_t)b * k.width + (o->pos0 >> c.page_shift)];
  o->page = page >= 0 && page < c.pages ? page : -1;
  o->in_page = o->pos0 & ((1 << c.page_shift) - 1);
  return true;
}

// grid: (kv head, keys or values, block of the chunk), sequence
template <int DT>
__global__ __launch_bounds__(kThreads) void append_kernel(CacheView c, ChunkView k, RowsView kr, RowsView vr) {
  using El = Elem<DT>;
  using T = typename El::data;
  constexpr int E = El::E, kWords = sizeof(T) == 4 ? 8 : 4;  // words of eight elements
  extern __shared__ __align__(16) char tile[];
  const int head = blockIdx.x % c.kv, vals = blockIdx.x / c.kv & 1;
  Block bl;
  if (!block_of(c, k, blockIdx.y, blockIdx.x / (2 * c.kv), &bl) || bl.page < 0) return;
  const int D = c.D, stride = D * El::bytes + kPad, tid = threadIdx.x;
  char *page = c.base + bl.page * c.page_bytes + head * c.head_bytes;
  const RowsView &src = vals ? vr : kr;
  const int r = tid >> 3, sub = tid & 7;  // eight lanes a row
  const bool mine = r >= bl.lo && r < bl.hi;
  uint32_t w[4][kWords];
  if (mine) {
    const T *p = reinterpret_cast<const T *>(src.p) + (int64_t)(bl.q.row0 + bl.pos0 + r - bl.q.base) * src.row +
                 (int64_t)head * src.head;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (sub + 8 * i < D / 8) load8(p + 8 * (sub + 8 * i), src.vec, w[i]);
  }
  char *row = tile + r * stride;
  if constexpr (DT == DT_F8) {
    // the row's largest finite magnitude (bf16 bits order like the values), over its eight lanes
    uint32_t top = 0;
    if (mine)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (sub + 8 * i < D / 8)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t a = w[i][j] & 0x7fffu, b = w[i][j] >> 16 & 0x7fffu;
            top = max(top, a < 0x7f80u ? a : 0u);
            top = max(top, b < 0x7f80u ? b : 0u);
          }
    for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    // top = 1.m 2^(x - 127) <= 448 2^e = 1.75 2^(8 + e): e = x - 135, one more where 1.m > 1.75
    const int byte = min(max((int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), 7), 247);  // e + 127
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);                             // 2^-e
    if (mine) {
      if (sub == 0) page[c.s_off + (vals ? (1 << c.page_shift) : 0) + bl.in_page + r] = (char)byte;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (sub + 8 * i < D / 8) {
          uint32_t code[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            uint32_t v = 0, bad = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t x = w[i][2 * u + j], lo = x << 16, hi = x & 0xffff0000u;
              // (the products are exact; the conversion rounds to nearest even)
              const int two = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(lo) * inv, __uint_as_float(hi) * inv,
                                                              0, false);
              v |= (two & 0xffff) << (16 * j);
              bad |= ((finite_bits(lo) ? 0u : 0x7fu) | (finite_bits(hi) ? 0u : 0x7f00u)) << (16 * j);
            }
            code[u] = v | bad;  // (0x7f and 0xff are the codes of NaN)
          }
          *reinterpret_cast<uint2 *>(row + 8 * (sub + 8 * i)) = make_uint2(code[0], code[1]);
        }
    }
  } else if (mine) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (sub + 8 * i < D / 8) {
        u32x4 *d = reinterpret_cast<u32x4 *>(row + 8 * El::bytes * (sub + 8 * i));
#pragma unroll
        for (int j = 0; j < kWords / 4; ++j)
          d[j] = u32x4{w[i][4 * j], w[i][4 * j + 1], w[i][4 * j + 2], w[i][4 * j + 3]};
      }
  }
  __syncthreads();
  if (!vals) {
    char *out = page + (int64_t)bl.in_page * D * El::bytes;
    for (int i = tid; i < kBlk * D / E; i += kThreads) {
      const int rr = i & (kBlk - 1);
      if (rr >= bl.lo && rr < bl.hi)
        reinterpret_cast<u32x4 *>(out)[i] = *reinterpret_cast<const u32x4 *>(tile + rr * stride + (i / kBlk) * 16);
    }
    return;
  }
  char *out = page + c.v_off + (int64_t)bl.in_page * D * El::bytes;
  const bool whole = bl.lo == 0 && bl.hi == kBlk;
  for (int i = tid; i < kBlk / E * D; i += kThreads) {
    const int g = i / D, d = i - g * D;
    if (whole) {
      u32x4 v = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const char *s = tile + v_token<E>(g, j) * stride + d * El::bytes;
        if constexpr (El::bytes == 4)
          v[j] = *reinterpret_cast<const uint32_t *>(s);
        else if constexpr (El::bytes == 2)
          v[j >> 1] |= (uint32_t) * reinterpret_cast<const uint16_t *>(s) << (16 * (j & 1));
        else
          v[j >> 2] |= (uint32_t) * reinterpret_cast<const uint8_t *>(s) << (8 * (j & 3));
      }
      reinterpret_cast<u32x4 *>(out)[i] = v;
    } else {
      // (the piece's other tokens keep their elements)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const int rr = v_token<E>(g, j);
        if (rr < bl.lo || rr >= bl.hi) continue;
        const char *s = tile + rr * stride + d * El::bytes;
        char *o = out + (int64_t)i * 16 + j * El::bytes;
        if constexpr (El::bytes == 4)
          *reinterpret_cast<uint32_t *>(o) = *reinterpret_cast<const uint32_t *>(s);
        else if constexpr (El::bytes == 2)
          *reinterpret_cast<uint16_t *>(o) = *reinterpret_cast<const uint16_t *>(s);
        else
          *o = *s;
      }
    }
  }
}

// grid as append_kernel's; the tile holds the data type
template <int DT>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheView c, ChunkView k, RowsView kr, RowsView vr) {
  using El = Elem<DT>;
  using T = typename El::data;
  constexpr int E = El::E;
  extern __shared__ __align__(16) char tile[];
  const int head = blockIdx.x % c.kv, vals = blockIdx.x / c.kv & 1;
  Block bl;
  if (!block_of(c, k, blockIdx.y, blockIdx.x / (2 * c.kv), &bl)) return;
  const int D = c.D, stride = D * (int)sizeof(T) + kPad, tid = threadIdx.x;
  const char *page = c.base + (bl.page < 0 ? 0 : bl.page) * c.page_bytes + head * c.head_bytes;
  const char *in = page + (vals ? c.v_off : 0) + (int64_t)bl.in_page * D * El::bytes;
  const uint8_t *ex = reinterpret_cast<const uint8_t *>(page + c.s_off) + (vals ? (1 << c.page_shift) : 0) + bl.in_page;
  for (int i = tid; i < kBlk * D / E; i += kThreads) {
    u32x4 v = {0, 0, 0, 0};
    if (bl.page >= 0) v = reinterpret_cast<const u32x4 *>(in)[i];
    const int g = vals ? i / D : i / kBlk, d = vals ? i - g * D : g * E, rr = i & (kBlk - 1);
    if constexpr (DT == DT_F8) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(v[u], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(v[u], true);
        const float f[4] = {a[0], a[1], b[0], b[1]};
        if (vals) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = v_token<E>(g, 4 * u + j);
            const uint32_t two = pack_bf16(bl.page < 0 ? 0.0f : f[j] * exp_of(ex[t]), 0.0f);
            *reinterpret_cast<uint16_t *>(tile + t * stride + d * 2) = (uint16_t)two;
          }
        } else {
          const float s = bl.page < 0 ? 0.0f : exp_of(ex[rr]);
          *reinterpret_cast<uint2 *>(tile + rr * stride + (d + 4 * u) * 2) =
              make_uint2(pack_bf16(f[0] * s, f[1] * s), pack_bf16(f[2] * s, f[3] * s));
        }
      }
    } else if (!vals) {
      *reinterpret_cast<u32x4 *>(tile + rr * stride + d * El::bytes) = v;
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        char *o = tile + v_token<E>(g, j) * stride + d * El::bytes;
        if constexpr (El::bytes == 4)
          *reinterpret_cast<uint32_t *>(o) = v[j];
        else
          *reinterpret_cast<uint16_t *>(o) = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
  __syncthreads();
  const RowsView &dst = vals ? vr : kr;
  const int r = tid >> 3, sub = tid & 7;
  if (r < bl.lo || r >= bl.hi) return;
  T *p = reinterpret_cast<T *>(dst.p) + (int64_t)(bl.q.row0 + bl.pos0 + r - bl.q.base) * dst.row +
         (int64_t)head * dst.head;
  constexpr int n = 16 / (int)sizeof(T);  // elements of a 16-byte store
  for (int i = sub; i < D / n; i += 8) {
    const u32x4 v = *reinterpret_cast<const u32x4 *>(tile + r * stride + i * 16);
    if (dst.vec) {
      *reinterpret_cast<u32x4 *>(p + n * i) = v;
    } else {
#pragma unroll
      for (int j = 0; j < n; ++j) {
        if constexpr (sizeof(T) == 4)
          p[n * i + j] = __uint_as_float(v[j]);
        else
          p[n * i + j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
}

// One wave per tree: at every step the lanes look for the child among their nodes (four
// each at most); the lowest index counts.
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
// stores, and a row is read (path[i] >= i) before or when it is written.
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

hipError_t launch_append(const CacheView &c, int dtype, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                         hipStream_t s) {
  const dim3 grid(c.kv * 2 * chunk_blocks(k), k.batch);
  const size_t lds = (size_t)kBlk * (c.D * elem_bytes(dtype) + kPad);
  auto f = dtype == DT_F32 ? append_kernel<DT_F32> : dtype == DT_BF16 ? append_kernel<DT_BF16> : append_kernel<DT_F8>;
  f<<<grid, kThreads, lds, s>>>(c, k, kr, vr);
  return hipGetLastError();
}

hipError_t launch_read(const CacheView &c, int dtype, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                       hipStream_t s) {
  const dim3 grid(c.kv * 2 * chunk_blocks(k), k.batch);
  const size_t lds = (size_t)kBlk * (c.D * (dtype == DT_F32 ? 4 : 2) + kPad);
  auto f = dtype == DT_F32 ? read_kernel<DT_F32> : dtype == DT_BF16 ? read_kernel<DT_BF16> : read_kernel<DT_F8>;
  f<<<grid, kThreads, lds, s>>>(c, k, kr, vr);
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
