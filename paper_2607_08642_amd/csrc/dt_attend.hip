// Attention over the paged cache for few rows (single tokens, small trees; fp32 of any
// size), the join of split calls, and the choice of kernel and split.
//
// stream_kernel: a workgroup of four waves holds 32 rows of one kv head; each wave
// walks key blocks of its own (every fourth) with its own running softmax, the
// blocks' pieces going from memory into the registers of the matrix operands.
// Nothing passes through LDS and no wave waits for another until the four partial
// results meet at the end.  Bound by memory: a block of 32 tokens (16 KB at bf16, D =
// 128) takes about a thousand cycles of a wave, a CU's eight waves then ask for four
// times the bytes that it can get.
#include "dt_attend.h"

namespace dt {
namespace {
using namespace att;

constexpr int kStreamWaves = 4, kStreamRows = 32;

// One block's keys and values in a wave's registers.
template <int DT, int D>
struct BlockRegs {
  static constexpr int N = D * (DT == DT_F32 ? 4 : DT == DT_BF16 ? 2 : 1) / 32;  // 16-byte pieces of a lane
  u32x4 k[N], v[N];
  uint32_t ke, ve[4];  // DT_F8: the key's exponent; of the values, tokens 8 t + 4 h + 0..3 in ve[t]
};

template <int DT, int D>
struct Stream {
  static constexpr int N = BlockRegs<DT, D>::N, ES = DT == DT_F32 ? 4 : DT == DT_BF16 ? 2 : 1;
  // (fp32 at D = 256: keys and values would not fit beside the sums)
  static constexpr bool kAhead = N * 8 <= 128;
};

template <int DT, int D>
__device__ inline void load_k(BlockRegs<DT, D> &r, const char *kb, const char *ex, int lane) {
#pragma unroll
  for (int n = 0; n < BlockRegs<DT, D>::N; ++n) r.k[n] = *reinterpret_cast<const u32x4 *>(kb + lane * 16 + n * 1024);
  if (DT == DT_F8) r.ke = reinterpret_cast<const uint8_t *>(ex)[lane & 31];
}
// piece of values n: the n-th run of 32 d of the lane's tokens
template <int DT, int D>
__device__ inline int v_piece(int n, int h, int l32) {
  constexpr int T = D / 32;
  const int x = n / T, d = 32 * (n % T) + l32;  // bf16: step x; 8 bits: x = 0; fp32: tokens 8 x + 4 h ..
  return ((DT == DT_F8 ? h : 2 * x + h) * D + d) * 16;
}
template <int DT, int D>
__device__ inline void load_v(BlockRegs<DT, D> &r, const char *vb, const char *ex, int h, int l32) {
#pragma unroll
  for (int n = 0; n < BlockRegs<DT, D>::N; ++n)
    r.v[n] = *reinterpret_cast<const u32x4 *>(vb + v_piece<DT, D>(n, h, l32));
  if (DT == DT_F8)
#pragma unroll
    for (int t = 0; t < 4; ++t) r.ve[t] = *reinterpret_cast<const uint32_t *>(ex + 8 * t + 4 * h);
}

// eight 8-bit elements (words a, b) times a power of two
__device__ inline bf16x8 widen8(uint32_t a, uint32_t b, float scale) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false),
               y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
               z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false),
               w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

template <int DT, int D>
__device__ inline f32x16 scores(const BlockRegs<DT, D> &r, const QRegs<DT, D> &q) {
  f32x16 s = zero16();
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = mfma(__uint_as_float(r.k[n][j]), __uint_as_float(q.v[n][j]), s);
  } else if constexpr (DT == DT_BF16) {
#pragma unroll
    for (int n = 0; n < D / 16; ++n) s = mfma(as_bf16x8(r.k[n]), as_bf16x8(q.v[n]), s);
  } else {
    const float e = exp_of(r.ke);
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int u = 0; u < 2; ++u)
        s = mfma(widen8(r.k[n][2 * u], r.k[n][2 * u + 1], e), as_bf16x8(q.v[2 * n + u]), s);
  }
  return s;
}

// O^T += V^T P^T; with MASKED, non-finite values of tokens that a row does not see stay out
template <int DT, int D, bool MASKED>
__device__ inline void add_values(const BlockRegs<DT, D> &r, float (&p)[16], uint32_t seen, f32x16 (&o)[D / 32]) {
  constexpr int T = D / 32;
  if constexpr (DT == DT_F32) {
    bool bad = false;
    if (MASKED)
#pragma unroll
      for (int n = 0; n < 4 * T; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= (r.v[n][j] & 0x7f800000u) == 0x7f800000u;
    if (MASKED && __ballot(bad)) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        f32x16 hit = zero16();
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t v = r.v[x * T + t][j];
            const bool b = (v & 0x7f800000u) == 0x7f800000u;
            o[t] = mfma(__uint_as_float(b ? 0u : v), p[4 * x + j], o[t]);
            hit = mfma(b ? 1.0f : 0.0f, seen >> reg_token(4 * x + j) & 1 ? 1.0f : 0.0f, hit);
          }
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = hit[i] > 0.0f ? __builtin_nanf("") : o[t][i];
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int t = 0; t < T; ++t) o[t] = mfma(__uint_as_float(r.v[x * T + t][j]), p[4 * x + j], o[t]);
  } else {
    if constexpr (DT == DT_F8) {
      // the tokens' exponents go to the probabilities (a product with a power of two: exact)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __uint_as_float((i % 4 == 3 ? r.ve[i / 4] >> 1 : r.ve[i / 4] << (23 - 8 * (i % 4))) & 0x7f800000u);
        p[i] = MASKED ? (seen >> reg_token(i) & 1 ? p[i] * e : 0.0f) : p[i] * e;
      }
    }
    bf16x8 pf[2] = {pack_p(p, 0), pack_p(p, 1)};
    auto frag = [&](int s, int t) {
      if constexpr (DT == DT_F8)
        return widen8(r.v[t][2 * s], r.v[t][2 * s + 1], 1.0f);
      else
        return as_bf16x8(r.v[s * T + t]);
    };
    auto raw = [&](int s, int t) {
      const bf16x8 f = frag(s, t);
      u32x4 u;
      __builtin_memcpy(&u, &f, 16);
      return u;
    };
    if (MASKED) {
      bool bad = false;
#pragma unroll
      for (int n = 0; n < 2 * T; ++n) bad |= has_bad(raw(n / T, n % T));
      if (__ballot(bad)) {
        const bf16x8 sf[2] = {pack_seen(seen, 0), pack_seen(seen, 1)};
#pragma unroll
        for (int t = 0; t < T; ++t) {
          f32x16 hit = zero16();
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            u32x4 clean, b;
            split_bad(raw(s, t), clean, b);
            o[t] = mfma(as_bf16x8(clean), pf[s], o[t]);
            hit = mfma(as_bf16x8(b), sf[s], hit);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][i] = hit[i] > 0.0f ? __builtin_nanf("") : o[t][i];
        }
        return;
      }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int t = 0; t < T; ++t) o[t] = mfma(frag(s, t), pf[s], o[t]);
  }
}

// grid: kv head (fastest: the workgroups of a head share an XCD's cache where there are
// eight heads), tile, split; sequence
template <int DT, int D>
__global__ __launch_bounds__(64 * kStreamWaves, DT != DT_F32 && D <= 128 ? 2 : 1) void stream_kernel(AttendArgs a,
                                                                                                      int tiles) {
  using St = Stream<DT, D>;
  constexpr int T = D / 32, ES = St::ES;
  __shared__ uint32_t words[kStreamRows * kTreeWords];
  __shared__ float ml[kStreamWaves][2][32];
  __shared__ float meet[2][D][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int head = blockIdx.x % a.cache.kv, tile = blockIdx.x / a.cache.kv % tiles,
            split = blockIdx.x / (a.cache.kv * tiles), b = blockIdx.y;
  Tile t;
  if (!tile_of(a, b, tile * kStreamRows, kStreamRows, &t)) return;
  const int active = active_splits(a, t);
  if (split >= active) return;
  const int it0 = split * a.split_blocks, it1 = split == active - 1 ? t.n_iter : it0 + a.split_blocks;
  if (a.nodes > 0) {
    tree_words(a, t, b, words, 64 * kStreamWaves);
    __syncthreads();
  }
  const Row w = row_of(a, t, b, t.r0 + l32, words);
  const float c = __builtin_fabsf(a.scale_log2e);
  QRegs<DT, D> q;
  load_q<DT, D>(a, t, w, head, h, DT == DT_F8, q);
  f32x16 o[T];
#pragma unroll
  for (int n = 0; n < T; ++n) o[n] = zero16();
  float m = kFloor, l = 0.0f;

  const int32_t *table = a.chunk.table + (int64_t)b * a.chunk.width;
  const int shift = a.cache.page_shift;
  auto page_of = [&](int it) { return it < it1 ? table[t.block(it) * kBlk >> shift] : 0; };
  // the head page of a block (an out-of-range page: page 0, whose tokens then count as unseen)
  auto page_at = [&](int page) {
    const int p = __builtin_amdgcn_readfirstlane(page);
    return a.cache.base + (int64_t)((uint32_t)p < (uint32_t)a.cache.pages ? p : 0) * a.cache.page_bytes +
           head * a.cache.head_bytes;
  };
  auto in_page = [&](int it) { return t.block(it) * kBlk & ((1 << shift) - 1); };
  BlockRegs<DT, D> r;
  auto fetch_k = [&](int it, int page) {
    const char *hp = page_at(page);
    const int n = in_page(it);
    load_k<DT, D>(r, hp + (int64_t)n * D * ES, hp + a.cache.s_off + n, lane);
  };
  auto fetch_v = [&](int it, int page) {
    const char *hp = page_at(page);
    const int n = in_page(it);
    load_v<DT, D>(r, hp + a.cache.v_off + (int64_t)n * D * ES, hp + a.cache.s_off + (1 << shift) + n, h, l32);
  };
  int it = it0 + wave;
  int page = page_of(it), next = page_of(it + kStreamWaves);
  if (St::kAhead && it < it1) {
    fetch_k(it, page);
    fetch_v(it, page);
  }
  for (; it < it1; it += kStreamWaves) {
    const int after = page_of(it + 2 * kStreamWaves), k0 = t.block(it) * kBlk;
    const bool more = it + kStreamWaves < it1, skip = sees_none(a, w, k0);
    const bool all = sees_all(a, w, k0) && (uint32_t)page < (uint32_t)a.cache.pages;
    if (!St::kAhead && !skip) {
      fetch_k(it, page);
      fetch_v(it, page);
    }
    f32x16 s;
    if (!skip) s = scores<DT, D>(r, q);
    if (St::kAhead && more) fetch_k(it + kStreamWaves, next);
    if (!skip) {
      float p[16];
      uint32_t seen = 0;
      float f;
      if (all) {
        f = softmax_block<false>(s, 0, c, m, l, p);
      } else {
        seen = (uint32_t)page < (uint32_t)a.cache.pages ? seen_word(a, t, w, k0) >> (4 * h) : 0;
        f = softmax_block<true>(s, seen, c, m, l, p);
      }
      if (__ballot(f != 1.0f))
#pragma unroll
        for (int n = 0; n < T; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[n][i] *= f;
      if (all)
        add_values<DT, D, false>(r, p, 0, o);
      else
        add_values<DT, D, true>(r, p, seen, o);
    }
    if (St::kAhead && more) fetch_v(it + kStreamWaves, next);
    page = next;
    next = after;
  }

  // the four waves' results meet: each scaled to the common maximum, then 2 + 2 and 1 + 1
  const float2 lh = halves(l);
  l = lh.x + lh.y;
  if (h == 0) {
    ml[wave][0][l32] = m;
    ml[wave][1][l32] = l;
  }
  __syncthreads();
  const float top = max2(max2(ml[0][0][l32], ml[1][0][l32]), max2(ml[2][0][l32], ml[3][0][l32]));
  l = 0.0f;
#pragma unroll
  for (int x = 0; x < kStreamWaves; ++x) l += ml[x][1][l32] * __builtin_amdgcn_exp2f(ml[x][0][l32] - top);
  const float f = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int n = 0; n < T; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] *= f;
  auto put = [&](int slot) {
#pragma unroll
    for (int n = 0; n < T; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) meet[slot][32 * n + reg_token(i) + 4 * h][l32] = o[n][i];
  };
  auto add = [&](int slot) {
#pragma unroll
    for (int n = 0; n < T; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][i] += meet[slot][32 * n + reg_token(i) + 4 * h][l32];
  };
  if (wave >= 2) put(wave - 2);
  __syncthreads();
  if (wave < 2) add(wave);
  if (wave == 1) put(1);  // (slot 1 is its own)
  __syncthreads();
  if (wave > 0) return;
  add(1);
  write_rows<DT, D>(a, t, w, head, split, active == 1, t.r0 + l32 < t.rows, h, o, top, l);
}

// One wave per (query, head): the splits' parts scaled to their common maximum and summed
// in order.  Rows of a tile with one split were written by it.
template <int DT>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a, int tile_rows) {
  const int lane = threadIdx.x & 63, D = a.cache.D, b = blockIdx.y;
  const int x = blockIdx.x * 4 + (threadIdx.x >> 6);  // query * heads + head
  const int i = x / a.heads, hq = x - i * a.heads;
  const int r = i * a.group + hq % a.group;
  Tile t;
  if (!tile_of(a, b, r / tile_rows * tile_rows, tile_rows, &t) || r >= t.rows) return;
  const int active = active_splits(a, t);
  if (active == 1) return;
  const int64_t row = t.q.row0 + i, at = (row * a.heads + hq) * a.splits;
  const float2 p = lane < active ? a.part_ml[at + lane] : make_float2(kFloor, 0.0f);
  float top = p.x;
  for (int o = 1; o < 64; o <<= 1) top = max2(top, __shfl_xor(top, o));
  const float f = __builtin_amdgcn_exp2f(p.x - top);
  float l = p.y * f;
  for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const float *part = a.part + at * D;
  for (int d = lane; d < D; d += 64) {
    float y = 0.0f;
#pragma unroll 8
    for (int s = 0; s < active; ++s) y += part[(int64_t)s * D + d] * __shfl(f, s);
    y *= inv;
    const int64_t o = row * a.out.row + (int64_t)hq * a.out.head + d;
    if (DT == DT_F32)
      reinterpret_cast<float *>(a.out.p)[o] = y;
    else
      reinterpret_cast<__bf16 *>(a.out.p)[o] = (__bf16)y;
  }
}

template <int DT>
hipError_t launch_stream(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  const dim3 grid(a.cache.kv * p.tiles * p.splits, a.chunk.batch);
  auto f = a.cache.D == 64    ? stream_kernel<DT, 64>
           : a.cache.D == 96  ? stream_kernel<DT, 96>
           : a.cache.D == 128 ? stream_kernel<DT, 128>
                              : stream_kernel<DT, 256>;
  f<<<grid, 64 * kStreamWaves, 0, s>>>(a, p.tiles);
  return hipGetLastError();
}

}  // namespace

AttendPlan attend_plan(const CacheView &c, const ChunkView &k, int dtype, int heads, int window, int sinks, int nodes) {
  const int group = heads / c.kv, rows = k.max_chunk * group;
  AttendPlan p;
  p.tile_rows = kStreamRows;
  p.tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  // blocks of a tile at most
  const int all = (k.max_len + kBlk - 1) / kBlk;
  int most = all;
  if (window > 0) {
    const int span = window + (p.tile_rows + group - 1) / group + 1 + nodes;
    const int64_t near = (span + kBlk - 1) / kBlk + 1 + (sinks + kBlk - 1) / kBlk;
    most = near < all ? (int)near : all;
  }
  // enough workgroups for two rounds of the chip (512 slots), a split no shorter than two
  // blocks a wave
  const int64_t wgs = (int64_t)c.kv * p.tiles * k.batch;
  int64_t want = (1024 + wgs - 1) / wgs;
  if (want > kMaxSplits) want = kMaxSplits;
  int blocks = (int)((most + want - 1) / want);
  if (blocks < 2 * kStreamWaves) blocks = 2 * kStreamWaves;
  p.splits = (most + blocks - 1) / blocks;
  p.blocks = blocks;
  return p;
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  hipError_t e = a.dtype == DT_F32    ? launch_stream<DT_F32>(a, p, s)
                 : a.dtype == DT_BF16 ? launch_stream<DT_BF16>(a, p, s)
                                      : launch_stream<DT_F8>(a, p, s);
  if (e != hipSuccess || p.splits == 1) return e;
  const dim3 grid(((int64_t)a.chunk.max_chunk * a.heads + 3) / 4, a.chunk.batch);
  (a.dtype == DT_F32 ? join_kernel<DT_F32> : join_kernel<DT_BF16>)<<<grid, 256, 0, s>>>(a, p.tile_rows);
  return hipGetLastError();
}

}  // namespace dt
