// Attention over the paged cache for few rows (single tokens, small trees; fp32 of any
// size), the join of split calls, and the choice of kernel and split.
//
// A row's result is sum_j p_j v_j / sum_j p_j with p_j = 2^(c s_j - m), s_j = q k_j, c = scale log2 e, in one
// pass over the keys: m is a running reference at or above the maximum of c s, and what was summed under an
// older one is scaled by 2^(old - new).  Two parts (m1, l1, o1), (m2, l2, o2) of the keys join the same way, which
// is what the waves, and the splits of a long sequence, do.
//
// stream_kernel: the waves of a workgroup hold the same 32 rows of one kv head; each walks key
// blocks of its own (every W-th) with its own running softmax and its own ring of LDS slots,
// which it fills by copies from memory that pass no registers: keys of block n + slots are
// asked for when those of block n have been used, and the values after them.  No wave waits
// for another until their partial results meet at the end.
//
// What bounds it: memory, from some thousand tokens a sequence on.  One token of 32 sequences of
// 2,580 to 8,192 (8 kv heads of 128, bf16): 709 MB in 133 us, 5.3 TB/s (a copy of 2 GiB: 4.7, a sum: 4.0); in 8 bits
// 357 MB in 88 us, 4.1 TB/s.  Below that the
// time of a chain: arguments, lengths, page, keys, the meeting of the waves (37 tokens of two heads
// of 64 in fp32: 7.4 us).  In fp32 the products of 32 rows are taken whatever the rows that are there: one
// token of 32 sequences of 4,096, 4 kv heads of 128: 110 us, 4.9 TB/s; 1,024 rows of 32 heads of 128 over 4,096: 539 us, 112
// TFLOP/s of the 153 of a large product (one wave a SIMD: its waits are not filled).
#include <math.h>

#include "dt_attend.h"

namespace dt {
namespace {
using namespace att;

constexpr int kStreamRows = 32;

// Waves that walk a block together, each with its share of the head's elements: two where there are
// 256 (by itself a wave's queries and sums leave too few registers; two kv heads of four, one token,
// single waves and pairs in the same splits: 32 sequences of 4,096 in fp32 384 and 193 us, bf16 66 and 72, 8 bits
// 40 and 38; one of 300 in bf16 19.5 and 14.6; with splits for pairs fp32 119, bf16 56).
constexpr int stream_share(int D) { return D == 256 ? 2 : 1; }
// Blocks that a workgroup works on at a time.
constexpr int stream_blocks(int D) { return D <= 128 ? 4 : 2; }

// Shape of a workgroup: waves, and blocks in a wave's ring, for at most 144 KB of LDS.
template <int DT, int D>
struct Stream {
  static constexpr int P = stream_share(D), DH = D / P, W = stream_blocks(D), kWaves = W * P;
  static constexpr int kPart = kBlk * DH * elem_bytes(DT);          // a wave's keys of a block, or values
  static constexpr int kExps = DT == DT_F8 ? 256 : 0;               // its exponents, as copied
  static constexpr int kFit = 147456 / (kWaves * (2 * kPart + kExps));
  static constexpr int kSlots = kFit > 4 ? 4 : kFit;
  static constexpr int kLds = kWaves * kSlots * (2 * kPart + kExps);
  static constexpr int kOps = kPart / 1024;                         // copies of a part
  static constexpr int kSwap = P > 1 ? kWaves * 4096 : 16;          // scores on their way between two waves
};

// grid: kv head (fastest: the workgroups of a head share an XCD's cache where there are
// eight heads), tile, split; sequence
template <int DT, int D>
__global__ __launch_bounds__((64 * Stream<DT, D>::kWaves)) void stream_kernel(AttendArgs a, int tiles) {
  using St = Stream<DT, D>;
  constexpr int P = St::P, DH = St::DH, T = DH / 32, W = St::W, WT = St::kWaves, NS = St::kSlots;
  __shared__ uint32_t words[kStreamRows * kTreeWords];
  __shared__ float2 ml[W][32];  // maximum and sum
  __shared__ __align__(16) char ring[St::kLds];
  __shared__ __align__(16) char swap[St::kSwap];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31, which = wave / P, share = wave % P;  // block of the turn, part of it
  const int head = blockIdx.x % a.cache.kv, tile = blockIdx.x / a.cache.kv % tiles,
            split = blockIdx.x / (a.cache.kv * tiles), b = blockIdx.y;
  Tile t;
  if (!tile_of(a, b, tile * kStreamRows, kStreamRows, &t)) return;
  const int active = active_splits(a, t);
  if (split >= active) return;
  const int it0 = split * a.split_blocks, it1 = split == active - 1 ? t.n_iter : it0 + a.split_blocks;

  // ---- its rows (q asked for before the blocks: it comes first)
  const Row w = row_of(a, t, b, t.r0 + l32, words);
  const float c = __builtin_fabsf(a.scale_log2e);
  QRegs<DT, DH> q;
  load_q<DT, DH>(a, t, w, head, h, share * DH, q);

  f32x16 o[T];
#pragma unroll
  for (int n = 0; n < T; ++n) o[n] = zero16();
  float m = kFloor, l = 0.0f;

  // ---- the wave's blocks: copies into its ring
  char *mine = ring + wave * (St::kLds / WT);
  constexpr int kSlot = 2 * St::kPart + St::kExps;
  const uint32_t off16 = lane * 16;
  // exponents: lanes 0-7 (mod 16) the keys' 32, lanes 8-15 the values'
  const uint32_t off4 = (lane & 7) * 4 + (lane & 8 ? 1 << a.cache.page_shift : 0);
  auto copy_keys = [&](const char *keys, const char *exps, char *slot) {
    if (DT == DT_F8) copy4(exps, off4, slot + 2 * St::kPart);
#pragma unroll
    for (int x = 0; x < St::kOps; ++x) copy16(keys + share * St::kPart + x * 1024, off16, slot + x * 1024);
  };
  auto copy_vals = [&](const char *keys, char *slot) {
#pragma unroll
    for (int x = 0; x < St::kOps; ++x) {
      const int group = x * 1024 / (DH * 16), in = x * 1024 % (DH * 16);  // (the tokens of 16 bytes: one run of D)
      static_assert(P == 1 || DH * 16 % 1024 == 0, "");
      copy16(keys + a.cache.v_off + (P == 1 ? x * 1024 : group * D * 16 + share * DH * 16 + in), off16,
             slot + St::kPart + x * 1024);
    }
  };
  constexpr int kK = St::kOps + (DT == DT_F8 ? 1 : 0), kV = St::kOps;
  int it = it0 + which;
  Walk<W> walk(a, t, b, head, it, it1);
  uint32_t there = 0;  // bit x: block (the last one asked for) - x W has a page
  auto asked = [&]() {
    there = there << 1 | (walk.there ? 1u : 0u);
    walk.step(P * St::kPart);
  };
#pragma unroll
  for (int x = 0; x < NS; ++x) {
    if (!walk.done()) {
      walk.open(a, t, P * St::kPart);
      copy_keys(walk.keys, walk.exps, mine + x * kSlot);
      copy_vals(walk.keys, mine + x * kSlot);
    }
    asked();
  }
  if (a.nodes > 0) {
    tree_words(a, t, b, words, 64 * WT);
    __syncthreads();
  }

  // One turn: the block's keys are there (every slot asked for: when the later copies are all
  // that is on its way; else when nothing is); as they are done with, their place takes the
  // keys of block it + NS W; the same with the values.
  char *slot = mine;
  // A pair's scores are the sums of its waves' (each takes the same sum).  Every wave comes by once a turn.
  auto meet_scores = [&](f32x16 &s) __attribute__((always_inline)) {
    if constexpr (P > 1) {
      wait_copies<63>();
      __builtin_amdgcn_s_barrier();  // (the last turn's are read)
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4 *>(swap + wave * 4096 + i * 1024 + lane * 16) =
            f32x4{s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]};
      wait_copies<63>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 z = *reinterpret_cast<const f32x4 *>(swap + (wave ^ 1) * 4096 + i * 1024 + lane * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * i + j] += z[j];
      }
    }
  };
  auto turn = [&](auto block_step) {
    const bool more = !walk.done();
    if (it + (NS - 1) * W < it1)
      wait_copies<kV + (NS - 1) * (kK + kV)>();
    else
      wait_copies<0>();
    auto between = [&](f32x16 &s) __attribute__((always_inline)) {
      meet_scores(s);
      wait_copies<63>();  // (LDS reads done)
      // (DT_F8: the values' exponents come with the keys, so those wait until the values are done with)
      if (more) {
        walk.open(a, t, P * St::kPart);
        if (DT != DT_F8) copy_keys(walk.keys, walk.exps, slot);
        wait_copies<(NS - 1) * (kK + kV) + (DT != DT_F8 ? kK : 0)>();
      } else {
        wait_copies<0>();
      }
    };
    block_step(between);
    wait_copies<63>();
    if (more) {
      if (DT == DT_F8) copy_keys(walk.keys, walk.exps, slot);
      copy_vals(walk.keys, slot);
    }
    asked();
    it += W;
    slot = slot == mine + (NS - 1) * kSlot ? mine : slot + kSlot;
  };
  while (it < it1) {
    // (a loop of its own for the blocks that every row sees whole: with the masks in it, the
    // sums would move between two sets of registers in every turn)
    const int full = min(full_end(a, t, w, it), it1);
    while (it < full && there >> (NS - 1) & 1)
      turn([&](const auto &between) __attribute__((always_inline)) {
        full_block<DT, DH>(slot, slot + St::kPart, slot + 2 * St::kPart, q, c, lane, m, l, o, between);
      });
    if (it >= it1) break;
    turn([&](const auto &between) __attribute__((always_inline)) {
      const int k0 = t.block(it) * kBlk;
      f32x16 none = zero16();
      if (sees_none(a, w, k0))
        between(none);
      else
        masked_block<DT, DH>(slot, slot + St::kPart, slot + 2 * St::kPart, q,
                             there >> (NS - 1) & 1 ? seen_word(a, t, w, k0) >> (4 * h) : 0, c, lane, m, l, o, between);
    });
  }

  if (P > 1 && (it1 - it0 - 1) % W < which) {  // (one block fewer than the others)
    f32x16 none = zero16();
    meet_scores(none);
  }

  // ---- the waves' results meet in LDS as rows; all threads scale them to the common maximum, sum
  // and write (in loops that stay short: of a small call most of the time is code coming in)
#pragma unroll
  for (int n = 0; n < T; ++n) settle(o[n]);
  const float2 lh = halves(l);
  if (h == 0 && share == 0) ml[which][l32] = make_float2(m, lh.x + lh.y);
  // (every wave is past its last block: the rings are free.  Rows of D floats, apart by one
  // 16-byte column where that fits.)
  constexpr int kRow = W * 32 * (D + 4) * 4 <= St::kLds ? D + 4 : D;
  static_assert(W * 32 * kRow * 4 <= St::kLds, "");
  float *meet = reinterpret_cast<float *>(ring);
  __syncthreads();
#pragma unroll
  for (int n = 0; n < T; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4 *>(meet + (which * 32 + l32) * kRow + share * DH + 32 * n + 8 * i + 4 * h) =
          f32x4{o[n][4 * i], o[n][4 * i + 1], o[n][4 * i + 2], o[n][4 * i + 3]};
  __syncthreads();
  const int rows = min(kStreamRows, t.rows - t.r0);
#pragma unroll 1
  for (int x = threadIdx.x; x < rows * (D / 4); x += 64 * WT) {
    const int r = x / (D / 4), d = x % (D / 4) * 4, i = (t.r0 + r) / a.group, hq = head * a.group + t.r0 + r - i * a.group;
    float top = ml[0][r].x, sum = 0.0f;
#pragma unroll
    for (int v = 1; v < W; ++v) top = max2(top, ml[v][r].x);
    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float f = __builtin_amdgcn_exp2f(ml[v][r].x - top);
      const f32x4 z = *reinterpret_cast<const f32x4 *>(meet + (v * 32 + r) * kRow + d);
      sum += ml[v][r].y * f;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = __builtin_fmaf(z[j], f, y[j]);
    }
    write4<DT>(a, (int64_t)(t.q.row0 + i), hq, d, split, active, y, top, sum);
  }
}

// The splits' parts scaled to their common maximum and summed in order (bound by latency: 2,080 rows of
// 20 splits, 21 MB, 6 us): LANES (16, 32 or 64) lanes a
// (row, head), four elements each.  The lanes look at the splits' maxima and sums side by side, so a
// row waits for memory three times, not once a split.  How many splits a row has stands with its sums (1: the tile's
// one split has written the result), so nothing of the call's geometry is worked out again.
template <int DT, int LANES>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
  constexpr int kEach = kMaxSplits / LANES, kDeep = 8;  // splits a lane looks at; parts on their way at once
  const int D = a.cache.D, first = scalar_at(a.chunk.starts, 0), end = scalar_at(a.chunk.starts, a.chunk.batch);
  const int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;  // row * heads + head
  const int row = (int)(x / a.heads), lane = threadIdx.x % LANES, d = lane * 4;
  if (row >= a.chunk.rows || row < first || row >= end) return;  // (LANES lanes as one)
  const float2 *ml = a.part_ml + x * (a.splits + 1);
  const int n = min((int)ml[a.splits].x, a.splits);
  if (n <= 1) return;
  float2 mine[kEach];
  float top = kFloor;
#pragma unroll
  for (int e = 0; e < kEach; ++e) mine[e] = ml[min(lane + e * LANES, n - 1)];
#pragma unroll
  for (int e = 0; e < kEach; ++e) top = max2(top, mine[e].x);
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) top = max2(top, __shfl_xor(top, o));
#pragma unroll
  for (int e = 0; e < kEach; ++e) mine[e].x = __builtin_amdgcn_exp2f(mine[e].x - top);
  const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part + x * a.splits * D + min(d, D - 4));
  f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
  float l = 0.0f;
#pragma unroll
  for (int e = 0; e < kEach; ++e)
    for (int s0 = e * LANES; s0 < min(n, (e + 1) * LANES); s0 += kDeep) {
      f32x4 v[kDeep];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) v[j] = part[(int64_t)min(s0 + j, n - 1) * D / 4];
#pragma unroll
      for (int j = 0; j < kDeep; ++j) {
        const float f = s0 + j < n ? __shfl(mine[e].x, (s0 + j) % LANES, LANES) : 0.0f;
        const float sum = __shfl(mine[e].y, (s0 + j) % LANES, LANES);
        l = __builtin_fmaf(sum, f, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_fmaf(v[j][i], f, y[i]);
      }
    }
  if (d >= D) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  store4<DT>(a, row * a.out.row + (x - (int64_t)row * a.heads) * a.out.head + d, y[0] * inv, y[1] * inv, y[2] * inv,
             y[3] * inv);
}

template <int DT>
hipError_t launch_stream(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  const dim3 grid(a.cache.kv * p.tiles * p.splits, a.chunk.batch);
  auto f = a.cache.D == 64    ? stream_kernel<DT, 64>
           : a.cache.D == 96  ? stream_kernel<DT, 96>
           : a.cache.D == 128 ? stream_kernel<DT, 128>
                              : stream_kernel<DT, 256>;
  f<<<grid, 64 * p.waves * stream_share(a.cache.D), 0, s>>>(a, p.tiles);
  return hipGetLastError();
}

}  // namespace


AttendPlan attend_plan(const CacheView &c, const ChunkView &k, int dtype, int heads, int window, int sinks, int nodes) {
  const int group = heads / c.kv, rows = k.max_chunk * group, sets = (rows + 31) / 32;
  AttendPlan p;
  // Few rows, or fp32: every wave its own blocks; more rows share them through LDS (of 68 rows a head
  // each wave would read all keys three times over).  Eight waves a workgroup for one sequence that fills the
  // chip twice with them, but not under a window at up to 128 a head; else four.  One chunk over 16,384 tokens in
  // eight and in four (us; 4,096 rows of 32 heads over 8, at 256 8,192 rows of 16 over 8): bf16 64 a head 569 and 568,
  // 96 719 and 729, 128 859 and 889, 256 1,339 and 2,193 (four are one wave a SIMD there; eight spill 116 registers a
  // lane); 8 bits 812 and 788, 917 and 863, 1,009 and 1,016, 1,705 and 2,074; under a window of 1,024 60 and 57, 76
  // and 70, 94 and 85, 207 and 278.  Chunks that do not fill it twice: eight ragged ones of up to 509 86 and 67, one of
  // 2,047 under a window 29 and 23 (when the rule was set).
  p.stream = dtype == DT_F32 || sets == 1;
  const bool twice = k.batch == 1 && (int64_t)c.kv * ((sets + 7) / 8) >= 512;
  p.waves = p.stream ? stream_blocks(c.D) : twice && (c.D == 256 || window == 0 || window >= k.max_len) ? 8 : 4;
  const int full = p.stream ? 1 : p.waves;
  p.tiles = (sets + full - 1) / full;
  p.tile_rows = (sets + p.tiles - 1) / p.tiles * 32;  // (even tiles: 9 sets of 32 rows are 3 + 3 + 3, not 4 + 4 + 1)
  // blocks of a tile at most
  const int all = (k.max_len + kBlk - 1) / kBlk;
  int most = all;
  if (window > 0) {
    const int64_t span = (int64_t)window + (p.tile_rows + group - 1) / group + 1 + nodes;
    const int64_t near = (span + kBlk - 1) / kBlk + 1 + (sinks + kBlk - 1) / kBlk;
    most = near < all ? (int)near : all;
  }
  // The number of splits whose estimate is least, in units of one block's time in a workgroup by
  // itself (0.5 us with shared blocks; 1.1 us for one block of each wave, 1.6 where pairs share them, in fp32 2.5 to 4.5 with 64 to
  // 128 elements a wave; with 1.1 there too, the choice took 1.3 times as long as the best of eight shapes):
  //  - a workgroup takes its blocks and 2.5 or 5.5 us to start and end; two on a CU take 1.5 times as long a
  //    block, and from half the CUs on a block takes at least what its bytes do (5.2 TB/s for all of them);
  //  - one sequence: equal workgroups in whole rounds of the chip's slots.  A batch: its lengths
  //    are known on the device only; 0.6 of the longest's blocks on average are assumed, and of the
  //    chunks what the rows say; they fill gaps, with a tail of a third of a workgroup (powers of
  //    two: three splits took longer than two and four: 120, 104, 113 us for 32 trees of 16);
  //  - the join: its launch, and the parts written and read.
  const int64_t wgs = (int64_t)c.kv * p.tiles * k.batch;
  const bool paired = !p.stream && p.waves == 4 && c.D <= 128;
  const double base_us = p.stream ? 1.1 : 0.5;
  const double unit_us = dtype == DT_F32                       ? 0.5 + 0.031 * c.D / stream_share(c.D)
                         : p.stream && stream_share(c.D) > 1 ? 1.6
                                                             : base_us;
  const double start = 5.0 * base_us / unit_us;
  const int unit = p.stream ? p.waves : 1;  // blocks that a workgroup takes at a time
  const double memory = unit * 2.0 * kBlk * c.D * elem_bytes(dtype) * 256 / 5.2e6 / unit_us;
  const double share = k.batch == 1 ? 1.0 : 0.6 * k.rows / ((double)k.batch * k.max_chunk);
  const double part = (double)k.rows * heads * c.D * 8 / 4.5e6 / unit_us;
  double best = 1e30;
  p.splits = 1;
  p.blocks = most;
  for (int s = 1; s <= kMaxSplits && (s == 1 || (most + s - 1) / s >= 2 * unit); s = k.batch == 1 ? s + 1 : 2 * s) {
    const int blocks = ((most + s - 1) / s + unit - 1) / unit * unit;
    const int n = (most + blocks - 1) / blocks;
    const double cus = wgs * n * share / 256, turns = (double)blocks / unit;
    double slow = paired && cus > 1.0 ? 1.5 : 1.0;
    if (p.stream && cus > 0.5) slow = fmax(slow, memory * fmin(cus, 1.0));
    double cost = turns + start;
    const double rounds = paired ? cus / 2 : cus;
    if (k.batch == 1) {
      cost = ceil(rounds) * (turns * slow + start);
    } else {
      const double filled = rounds * (turns * slow + start) + 0.3 * cost;
      cost = filled > cost ? filled : cost;
    }
    if (n > 1) cost += (4.0 + 0.1 * n) * base_us / unit_us + part * n * (k.batch == 1 ? 1.0 : 0.7);
    if (cost < best * 0.98) {
      best = cost;
      p.splits = n;
      p.blocks = blocks;
    }
  }
  return p;
}

hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  hipError_t e = !p.stream ? launch_attend_tile(a, p, s)
                 : a.dtype == DT_F32  ? launch_stream<DT_F32>(a, p, s)
                 : a.dtype == DT_BF16 ? launch_stream<DT_BF16>(a, p, s)
                                      : launch_stream<DT_F8>(a, p, s);
  if (e != hipSuccess || p.splits == 1) return e;
  const int lanes = a.cache.D <= 64 ? 16 : a.cache.D <= 128 ? 32 : 64;
  const int64_t groups = ((int64_t)a.chunk.rows * a.heads * lanes + 255) / 256;
  auto f = a.dtype == DT_F32 ? lanes == 16   ? join_kernel<DT_F32, 16>
                               : lanes == 32 ? join_kernel<DT_F32, 32>
                                             : join_kernel<DT_F32, 64>
           : lanes == 16 ? join_kernel<DT_BF16, 16>
           : lanes == 32 ? join_kernel<DT_BF16, 32>
                         : join_kernel<DT_BF16, 64>;
  f<<<(unsigned)groups, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace dt
