// Attention over the paged cache for many rows (chunks of prompts, trees): bf16 data.
//
// The mathematics is the one-pass softmax of dt_attend.hip; a workgroup of NW waves holds 32 rows
// a wave of one kv head; all its waves walk the same key blocks, which every wave copies its share
// of from memory into a ring of LDS slots, three blocks ahead and past the registers.  The slots hold
// the blocks in the cache's order, so a wave's operand is 1,024 contiguous bytes and no bank is hit twice.
//
// What bounds it: the issue of instructions.  A wave by itself takes about five cycles an instruction,
// and a block of 32 tokens of 128 is 16 matrix products (512 cycles of the matrix unit) among
// some 175 others in bf16, 285 in 8 bits (64 of them widen codes, 36 bring in the values' scales): a
// block takes 0.5 us of a workgroup by itself, 0.65 in 8 bits, and two workgroups a CU fill each other's
// gaps.  4,096 rows of 32 heads over 16,384 tokens: 858 to 930 us from one card to another (graph-captured; 983
// under a kernel trace), 1,035 to 1,120 TFLOP/s of the 1,245 of a large product; in 8 bits 1,012 us.  8,192 rows of 16
// heads of 256 over as many: 1,337 us, 1,230 TFLOP/s.  Eight ragged chunks of 16 heads of 64 in 8 bits: 69 us, 260
// TFLOP/s (the longest tile's blocks, one after another); 65 rows of 32 heads over 30,011 tokens in 8 bits: 70 us, of which
// about 20 do not depend on the length (start, masked blocks, parts, join).
// Measured and not taken: two blocks a turn; the next block's scores between the instructions of
// the last one's softmax (881 -> 943 us then: the number of instructions counts, not their order); all keys of a
// block read before the first product (897); four waves a SIMD at 64 (a long chunk 303 -> 295, but
// one under a window 24 -> 26: registers).
#include "dt_attend.h"

namespace dt {
namespace {
using namespace att;

constexpr int kAhead = 3;  // blocks on their way from memory

// grid: kv head (fastest), tile (the last rows, which see most, first), split; sequence
template <int DT, int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((
    amdgpu_waves_per_eu(NW == 8 || D <= 128 ? 2 : 1, NW == 8 || D <= 128 ? 2 : 1))) void tile_kernel(AttendArgs a,
                                                                                                     int tiles,
                                                                                                     int tile_rows) {
  constexpr int T = D / 32, ES = DT == DT_F8 ? 1 : 2, kRows = 32 * NW, kPart = kBlk * D * ES;
  constexpr int kSlot = 2 * kPart + (DT == DT_F8 ? 256 : 0);  // keys, values, exponents
  __shared__ __align__(16) char ring[(kAhead + 1) * kSlot];
  __shared__ uint32_t words[kRows * kTreeWords];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, l32 = lane & 31;
  const int head = blockIdx.x % a.cache.kv, tile = tiles - 1 - blockIdx.x / a.cache.kv % tiles,
            split = blockIdx.x / (a.cache.kv * tiles), b = blockIdx.y;
  Tile t;
  if (!tile_of(a, b, tile * tile_rows, tile_rows, &t)) return;
  const int active = active_splits(a, t);
  if (split >= active) return;
  const int it0 = split * a.split_blocks, it1 = split == active - 1 ? t.n_iter : it0 + a.split_blocks;
  const int r = t.r0 + 32 * wave + l32;
  const bool idle = 32 * wave >= tile_rows || t.r0 + 32 * wave >= t.rows;  // (no rows: it copies only)
  const Row w = row_of(a, t, b, idle ? t.r0 : r, words);
  const float c = __builtin_fabsf(a.scale_log2e);
  QRegs<DT, D> q;
  load_q<DT, D>(a, t, w, head, h, 0, q);
  f32x16 o[T];
#pragma unroll
  for (int n = 0; n < T; ++n) o[n] = zero16();
  float m = kFloor, l = 0.0f;

  // kilobytes of a block, each one wave's copy; every wave copies as many (past the last:
  // again one that another wave copies, the same bytes), so all count alike
  constexpr int kPieces = 2 * kPart / 1024, kMine = (kPieces + NW - 1) / NW, kEach = kMine + (DT == DT_F8 ? 1 : 0);
  uint32_t from[kMine];  // of the block's keys, this lane's
  int to[kMine];         // in its slot
#pragma unroll
  for (int x = 0; x < kMine; ++x) {
    const int p = wave + x * NW, i = p < kPieces ? p : p - kPieces;
    from[x] = (i < kPieces / 2 ? i * 1024 : (int)a.cache.v_off + (i - kPieces / 2) * 1024) + lane * 16;
    to[x] = i * 1024;
  }
  // exponents: lanes 0-7 (mod 16) the keys' 32, lanes 8-15 the values'
  const uint32_t off4 = (lane & 7) * 4 + (lane & 8 ? 1 << a.cache.page_shift : 0);
  Walk<1> walk(a, t, b, head, it0, it1);
  uint32_t there = 0;  // bit x: block (the last one asked for) - x has a page
  auto ask = [&](char *slot) {
    if (!walk.done()) {
      walk.open(a, t, kPart);
      if (DT == DT_F8) copy4(walk.exps, off4, slot + 2 * kPart);
#pragma unroll
      for (int x = 0; x < kMine; ++x) copy16(walk.keys, from[x], slot + to[x]);
    }
    there = there << 1 | (walk.there ? 1u : 0u);
    walk.step(kPart);
  };
#pragma unroll
  for (int x = 0; x < kAhead; ++x) ask(ring + x * kSlot);
  if (a.nodes > 0) {
    tree_words(a, t, b, words, 64 * NW);
    __syncthreads();
  }
  int it = it0;
  char *slot = ring, *before = ring + kAhead * kSlot;  // of the present block and of the last
  const int steady = it1 - kAhead;  // up to there every turn asks for a block
  // (bit kAhead - 1 of `there` is the present block before its turn, bit kAhead after it.)
  // A turn: the present block is there (near the end: all that was asked for), for every wave, and every
  // wave has done with the last one, whose slot takes the next.
  auto turn = [&]() {
    if (__builtin_expect(it <= steady, 1))
      wait_copies<(kAhead - 1) * kEach>();
    else
      wait_copies<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    ask(before);
  };
  auto next = [&]() {
    before = slot;
    slot = slot == ring + kAhead * kSlot ? ring : slot + kSlot;
    ++it;
  };
  const Nothing nothing;
  if (idle)
    for (; it < it1; next()) turn();
  while (it < it1) {
    // (a loop of its own for the blocks that every row sees whole: with the masks in it, the
    // sums would move between two sets of registers in every turn)
    const int full = min(full_end(a, t, w, it), it1);
    for (; it < full && there >> (kAhead - 1) & 1; next()) {
      turn();
      full_block<DT, D>(slot, slot + kPart, slot + 2 * kPart, q, c, lane, m, l, o, nothing);
    }
    if (it >= it1) break;
    turn();
    const int k0 = t.block(it) * kBlk;
    if (!sees_none(a, w, k0))
      masked_block<DT, D>(slot, slot + kPart, slot + 2 * kPart, q,
                          there >> kAhead & 1 ? seen_word(a, t, w, k0) >> (4 * h) : 0, c, lane, m, l, o, nothing);
    next();
  }
#pragma unroll
  for (int n = 0; n < T; ++n) settle(o[n]);
  if (idle || r >= t.rows) return;
  const float2 lh = halves(l);
  const int hq = head * a.group + w.r % a.group;
#pragma unroll
  for (int n = 0; n < T; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      write4<DT_BF16>(a, t.q.row0 + w.i, hq, 32 * n + 8 * i + 4 * h, split, active,
                      f32x4{o[n][4 * i], o[n][4 * i + 1], o[n][4 * i + 2], o[n][4 * i + 3]}, m, lh.x + lh.y);
}

template <int DT, int NW>
hipError_t launch(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  const dim3 grid(a.cache.kv * p.tiles * p.splits, a.chunk.batch);
  auto f = a.cache.D == 64    ? tile_kernel<DT, 64, NW>
           : a.cache.D == 96  ? tile_kernel<DT, 96, NW>
           : a.cache.D == 128 ? tile_kernel<DT, 128, NW>
                              : tile_kernel<DT, 256, NW>;
  f<<<grid, 64 * NW, 0, s>>>(a, p.tiles, p.tile_rows);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_tile(const AttendArgs &a, const AttendPlan &p, hipStream_t s) {
  if (a.dtype == DT_F8) return p.waves == 4 ? launch<DT_F8, 4>(a, p, s) : launch<DT_F8, 8>(a, p, s);
  return p.waves == 4 ? launch<DT_BF16, 4>(a, p, s) : launch<DT_BF16, 8>(a, p, s);
}

}  // namespace dt
