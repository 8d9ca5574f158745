// Attention over the paged cache for many rows (chunks of prompts, trees): bf16 data.
//
// A workgroup of NW waves holds 32 NW rows of one kv head; all its waves walk the
// same key blocks, which pass through LDS once for the workgroup: pieces go from memory
// into registers one block ahead and into the other of two LDS slots while the
// present one is used (8-bit caches are widened to bf16 on the way, their powers of two
// applied).  The slots hold the pieces in the cache's order, so a wave's operand is 1,024
// contiguous bytes and no bank is hit twice.
#include "dt_attend.h"

namespace dt {
namespace {
using namespace att;

// Pieces of 16 bytes of one block that a thread carries from memory to LDS.
template <int DT, int D, int NW>
struct Carry {
  static constexpr int kThreads = 64 * NW;
  static constexpr int kPieces = DT == DT_F8 ? 2 * D : 4 * D;  // of the keys, and of the values
  static constexpr int N = (2 * kPieces + kThreads - 1) / kThreads;
  u32x4 v[N];
  uint32_t e[N][DT == DT_F8 ? 4 : 1];  // DT_F8: the exponents (keys: one byte, values: of 16 tokens)

  __device__ __forceinline__ void fetch(const char *kb, const char *vb, const char *ke, const char *ve) {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int i = threadIdx.x + x * kThreads;
      if (i >= 2 * kPieces) break;
      const bool val = i >= kPieces;
      const int j = val ? i - kPieces : i;
      v[x] = reinterpret_cast<const u32x4 *>(val ? vb : kb)[j];
      if (DT == DT_F8) {
        if (val) {
          const int g = j / D;
#pragma unroll
          for (int t = 0; t < 4; ++t) e[x][t] = *reinterpret_cast<const uint32_t *>(ve + 8 * t + 4 * g);
        } else {
          e[x][0] = reinterpret_cast<const uint8_t *>(ke)[j & (kBlk - 1)];
        }
      }
    }
  }
  // (the slot: keys [D / 8][32][8], values [4][D][8], bf16)
  __device__ __forceinline__ void store(char *slot) const {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int i = threadIdx.x + x * kThreads;
      if (i >= 2 * kPieces) break;
      const bool val = i >= kPieces;
      const int j = val ? i - kPieces : i;
      if (DT != DT_F8) {
        reinterpret_cast<u32x4 *>(slot)[i] = v[x];
      } else if (!val) {
        // sixteen elements of token j % 32: pieces 2 c and 2 c + 1 of the slot
        const float s = exp_of(e[x][0]);
        u32x4 w[2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[x][u], s, false),
                       b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[x][u], s, true);
          uint32_t ua, ub;
          __builtin_memcpy(&ua, &a, 4);
          __builtin_memcpy(&ub, &b, 4);
          w[u >> 1][2 * (u & 1)] = ua;
          w[u >> 1][2 * (u & 1) + 1] = ub;
        }
        const int c = j / kBlk, r = j & (kBlk - 1);
        u32x4 *p = reinterpret_cast<u32x4 *>(slot) + 2 * c * kBlk + r;
        p[0] = w[0];
        p[kBlk] = w[1];
      } else {
        // element d of the 16 tokens 8 t + 4 g + 0..3: pieces (2 s + g, d), s = 0, 1
        const int g = j / D, d = j - g * D;
        u32x4 w[2];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(v[x][t], false),
                      b = __builtin_amdgcn_cvt_pk_f32_fp8(v[x][t], true);
          const uint32_t q = e[x][t];
          const bf16x2 lo = {(__bf16)(a[0] * __uint_as_float(q << 23 & 0x7f800000u)),
                             (__bf16)(a[1] * __uint_as_float(q << 15 & 0x7f800000u))},
                       hi = {(__bf16)(b[0] * __uint_as_float(q << 7 & 0x7f800000u)),
                             (__bf16)(b[1] * __uint_as_float(q >> 1 & 0x7f800000u))};
          uint32_t ul, uh;
          __builtin_memcpy(&ul, &lo, 4);
          __builtin_memcpy(&uh, &hi, 4);
          w[t >> 1][2 * (t & 1)] = ul;
          w[t >> 1][2 * (t & 1) + 1] = uh;
        }
        u32x4 *p = reinterpret_cast<u32x4 *>(slot) + 4 * D + d;
        p[g * D] = w[0];
        p[(2 + g) * D] = w[1];
      }
    }
  }
};

// Blocks on their way from memory: bf16 pieces are copied into a ring of LDS slots without
// passing through registers, 8-bit ones wait in registers to be widened.
constexpr int kCopies = 3, kCarried = 2;

// grid: kv head (fastest), tile (the last rows, which see most, first), split; sequence
template <int DT, int D, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((
    amdgpu_waves_per_eu(NW == 8 || D <= 128 ? 2 : 1, NW == 8 || D <= 128 ? 2 : 1))) void tile_kernel(AttendArgs a, int tiles, int tile_rows) {
  constexpr int T = D / 32, ES = DT == DT_F8 ? 1 : 2, kRows = 32 * NW;
  constexpr int kSlots = DT == DT_F8 ? 2 : kCopies + 1, kSlot = 128 * D;
  __shared__ __align__(16) char slots[kSlots][kSlot];
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
  if (a.nodes > 0) tree_words(a, t, b, words, 64 * NW);
  __syncthreads();
  const int r = t.r0 + 32 * wave + l32;
  const bool idle = 32 * wave >= tile_rows || t.r0 + 32 * wave >= t.rows;  // (no rows: it carries blocks only)
  const Row w = row_of(a, t, b, idle ? t.r0 : r, words);
  const float c = __builtin_fabsf(a.scale_log2e);
  QRegs<DT_BF16, D> q;
  load_q<DT_BF16, D>(a, t, w, head, h, false, q);
  f32x16 o[T];
#pragma unroll
  for (int n = 0; n < T; ++n) o[n] = zero16();
  float m = kFloor, l = 0.0f;

  const int32_t *table = a.chunk.table + (int64_t)b * a.chunk.width;
  const int shift = a.cache.page_shift;
  auto page_of = [&](int it) { return it < it1 ? scalar_at(table, t.block(it) * kBlk >> shift) : 0; };
  // head page of a block (out of range: page 0, whose tokens then count as unseen), token in it
  auto place = [&](int it, int page, int *n) {
    const int p = __builtin_amdgcn_readfirstlane(page);
    *n = t.block(it) * kBlk & ((1 << shift) - 1);
    return a.cache.base + (int64_t)((uint32_t)p < (uint32_t)a.cache.pages ? p : 0) * a.cache.page_bytes +
           head * a.cache.head_bytes;
  };
  auto use = [&](int it, int page, const char *slot) __attribute__((always_inline)) {
    const int k0 = t.block(it) * kBlk;
    if (idle || sees_none(a, w, k0)) return;
    const bool there = (uint32_t)page < (uint32_t)a.cache.pages;
    const f32x16 s = scores<DT_BF16, D>(slot, nullptr, q, lane);
    float p[16];
    if (there && sees_all(a, w, k0)) {
      softmax_block<false>(s, 0, c, m, l, o, p);
      add_values<DT_BF16, D, false>(slot + kSlot / 2, nullptr, p, 0, lane, o);
    } else {
      const uint32_t seen = there ? seen_word(a, t, w, k0) >> (4 * h) : 0;
      softmax_block<true>(s, seen, c, m, l, o, p);
      add_values<DT_BF16, D, true>(slot + kSlot / 2, nullptr, p, seen, lane, o);
    }
  };

  if constexpr (DT == DT_BF16) {
    // kilobytes of a block, each one wave's copy; every wave copies as many (past the last:
    // again one that another wave copies, the same bytes), so all count alike
    constexpr int kPieces = kSlot / 1024, kEach = (kPieces + NW - 1) / NW;
    auto copy = [&](int it, int page, char *slot) {
      int n;
      const char *hp = place(it, page, &n);
      hp += (int64_t)n * D * ES;
#pragma unroll
      for (int x = 0; x < kEach; ++x) {
        int i = wave + x * NW;
        if (kPieces % NW) i = i < kPieces ? i : i - kPieces;
        copy16((i < kPieces / 2 ? hp + i * 1024 : hp + a.cache.v_off + (i - kPieces / 2) * 1024) + lane * 16,
               slot + i * 1024);
      }
    };
    int pages[kCopies + 1];  // of blocks it .. it + kCopies
#pragma unroll
    for (int x = 0; x <= kCopies; ++x) pages[x] = page_of(it0 + x);
#pragma unroll
    for (int x = 0; x < kCopies; ++x)
      if (it0 + x < it1) copy(it0 + x, pages[x], slots[x]);
    int slot = 0, free_slot = kCopies;
    for (int it = it0; it < it1; ++it) {
      // this wave's copies of the block are there (near the end: all of them), then every wave's
      if (it + kCopies <= it1)
        wait_copies<(kCopies - 1) * kEach>();
      else
        wait_copies<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      // (every wave has done with the last block: its slot is free)
      if (it + kCopies < it1) copy(it + kCopies, pages[kCopies], slots[free_slot]);
      const int after = page_of(it + kCopies + 1);
      use(it, pages[0], slots[slot]);
#pragma unroll
      for (int x = 0; x < kCopies; ++x) pages[x] = pages[x + 1];
      pages[kCopies] = after;
      slot = slot == kCopies ? 0 : slot + 1;
      free_slot = free_slot == kCopies ? 0 : free_slot + 1;
    }
  } else {
    Carry<DT, D, NW> carry[kCarried];
    auto fetch = [&](Carry<DT, D, NW> &to, int it, int page) {
      int n;
      const char *hp = place(it, page, &n);
      to.fetch(hp + (int64_t)n * D * ES, hp + a.cache.v_off + (int64_t)n * D * ES, hp + a.cache.s_off + n,
               hp + a.cache.s_off + (1 << shift) + n);
    };
    int pages[kCarried + 2];  // of blocks it .. it + kCarried + 1
#pragma unroll
    for (int x = 0; x < kCarried + 2; ++x) pages[x] = page_of(it0 + x);
    if (it0 < it1) {
      fetch(carry[0], it0, pages[0]);
      carry[0].store(slots[0]);
#pragma unroll
      for (int x = 1; x <= kCarried; ++x)
        if (it0 + x < it1) fetch(carry[x % kCarried], it0 + x, pages[x]);
    }
    __syncthreads();
    for (int it = it0; it < it1; it += kCarried) {
#pragma unroll
      for (int u = 0; u < kCarried; ++u) {
        const int now = it + u;
        if (now >= it1) break;
        const int at = (now - it0) & 1, after = page_of(now + kCarried + 2);
        if (now + 1 < it1) {
          Carry<DT, D, NW> &cr = carry[(u + 1) % kCarried];
          cr.store(slots[at ^ 1]);
          if (now + 1 + kCarried < it1) fetch(cr, now + 1 + kCarried, pages[kCarried + 1]);
        }
        use(now, pages[0], slots[at]);
        __syncthreads();
#pragma unroll
        for (int x = 0; x <= kCarried; ++x) pages[x] = pages[x + 1];
        pages[kCarried + 1] = after;
      }
    }
  }
  if (idle) return;
  const float2 lh = halves(l);
  write_rows<DT_BF16, D>(a, t, w, head, split, active == 1, r < t.rows, h, o, m, lh.x + lh.y);
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
