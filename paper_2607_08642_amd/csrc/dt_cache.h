// The paged cache of the verification calls: where its elements lie.
//
// A layer is pages x kv heads x one head page: the keys of page_size tokens, their
// values, and for DT_F8 an exponent byte for each token's keys and each token's
// values.  Tokens come in blocks of 32, stored in 16-byte pieces of E elements (E = 4,
// 8, 16 for 4-, 2- and 1-byte elements) in the operand order of the 32x32 matrix
// instructions, so that a wave's operand is one or two contiguous runs of a block
// and no transpose stands between the cache and the matrix unit:
//   keys    [D / E][32 tokens][E]: piece (c, r) = elements c E .. c E + E - 1 of token r
//           (A of S^T = K Q^T: a lane holds one token and a run of D);
//   values  [32 / E][D][E]: piece (g, d) = element d of E tokens (A of O^T = V^T P^T: a
//           lane holds one d and a run of tokens).  S^T leaves a lane of column q
//           with the tokens 8 t + 4 h + 0..3 (t = 0..3, h = the lane's half), and the
//           tokens of a piece are those of one h, so the probabilities are B of the
//           second product without moving between lanes:
//             token r: s = r >> 4, b = r >> 3 & 1, h = r >> 2 & 1, e = r & 3
//             4-byte: g = r >> 2, element e; 2-byte: g = 2 s + h, element 4 b + e;
//             1-byte: g = h, element 8 s + 4 b + e.
#pragma once

#include "dt_internal.h"

namespace dt {

constexpr int kBlk = 32;  // tokens of a block

struct CacheView {  // one layer
  char *base;
  int64_t head_bytes, page_bytes;  // a head page, a page (kv head pages)
  int64_t v_off, s_off;            // values and exponents within a head page
  int pages, page_shift, kv, D;
};

struct ChunkView {
  int batch, rows, max_chunk, max_len, width;
  const int32_t *starts, *lens, *table;
};

struct RowsView {
  char *p;
  int64_t row, head;  // strides in elements
  int vec;            // 16-byte aligned throughout
};

constexpr int elem_bytes(int dtype) { return dtype == DT_F32 ? 4 : dtype == DT_BF16 ? 2 : 1; }
inline int data_dtype(int cache_dtype) { return cache_dtype == DT_F32 ? DT_F32 : DT_BF16; }

// bytes of a head page
inline int64_t head_page_bytes(int page_size, int D, int dtype) {
  return (int64_t)2 * page_size * D * elem_bytes(dtype) + (dtype == DT_F8 ? 2 * page_size : 0);
}

inline CacheView cache_view(const dt_cache &c, int layer) {
  CacheView v;
  v.head_bytes = head_page_bytes(c.page_size, c.head_dim, c.dtype);
  v.page_bytes = v.head_bytes * c.kv_heads;
  v.base = static_cast<char *>(c.data) + (int64_t)layer * v.page_bytes * c.pages;
  v.v_off = (int64_t)c.page_size * c.head_dim * elem_bytes(c.dtype);
  v.s_off = 2 * v.v_off;
  v.pages = c.pages;
  v.page_shift = __builtin_ctz((unsigned)c.page_size);
  v.kv = c.kv_heads;
  v.D = c.head_dim;
  return v;
}

inline ChunkView chunk_view(const dt_chunk &c) {
  return ChunkView{c.batch, c.rows, c.max_chunk, c.max_len, c.table_width, c.starts, c.lens, c.table};
}

// An index that is the same for the whole wave, read through the scalar cache.
__device__ __forceinline__ int32_t scalar_at(const int32_t *p, int64_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(p))[i];
}

// A sequence's rows and tokens, kept within the tensors whatever starts and lens hold.
struct Seq {
  int row0, n;  // rows [row0, row0 + n)
  int base;     // position of row0's token (negative only where lens < n)
  int len;      // tokens that the table can hold
};
__device__ inline Seq seq_of(const ChunkView &c, int page_shift, int b) {
  Seq s;
  const int a = scalar_at(c.starts, b), e = scalar_at(c.starts, b + 1), len = scalar_at(c.lens, b);
  s.row0 = min(max(a, 0), c.rows);
  s.n = min(max(e, s.row0), c.rows) - s.row0;
  s.base = min(max(len, 0), 1 << 30) - s.n;
  s.len = min(max(len, 0), c.width << page_shift);
  return s;
}

// Position of token r (0..31) of a block in a values piece: piece row g, element j.
template <int E>
__host__ __device__ inline int v_group(int r) {
  return E == 4 ? r >> 2 : E == 8 ? ((r >> 4) << 1) | ((r >> 2) & 1) : (r >> 2) & 1;
}
template <int E>
__host__ __device__ inline int v_elem(int r) {
  return E == 4 ? r & 3 : E == 8 ? (((r >> 3) & 1) << 2) | (r & 3) : ((r >> 3) << 2) | (r & 3);
}
// its inverse: the token of element j of piece row g
template <int E>
__host__ __device__ inline int v_token(int g, int j) {
  return E == 4 ? 4 * g + j : E == 8 ? 16 * (g >> 1) + 8 * (j >> 2) + 4 * (g & 1) + (j & 3)
                                     : 8 * (j >> 2) + 4 * g + (j & 3);
}

// exponents of DT_F8: byte e + 127 of 2^e
__device__ inline float exp_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Whether a cache is one (dt_verify.hip); data: its memory too.
dt_status check_cache(const dt_cache *c, bool data);

// launchers (dt_cache.hip, dt_attend*.hip)
struct AttendArgs {
  CacheView cache;
  ChunkView chunk;
  RowsView q, out;
  int dtype, heads, group;
  float scale_log2e;
  int window, sinks, nodes;
  const uint8_t *mask;
  const int32_t *depth;
  float *part;     // [rows * heads][splits][D] partial sums
  float2 *part_ml;  // [rows * heads][splits + 1] maximum and sum; how many splits there are
  int splits, split_blocks;
};

// How a call is cut up: tiles of tile_rows (query, head) rows of a kv head, the key blocks
// of a tile dealt to `splits` workgroups of `waves` waves, `blocks` blocks each.
struct AttendPlan {
  bool stream;  // each wave its own blocks (stream_kernel), not all of them the same (tile_kernel)
  int waves, tile_rows, tiles, splits, blocks;
};
AttendPlan attend_plan(const CacheView &c, const ChunkView &k, int dtype, int heads, int window, int sinks, int nodes);
hipError_t launch_attend(const AttendArgs &a, const AttendPlan &p, hipStream_t s);
hipError_t launch_append(const CacheView &c, int dtype, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                         hipStream_t s);
hipError_t launch_read(const CacheView &c, int dtype, const ChunkView &k, const RowsView &kr, const RowsView &vr,
                       hipStream_t s);
hipError_t launch_accept(const dt_tree &t, int batch, int B, const int32_t *target, int32_t *path, int32_t *n,
                         int32_t *next, hipStream_t s);
hipError_t launch_commit(const CacheView &c, int dtype, int layers, const ChunkView &k, int nodes,
                         const int32_t *path, const int32_t *n, hipStream_t s);

}  // namespace dt
