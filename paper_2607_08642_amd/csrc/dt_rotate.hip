// Heads normed and rotated by position, as rows (dt_rotate): how rows are dealt to waves, the kernel.
// (With the pages of a cache: append_rotated_kernel of dt_cache.hip.)
//
// y = w x / sqrt(mean x^2 + eps), then pairs turned by pos f_j: a copy with some forty instructions an access, bound by memory
// for prompts (16,000 rows of 40 heads of 128 in bf16 66 us, 5.0 TB/s; 8,000 in fp32 64, 5.1; a copy of 1 GiB: 5.0) and by
// latency for few rows (3.1 us for one row of a small model).  A wave takes a row, so that its angles are computed once, a pair a
// lane, in 64 bits up to the turn's remainder, and are read from LDS for all heads.
#include <math.h>

#include "dt_rotate.h"

namespace dt {
namespace {

template <typename T, bool kNear>
__global__ __launch_bounds__(64 * kRotWaves) void rotate_kernel(RotaryView r, HeadsView q, HeadsView k, RotatePlan plan,
                                                                int rows, int D) {
  __shared__ float2 cs[kRotWaves][kMaxPairs];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t at = (int64_t)blockIdx.x * kRotWaves + wave;
  const int64_t row = at / plan.splits;
  if (row >= rows) return;
  const int first = (int)(at % plan.splits) * plan.per, last = min(first + plan.per, plan.passes);
  if (q.in.vec && q.out.vec && k.in.vec && k.out.vec)
    rotate_row<T, true, kNear>(r, q, k, D, plan.lanes, row, first, last, cs[wave]);
  else
    rotate_row<T, false, kNear>(r, q, k, D, plan.lanes, row, first, last, cs[wave]);
}

}  // namespace

RotatePlan rotate_plan(int64_t rows, int heads, int kv_heads, int D) {
  RotatePlan p;
  p.lanes = 1;
  while (16 * p.lanes < D) p.lanes *= 2;
  const int wide = 64 / p.lanes;
  p.passes = (heads + wide - 1) / wide + (kv_heads + wide - 1) / wide;
  // Few rows: a row's passes are dealt to several waves, each of which computes the angles again.  40 heads of 128 in bf16,
  // graph-captured, a wave a row / up to 4,096 waves / up to 16,384: 1 row 6.9 / 3.7 / 3.8 us, 544 8.5 / 5.3 / 5.4, 2,000
  // 11.5 / 12.2 / 11.5, 4,000 16.6 / 17.2 / 19.7.
  p.splits = 1;
  while (p.splits < p.passes && rows * p.splits < 4096) ++p.splits;
  p.per = (p.passes + p.splits - 1) / p.splits;
  p.splits = (p.passes + p.per - 1) / p.per;
  return p;
}

hipError_t launch_rotate(const RotaryView &r, const HeadsView &q, const HeadsView &k, int rows, int D, int dtype,
                         hipStream_t s) {
  const RotatePlan plan = rotate_plan(rows, q.heads, k.heads, D);
  const int64_t groups = ((int64_t)rows * plan.splits + kRotWaves - 1) / kRotWaves;
  auto f = dtype == DT_F32 ? r.interleaved ? rotate_kernel<float, true> : rotate_kernel<float, false>
           : r.interleaved ? rotate_kernel<uint16_t, true> : rotate_kernel<uint16_t, false>;
  f<<<(unsigned)groups, 64 * kRotWaves, 0, s>>>(r, q, k, plan, rows, D);
  return hipGetLastError();
}

}  // namespace dt
