// Sampling (dt_sample): a token of each row of logits, by given random numbers.
//
// The row's order is (logit desc, id asc), weights are w = exp((x - max) / T).  What top-k, top-p and min-p keep is
// a prefix of that order, so it is found as a border (a logit, and how many of the logits equal to it are kept),
// not by a sort; the token is found by running sums in the order of ids.  A token is an answer that is right
// or wrong, and of 150,000 borders between tokens some lie within fp32's error of any random number, so
// weights and sums are held in 64 bits throughout.
//
// segments_kernel reads the logits once: a wave takes a segment of 2048 elements and leaves its maximum and, where
// the row needs it, its sum of weights.  row_kernel finishes a row: only segments that can matter are read again.
#include <cmath>
#include <type_traits>

#include "dt_internal.h"

namespace dt {
namespace {

constexpr int kSeg = 2048;          // elements of a segment
constexpr int kLane = kSeg / 64;    // of them with one lane
constexpr int kMaxV = 1 << 19;
constexpr int kMaxSegs = kMaxV / kSeg + 1;   // (a row may begin inside a 16-byte piece)
constexpr int kWaves = 4;           // of a workgroup of segments_kernel
constexpr int kRowThreads = 512, kRowWaves = kRowThreads / 64;
constexpr int kBins = 2048;
constexpr int kMaxGroups = 1 << 24;
constexpr double kOne = 17592186044416.0;  // 2^44: masses in the bins are whole numbers of 2^-44 (2^19 of them fit 63 bits)

struct Settings {
  float temperature, top_p, min_p;
  int top_k;
  const float *temperatures, *top_ps, *min_ps;
  const int32_t *top_ks;
};

struct Logits {
  const char *p;
  int64_t stride;  // bytes
  int rows, V, segs;
};

// What a row asks for.  Off: k = 0, p = 2, q = 0.
struct Row {
  double a;   // log2 e / T
  double p, q;
  int k;
  bool greedy;
};
__device__ inline Row row_of(const Settings &s, int row, int V) {
  const float t = s.temperatures ? s.temperatures[row] : s.temperature;
  const float p = s.top_ps ? s.top_ps[row] : s.top_p, q = s.min_ps ? s.min_ps[row] : s.min_p;
  Row r;
  r.k = s.top_ks ? s.top_ks[row] : s.top_k;
  if (r.k < 0 || r.k >= V) r.k = 0;
  r.greedy = !(t > 0.0f) || r.k == 1 || p <= 0.0f;
  r.a = 1.44269504088896340736 / (double)t;
  r.p = p < 1.0f ? (double)p : 2.0;  // (NaN: off)
  r.q = q > 0.0f ? fmin((double)q, 1.0) : 0.0;
  return r;
}

// 2^t, t <= 0 (NaN and less than -2000 as -2000: 0).  2^f = 1 + f g(f) for |f| <= 1/2, g interpolated at the nine
// Chebyshev points: 4e-14 of the result at most, and 2^0 is 1.
__device__ __forceinline__ double pow2(double t) {
  t = fmax(t, -2000.0);
  const double n = rint(t), f = t - n;
  double g = 1.0203121063391729e-07;
  g = fma(g, f, 1.3255224878668817e-06);
  g = fma(g, f, 1.525268684626772e-05);
  g = fma(g, f, 0.00015403455852453838);
  g = fma(g, f, 0.0013333558179043112);
  g = fma(g, f, 0.009618129159402558);
  g = fma(g, f, 0.055504108664760424);
  g = fma(g, f, 0.2402265069581299);
  g = fma(g, f, 0.6931471805599453);
  return ldexp(fma(g, f, 1.0), (int)n);
}

// the weight of x against a maximum m (an infinite maximum: its equals alone)
__device__ __forceinline__ double weight(float x, float m, double a) {
  if (m == INFINITY) return x == m ? 1.0 : 0.0;
  return pow2(((double)x - (double)m) * a);
}

template <typename T>
__device__ __forceinline__ float value(T x) {
  float v;
  if constexpr (sizeof(T) == 4)
    v = __uint_as_float(x);
  else
    v = bf16_to_f32(x);
  return v == v ? v : -INFINITY;  // (NaN: never chosen)
}

// A row as segments of aligned 16-byte pieces: element i of segment s has the id s * kSeg + i - before.
template <typename T>
struct RowAt {
  const T *base;
  int before, V;
};
template <typename T>
__device__ inline RowAt<T> row_at(const Logits &l, int row) {
  const char *p = l.p + row * l.stride;
  RowAt<T> r;
  r.before = (int)(reinterpret_cast<uintptr_t>(p) % 16) / (int)sizeof(T);
  r.base = reinterpret_cast<const T *>(p) - r.before;
  r.V = l.V;
  return r;
}

// N elements from `at` (a multiple of a piece) of the row's pieces on; those that are not the row's: -infinity
template <int N, typename T>
__device__ __forceinline__ void load_run(const RowAt<T> &r, int at, float *x) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  constexpr int kPiece = 16 / sizeof(T);
  static_assert(N <= kPiece, "one piece at most");
  const int lo = r.before, hi = r.before + r.V;
  if (N == kPiece && at >= lo && at + N <= hi) {
    const u32x4 w = *reinterpret_cast<const u32x4 *>(r.base + at);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(T) == 4)
        x[i] = value<uint32_t>(w[i]);
      else
        x[i] = value<uint16_t>((uint16_t)(w[i / 2] >> (16 * (i & 1))));
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = at + i >= lo && at + i < hi ? value<T>(r.base[at + i]) : -INFINITY;
  }
}

// A segment by a wave: lane l holds piece l + 64 j as x[j * piece ..]; its first element's place
template <typename T>
__device__ __forceinline__ void load_segment(const RowAt<T> &r, int seg, float (&x)[kLane]) {
  constexpr int kPiece = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < kLane / kPiece; ++j)
    load_run<kPiece>(r, seg * kSeg + (j * 64 + (threadIdx.x & 63)) * kPiece, x + j * kPiece);
}

__device__ inline double wave_sum(double x) {
  for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
  return x;
}

// grid: rows x groups of kWaves segments
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void segments_kernel(Logits l, Settings s, int groups, float *maxima,
                                                               double *sums) {
  const int row = blockIdx.x / groups;
  const int seg = (int)(blockIdx.x % groups) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (seg >= l.segs) return;
  const RowAt<T> r = row_at<T>(l, row);
  float x[kLane];
  load_segment(r, seg, x);
  float m = x[0];
#pragma unroll
  for (int i = 1; i < kLane; ++i) m = fmaxf(m, x[i]);
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const Row ask = row_of(s, row, l.V);
  const int64_t at = (int64_t)row * l.segs + seg;
  if ((threadIdx.x & 63) == 0) maxima[at] = m;
  if (ask.greedy || ask.k || (ask.q > 0.0 && ask.p > 1.0)) return;  // (no sum over all is asked for)
  double z = 0.0;
  if (m > -INFINITY) {
#pragma unroll
    for (int i = 0; i < kLane; ++i) z += weight(x[i], m, ask.a);
    z = wave_sum(z);
  }
  if ((threadIdx.x & 63) == 0) sums[at] = z;
}

// Sums over a workgroup of row_kernel in the order of its threads: what comes before a thread, and the whole.
template <typename N>
__device__ N before_thread(N x, N *tmp, N *whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  N run = x;
  for (int o = 1; o < 64; o <<= 1) {
    const N y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = run;
  __syncthreads();
  N first = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    if (w < wave) first += tmp[w];
    all += tmp[w];
  }
  *whole = all;
  return first + (run - x);
}

__device__ inline int block_min(int x, int *tmp) {
  for (int o = 1; o < 64; o <<= 1) x = min(x, __shfl_xor(x, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) x = min(x, tmp[w]);
  return x;
}

struct Shared {
  float maxima[kMaxSegs];
  double mass[kMaxSegs];   // of a segment's kept elements
  int ties[kMaxSegs];      // its elements at the border
  uint32_t count[kBins];
  unsigned long long bin[kBins];
  double tmp_d[kRowWaves];
  unsigned long long tmp_u[kRowWaves];
  int tmp_i[kRowWaves];
  int at;
  double before;
};

// Where an order's prefix ends: elements above `key` are kept, and `ties` of those equal to it.
struct Border {
  uint32_t key;
  int ties;
  double mass;  // of what is kept
};

// One workgroup's view of its row.
template <typename T>
struct Finish {
  Shared &sh;
  RowAt<T> r;
  Row ask;
  int segs;
  float m;

  // f(segment, elements) by the waves for every segment with an element >= lo
  template <typename F>
  __device__ void each_segment(float lo, F f) {
    for (int seg = threadIdx.x >> 6; seg < segs; seg += kRowWaves) {
      if (sh.maxima[seg] < lo || sh.maxima[seg] == -INFINITY) continue;
      float x[kLane];
      load_segment(r, seg, x);
      f(seg, x);
    }
  }

  // The border of the first `want` elements (by_mass: of the elements before which the mass is below `want`), known to
  // lie at keys >= key(lo).  Bins of equal ranges of keys, then of the border's bin, until a bin is a key.
  __device__ Border select(bool by_mass, double want, float lo_value) {
    uint32_t lo = ordered_bits(lo_value), hi = ordered_bits(m);
    double above_n = 0.0;
    unsigned long long above_m = 0;
    for (;;) {
      const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
      for (int i = threadIdx.x; i < kBins; i += kRowThreads) sh.count[i] = 0, sh.bin[i] = 0;
      __syncthreads();
      each_segment(ordered_to_float(lo), [&](int, const float (&x)[kLane]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
          const uint32_t key = ordered_bits(x[i]);
          if (key < lo || key > hi || x[i] == -INFINITY) continue;
          const int b = (int)((key - lo) >> shift);
          atomicAdd(&sh.count[b], 1u);
          atomicAdd(&sh.bin[b], (unsigned long long)(weight(x[i], m, ask.a) * kOne + 0.5));
        }
      });
      __syncthreads();
      // the bins from the top: thread t has bins top - 4 t .. top - 4 t - 3
      constexpr int kEach = kBins / kRowThreads;
      uint32_t n[kEach];
      unsigned long long w[kEach], sum_w = 0, all_w;
      int sum_n = 0, all_n;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int b = kBins - 1 - (kEach * (int)threadIdx.x + i);
        n[i] = sh.count[b];
        w[i] = sh.bin[b];
        sum_n += (int)n[i];
        sum_w += w[i];
      }
      int run_n = before_thread(sum_n, sh.tmp_i, &all_n);
      unsigned long long run_w = before_thread(sum_w, sh.tmp_u, &all_w);
      // the first bin (from the top) whose elements reach the wanted number or mass; else the last that has any
      int mine = kBins;
      const bool reaches = by_mass ? (double)(above_m + all_w) / kOne >= want : above_n + all_n >= want;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        run_n += (int)n[i];
        run_w += w[i];
        const bool there = reaches ? (by_mass ? (double)(above_m + run_w) / kOne >= want : above_n + run_n >= want)
                                   : run_n == all_n;
        if (there && n[i] && mine == kBins) mine = kEach * (int)threadIdx.x + i;
      }
      const int found = block_min(mine, sh.tmp_i);   // (counted from the top)
      if (mine == found && found < kBins) {
        const int i = found - kEach * (int)threadIdx.x;
        int n_above = run_n;
        unsigned long long w_above = run_w;
#pragma unroll
        for (int j = kEach - 1; j >= 0; --j)
          if (j >= i) n_above -= (int)n[j], w_above -= w[j];
        sh.at = n_above;
        sh.tmp_u[0] = w_above;
      }
      __syncthreads();
      const int b = kBins - 1 - found;
      above_n += sh.at;
      above_m += sh.tmp_u[0];
      const int here = (int)sh.count[b];
      __syncthreads();
      lo += (uint32_t)b << shift;
      hi = min(hi, lo + ((1u << shift) - 1));
      if (shift == 0) {
        Border o;
        o.key = lo;
        const double w1 = weight(ordered_to_float(lo), m, ask.a), mass = (double)above_m / kOne;
        double ties = by_mass ? ceil((want - mass) / w1) : want - above_n;
        if (!(ties < (double)here)) ties = here;   // (NaN: a weight of 0)
        o.ties = max((int)ties, above_n > 0.0 ? 0 : 1);
        o.mass = mass + o.ties * w1;
        return o;
      }
    }
  }

  // The element where the running sum of kept weights, in the order of ids, passes u of the whole: segment masses are in
  // sh.mass, ties in sh.ties.  All threads return it; weight: its own, whole: of all kept.
  __device__ int pick(double u, const Border &edge, double *own, double *whole) {
    double z = 0.0, left = 0.0;
    int tied = 0;
    // (a few hundred segments: every thread would add the same numbers; one wave's lanes take a run each)
    const int each = (segs + kRowThreads - 1) / kRowThreads;
    double x = 0.0;
    int t = 0, n_all;
    for (int i = 0; i < each; ++i) {
      const int s = (int)threadIdx.x * each + i;
      if (s < segs) x += sh.mass[s], t += sh.ties[s];
    }
    double run = before_thread(x, sh.tmp_d, &z);
    int run_t = before_thread(t, sh.tmp_i, &n_all);
    const double at = u * z;
    int mine = segs, last = 0;
    for (int i = 0; i < each; ++i) {
      const int s = (int)threadIdx.x * each + i;
      if (s >= segs) break;
      if (run + sh.mass[s] > at && sh.mass[s] > 0.0 && mine == segs) {
        mine = s;
        left = run;
        tied = run_t;
      }
      run += sh.mass[s];
      run_t += sh.ties[s];
    }
    int seg = block_min(mine, sh.tmp_i);
    if (seg == segs) return -1;   // (no weight anywhere: not with a maximum)
    if (mine == seg) sh.before = left, sh.at = tied;
    __syncthreads();
    left = sh.before;
    tied = sh.at;
    // four neighbours a thread
    constexpr int kEach = kSeg / kRowThreads;
    float v[kEach];
    load_run<kEach>(r, seg * kSeg + kEach * (int)threadIdx.x, v);
    int equal = 0, all_equal;
    uint32_t key[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      key[i] = ordered_bits(v[i]);
      equal += key[i] == edge.key && v[i] > -INFINITY;
    }
    int rank = tied + before_thread(equal, sh.tmp_i, &all_equal);
    double w[kEach], sum = 0.0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      w[i] = 0.0;
      if (v[i] == -INFINITY) continue;
      if (key[i] > edge.key || (key[i] == edge.key && rank < edge.ties)) {
        w[i] = weight(v[i], m, ask.a);
        if (w[i] < ask.q) w[i] = 0.0;
      }
      rank += key[i] == edge.key;
      sum += w[i];
    }
    run = left + before_thread(sum, sh.tmp_d, &all);
    mine = kSeg;
    last = -1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      run += w[i];
      if (w[i] > 0.0) last = kEach * (int)threadIdx.x + i;
      if (run > at && w[i] > 0.0 && mine == kSeg) mine = kEach * (int)threadIdx.x + i;
    }
    int found = block_min(mine, sh.tmp_i);
    if (found == kSeg) found = -block_min(-last, sh.tmp_i);   // (the sums' last bits: the segment's last kept element)
    if (found / kEach == (int)threadIdx.x) {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (i == found % kEach) sh.before = w[i];
    }
    __syncthreads();
    *own = sh.before;
    *whole = z;
    return seg * kSeg + found - r.before;
  }
};

// grid: rows
template <typename T>
__global__ __launch_bounds__(kRowThreads) void row_kernel(Logits l, Settings s, const float *u, const float *maxima,
                                                          const double *sums, int32_t *tokens, float *logprobs) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  Finish<T> f{sh, row_at<T>(l, row), row_of(s, row, l.V), l.segs, 0.0f};
  Row &ask = f.ask;
  const int64_t first = (int64_t)row * l.segs;
  float m = -INFINITY;
  for (int i = tid; i < l.segs; i += kRowThreads) {
    const float x = maxima[first + i];
    sh.maxima[i] = x;
    m = fmaxf(m, x);
  }
  // (ordered bits' top: as a signed whole number, smallest first)
  const int top = block_min(~(int)(ordered_bits(m) ^ 0x80000000u), sh.tmp_i);
  m = f.m = ordered_to_float((uint32_t)~top ^ 0x80000000u);
  int token = -1;
  double own = 1.0, whole = 1.0;
  if (m == -INFINITY) {
    own = 0.0;
  } else if (ask.greedy) {
    int seg = l.segs;
    for (int i = tid; i < l.segs && seg == l.segs; i += kRowThreads)
      if (sh.maxima[i] == m) seg = i;
    seg = block_min(seg, sh.tmp_i);
    constexpr int kEach = kSeg / kRowThreads;
    float v[kEach];
    load_run<kEach>(f.r, seg * kSeg + kEach * tid, v);
    int mine = kSeg;
#pragma unroll
    for (int i = kEach - 1; i >= 0; --i)
      if (v[i] == m) mine = kEach * tid + i;
    token = seg * kSeg + block_min(mine, sh.tmp_i) - f.r.before;
  } else {
    const double at = fmin(fmax((double)u[row], 0.0), 0.99999999999);   // (NaN: 0)
    Border edge{0u, 0, 0.0};
    const bool sums_there = !ask.k && !(ask.q > 0.0 && ask.p > 1.0);
    if (sums_there) {
      double z = 0.0;
      for (int i = tid; i < l.segs; i += kRowThreads) {
        const double x = sh.maxima[i] > -INFINITY ? sums[first + i] * weight(sh.maxima[i], m, ask.a) : 0.0;
        sh.mass[i] = x;
        sh.ties[i] = 0;
        z += x;
      }
      before_thread(z, sh.tmp_d, &whole);
    }
    if (ask.k || ask.p <= 1.0 || ask.q > 0.0) {
      // below these nothing is kept: weights under min_p (and a little less), weights that all together are
      // less than 1 - top_p of the whole
      float lo = -INFINITY;
      if (m < INFINITY) {
        // (top-p after top-k is of the mass of all k, those under min_p among them)
        double t = ask.q > 0.0 && !(ask.k && ask.p <= 1.0) ? log2(ask.q) - 1e-6 : -INFINITY;
        if (ask.p <= 1.0 && sums_there) t = fmax(t, log2((1.0 - ask.p) * whole / l.V) - 1e-6);
        const double x = (double)m + t / ask.a;
        lo = (float)(x - 1e-6 * fabs(x));
        if (!(lo <= m)) lo = -INFINITY;
      }
      lo = fmaxf(lo, -3.4028235e38f);
      if (ask.k) edge = f.select(false, (double)ask.k, lo);
      if (ask.k && ask.p <= 1.0) {
        whole = edge.mass;
        lo = ordered_to_float(edge.key);
      }
      if (ask.p <= 1.0) edge = f.select(true, ask.p * whole, lo);
      for (int i = tid; i < l.segs; i += kRowThreads) sh.mass[i] = 0.0, sh.ties[i] = 0;
      __syncthreads();
      // the kept mass of every segment: what lies above the border, and the ties
      const float border = fmaxf(edge.key ? ordered_to_float(edge.key) : lo, lo);
      f.each_segment(border, [&](int seg, const float (&x)[kLane]) __attribute__((always_inline)) {
        double z = 0.0;
        int ties = 0;
#pragma unroll
        for (int i = 0; i < kLane; ++i) {
          const uint32_t key = ordered_bits(x[i]);
          if (x[i] < border || x[i] == -INFINITY) continue;
          if (key == edge.key) {
            ++ties;
          } else if (key > edge.key) {
            const double w = weight(x[i], m, ask.a);
            if (w >= ask.q) z += w;
          }
        }
        z = wave_sum(z);
        for (int o = 1; o < 64; o <<= 1) ties += __shfl_xor(ties, o);
        if ((tid & 63) == 0) sh.mass[seg] = z, sh.ties[seg] = ties;
      });
      __syncthreads();
      if (edge.key) {
        double w = weight(ordered_to_float(edge.key), m, ask.a);
        if (w < ask.q) w = 0.0;
        int t = 0, all;
        const int each = (l.segs + kRowThreads - 1) / kRowThreads;
        for (int i = 0; i < each; ++i)
          if (tid * each + i < l.segs) t += sh.ties[tid * each + i];
        int run = before_thread(t, sh.tmp_i, &all);
        for (int i = 0; i < each; ++i) {
          const int seg = tid * each + i;
          if (seg >= l.segs) break;
          sh.mass[seg] += min(max(edge.ties - run, 0), sh.ties[seg]) * w;
          run += sh.ties[seg];
        }
      }
    }
    __syncthreads();
    token = f.pick(at, edge, &own, &whole);
  }
  if (tid == 0) {
    tokens[row] = token;
    if (logprobs) logprobs[row] = (float)log(own / whole);
  }
}

int segments(int V) { return (V + 15 + kSeg - 1) / kSeg; }

}  // namespace
}  // namespace dt

using namespace dt;

extern "C" {

dt_status dt_sample_workspace_size(int rows, int V, size_t *bytes) {
  if (!bytes) return fail(DT_ERR_NULL, "bytes is required");
  if (rows < 1 || V < 1) return fail(DT_ERR_SHAPE, "sizes must be positive (rows=%d V=%d)", rows, V);
  if (V > kMaxV) return fail(DT_ERR_UNSUPPORTED, "V must be <= %d (%d)", kMaxV, V);
  const int64_t groups = (segments(V) + kWaves - 1) / kWaves;
  if (rows * groups >= kMaxGroups) return fail(DT_ERR_UNSUPPORTED, "rows and V are too large together");
  const size_t n = (size_t)rows * segments(V);
  *bytes = align_up(n * sizeof(double), 256) + align_up(n * sizeof(float), 256);
  return DT_OK;
}

dt_status dt_sample(const void *logits, int64_t row_stride, int rows, int V, int logits_dtype, const float *u,
                    const dt_sampling *how, int32_t *tokens, float *logprobs, void *workspace, size_t ws_bytes,
                    void *stream) {
  if (!logits || !u || !how || !tokens) return fail(DT_ERR_NULL, "logits, u, the settings and tokens are required");
  if (logits_dtype != DT_F32 && logits_dtype != DT_BF16)
    return fail(DT_ERR_DTYPE, "logits_dtype must be DT_F32 or DT_BF16");
  size_t need = 0;
  const dt_status st = dt_sample_workspace_size(rows, V, &need);
  if (st != DT_OK) return st;
  if (row_stride < 0) return fail(DT_ERR_SHAPE, "row_stride must be >= 0");
  if (!how->temperatures && !(how->temperature >= 0.0f)) return fail(DT_ERR_SHAPE, "temperature must be >= 0");
  if (!how->top_ks && how->top_k < 0) return fail(DT_ERR_SHAPE, "top_k must be >= 0 (0: off)");
  if (!how->top_ps && !(how->top_p >= 0.0f)) return fail(DT_ERR_SHAPE, "top_p must be >= 0 (1: off)");
  if (!how->min_ps && !(how->min_p >= 0.0f && how->min_p <= 1.0f))
    return fail(DT_ERR_SHAPE, "min_p must be within [0, 1] (0: off)");
  const size_t es = logits_dtype == DT_F32 ? 4 : 2;
  for (const void *p : {(const void *)u, (const void *)tokens, (const void *)logprobs, (const void *)how->temperatures,
                        (const void *)how->top_ks, (const void *)how->top_ps, (const void *)how->min_ps})
    if (reinterpret_cast<uintptr_t>(p) % 4) return fail(DT_ERR_ALIGN, "tensors must be naturally aligned");
  if (reinterpret_cast<uintptr_t>(logits) % es) return fail(DT_ERR_ALIGN, "logits must be naturally aligned");
  if (!workspace || ws_bytes < need)
    return fail(DT_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", need, workspace ? ws_bytes : 0);
  if (reinterpret_cast<uintptr_t>(workspace) % 256) return fail(DT_ERR_ALIGN, "workspace must be 256-byte aligned");
  const Logits l{static_cast<const char *>(logits), row_stride * (int64_t)es, rows, V, segments(V)};
  const Settings s{how->temperature, how->top_p, how->min_p, how->top_k, how->temperatures, how->top_ps, how->min_ps,
                   how->top_ks};
  double *sums = static_cast<double *>(workspace);
  float *maxima = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                            align_up((size_t)rows * l.segs * sizeof(double), 256));
  const int groups = (l.segs + kWaves - 1) / kWaves;
  hipStream_t q = static_cast<hipStream_t>(stream);
  auto launch = [&](auto t) {
    using T = decltype(t);
    segments_kernel<T><<<(unsigned)(rows * groups), 64 * kWaves, 0, q>>>(l, s, groups, maxima, sums);
    row_kernel<T><<<rows, kRowThreads, 0, q>>>(l, s, u, maxima, sums, tokens, logprobs);
  };
  if (logits_dtype == DT_F32)
    launch(uint32_t());
  else
    launch(uint16_t());
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DT_OK : hip_fail(e, "sampling launch");
}

}  // extern "C"
