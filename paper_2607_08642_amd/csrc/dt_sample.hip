// Sampling (dt_sample): a token of each row of logits, by given random numbers.
//
// The row's order is (logit desc, id asc), weights are w = exp((x - max) / T).  What top-k, top-p and min-p keep is
// a prefix of that order, so it is found as a border (a logit, and how many of the logits equal to it are kept),
// not by a sort; the token is found by running sums in the order of ids.  A token is an answer that is right
// or wrong, and of 150,000 borders between tokens some lie within fp32's error of any random number (running sums in
// fp32 drew another token in 47 of 3,264 peaked rows and in 100 of 3,264 flat ones), so weights and sums are held in 64 bits.
//
// segments_kernel reads the logits once: a wave takes a segment of 2048 elements and leaves the maxima of its groups and,
// where the row needs it, its sum of weights.  Segments lie where they lie whatever else a call holds, so a row's
// sums do not depend on the other rows.  row_kernel finishes a row, a workgroup each: the groups' maxima bound from below what can
// be kept, and only groups that reach the bound are read again; a list of at most 1024 elements in LDS is put
// in order.  Rows of which more is kept by top-p or min-p go on in three launches over the whole card: masses in bins of values, the
// border's bin and each segment's mass above it, the border among the bin's elements.  What none of this fits (top-k of
// thousands; more than kList elements in the border's bin, as where thousands of logits are equal) is found by passes of the
// row's own workgroup (Finish::select).  In bf16 such equals are common away from zero: of 151,936 logits about +10 with a
// spread of 2, whose values there are 1/16 apart, some 1,500 are equal at the border of top-p 0.9 (17 rows: 503 us, where those
// about 0 take 47); of logits about -10 with a spread of 2.5 that is so for T 1.3 and top-p 0.97 (542), not for T 1 and 0.9 (55).
// Rows of up to 16 segments (32,753 logits, as a row may begin inside a piece) are read by the workgroup that finishes them.
//
// Measured, 151,936 logits in bf16, kernels alone: segments_kernel over 544 rows 26 us without sums (6.4 TB/s: memory), 65 with
// sums (64-bit arithmetic: 15 instructions of about five cycles an element); row_kernel at one row 3 us for the
// largest, 6 for all, 9 for top-k 20, 11 for top-p 0.9, 19 for top-k 200; at 544 rows 4, 9, 12, 17, 28: bound by latency, of
// memory (two reads that wait for one another) and of instructions, which a workgroup runs once.  The launches for large rows add
// 5 us where there is none (1, 32 and 544 rows with top-k 20, graph-captured), and take 34 for 17 flat rows of fp32.
#include <cmath>
#include <type_traits>

#include "dt_internal.h"

namespace dt {
namespace {

typedef unsigned long long u64;

constexpr int kSeg = 2048;          // elements of a segment
constexpr int kLane = kSeg / 64;    // of them with one lane
constexpr int kMaxV = 1 << 19;
constexpr int kMaxSegs = kMaxV / kSeg + 1;   // (a row may begin inside a 16-byte piece)
constexpr int kWaves = 4;           // of a workgroup of segments_kernel
constexpr int kRowThreads = 256, kRowWaves = kRowThreads / 64;
// A segment's maxima are kept for groups of elements: those of four lanes (128), or of each lane in a short row.
template <bool kShort>
struct Groups {
  static constexpr int lanes = kShort ? 1 : 4, n = 64 / lanes;   // n in a segment
};
// Rows of no more segments are read by the workgroup that finishes them, in one launch (graph-captured calls, two launches / one:
// 8,000 logits 13 / 10 us for a row, 47 / 32 for 2,048 of them with top-k 20; 32,000: 13 / 12, 47 / 46, with top-p 0.9 141 / 97;
// one row of 32,000 as it is 11 / 14), and are not large: their workgroup's own passes are short.
constexpr int kFewSegs = 16;
constexpr int kBins = 2048;
constexpr int kPad = 64;
constexpr int kList = 1024;  // elements that a row's end is found among in LDS
constexpr int kPart = 4;     // waves of a workgroup of the passes for large rows
constexpr int kMaxGroups = 1 << 24;
constexpr int kSpread = 1024;   // workgroups of the passes for large rows (four a CU): launches that find no such row end soon
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
  __device__ __forceinline__ bool filters() const { return k || p <= 1.0 || q > 0.0; }
  // whether the weights of all elements are summed: nothing is left out, or top-p is of all
  __device__ __forceinline__ bool sums() const { return !greedy && !k && (p <= 1.0 || !(q > 0.0)); }
};
__device__ __forceinline__ Row row_of(const Settings &s, int row, int V) {
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
// Chebyshev points: 4e-14 of the result at most, and 2^0 is 1.  The coefficients are kept in scalar registers (as
// literals each step would move one to the vector registers first: half of all instructions).
struct Pow2 {
  double c[9] = {1.0203121063391729e-07, 1.3255224878668817e-06, 1.525268684626772e-05, 0.00015403455852453838,
                 0.0013333558179043112,  0.009618129159402558,   0.055504108664760424,  0.2402265069581299,
                 0.6931471805599453};
  __device__ __forceinline__ Pow2() {
#pragma unroll
    for (int i = 0; i < 9; ++i) asm("" : "+s"(c[i]));
  }
  __device__ __forceinline__ double operator()(double t) const {
    t = fmax(t, -2000.0);
    const double n = rint(t), f = t - n;
    double g = c[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) g = fma(g, f, c[i]);
    return ldexp(fma(g, f, 1.0), (int)n);
  }
  // 2^((x - m) a) for x with (x - m) a >= -1000, in three steps less: the nearest whole number is left in the low bits of a
  // sum with 1.5 2^52, and added to the exponent.
  __device__ __forceinline__ double near(float x, double m, double a) const {
    constexpr double kWhole = 6755399441055744.0;
    const double d = (double)x - m, u = fma(d, a, kWhole), f = fma(d, a, kWhole - u);
    double g = c[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) g = fma(g, f, c[i]);
    g = fma(g, f, 1.0);
    return __hiloint2double(__double2hiint(g) + (__double2loint(u) << 20), __double2loint(g));
  }
};

// the weight of x against a finite maximum m
__device__ __forceinline__ double weight(float x, float m, double a, const Pow2 &pow2 = Pow2()) {
  return pow2(((double)x - (double)m) * a);
}

__device__ __forceinline__ float widen(uint32_t x) { return __uint_as_float(x); }
__device__ __forceinline__ float widen(uint16_t x) { return bf16_to_f32(x); }

// A row as segments of aligned 16-byte pieces: element i of segment s has the id s * kSeg + i - before.  Where the
// maximum is +infinity, its equals are read as 0 and the rest as -infinity.
// raw: as they are, NaN too (a maximum and pow2 take no notice of it).
template <typename T, bool raw = false>
struct RowAt {
  static constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;   // -infinity in every element of a word
  const T *base;
  int before, V;
  bool infinite;

  __device__ __forceinline__ float at(T x) const {
    const float v = widen(x);
    if (raw) return v;
    if (infinite) return v == INFINITY ? 0.0f : -INFINITY;
    return v == v ? v : -INFINITY;   // (NaN: never chosen)
  }
};
template <typename T, bool raw = false>
__device__ __forceinline__ RowAt<T, raw> row_at(const Logits &l, int row) {
  const char *p = l.p + row * l.stride;
  RowAt<T, raw> r;
  r.before = (int)(reinterpret_cast<uintptr_t>(p) % 16) / (int)sizeof(T);
  r.base = reinterpret_cast<const T *>(p) - r.before;
  r.V = l.V;
  r.infinite = false;
  return r;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int N, typename T, bool raw>
__device__ __forceinline__ void unpack(const RowAt<T, raw> &r, u32x4 w, float *x) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 4)
      x[i] = r.at(w[i]);
    else
      x[i] = r.at((uint16_t)(w[i / 2] >> (16 * (i & 1))));
  }
}

template <int N, typename T, bool raw>
__device__ __forceinline__ bool inside(const RowAt<T, raw> &r, int at) {
  return at >= r.before && at + N <= r.before + r.V;
}

// A piece at the row's beginning or end: the elements that are not the row's are -infinity.
template <typename T, bool raw>
__device__ __forceinline__ u32x4 edge_piece(const RowAt<T, raw> &r, int at) {
  constexpr int kPiece = 16 / sizeof(T);
  u32x4 w = {r.none, r.none, r.none, r.none};
#pragma unroll
  for (int i = 0; i < kPiece; ++i)
    if (at + i >= r.before && at + i < r.before + r.V) {
      const uint32_t x = r.base[at + i];
      if constexpr (sizeof(T) == 4)
        w[i] = x;
      else
        w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | x << 16 : (w[i / 2] & 0xffff0000u) | x;
    }
  return w;
}

// A piece's elements from place `at`; those that are not the row's: -infinity
template <int N, typename T, bool raw>
__device__ __forceinline__ void load_run(const RowAt<T, raw> &r, int at, float *x) {
  static_assert(N == 16 / sizeof(T), "a piece");
  unpack<N>(r, inside<N>(r, at) ? *reinterpret_cast<const u32x4 *>(r.base + at) : edge_piece(r, at), x);
}

// a thread's share of a segment, in the order of ids
constexpr int kOwn = kSeg / kRowThreads;
template <typename T>
__device__ __forceinline__ void load_own(const RowAt<T> &r, int seg, float (&x)[kOwn]) {
  constexpr int kPiece = 16 / sizeof(T);
#pragma unroll
  for (int j = 0; j < kOwn; j += kPiece) load_run<kPiece>(r, seg * kSeg + kOwn * (int)threadIdx.x + j, x + j);
}

// The place of piece j of a lane in a segment's order: lane l holds pieces l + 64 j.
template <typename T>
__device__ __forceinline__ int piece_at(int seg, int lane, int j) {
  return seg * kSeg + (j * 64 + lane) * (16 / (int)sizeof(T));
}
template <typename T, bool raw>
__device__ __forceinline__ void load_segment(const RowAt<T, raw> &r, int seg, float (&x)[kLane]) {
  constexpr int kPiece = 16 / sizeof(T);
  if (seg * kSeg >= r.before && (seg + 1) * kSeg <= r.before + r.V) {   // (the same for the whole wave)
    u32x4 w[kLane / kPiece];
#pragma unroll
    for (int j = 0; j < kLane / kPiece; ++j)
      w[j] = *reinterpret_cast<const u32x4 *>(r.base + piece_at<T>(seg, threadIdx.x & 63, j));
#pragma unroll
    for (int j = 0; j < kLane / kPiece; ++j) unpack<kPiece>(r, w[j], x + j * kPiece);
    return;
  }
#pragma unroll 1
  for (int j = 0; j < kLane / kPiece; ++j) {
    float y[kPiece];
    load_run<kPiece>(r, piece_at<T>(seg, threadIdx.x & 63, j), y);
#pragma unroll
    for (int i = 0; i < kLane; ++i)
      if (i / kPiece == j) x[i] = y[i % kPiece];
  }
}

// A segment, or a part of it, by a wave, piece by piece from the wave's own LDS: short code for kernels that run once on most CUs
// (bins_kernel at 17 rows of 151,936 in fp32: 12.2 -> 11.0 us).
template <typename T, int kWavesEach>
struct Staged {
  static constexpr int kPiece = 16 / sizeof(T), kPieces = kLane / kPiece / kWavesEach;
  u32x4 *at;   // [kPieces][64]
  int first;   // piece

  __device__ __forceinline__ Staged(u32x4 *lds, const RowAt<T> &r, int seg, int part)
      : at(lds + (threadIdx.x & 63)), first(part * kPieces) {
    u32x4 w[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int place = piece_at<T>(seg, threadIdx.x & 63, first + j);
      w[j] = u32x4{r.none, r.none, r.none, r.none};
      if (inside<kPiece>(r, place)) w[j] = *reinterpret_cast<const u32x4 *>(r.base + place);
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) at[j * 64] = w[j];
    if (seg * kSeg >= r.before && (seg + 1) * kSeg <= r.before + r.V) return;
#pragma unroll 1
    for (int j = 0; j < kPieces; ++j) {
      const int place = piece_at<T>(seg, threadIdx.x & 63, first + j);
      if (!inside<kPiece>(r, place)) at[j * 64] = edge_piece(r, place);
    }
  }
  // f(element, its place) for all of the lane's
  template <typename F>
  __device__ __forceinline__ void each(const RowAt<T> &r, int seg, F f) const {
#pragma unroll 1
    for (int j = 0; j < kPieces; ++j) {
      float x[kPiece];
      unpack<kPiece>(r, at[j * 64], x);
#pragma unroll
      for (int i = 0; i < kPiece; ++i) f(x[i], piece_at<T>(seg, threadIdx.x & 63, first + j) + i);
    }
  }
};

// ---- over a wave, by moves between its lanes ----
template <int ctrl, int rows>
__device__ __forceinline__ int moved(int x, int none) {
  return __builtin_amdgcn_update_dpp(none, x, ctrl, rows, 0xf, false);
}
template <int ctrl, int rows>
__device__ __forceinline__ double moved(double x, double none) {
  return __hiloint2double(moved<ctrl, rows>(__double2hiint(x), __double2hiint(none)),
                          moved<ctrl, rows>(__double2loint(x), __double2loint(none)));
}
template <int ctrl, int rows>
__device__ __forceinline__ u64 moved(u64 x, u64 none) {
  return (u64)(uint32_t)moved<ctrl, rows>((int)(x >> 32), (int)(none >> 32)) << 32 |
         (uint32_t)moved<ctrl, rows>((int)x, (int)none);
}
// f over the lanes up to and with this one (rows of 16 lanes, then across them); none: f's neutral element
template <typename N, typename F>
__device__ __forceinline__ N wave_scan(N x, N none, F f) {
  x = f(x, moved<0x111, 0xf>(x, none));
  x = f(x, moved<0x112, 0xf>(x, none));
  x = f(x, moved<0x114, 0xf>(x, none));
  x = f(x, moved<0x118, 0xf>(x, none));
  x = f(x, moved<0x142, 0xa>(x, none));
  return f(x, moved<0x143, 0xc>(x, none));
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }
__device__ __forceinline__ double last_lane(double x) {
  return __hiloint2double(last_lane(__double2hiint(x)), last_lane(__double2loint(x)));
}
__device__ __forceinline__ double wave_sum(double x) {
  return last_lane(wave_scan(x, 0.0, [](double a, double b) { return a + b; }));
}

// A segment by a wave: the maxima of its groups to maxima[0 .. n), and where the row needs it the sum of its
// weights against its own maximum to *sum (a short row's segment: its maximum to *top).
template <bool kShort, typename T>
__device__ __forceinline__ void summarise(const RowAt<T, true> &r, int seg, const Row &ask, float *maxima, double *sum,
                                          float *top = nullptr) {
  constexpr int kGroupLanes = Groups<kShort>::lanes;
  const int lane = threadIdx.x & 63;
  float x[kLane];
  load_segment(r, seg, x);
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kLane; ++i) m = fmaxf(m, x[i]);
  for (int o = 1; o < kGroupLanes; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (lane % kGroupLanes == 0) maxima[lane / kGroupLanes] = m;
  if (!kShort && !ask.sums()) return;
  for (int o = kGroupLanes; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  if (kShort && lane == 0) *top = m;
  if (kShort && !ask.sums()) return;
  double z = 0.0;
  m = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(m)));
  if (m > -INFINITY) {
    const Pow2 pow2;
    if (m == INFINITY) {
#pragma unroll
      for (int i = 0; i < kLane; ++i) z += x[i] == m;
    } else {
      // (what lies further below counts as 2^-990: masked elements, NaN; the sum is 1 or more)
      const float lo = (float)((double)m - 990.0 / ask.a);
      const double down = ((double)lo - (double)m) * ask.a;
      if (down >= -1000.0 && down <= -900.0) {   // (not where fp32 has no such value)
#pragma unroll
        for (int i = 0; i < kLane; ++i) z += pow2.near(fmaxf(x[i], lo), m, ask.a);
      } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i) z += pow2(((double)x[i] - (double)m) * ask.a);
      }
    }
    z = wave_sum(z);
  }
  if (lane == 0) *sum = z;
}

// grid: rows x groups of kWaves segments
template <typename T>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(7))) void segments_kernel(
    Logits l, Settings s, int groups, float *maxima, double *sums, int *large) {
  if (blockIdx.x == 0 && threadIdx.x == 0) *large = 0;
  const int row = blockIdx.x / groups;
  const int seg = (int)(blockIdx.x % groups) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (seg >= l.segs) return;
  const int64_t at = (int64_t)row * l.segs + seg;
  summarise<false>(row_at<T, true>(l, row), seg, row_of(s, row, l.V), maxima + at * Groups<false>::n, sums + at);
}

// Sums over a workgroup in the order of its threads: what comes before a thread, and the whole.
template <typename N>
__device__ __forceinline__ N before_thread(N x, N *tmp, N *whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const N run = wave_scan(x, (N)0, [](N a, N b) { return a + b; });
  __syncthreads();
  if (lane == 63) tmp[wave] = run;
  __syncthreads();
  N first = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    const N t = tmp[w];
    if (w < wave) first += t;
    all += t;
  }
  *whole = all;
  return first + (run - x);
}

__device__ __forceinline__ int block_min(int x, int *tmp) {
  x = last_lane(wave_scan(x, 0x7fffffff, [](int a, int b) { return min(a, b); }));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) x = min(x, tmp[w]);
  return x;
}
// floats by their order (no NaN)
__device__ __forceinline__ float block_max(float x, int *tmp) {
  const int top = block_min(~(int)(ordered_bits(x) ^ 0x80000000u), tmp);
  return ordered_to_float((uint32_t)~top ^ 0x80000000u);
}
__device__ __forceinline__ float block_min(float x, int *tmp) {
  const int low = block_min((int)(ordered_bits(x) ^ 0x80000000u), tmp);
  return ordered_to_float((uint32_t)low ^ 0x80000000u);
}

// Whole numbers in bins, found again by their running sums.
struct Bins {
  uint32_t count[kBins];
  u64 mass[kBins];
};

struct Shared {
  float groups[kMaxSegs * Groups<false>::n];  // maxima
  double mass[kMaxSegs];             // of a segment's kept elements
  double sums[kFewSegs];             // of a short row's segments: sums, maxima
  float tops[kFewSegs];
  int ties[kMaxSegs];                // its elements at the border
  Bins bins;                         // or arrays of their size
  u64 list[kList + kPad];            // keys (make_key) of candidates
  double tmp_d[kRowWaves];
  u64 tmp_u[kRowWaves];
  int tmp_i[kRowWaves];
  int at, n;
  u64 u;
  double before;
};

// What the large rows of a call pass from one launch to the next, in the order in which they are found.
struct Large {
  int row;
  int on;            // 1: the border is looked for in bins; 2: all from `lo` on is kept
  float m, lo, scale;
  double whole;
  int infinite, listed;
};

struct Work {
  Large *large;  // [rows], NULL: no row of the call can be one
  int *count;    // of them
  u64 *bins;     // of each: [kBins]
  u64 *list;     // [kList] the elements in the border's bin
  u64 *above;    // the mass before that bin
};

// Where an order's prefix ends: elements above `key` are kept, and `ties` of those equal to it.
struct Border {
  uint32_t key;
  int ties;
};

__device__ __forceinline__ u64 whole_number(double w) { return (u64)(w * kOne + 0.5); }

// bins of equal ranges of values from m down, monotone in x (differences past fp32's range, which meet a scale of 0: the last)
__device__ __forceinline__ int bin_of(float x, float m, float scale) {
  return (int)fminf((m - x) * scale, (float)(kBins - 1));
}
// the scale with which they reach down to lo: 2^100 at most, so that it is finite and a bin's range a normal number where
// all values lie within a hair of m
__device__ __forceinline__ float scale_of(float m, float lo) {
  return m > lo ? fminf((float)(kBins - 1) / (m - lo), 0x1p100f) : 0.0f;
}

// One workgroup's view of its row.
template <typename T, bool kShort>
struct Finish {
  static constexpr int kGroupLanes = Groups<kShort>::lanes, kGroups = Groups<kShort>::n;
  Shared &sh;
  RowAt<T> r;
  Row ask;
  int segs;
  float m;
  Pow2 pow2;

  __device__ __forceinline__ double weight_of(float x) const { return pow2(((double)x - (double)m) * ask.a); }

  __device__ __forceinline__ float segment_max(int seg) const {
    if (kShort) return sh.tops[seg];
    float x = sh.groups[seg * kGroups];
#pragma unroll 8
    for (int g = 1; g < kGroups; ++g) x = fmaxf(x, sh.groups[seg * kGroups + g]);
    return x;
  }

  // By the waves, for every segment with an element >= lo: piece(its elements) by every lane, piece after piece, then
  // done(segment).  All pieces are asked for first; they are kept apart, so that few registers are in use at once (these are
  // the slow rows' loops, and share a kernel with the others).
  template <typename F, typename G>
  __device__ __forceinline__ void each_segment(float lo, F piece, G done) {
    constexpr int kPiece = 16 / sizeof(T), kPieces = kLane / kPiece;
    for (int seg = threadIdx.x >> 6; seg < segs; seg += kRowWaves) {
      const float top = segment_max(seg);
      if (top < lo || top == -INFINITY) continue;
      u32x4 w[kPieces];
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        const int place = piece_at<T>(seg, threadIdx.x & 63, j);
        w[j] = u32x4{r.none, r.none, r.none, r.none};
        if (inside<kPiece>(r, place)) w[j] = *reinterpret_cast<const u32x4 *>(r.base + place);
      }
      const bool whole = seg * kSeg >= r.before && (seg + 1) * kSeg <= r.before + r.V;
#pragma unroll 1
      for (int j = 0; j < kPieces; ++j) {
        u32x4 now = w[0];
#pragma unroll
        for (int i = 0; i + 1 < kPieces; ++i) w[i] = w[i + 1];   // (the next one's turn)
        const int place = piece_at<T>(seg, threadIdx.x & 63, j);
        if (!whole && !inside<kPiece>(r, place)) now = edge_piece(r, place);
        float x[kPiece];
        unpack<kPiece>(r, now, x);
        piece(x);
      }
      done(seg);
    }
  }

  __device__ __forceinline__ void clear_bins() {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kRowThreads) sh.bins.count[i] = 0, sh.bins.mass[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void add(int bin, double w) {
    atomicAdd(&sh.bins.count[bin], 1u);
    atomicAdd(&sh.bins.mass[bin], whole_number(w));
  }
  // The same by all lanes of a wave that are here, whose elements may be equal: the equals of the first lane's are added once
  // (a row of equal logits would have its lanes wait for one another: 870 us for 151,936).
  __device__ __forceinline__ void add_equals(uint32_t key, int bin, bool by_mass, float x) {
    const u64 same = __ballot(key == (uint32_t)__builtin_amdgcn_readfirstlane((int)key));
    const int lane = threadIdx.x & 63;
    int n = 1;
    if (same >> lane & 1) n = lane == __ffsll((long long)same) - 1 ? __popcll(same) : 0;
    if (n == 0) return;
    atomicAdd(&sh.bins.count[bin], (uint32_t)n);
    if (by_mass) atomicAdd(&sh.bins.mass[bin], (u64)n * whole_number(weight_of(x)));
  }

  // The first bin at which f(elements, mass up to and with it) holds; the last that has any, if none.  *n_before,
  // *w_before: what lies before it; *all: all masses.
  template <typename F>
  __device__ __forceinline__ int find_bin(F f, int *n_before, u64 *w_before, u64 *all) {
    __syncthreads();
    constexpr int kEach = kBins / kRowThreads;
    uint32_t n[kEach];
    u64 w[kEach], sum_w = 0, all_w;
    int sum_n = 0, all_n;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      n[i] = sh.bins.count[kEach * threadIdx.x + i];
      w[i] = sh.bins.mass[kEach * threadIdx.x + i];
      sum_n += (int)n[i];
      sum_w += w[i];
    }
    const int before_n = before_thread(sum_n, sh.tmp_i, &all_n);
    const u64 before_w = before_thread(sum_w, sh.tmp_u, &all_w);
    int mine = 2 * kBins, run_n = before_n;
    u64 run_w = before_w;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      run_n += (int)n[i];
      run_w += w[i];
      if (!n[i]) continue;
      const int at = kEach * (int)threadIdx.x + i;
      if (f(run_n, run_w)) mine = min(mine, at);
      else if (run_n == all_n) mine = min(mine, at + kBins);   // (the last)
    }
    const int found = block_min(mine, sh.tmp_i), bin = found % kBins;
    if (mine == found && found < 2 * kBins) {
      int at_n = before_n;
      u64 at_w = before_w;
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (kEach * (int)threadIdx.x + i < bin) at_n += (int)n[i], at_w += w[i];
      sh.at = at_n;
      sh.u = at_w;
    }
    __syncthreads();
    *n_before = sh.at;
    *w_before = sh.u;
    *all = all_w;
    return found < 2 * kBins ? bin : -1;
  }

  // The border of the first `want` elements (by_mass: of the elements before which the mass is below `want`), known to
  // lie at keys >= key(lo), by passes over the row: bins of equal ranges of keys, then of the border's
  // bin, until a bin is a key.  Right for every row, and the slowest way.
  __device__ __forceinline__ Border select(bool by_mass, double want, float lo_value) {
    uint32_t lo = ordered_bits(lo_value), hi = ordered_bits(m);
    int above_n = 0;
    u64 above_w = 0;
    for (;;) {
      const int shift = max(0, 32 - __clz((int)(hi - lo)) - 11);
      clear_bins();
      each_segment(ordered_to_float(lo), [&](const float(&x)[16 / sizeof(T)]) __attribute__((always_inline)) {
#pragma unroll
        for (const float v : x) {
          const uint32_t key = ordered_bits(v);
          if (key < lo || key > hi || v == -INFINITY) continue;
          add_equals(key, (int)((hi - key) >> shift), by_mass, v);
        }
      }, [](int) {});
      int n;
      u64 w, all;
      const int b = find_bin([&](int run_n, u64 run_w) {
        return by_mass ? (double)(above_w + run_w) / kOne >= want : (double)above_n + run_n >= want;
      }, &n, &w, &all);
      above_n += n;
      above_w += w;
      const int here = (int)sh.bins.count[b];
      __syncthreads();
      hi -= (uint32_t)b << shift;
      lo = max(lo, hi - min(hi, (1u << shift) - 1));
      if (shift == 0) {
        Border o;
        o.key = lo;
        const double w1 = weight_of(ordered_to_float(lo)), mass = (double)above_w / kOne;
        double ties = by_mass ? ceil((want - mass) / w1) : want - above_n;
        if (!(ties < (double)here)) ties = here;   // (NaN: a weight of 0)
        o.ties = max((int)ties, above_n > 0 ? 0 : 1);
        return o;
      }
    }
  }

  // The kept mass of every segment: what lies above the border and, in the order of ids, the ties.
  __device__ __forceinline__ void segment_masses(const Border &edge, float lo) {
    __syncthreads();
    for (int i = threadIdx.x; i < segs; i += kRowThreads) sh.mass[i] = 0.0, sh.ties[i] = 0;
    __syncthreads();
    double z = 0.0;
    int ties = 0;
    each_segment(lo, [&](const float(&x)[16 / sizeof(T)]) __attribute__((always_inline)) {
#pragma unroll
      for (const float v : x) {
        const uint32_t key = ordered_bits(v);
        if (v < lo || v == -INFINITY) continue;
        if (key == edge.key) {
          ++ties;
        } else if (key > edge.key) {
          const double w = weight_of(v);
          if (w >= ask.q) z += w;
        }
      }
    }, [&](int seg) {
      z = wave_sum(z);
      for (int o = 1; o < 64; o <<= 1) ties += __shfl_xor(ties, o);
      if ((threadIdx.x & 63) == 0) sh.mass[seg] = z, sh.ties[seg] = ties;
      z = 0.0;
      ties = 0;
    });
    __syncthreads();
    if (!edge.key) return;
    double w = weight_of(ordered_to_float(edge.key));
    if (w < ask.q) w = 0.0;
    int t = 0, all;
    const int each = (segs + kRowThreads - 1) / kRowThreads, first = (int)threadIdx.x * each;
    for (int i = first; i < min(first + each, segs); ++i) t += sh.ties[i];
    int run = before_thread(t, sh.tmp_i, &all);
    for (int i = first; i < min(first + each, segs); ++i) {
      sh.mass[i] += min(max(edge.ties - run, 0), sh.ties[i]) * w;
      run += sh.ties[i];
    }
    __syncthreads();
  }

  // The element where the running sum of kept weights, in the order of ids, passes u of the whole: segment masses are in
  // sh.mass, ties in sh.ties.  All threads return it; own: its weight, whole: of all kept.
  __device__ __forceinline__ int pick(double u, const Border &edge, double *own, double *whole) {
    double z = 0.0, left = 0.0;
    int tied = 0;
    const int each = (segs + kRowThreads - 1) / kRowThreads, first = (int)threadIdx.x * each;
    double x = 0.0;
    int t = 0, n_all;
    for (int i = first; i < min(first + each, segs); ++i) x += sh.mass[i], t += sh.ties[i];
    double run = before_thread(x, sh.tmp_d, &z);
    int run_t = before_thread(t, sh.tmp_i, &n_all);
    const double at = u * z;
    int mine = segs, last = 0;
    for (int i = first; i < min(first + each, segs); ++i) {
      if (run + sh.mass[i] > at && sh.mass[i] > 0.0 && mine == segs) {
        mine = i;
        left = run;
        tied = run_t;
      }
      run += sh.mass[i];
      run_t += sh.ties[i];
    }
    const int seg = block_min(mine, sh.tmp_i);
    if (seg == segs) return -1;   // (no weight anywhere: not with a maximum)
    if (mine == seg) sh.before = left, sh.at = tied;
    __syncthreads();
    left = sh.before;
    tied = sh.at;
    constexpr int kEach = kOwn;
    float v[kEach];
    load_own(r, seg, v);
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
        w[i] = weight_of(v[i]);
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

  // ---- rows of which few elements can be kept: a list of them in LDS ----

  // Of the list's elements, in their order, the last one before which the mass is below `want`.
  __device__ __forceinline__ u64 last_below(double want) {
    constexpr int kEach = kList / kRowThreads;
    const int tid = threadIdx.x, n = sh.n;
    put_in_order(sh.list, n, (u64)0, [](u64 a, u64 b) { return a > b; });
    double w[kEach], sum = 0.0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = kEach * tid + i;
      w[i] = at < n ? weight_of(key_value(sh.list[at])) : 0.0;
      sum += w[i];
    }
    double before = before_thread(sum, sh.tmp_d, &all);
    int first_out = n;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = kEach * tid + i;
      if (at > 0 && !(before < want)) first_out = min(first_out, at);
      before += w[i];
    }
    return sh.list[block_min(first_out, sh.tmp_i) - 1];
  }

  // n numbers of LDS, all different, in order (more(a, b): a comes first), by counting those before each one.  kMine
  // numbers a thread; where there are fewer, several threads share a number's count.  `last`: a number that comes after all,
  // which fills the list up to whole 16-byte reads (kPad numbers more than n).
  template <int kMine, typename N, typename F>
  __device__ __forceinline__ void put_in_order(N *list, int n, N last, F more) {
    constexpr int kRead = 16 / sizeof(N);
    const int tid = threadIdx.x;
    int split = 1;
    if (kMine == 1)
      while (split < 16 && n * split * 2 <= kRowThreads) split *= 2;
    if (tid < kPad) list[n + tid] = last;
    __syncthreads();
    const int e = tid / split, part = tid % split, reads = (n + split * kRead - 1) / (split * kRead);
    N mine[kMine];
    int rank[kMine] = {};
#pragma unroll
    for (int i = 0; i < kMine; ++i) mine[i] = list[min(e + i * kRowThreads, n)];
    typedef N Read __attribute__((ext_vector_type(kRead)));
#pragma unroll 4
    for (int j = 0; j < reads; ++j) {
      const Read x = *reinterpret_cast<const Read *>(list + (j * split + part) * kRead);
#pragma unroll
      for (int v = 0; v < kRead; ++v)
#pragma unroll
        for (int i = 0; i < kMine; ++i) rank[i] += more(x[v], mine[i]);
    }
    if (kMine == 1)
      for (int o = 1; o < split; o <<= 1) rank[0] += __shfl_xor(rank[0], o);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if (e + i * kRowThreads < n && part == 0) list[rank[i]] = mine[i];
    __syncthreads();
  }
  template <typename N, typename F>
  __device__ __forceinline__ void put_in_order(N *list, int n, N last, F more) {
    if (n <= kRowThreads)
      put_in_order<1>(list, n, last, more);
    else if (n <= 2 * kRowThreads)
      put_in_order<2>(list, n, last, more);
    else
      put_in_order<kList / kRowThreads>(list, n, last, more);
  }

  // Of the list (all elements >= lo of the row): the token.  kEach elements a thread.
  template <int kEach>
  __device__ __forceinline__ void from_list(double u, double whole, int *token, double *own, double *kept) {
    const int tid = threadIdx.x, n = sh.n;
    put_in_order(sh.list, n, (u64)0, [](u64 a, u64 b) { return a > b; });
    uint32_t *const by_id = sh.bins.count;
    double *const weights = reinterpret_cast<double *>(sh.bins.mass);
    u64 key[kEach];
    double w[kEach], sum = 0.0, z;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = kEach * tid + i;
      key[i] = at < n ? sh.list[at] : 0;
      w[i] = at < n && (!ask.k || at < ask.k) ? weight_of(key_value(key[i])) : 0.0;
      sum += w[i];
    }
    double before = 0.0, want = INFINITY;
    if (ask.p <= 1.0) {
      before = before_thread(sum, sh.tmp_d, &z);
      want = ask.p * (ask.k ? z : whole);
    }
    // what is kept is the first few of the order
    int first_out = n;
#pragma unroll
    for (int i = kEach - 1; i >= 0; --i) {
      const int at = kEach * tid + i;
      double b = before;
#pragma unroll
      for (int j = 0; j < i; ++j) b += w[j];
      const bool in = at < n && (!ask.k || at < ask.k) && w[i] >= ask.q && (at == 0 || b < want);
      if (!in) first_out = min(first_out, at);
    }
    const int c = block_min(first_out, sh.tmp_i);
    // their running sums in the order of ids: an id with its place in the order
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = kEach * tid + i;
      if (at >= c) continue;
      weights[at] = w[i];
      by_id[at] = key_index(key[i]) << 10 | (uint32_t)at;
    }
    __syncthreads();
    put_in_order(by_id, c, 0xffffffffu, [](uint32_t a, uint32_t b) { return a < b; });
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = kEach * tid + i;
      w[i] = at < c ? weights[by_id[at] & (kList - 1)] : 0.0;
      sum += w[i];
    }
    double run = before_thread(sum, sh.tmp_d, &z);
    const double at = u * z;
    int mine = kList, last = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      run += w[i];
      if (w[i] > 0.0) last = kEach * tid + i;
      if (run > at && w[i] > 0.0 && mine == kList) mine = kEach * tid + i;
    }
    int found = block_min(mine, sh.tmp_i);
    if (found == kList) found = -block_min(-last, sh.tmp_i);   // (the sums' last bits)
    const uint32_t id = by_id[found];
    *own = weights[id & (kList - 1)];
    *token = (int)(id >> 10);
    *kept = z;
  }

  // The elements >= lo into the list, from the groups that have any; false: they are too many.
  __device__ __forceinline__ bool gather(float lo) {
    const int tid = threadIdx.x, n_groups = segs * kGroups;
    __syncthreads();
    if (tid == 0) sh.n = 0;
    int *const found = reinterpret_cast<int *>(sh.bins.mass);   // groups
    int mine = 0, c;
    for (int g = tid; g < n_groups; g += kRowThreads) mine += sh.groups[g] >= lo && sh.groups[g] > -INFINITY;
    int to = before_thread(mine, sh.tmp_i, &c);
    if (c > kList) return false;   // (an element each)
    for (int g = tid; g < n_groups; g += kRowThreads)
      if (sh.groups[g] >= lo && sh.groups[g] > -INFINITY) found[to++] = g;
    __syncthreads();
    // a group's pieces with neighbouring lanes.  (The code is kept short here and in what follows: a row passes through
    // once, so fetching instructions counts for more than running them.)
    constexpr int kPiece = 16 / sizeof(T), kPieces = kLane / kPiece * kGroupLanes, kAtOnce = 64 / kPiece;
    const auto place_of = [&](int i) {
      const int g = found[i / kPieces], piece = i % kPieces;
      return piece_at<T>(g / kGroups, g % kGroups * kGroupLanes + piece % kGroupLanes, piece / kGroupLanes);
    };
    const float bound = r.infinite ? INFINITY : lo;   // (of the elements as they are; NaN is not above it)
    for (int i0 = tid; i0 < (c * kPieces + kRowThreads - 1) / kRowThreads * kRowThreads; i0 += kAtOnce * kRowThreads) {
      u32x4 w[kAtOnce];   // (all in flight: a round takes as long as memory does)
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n) {
        const int i = i0 + n * kRowThreads;
        w[n] = u32x4{r.none, r.none, r.none, r.none};
        if (i >= c * kPieces) continue;
        const int at = place_of(i);
        if (inside<kPiece>(r, at)) w[n] = *reinterpret_cast<const u32x4 *>(r.base + at);
      }
      // 64 elements a lane: a bit each, the first element in the highest
      constexpr int kWords = kAtOnce * kPiece / 32;
      uint32_t hits[kWords] = {};
#pragma unroll
      for (int n = 0; n < kAtOnce; ++n)
#pragma unroll
        for (int j = 0; j < kPiece; ++j) {
          float x;
          if constexpr (sizeof(T) == 4)
            x = __uint_as_float(w[n][j]);
          else
            x = __uint_as_float(j & 1 ? w[n][j / 2] & 0xffff0000u : w[n][j / 2] << 16);
          uint32_t &h = hits[(n * kPiece + j) / 32];
          h = h + h + (x >= bound);
        }
      mine = 0;
#pragma unroll
      for (int h = 0; h < kWords; ++h) mine += __popc(hits[h]);
      int place = wave_scan(mine, 0, [](int a, int b) { return a + b; });
      const int all = last_lane(place);
      if (!all) continue;
      int base = 0;
      if ((tid & 63) == 0) base = atomicAdd(&sh.n, all);
      place += __builtin_amdgcn_readfirstlane(base) - mine;
#pragma unroll
      for (int h = 0; h < kWords; ++h)
        for (uint32_t left = hits[h]; left;) {
          const int bit = __clz((int)left), e = 32 * h + bit;
          left &= ~(0x80000000u >> bit);
          const int at = place_of(i0 + e / kPiece * kRowThreads) + e % kPiece;
          if (place < kList) sh.list[place] = make_key(r.at(r.base[at]), (uint32_t)(at - r.before));
          ++place;
        }
    }
    // the pieces at the row's beginning and end
#pragma unroll 1
    for (int i = tid; i < c * kPieces; i += kRowThreads) {
      const int at = place_of(i);
      if (inside<kPiece>(r, at)) continue;
#pragma unroll 1
      for (int e = max(at, r.before); e < min(at + kPiece, r.before + r.V); ++e) {
        const float x = r.at(r.base[e]);
        if (!(x >= lo)) continue;
        const int place = atomicAdd(&sh.n, 1);
        if (place < kList) sh.list[place] = make_key(x, (uint32_t)(e - r.before));
      }
    }
    __syncthreads();
    return sh.n <= kList;
  }

  // reach() by the order of the maxima of kTops parts of the groups, where they suffice.
  template <int kTops>
  __device__ __forceinline__ float reach_of_few(bool by_mass, double want, bool *far) {
    constexpr int kSplit = kRowThreads / kTops;   // threads a maximum
    const int tid = threadIdx.x, e = tid / kSplit, part = tid % kSplit;
    float top = -INFINITY;
    for (int g = tid; g < segs * kGroups; g += kRowThreads) top = fmaxf(top, sh.groups[g]);
    for (int o = 1; o < kSplit; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    // (their ordered bits with a number in the last eight: all different, and no value is above its maximum)
    static_assert(kTops <= 256, "eight bits of a number");
    uint32_t *const tops = sh.bins.count, *const order = tops + kTops;
    const uint32_t mine = (ordered_bits(top) & ~255u) | (uint32_t)e;
    if (part == 0) tops[e] = mine;
    __syncthreads();
    int rank = 0;
#pragma unroll 4
    for (int i = part * 4; i < kTops; i += 4 * kSplit) {
      const uint4 v = *reinterpret_cast<const uint4 *>(tops + i);
      rank += (v.x > mine) + (v.y > mine) + (v.z > mine) + (v.w > mine);
    }
    for (int o = 1; o < kSplit; o <<= 1) rank += __shfl_xor(rank, o);
    if (part == 0) order[rank] = mine;
    __syncthreads();
    const auto value_at = [&](int i) {
      const uint32_t bits = order[i] & ~255u;
      return bits > ordered_bits(-INFINITY) ? ordered_to_float(bits) : -INFINITY;
    };
    *far = false;
    if (!by_mass) return value_at((int)want - 1);
    const float x = tid < kTops ? value_at(tid) : -INFINITY;
    double all;
    const double w = x > -INFINITY ? weight_of(x) : 0.0, run = w + before_thread(w, sh.tmp_d, &all);
    *far = all < want * 0.25;
    const int at = block_min(run >= want ? tid : kRowThreads, sh.tmp_i);
    return at < kTops ? value_at(at) : -INFINITY;
  }

  // A value such that the elements >= it reach `want` (their number, or by_mass their weights): by the groups' maxima
  // alone, which is less than there is.  -infinity: not reached.
  __device__ __forceinline__ float reach(bool by_mass, double want) {
    // (few first, but for large numbers: 128 maxima are put in order sooner than all are put in bins, and bound fewer
    // elements as the number rises; one row of 151,936, in order / in bins: top-k 5 12.7 / 15.2 us, 50 13.3 / 16.0, and by the
    // order of 256 maxima top-k 100 17.5 / 18.1, 200 32.3 / 25.0; top-p 0.9 20.5 / 23.2; 544 rows 38 / 42, 40 / 44, 49 / 46,
    // 71 / 57, 167 / 166)
    bool far = false;
    float x = -INFINITY;
    if (by_mass || want <= 64.0) x = reach_of_few<128>(by_mass, want, &far);
    if (x > -INFINITY || far) return x;   // (far: more than the list holds are kept, as a rule)
    float low = m;
    const int n_groups = segs * kGroups;
    for (int g = threadIdx.x; g < n_groups; g += kRowThreads)
      if (sh.groups[g] > -INFINITY) low = fminf(low, sh.groups[g]);
    low = block_min(low, sh.tmp_i);
    const float scale = scale_of(m, low);
    clear_bins();
    for (int g = threadIdx.x; g < n_groups; g += kRowThreads)
      if (sh.groups[g] > -INFINITY) add(bin_of(sh.groups[g], m, scale), by_mass ? weight_of(sh.groups[g]) : 0.0);
    int n;
    u64 w, all;
    const auto holds = [&](int run_n, u64 run_w) { return by_mass ? (double)run_w / kOne >= want : (double)run_n >= want; };
    const int b = find_bin(holds, &n, &w, &all);
    if (holds(n + (int)sh.bins.count[b], w + sh.bins.mass[b])) {
      float least = m;
      for (int g = threadIdx.x; g < n_groups; g += kRowThreads)
        if (sh.groups[g] > -INFINITY && bin_of(sh.groups[g], m, scale) <= b) least = fminf(least, sh.groups[g]);
      return block_min(least, sh.tmp_i);
    }
    return kShort && !by_mass ? reach_of_all(want) : -INFINITY;
  }

  // reach() of a number by all elements (of a short row: two passes over it).
  __device__ __forceinline__ float reach_of_all(double want) {
    float low = m;
    each_segment(-INFINITY, [&](const float(&x)[16 / sizeof(T)]) __attribute__((always_inline)) {
#pragma unroll
      for (const float v : x) low = v > -INFINITY ? fminf(low, v) : low;
    }, [](int) {});
    low = block_min(low, sh.tmp_i);
    const float scale = scale_of(m, low);
    clear_bins();
    each_segment(-INFINITY, [&](const float(&x)[16 / sizeof(T)]) __attribute__((always_inline)) {
#pragma unroll
      for (const float v : x)
        if (v > -INFINITY) atomicAdd(&sh.bins.count[bin_of(v, m, scale)], 1u);
    }, [](int) {});
    int n;
    u64 w, all;
    const int b = find_bin([&](int run_n, u64) { return (double)run_n >= want; }, &n, &w, &all);
    // (below every value of the bin: what lies further down only makes the list longer)
    return scale > 0.0f ? m - (float)(b + 2) / scale : -INFINITY;
  }

  // The row by passes over it.
  __device__ __forceinline__ int by_passes(double u, double whole, float lo, double *own, double *kept) {
    Border edge{0u, 0};
#pragma unroll 1
    for (int step = 0; step < 2; ++step) {   // top-k, then top-p (the passes' code once)
      if (step ? !(ask.p <= 1.0) : !ask.k) continue;
      edge = select(step, step ? ask.p * whole : (double)ask.k, lo);
      lo = fmaxf(ordered_to_float(edge.key), lo);
      if (step == 0 && ask.p <= 1.0) {   // (top-p's whole: the mass of all k, whatever min_p leaves of it)
        const double q = ask.q;
        ask.q = 0.0;
        segment_masses(edge, lo);
        ask.q = q;
        double x = 0.0;
        for (int i = threadIdx.x; i < segs; i += kRowThreads) x += sh.mass[i];
        before_thread(x, sh.tmp_d, &whole);
      }
    }
    segment_masses(edge, lo);
    return pick(u, edge, own, kept);
  }
};

__device__ __forceinline__ double number_of(const float *u, int row) { return fmin(fmax((double)u[row], 0.0), 0.99999999999); }

__device__ __forceinline__ void answer(int row, int token, double own, double whole, int32_t *tokens, float *logprobs) {
  if (threadIdx.x != 0) return;
  tokens[row] = token;
  if (logprobs) logprobs[row] = (float)log(own / whole);
}

// grid: rows.  kShort: the row is read here, and no segments_kernel came before (maxima, sums: not looked at).
template <typename T, bool kShort>
__global__ __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(3))) void row_kernel(Logits l, Settings s, const float *u, const float *maxima,
                                                          const double *sums, Work work, int32_t *tokens,
                                                          float *logprobs) {
  __shared__ Shared sh;
  const int row = blockIdx.x, tid = threadIdx.x;
  constexpr int kGroups = Groups<kShort>::n;
  Finish<T, kShort> f{sh, row_at<T>(l, row), row_of(s, row, l.V), l.segs, 0.0f};
  Row &ask = f.ask;
  const int64_t first = (int64_t)row * l.segs;
  float m = -INFINITY;
  if constexpr (kShort) {
    const RowAt<T, true> raw = row_at<T, true>(l, row);
    for (int seg = __builtin_amdgcn_readfirstlane(tid >> 6); seg < l.segs; seg += kRowWaves)
      summarise<kShort>(raw, seg, ask, sh.groups + seg * kGroups, sh.sums + seg, sh.tops + seg);
    __syncthreads();
    if (tid < l.segs) m = sh.tops[tid];
  } else {
    for (int i0 = tid; i0 < l.segs * kGroups; i0 += 8 * kRowThreads) {
      float x[8];
  #pragma unroll
      for (int n = 0; n < 8; ++n) {
        const int i = i0 + n * kRowThreads;
        x[n] = i < l.segs * kGroups ? maxima[first * kGroups + i] : -INFINITY;
      }
  #pragma unroll
      for (int n = 0; n < 8; ++n) {
        const int i = i0 + n * kRowThreads;
        if (i < l.segs * kGroups) sh.groups[i] = x[n];
        m = fmaxf(m, x[n]);
      }
    }
  }
  m = block_max(m, sh.tmp_i);
  if (m == INFINITY) {
    f.r.infinite = true;
    for (int i = tid; i < l.segs * kGroups; i += kRowThreads) sh.groups[i] = sh.groups[i] == INFINITY ? 0.0f : -INFINITY;
    if (kShort && tid < l.segs) sh.tops[tid] = sh.tops[tid] == INFINITY ? 0.0f : -INFINITY;
    m = 0.0f;
  }
  f.m = m;
  __syncthreads();
  int token = -1;
  double own = 1.0, whole = 1.0;
  bool large = false;
  if (m == -INFINITY) {
    own = 0.0;
  } else if (ask.greedy) {
    int group = l.segs * kGroups;
    for (int i = tid; i < l.segs * kGroups; i += kRowThreads)
      if (sh.groups[i] == m) group = min(group, i);
    const int seg = block_min(group, sh.tmp_i) / kGroups;
    constexpr int kEach = kOwn;
    float v[kEach];
    load_own(f.r, seg, v);
    int mine = kSeg;
#pragma unroll
    for (int i = kEach - 1; i >= 0; --i)
      if (v[i] == m) mine = kEach * tid + i;
    token = seg * kSeg + block_min(mine, sh.tmp_i) - f.r.before;
  } else {
    const double at = number_of(u, row);
    if (ask.sums()) {
      double z = 0.0;
      for (int i = tid; i < l.segs; i += kRowThreads) {
        const float top = f.segment_max(i);
        const double x = top > -INFINITY ? (kShort ? sh.sums[i] : sums[first + i]) * f.weight_of(top) : 0.0;
        sh.mass[i] = x;
        sh.ties[i] = 0;
        z += x;
      }
      before_thread(z, sh.tmp_d, &whole);
    }
    if (ask.filters()) {
      // below these nothing is kept: weights under min_p (and a little less), weights that all together are
      // less than 1 - top_p of the whole.  (top-p after top-k is of the mass of all k, those under min_p among them)
      double t = ask.q > 0.0 && !(ask.k && ask.p <= 1.0) ? log2(ask.q) - 1e-6 : -INFINITY;
      if (ask.p <= 1.0 && !ask.k) t = fmax(t, log2((1.0 - ask.p) * whole / l.V) - 1e-6);
      const double x = (double)m + t / ask.a;
      float lo = (float)(x - 1e-6 * fabs(x));
      if (!(lo <= m)) lo = -INFINITY;
      lo = fmaxf(lo, -3.4028235e38f);
      float near = lo;
      if (ask.k)
        near = fmaxf(near, f.reach(false, (double)ask.k));
      else if (ask.p <= 1.0)
        near = fmaxf(near, f.reach(true, ask.p * whole * (1.0 + 1e-9)));
      if (f.gather(near)) {
        if (sh.n <= kRowThreads)
          f.template from_list<1>(at, whole, &token, &own, &whole);
        else
          f.template from_list<kList / kRowThreads>(at, whole, &token, &own, &whole);
      } else {
        if (work.large && !ask.k) {
          large = true;
          __syncthreads();
          if (tid == 0) sh.at = atomicAdd(work.count, 1);
          __syncthreads();
          const int at_large = sh.at;
          if (tid == 0)
            work.large[at_large] = Large{row, ask.p <= 1.0 ? 1 : 2, m, lo, scale_of(m, lo), whole, f.r.infinite, 0};
          for (int i = tid; i < kBins; i += kRowThreads) work.bins[(int64_t)at_large * kBins + i] = 0;
        } else {
          token = f.by_passes(at, whole, near, &own, &whole);
        }
      }
    } else {
      token = f.pick(at, Border{0u, 0}, &own, &whole);
    }
  }
  if (!large) answer(row, token, own, whole, tokens, logprobs);
}

// ---- rows of which many elements are kept: the passes over all workgroups ----

// (each over the parts of the rows found, or the rows, by as many workgroups as are useful at once)

// The i-th of them; false: there are fewer.  (Asked for together with their number.)
__device__ __forceinline__ bool large_at(const Work &work, int rows, int i, Large *x) {
  if (i >= rows) return false;
  const int count = *work.count;
  *x = work.large[i];
  asm volatile("" : "+v"(x->row), "+v"(x->on), "+v"(x->lo));
  return i < count;
}

// Masses in bins of values, from m down to lo (17 rows of 151,936 in fp32: 11 us, of them a third its launch, reads that wait
// for one another; then 32 exponentials a lane and the bins' sums over the card).
template <typename T>
__global__ __launch_bounds__(64 * kPart) void bins_kernel(Logits l, Settings s, int parts, Work work) {
  __shared__ u64 bins[kBins];
  __shared__ u32x4 staged[kPart][kSeg * sizeof(T) / 16];
  for (int item = blockIdx.x;; item += gridDim.x) {
    Large x;
    const int at = item / parts;
    if (!large_at(work, l.rows, at, &x)) return;
    if (x.on != 1) continue;
    const int row = x.row;
    const int wave = threadIdx.x >> 6, seg = item % parts * kPart + wave;
    RowAt<T> r = row_at<T>(l, row);
    r.infinite = x.infinite;
    const Staged<T, 1> v(staged[wave], r, min(seg, l.segs - 1), 0);
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += 64 * kPart) bins[i] = 0;
    __syncthreads();
    if (seg < l.segs) {
      const Row ask = row_of(s, row, l.V);
      const Pow2 pow2;
      v.each(r, seg, [&](float y, int) __attribute__((always_inline)) {
        if (y >= x.lo) atomicAdd(&bins[bin_of(y, x.m, x.scale)], whole_number(weight(y, x.m, ask.a, pow2)));
      });
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += 64 * kPart)
      if (bins[i]) atomicAdd(&work.bins[(int64_t)at * kBins + i], bins[i]);
  }
}

// The border's bin (each workgroup finds it again); the mass of each segment's elements before it, and the elements in it into a
// list.
template <typename T>
__global__ __launch_bounds__(64 * kPart) void masses_kernel(Logits l, Settings s, int parts, double *masses, Work work) {
  __shared__ u64 tmp[kRowWaves];
  __shared__ int tmp_i[kRowWaves];
  __shared__ double halves[kPart];
  __shared__ u32x4 staged[kPart][kSeg * sizeof(T) / 32];
  static_assert(kPart == kRowWaves, "sums over a workgroup");
  const int tid = threadIdx.x;
  for (int item = blockIdx.x;; item += gridDim.x) {
    Large x;
    const int at = item / parts;
    if (!large_at(work, l.rows, at, &x)) return;
    const int row = x.row;
    const int wave = tid >> 6, seg = item % parts * (kPart / 2) + wave / 2;
    RowAt<T> r = row_at<T>(l, row);
    r.infinite = x.infinite;
    const Staged<T, 2> v(staged[wave], r, min(seg, l.segs - 1), wave & 1);   // (few rows: more SIMDs at work, 14.4 -> 12.0 us)
    const Row ask = row_of(s, row, l.V);
    int border = kBins;
    if (x.on == 1) {
      constexpr int kEach = kBins / (64 * kPart);
      u64 w[kEach], sum = 0, above = 0, all;
#pragma unroll
      for (int i = 0; i < kEach; ++i) sum += w[i] = work.bins[(int64_t)at * kBins + kEach * tid + i];
      u64 run = before_thread(sum, tmp, &all);
      const double want = ask.p * x.whole;
      int mine = kBins;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const u64 before = run;
        run += w[i];
        if (w[i] && (double)run / kOne >= want && mine == kBins) mine = kEach * tid + i, above = before;
      }
      border = block_min(mine, tmp_i);
      // (never reached: all is kept)
      if (border < kBins && border == mine && item % parts == 0) work.above[at] = above;
    }
    double z = 0.0;
    if (seg < l.segs) {
      const Pow2 pow2;
      int mine = 0;
      v.each(r, seg, [&](float y, int) __attribute__((always_inline)) {
        if (!(y >= x.lo)) return;
        const int b = bin_of(y, x.m, x.scale);
        if (b < border) {
          const double w = weight(y, x.m, ask.a, pow2);
          if (w >= ask.q) z += w;
        }
        mine += b == border;
      });
      int place = wave_scan(mine, 0, [](int a, int b) { return a + b; });
      const int listed = last_lane(place);
      if (listed) {   // (one atomic for the wave)
        int base = 0;
        if ((tid & 63) == 0) base = atomicAdd(&work.large[at].listed, listed);
        place += __builtin_amdgcn_readfirstlane(base) - mine;
        v.each(r, seg, [&](float y, int where) __attribute__((always_inline)) {
          if (!(y >= x.lo) || bin_of(y, x.m, x.scale) != border) return;
          if (place < kList) work.list[(int64_t)at * kList + place] = make_key(y, (uint32_t)(where - r.before));
          ++place;
        });
      }
      z = wave_sum(z);
    }
    __syncthreads();   // (the last item's halves have been read)
    if ((tid & 63) == 0) halves[wave] = z;
    __syncthreads();
    if ((tid & 127) == 0 && seg < l.segs) masses[(int64_t)row * l.segs + seg] = halves[wave] + halves[wave + 1];
  }
}

// The border among its bin's elements, and the token.
template <typename T>
__device__ __forceinline__ void finish_large(Shared &sh, int index, const Large &x, const Logits &l, const Settings &s, const float *u, const float *maxima,
                             const double *masses, const Work &work, int32_t *tokens, float *logprobs) {
  const int tid = threadIdx.x, row = x.row;
  __syncthreads();
  constexpr int kGroups = Groups<false>::n;
  Finish<T, false> f{sh, row_at<T>(l, row), row_of(s, row, l.V), l.segs, x.m};
  f.r.infinite = x.infinite;
  const int64_t first = (int64_t)row * l.segs;
  const double at = number_of(u, row);
  double own = 1.0, whole = x.whole;
  int token;
  const bool fits = x.listed <= kList;
  Border edge{0u, 0};
  if (fits) {
    if (tid == 0) sh.n = x.listed;
    for (int i = tid; i < x.listed; i += kRowThreads) sh.list[i] = work.list[(int64_t)index * kList + i];
    for (int i = tid; i < l.segs; i += kRowThreads) sh.mass[i] = masses[first + i], sh.ties[i] = 0;
    __syncthreads();
    if (x.listed) {
      const u64 border = f.last_below(f.ask.p * x.whole - (double)work.above[index] / kOne);
      {
        // the kept ones of the bin join their segments (whole numbers: in any order); of the border's equals only those
        // up to it are kept
        u64 *const more = sh.bins.mass;
        __syncthreads();
        for (int i = tid; i < l.segs; i += kRowThreads) more[i] = 0;
        __syncthreads();
        if (tid == 0) sh.at = 0;
        __syncthreads();
        edge.key = ordered_bits(key_value(border));
        for (int i = tid; i < x.listed; i += kRowThreads) {
          const u64 key = sh.list[i];
          const uint32_t bits = (uint32_t)(key >> 32);
          const int seg = ((int)key_index(key) + f.r.before) / kSeg;
          if (bits == edge.key) atomicAdd(&sh.ties[seg], 1);
          if (key < border) continue;
          if (bits == edge.key) atomicAdd(&sh.at, 1);
          const double w = f.weight_of(key_value(key));
          if (w >= f.ask.q) atomicAdd(&more[seg], whole_number(w));
        }
        __syncthreads();
        edge.ties = sh.at;
        for (int i = tid; i < l.segs; i += kRowThreads) sh.mass[i] += (double)more[i] / kOne;
        __syncthreads();
      }
    }
  }
  if (fits) {
    if (!edge.key) edge = Border{ordered_bits(x.lo), 1 << 30};   // (all from lo on)
    token = f.pick(at, edge, &own, &whole);
  } else {
    __syncthreads();
    for (int i = tid; i < l.segs * kGroups; i += kRowThreads) {
      const float g = maxima[first * kGroups + i];
      sh.groups[i] = x.infinite ? g == INFINITY ? 0.0f : -INFINITY : g;
    }
    __syncthreads();
    token = f.by_passes(at, x.whole, x.lo, &own, &whole);
  }
  answer(row, token, own, whole, tokens, logprobs);
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void large_kernel(Logits l, Settings s, const float *u, const float *maxima,
                                                            const double *masses, Work work, int32_t *tokens,
                                                            float *logprobs) {
  __shared__ Shared sh;
  for (int i = blockIdx.x;; i += gridDim.x) {
    Large x;
    if (!large_at(work, l.rows, i, &x)) return;
    finish_large<T>(sh, i, x, l, s, u, maxima, masses, work, tokens, logprobs);
  }
}

int segments(int V) { return (V + 15 + kSeg - 1) / kSeg; }

struct Layout {
  size_t sums, maxima, count, large, above, bins, list, bytes;
};
Layout layout(int rows, int V) {
  Layout w{};
  size_t n = 0;
  auto take = [&](size_t bytes) {
    const size_t at = n;
    n += align_up(bytes, 256);
    return at;
  };
  const size_t segs = (size_t)rows * segments(V);
  w.sums = take(segs * sizeof(double));
  w.maxima = take(segs * Groups<false>::n * sizeof(float));
  w.count = take(sizeof(int));
  if (segments(V) <= kFewSegs) {   // (no large rows)
    w.bytes = n;
    return w;
  }
  w.large = take(rows * sizeof(Large));
  w.above = take(rows * sizeof(u64));
  w.bins = take((size_t)rows * kBins * sizeof(u64));
  w.list = take((size_t)rows * kList * sizeof(u64));
  w.bytes = n;
  return w;
}

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
  *bytes = layout(rows, V).bytes;
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
  const Layout w = layout(rows, V);
  char *const at = static_cast<char *>(workspace);
  double *sums = reinterpret_cast<double *>(at + w.sums);
  float *maxima = reinterpret_cast<float *>(at + w.maxima);
  // (thousands of tokens are kept by top-p or min-p, if by anything; top-k's passes, where its elements are too many, are
  // its row's workgroup's)
  const bool can_be_large = l.segs > kFewSegs && (how->top_ks || how->top_k == 0 || how->top_k >= V) &&
                            (how->top_ps || how->top_p < 1.0f || how->min_ps || how->min_p > 0.0f);
  const Work work{can_be_large ? reinterpret_cast<Large *>(at + w.large) : nullptr, reinterpret_cast<int *>(at + w.count),
                  reinterpret_cast<u64 *>(at + w.bins), reinterpret_cast<u64 *>(at + w.list),
                  reinterpret_cast<u64 *>(at + w.above)};
  const int groups = (l.segs + kWaves - 1) / kWaves, parts = (l.segs + kPart - 1) / kPart,
            halves = (l.segs + kPart / 2 - 1) / (kPart / 2);
  hipStream_t q = static_cast<hipStream_t>(stream);
  auto launch = [&](auto t) {
    using T = decltype(t);
    if (l.segs <= kFewSegs) {
      row_kernel<T, true><<<rows, kRowThreads, 0, q>>>(l, s, u, maxima, sums, work, tokens, logprobs);
      return;
    }
    segments_kernel<T><<<(unsigned)(rows * groups), 64 * kWaves, 0, q>>>(l, s, groups, maxima, sums, work.count);
    row_kernel<T, false><<<rows, kRowThreads, 0, q>>>(l, s, u, maxima, sums, work, tokens, logprobs);
    if (can_be_large) {
      const auto some = [&](int64_t all) { return (unsigned)(all < kSpread ? all : kSpread); };
      bins_kernel<T><<<some((int64_t)rows * parts), 64 * kPart, 0, q>>>(l, s, parts, work);
      masses_kernel<T><<<some((int64_t)rows * halves), 64 * kPart, 0, q>>>(l, s, halves, sums, work);
      large_kernel<T><<<some(rows), kRowThreads, 0, q>>>(l, s, u, maxima, sums, work, tokens, logprobs);
    }
  };
  if (logits_dtype == DT_F32)
    launch(uint32_t());
  else
    launch(uint16_t());
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DT_OK : hip_fail(e, "sampling launch");
}

}  // extern "C"
