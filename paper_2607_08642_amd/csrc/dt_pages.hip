// Pages of a cache (dt_pages): which of them the sequences of a batch hold, and copies of whole pages.
//
// The books are a few thousand numbers and every decision depends on all of them (the lowest free pages, in the order
// of the sequences), so one workgroup keeps them: bound by latency (64 sequences over 16,384 pages: 9 us; the plan of a
// compaction of 2,048 pages 5, of a fork 5).  Data moves in launches of their own over the whole card, bound by
// memory traffic (500 pages of 512 KB: 104 us, 5.0 TB/s, as a copy of 1 GiB).
#include "dt_cache.h"

namespace dt {
namespace {

constexpr int kBookThreads = 1024, kBookWaves = kBookThreads / 64;
constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = kCopyThreads * 16 * 4;  // of a workgroup's step
constexpr int kMaxGroups = 1 << 24;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Book {
  int pages, page_size, batch, width;
  int32_t *uses, *held, *lens, *table, *missing;
};

// What a call needs besides: lists of pages, one plan a sequence, and a new table.
struct Scratch {
  int32_t *head;          // [64]: how many copies, the pages in use
  int32_t *from, *to;     // [pages] copies (fit, fork: `to` holds the free pages taken)
  int32_t *rank;          // [pages] a moving page's place in `from`
  int32_t *first;         // [batch] a sequence's first place in `to`
  int32_t *source, *full; // [batch] fork: where a sequence's pages come from (-1: it keeps its own), how many are shared
  int32_t *len;           // [batch] fork: new lengths
  int32_t *rows;          // [batch, width] fork: new rows
};

size_t scratch(const dt_pages &p, char *at, Scratch *s) {
  size_t n = 0;
  auto take = [&](size_t ints) {
    int32_t *q = reinterpret_cast<int32_t *>(at + n);
    n += align_up(ints * 4, 256);
    return q;
  };
  s->head = take(64);
  s->from = take(p.pages);
  s->to = take(p.pages);
  s->rank = take(p.pages);
  s->first = take(p.batch);
  s->source = take(p.batch);
  s->full = take(p.batch);
  s->len = take(p.batch);
  s->rows = take((size_t)p.batch * p.table_width);
  return n;
}

// The sum over the workgroup's threads before this one, and over all.
__device__ int before_thread(int x, int *tmp, int *whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int run = x;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(run, o);
    if (lane >= o) run += y;
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = run;
  __syncthreads();
  int first = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kBookWaves; ++w) {
    const int t = tmp[w];
    if (w < wave) first += t;
    all += t;
  }
  *whole = all;
  return first + run - x;
}

__device__ inline int held_of(const Book &k, int b) { return min(max(k.held[b], 0), k.width); }
__device__ inline int len_of(const Book &k, int b) { return min(max(k.lens[b], 0), k.width * k.page_size); }

// The `want` lowest free pages: the first kTaken of them in LDS, the rest in list[]; how many there are (all
// of them counted only where they do not suffice).  What the workgroup wrote before is there after a barrier: it is one
// workgroup's memory.
constexpr int kTaken = 4096;
struct Taken {
  int pages[kTaken];
  __device__ int at(const int32_t *list, int i) const { return i < kTaken ? pages[i] : list[i]; }
};
__device__ int lowest_free(const Book &k, int want, int32_t *list, Taken &taken, int *tmp) {
  constexpr int kEach = 4;
  int found = 0;
  for (int p0 = 0; p0 < k.pages && found < want; p0 += kEach * kBookThreads) {
    const int p = p0 + kEach * (int)threadIdx.x;
    int free = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (p + i < k.pages && k.uses[p + i] <= 0) free |= 1 << i;
    int at = found + before_thread(__popc(free), tmp, &all);
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (free >> i & 1) {
        if (at < min(want, kTaken))
          taken.pages[at] = p + i;
        else if (at < want)
          list[at] = p + i;
        ++at;
      }
    found += all;
  }
  __syncthreads();
  return found;
}

// Items dealt to sequences: which one item i belongs to (the last whose first item is not after it).
__device__ inline int owner(const int *first, int n, int i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= i)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// One workgroup.  Every step over pages is dealt out evenly, a page a thread, so what counts is the number of times that one
// step waits for the memory of another: lengths; entries that go; uses; entries that come.
__global__ __launch_bounds__(kBookThreads) void fit_kernel(Book k, Scratch s) {
  __shared__ int tmp[kBookWaves];
  __shared__ int first[kBookThreads], start[kBookThreads];   // of a sequence: its first item, its first entry
  __shared__ Taken taken;
  const int tid = threadIdx.x;
  int total = 0;
  for (int b0 = 0; b0 < k.batch; b0 += kBookThreads) {
    const int b = b0 + tid, n = min(k.batch - b0, kBookThreads);
    int want = 0, held = 0, goes, lacks;
    if (b < k.batch) {
      want = (len_of(k, b) + k.page_size - 1) / k.page_size;
      held = held_of(k, b);
    }
    const int at = before_thread(max(held - want, 0), tmp, &goes);
    before_thread(max(want - held, 0), tmp, &lacks);
    first[tid] = at;
    start[tid] = want;
    total += lacks;
    __syncthreads();
    for (int i = tid; i < goes; i += kBookThreads) {
      const int q = owner(first, n, i);
      int32_t &entry = k.table[(int64_t)(b0 + q) * k.width + start[q] + i - first[q]];
      const int p = entry;
      if (p >= 0 && p < k.pages) atomicSub(k.uses + p, 1);
      entry = -1;
    }
    if (want < held) k.held[b] = want;
    __syncthreads();
  }
  const int found = total ? lowest_free(k, total, s.to, taken, tmp) : 0;
  if (tid == 0) *k.missing = max(total - found, 0);
  if (found < total || total == 0) return;
  int done = 0;
  for (int b0 = 0; b0 < k.batch; b0 += kBookThreads) {
    const int b = b0 + tid, n = min(k.batch - b0, kBookThreads);
    int want = 0, held = 0, comes;
    if (b < k.batch) {
      want = (len_of(k, b) + k.page_size - 1) / k.page_size;
      held = held_of(k, b);
    }
    const int at = before_thread(max(want - held, 0), tmp, &comes);
    first[tid] = at;
    start[tid] = held;
    __syncthreads();
    for (int i = tid; i < comes; i += kBookThreads) {
      const int q = owner(first, n, i), p = taken.at(s.to, done + i);
      k.table[(int64_t)(b0 + q) * k.width + start[q] + i - first[q]] = p;
      k.uses[p] = 1;
    }
    if (want > held) k.held[b] = want;
    done += comes;
    __syncthreads();
  }
}

// Fork, first: where each sequence's pages come from, and a free page for each partial one.
__global__ __launch_bounds__(kBookThreads) void fork_plan_kernel(Book k, Scratch s, const int32_t *source) {
  __shared__ int tmp[kBookWaves];
  __shared__ Taken taken;
  const int tid = threadIdx.x;
  int total = 0;
  for (int b0 = 0; b0 < k.batch; b0 += kBookThreads) {
    const int b = b0 + tid;
    int from = -1, full = 0, part = 0, len = 0, all;
    if (b < k.batch) {
      from = source[b];
      if (from < 0 || from >= k.batch || from == b) from = -1;
      if (from >= 0) {
        const int held = held_of(k, from);
        len = len_of(k, from);
        full = min(len / k.page_size, held);
        part = full < held && len > full * k.page_size;
      }
    }
    const int at = before_thread(part, tmp, &all);
    if (b < k.batch) {
      s.source[b] = from;
      s.full[b] = full;
      s.len[b] = len;
      s.first[b] = part ? total + at : -1;
    }
    total += all;
  }
  const int found = total ? lowest_free(k, total, s.to, taken, tmp) : 0;
  for (int i = tid; i < min(min(total, found), kTaken); i += kBookThreads) s.to[i] = taken.pages[i];
  if (tid == 0) {
    *k.missing = max(total - found, 0);
    s.head[0] = found >= total;
  }
}

// Copy `bytes` (a multiple of 16) by a workgroup, at most kCopyBytes of them.
__device__ __forceinline__ void copy_step(const char *from, char *to, int bytes) {
  u32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = ((int)threadIdx.x + i * kCopyThreads) * 16;
    if (at < bytes) v[i] = *reinterpret_cast<const u32x4 *>(from + at);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = ((int)threadIdx.x + i * kCopyThreads) * 16;
    if (at < bytes) *reinterpret_cast<u32x4 *>(to + at) = v[i];
  }
}

// Steps of a copy of a page in every layer, and one of them.
struct Copies {
  CacheView c;  // layer 0
  int layers, steps;  // steps of a page of a layer
  int64_t layer_bytes;
};
__device__ __forceinline__ void copy_part(const Copies &c, int from, int to, int part) {
  const int64_t at = (int64_t)(part / c.steps) * c.layer_bytes + (int64_t)(part % c.steps) * kCopyBytes;
  const int64_t left = c.c.page_bytes - (int64_t)(part % c.steps) * kCopyBytes;
  copy_step(c.c.base + from * c.c.page_bytes + at, c.c.base + to * c.c.page_bytes + at,
            left < kCopyBytes ? (int)left : kCopyBytes);
}

// Fork, second: new rows and their uses (workgroups [0, batch)), copies of partial pages.  Nothing that is read
// here changes here: pages copied into are free, rows are put together apart.
__global__ __launch_bounds__(kCopyThreads) void fork_copy_kernel(Book k, Scratch s, Copies c) {
  if (!s.head[0]) return;
  const int parts = c.layers * c.steps;
  if ((int)blockIdx.x < k.batch) {
    const int b = blockIdx.x, from = s.source[b];
    if (from < 0) return;
    const int full = s.full[b];
    const int32_t *old = k.table + (int64_t)from * k.width;
    int32_t *row = s.rows + (int64_t)b * k.width;
    for (int e = threadIdx.x; e < full; e += kCopyThreads) {
      const int p = old[e];
      row[e] = p;
      if (p >= 0 && p < k.pages) atomicAdd(k.uses + p, 1);
    }
    if (threadIdx.x == 0 && s.first[b] >= 0) {
      row[full] = s.to[s.first[b]];
      k.uses[row[full]] = 1;
    }
    return;
  }
  const int b = ((int)blockIdx.x - k.batch) / parts;
  if (s.source[b] < 0 || s.first[b] < 0) return;
  const int p = k.table[(int64_t)s.source[b] * k.width + s.full[b]];
  if (p >= 0 && p < k.pages) copy_part(c, p, s.to[s.first[b]], ((int)blockIdx.x - k.batch) % parts);
}

// Fork, third: the old rows' uses go, the new rows and lengths come.
__global__ __launch_bounds__(kCopyThreads) void fork_rows_kernel(Book k, Scratch s) {
  const int b = blockIdx.x;
  if (!s.head[0] || s.source[b] < 0) return;
  const int now = s.full[b] + (s.first[b] >= 0), held = held_of(k, b);
  int32_t *row = k.table + (int64_t)b * k.width;
  const int32_t *next = s.rows + (int64_t)b * k.width;
  for (int e = threadIdx.x; e < max(held, now); e += kCopyThreads) {
    const int p = row[e];
    if (e < held && p >= 0 && p < k.pages) atomicSub(k.uses + p, 1);
    row[e] = e < now ? next[e] : -1;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    k.held[b] = now;
    k.lens[b] = s.len[b];
  }
}
// Compact, first: the pages in use that lie beyond their number, and the free ones before it.
__global__ __launch_bounds__(kBookThreads) void compact_plan_kernel(Book k, Scratch s) {
  __shared__ int tmp[kBookWaves];
  constexpr int kEach = 8;
  const int tid = threadIdx.x;
  const auto used_of = [&](int p0) {   // kEach neighbouring pages: a bit each
    int32_t u[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) u[i] = p0 + i < k.pages ? k.uses[p0 + i] : 0;
    int used = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) used |= (u[i] > 0) << i;
    return used;
  };
  int mine = 0, live;
  const int used0 = used_of(kEach * tid);
  for (int p = kEach * tid; p < k.pages; p += kEach * kBookThreads) mine += __popc(p == kEach * tid ? used0 : used_of(p));
  before_thread(mine, tmp, &live);
  int moves = 0, holes = 0;
  for (int p0 = 0; p0 < k.pages; p0 += kEach * kBookThreads) {
    const int p = p0 + kEach * tid, used = p0 ? used_of(p) : used0;
    const int below = (1 << min(max(live - p, 0), kEach)) - 1;   // (the pages before `live`)
    const int high = used & ~below, hole = ~used & below;
    int all;   // (both counts in one sum: at most 8192 of each a step)
    const int at = before_thread(__popc(high) << 16 | __popc(hole), tmp, &all);
    int at_high = moves + (at >> 16), at_hole = holes + (at & 0xffff);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (high >> i & 1) {
        s.from[at_high] = p + i;
        s.rank[p + i] = at_high++;
      }
      if (hole >> i & 1) s.to[at_hole++] = p + i;
    }
    moves += all >> 16;
    holes += all & 0xffff;
  }
  if (tid == 0) {
    s.head[0] = moves;
    s.head[1] = live;
    *k.missing = 0;
  }
}

// Compact, second: the table's entries (workgroups [0, batch)), the pages' data and uses.
__global__ __launch_bounds__(kCopyThreads) void compact_copy_kernel(Book k, Scratch s, Copies c, int copiers) {
  const int moves = s.head[0], live = s.head[1];
  if (moves == 0) return;
  if ((int)blockIdx.x < k.batch) {
    int32_t *row = k.table + (int64_t)blockIdx.x * k.width;
    const int held = held_of(k, blockIdx.x);
    for (int e = threadIdx.x; e < held; e += kCopyThreads) {
      const int p = row[e];
      if (p >= live && p < k.pages) {
        const int r = s.rank[p];
        if (r >= 0 && r < moves && s.from[r] == p) row[e] = s.to[r];
      }
    }
    return;
  }
  const int parts = c.layers * c.steps;
  for (int64_t i = (int)blockIdx.x - k.batch; i < (int64_t)moves * parts; i += copiers) {
    const int from = s.from[i / parts], to = s.to[i / parts], part = (int)(i % parts);
    if (part == 0 && threadIdx.x == 0) {
      k.uses[to] = k.uses[from];
      k.uses[from] = 0;
    }
    copy_part(c, from, to, part);
  }
}

__global__ __launch_bounds__(kCopyThreads) void copy_pages_kernel(Copies c, const int32_t *from, const int32_t *to) {
  const int parts = c.layers * c.steps, i = blockIdx.x / parts, f = from[i], t = to[i];
  if (f >= 0 && f < c.c.pages && t >= 0 && t < c.c.pages && f != t) copy_part(c, f, t, blockIdx.x % parts);
}

Copies copies_of(const dt_cache &cache) {
  Copies c;
  c.c = cache_view(cache, 0);
  c.layers = cache.layers;
  c.steps = (int)((c.c.page_bytes + kCopyBytes - 1) / kCopyBytes);
  c.layer_bytes = c.c.page_bytes * cache.pages;
  return c;
}

dt_status check_pages(const dt_pages *p, bool data) {
  if (!p) return fail(DT_ERR_NULL, "pages is required");
  if (p->pages < 1 || p->batch < 1 || p->table_width < 1)
    return fail(DT_ERR_SHAPE, "sizes must be positive (pages=%d batch=%d table_width=%d)", p->pages, p->batch,
                p->table_width);
  if (p->page_size != 32 && p->page_size != 64 && p->page_size != 128 && p->page_size != 256)
    return fail(DT_ERR_UNSUPPORTED, "page_size must be 32, 64, 128 or 256 (%d)", p->page_size);
  if (p->pages > 1 << 28 || p->batch > 65535 || (int64_t)p->table_width * p->page_size >= (int64_t)1 << 30 ||
      (int64_t)p->batch * p->table_width >= (int64_t)1 << 31)   // (entries are counted in 32 bits)
    return fail(DT_ERR_UNSUPPORTED,
                "need pages <= 2^28, batch <= 65535, table_width * page_size < 2^30, batch * table_width < 2^31");
  if (!data) return DT_OK;
  for (const void *q : {(const void *)p->uses, (const void *)p->held, (const void *)p->lens, (const void *)p->table,
                        (const void *)p->missing}) {
    if (!q) return fail(DT_ERR_NULL, "uses, held, lens, table and missing are required");
    if (reinterpret_cast<uintptr_t>(q) % 4) return fail(DT_ERR_ALIGN, "tensors must be naturally aligned");
  }
  return DT_OK;
}

dt_status check_scratch(const dt_pages *p, void *workspace, size_t bytes, Scratch *s) {
  const size_t need = scratch(*p, static_cast<char *>(workspace), s);
  if (!workspace || bytes < need)
    return fail(DT_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", need, workspace ? bytes : 0);
  if (reinterpret_cast<uintptr_t>(workspace) % 256) return fail(DT_ERR_ALIGN, "workspace must be 256-byte aligned");
  return DT_OK;
}

dt_status check_both(const dt_pages *p, const dt_cache *cache) {
  dt_status st = check_pages(p, true);
  if (st == DT_OK) st = check_cache(cache, true);
  if (st == DT_OK && (cache->pages != p->pages || cache->page_size != p->page_size))
    st = fail(DT_ERR_SHAPE, "the cache has %d pages of %d tokens, the books %d of %d", cache->pages, cache->page_size,
              p->pages, p->page_size);
  return st;
}

Book book_of(const dt_pages &p) {
  return Book{p.pages, p.page_size, p.batch, p.table_width, p.uses, p.held, p.lens, p.table, p.missing};
}

}  // namespace
}  // namespace dt

using namespace dt;

extern "C" {

dt_status dt_pages_workspace_size(const dt_pages *pages, size_t *bytes) {
  if (!bytes) return fail(DT_ERR_NULL, "bytes is required");
  const dt_status st = check_pages(pages, false);
  if (st != DT_OK) return st;
  Scratch s;
  *bytes = scratch(*pages, nullptr, &s);
  return DT_OK;
}

dt_status dt_pages_fit(const dt_pages *pages, void *workspace, size_t ws_bytes, void *stream) {
  Scratch s;
  dt_status st = check_pages(pages, true);
  if (st == DT_OK) st = check_scratch(pages, workspace, ws_bytes, &s);
  if (st != DT_OK) return st;
  fit_kernel<<<1, kBookThreads, 0, static_cast<hipStream_t>(stream)>>>(book_of(*pages), s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DT_OK : hip_fail(e, "pages launch");
}

dt_status dt_pages_fork(const dt_pages *pages, const dt_cache *cache, const int32_t *source, void *workspace,
                        size_t ws_bytes, void *stream) {
  Scratch s;
  dt_status st = check_both(pages, cache);
  if (st == DT_OK) st = check_scratch(pages, workspace, ws_bytes, &s);
  if (st != DT_OK) return st;
  if (!source) return fail(DT_ERR_NULL, "source is required");
  if (reinterpret_cast<uintptr_t>(source) % 4) return fail(DT_ERR_ALIGN, "source must be naturally aligned");
  const Book k = book_of(*pages);
  const Copies c = copies_of(*cache);
  const int64_t groups = k.batch + (int64_t)k.batch * c.layers * c.steps;
  if (groups >= kMaxGroups) return fail(DT_ERR_UNSUPPORTED, "batch, layers and pages are too large together");
  hipStream_t q = static_cast<hipStream_t>(stream);
  fork_plan_kernel<<<1, kBookThreads, 0, q>>>(k, s, source);
  fork_copy_kernel<<<(unsigned)groups, kCopyThreads, 0, q>>>(k, s, c);
  fork_rows_kernel<<<k.batch, kCopyThreads, 0, q>>>(k, s);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DT_OK : hip_fail(e, "pages launch");
}

dt_status dt_pages_compact(const dt_pages *pages, const dt_cache *cache, void *workspace, size_t ws_bytes,
                           void *stream) {
  Scratch s;
  dt_status st = check_both(pages, cache);
  if (st == DT_OK) st = check_scratch(pages, workspace, ws_bytes, &s);
  if (st != DT_OK) return st;
  const Book k = book_of(*pages);
  const Copies c = copies_of(*cache);
  const int64_t most = (int64_t)(k.pages / 2) * c.layers * c.steps;  // (a page that moves leaves one for a hole)
  const int copiers = (int)(most < 8192 ? most : 8192);
  hipStream_t q = static_cast<hipStream_t>(stream);
  compact_plan_kernel<<<1, kBookThreads, 0, q>>>(k, s);
  compact_copy_kernel<<<(unsigned)(k.batch + copiers), kCopyThreads, 0, q>>>(k, s, c, copiers);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DT_OK : hip_fail(e, "pages launch");
}

dt_status dt_cache_copy_pages(const dt_cache *cache, const int32_t *from, const int32_t *to, int n, void *stream) {
  const dt_status st = check_cache(cache, true);
  if (st != DT_OK) return st;
  if (!from || !to) return fail(DT_ERR_NULL, "from and to are required");
  if (reinterpret_cast<uintptr_t>(from) % 4 || reinterpret_cast<uintptr_t>(to) % 4)
    return fail(DT_ERR_ALIGN, "from and to must be naturally aligned");
  if (n < 1) return fail(DT_ERR_SHAPE, "n must be positive (%d)", n);
  const Copies c = copies_of(*cache);
  if ((double)n * c.layers * c.steps >= kMaxGroups) return fail(DT_ERR_UNSUPPORTED, "too many pages in one call");
  copy_pages_kernel<<<(unsigned)(n * c.layers * c.steps), kCopyThreads, 0, static_cast<hipStream_t>(stream)>>>(c, from, to);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? DT_OK : hip_fail(e, "copy launch");
}

}  // extern "C"
