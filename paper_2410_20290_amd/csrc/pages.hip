// The paged candidate cache: forking rows, reserving and compacting pages, and
// writing rotated keys and values into them.  Which page goes where follows
// from counts and ascending page numbers alone, so results do not depend on
// the order in which work-groups run.
#include <algorithm>
#include <climits>

#include "common.h"
#include "kernels.h"
#include "paged.h"

namespace sr {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

__device__ __forceinline__ bool is_page(int pg, int n_pages) { return (uint32_t)pg < (uint32_t)n_pages; }
__device__ __forceinline__ int pages_of(int tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }

// Exclusive scan over the plan work-group; *total receives the sum.
__device__ int plan_scan(int v, int* wsum, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(inc, o, 64);
    if (lane >= o) inc += t;
  }
  __syncthreads();   // (wsum may still be read from the scan before)
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  int off = 0, tot = 0;
  for (int w = 0; w < kPlanWaves; ++w) {
    if (w < wave) off += wsum[w];
    tot += wsum[w];
  }
  *total = tot;
  return off + inc - v;
}

// The same of two counts below 2^31 each, in one round: x in the low half.
__device__ int2 plan_scan2(int2 v, uint64_t* wsum, int2* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t inc = (uint64_t)(uint32_t)v.y << 32 | (uint32_t)v.x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t lo = __shfl_up((uint32_t)inc, o, 64), hi = __shfl_up((uint32_t)(inc >> 32), o, 64);
    if (lane >= o) inc += (uint64_t)hi << 32 | lo;
  }
  __syncthreads();
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  uint64_t off = 0, tot = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const uint64_t x = wsum[w];
    if (w < wave) off += x;
    tot += x;
  }
  *total = make_int2((int)(uint32_t)tot, (int)(tot >> 32));
  off += inc;
  return make_int2((int)(uint32_t)off - v.x, (int)(off >> 32) - v.y);
}

// -------------------------------------------------------------------- fork
// Entries i, i + step, .. (U of them, those below n) of the new table, and their
// rows' lengths; the parents, lengths and entries of all are loaded together.
template <int U>
__device__ __forceinline__ void forked_entries(const PageForkArgs& a, int64_t i, int64_t step, int64_t n, int (&pg)[U],
                                               int (&len)[U]) {
  int par[U], c[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t k = i + u * step < n ? i + u * step : n - 1;
    const int j = (int)(k / a.max_pages);
    c[u] = (int)(k - (int64_t)j * a.max_pages);
    par[u] = a.parent[j];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) len[u] = (uint32_t)par[u] < (uint32_t)a.rows ? a.lens[par[u]] : 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    len[u] = clamp_len(len[u], a.max_pages, a.shift);
    // out of every later token's sight: the next one sits at position len
    const bool behind = ((c[u] + 1) << a.shift) <= window_start(len[u], a.window) && (c[u] << a.shift) >= a.sinks;
    const bool there = c[u] < pages_of(len[u], a.shift) && !behind;
    pg[u] = there ? a.table[(int64_t)par[u] * a.max_pages + c[u]] : -1;
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (!is_page(pg[u], a.n_pages)) pg[u] = -1;
}

// Small tables and pools: one work-group and one launch, the counts in LDS.  Us a
// call, and in a replayed graph, with 16384 pages, against the two launches below:
// 256 entries 5.9, 4.7 against 8.6, 4.6; 4096 6.5, 6.6 against 8.6, 5.1; 30720
// 20.2, 20.3 against 8.8, 5.5 (with 512 pages 256 entries 5.7, 3.6 against 8.2,
// 4.7).
constexpr int kForkSmallPages = 16384, kForkSmallEntries = 4096;
__global__ void __launch_bounds__(kPlanThreads) fork_small_kernel(PageForkArgs a) {
  __shared__ int refs[kForkSmallPages];
  for (int p = threadIdx.x; p < a.n_pages; p += kPlanThreads) refs[p] = 0;
  __syncthreads();
  const int n = a.new_rows * a.max_pages;
  constexpr int U = 8;
  for (int i = threadIdx.x; i < n; i += U * kPlanThreads) {
    int pg[U], len[U];
    forked_entries<U>(a, i, kPlanThreads, n, pg, len);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = i + u * kPlanThreads;
      if (k >= n) break;
      if (pg[u] >= 0) atomicAdd(&refs[pg[u]], 1);
      a.table_out[k] = pg[u];
      if (k % a.max_pages == 0) a.lens_out[k / a.max_pages] = len[u];
    }
  }
  __syncthreads();
  for (int p = threadIdx.x; p < a.n_pages; p += kPlanThreads) a.refs_out[p] = refs[p];
}

// One thread per entry of the new table; the counts start at 0.
__global__ void __launch_bounds__(256) fork_table_kernel(PageForkArgs a) {
  const int64_t tid = (int64_t)blockIdx.x * 256 + threadIdx.x, nthr = (int64_t)gridDim.x * 256;
  for (int64_t p = tid; p < a.n_pages; p += nthr) a.refs_out[p] = 0;
  const int64_t n = (int64_t)a.new_rows * a.max_pages;
  constexpr int U = 4;
  for (int64_t i = tid; i < n; i += U * nthr) {
    int pg[U], len[U];
    forked_entries<U>(a, i, nthr, n, pg, len);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = i + u * nthr;
      if (k >= n) break;
      a.table_out[k] = pg[u];
      if (k % a.max_pages == 0) a.lens_out[k / a.max_pages] = len[u];
    }
  }
}

// Counts of the new table.  A thread takes one column of kForkRows rows and
// adds runs of the same page at once: rows forked from one parent name the
// same pages, and their atomics would queue on one address.
constexpr int kForkRows = 16;
__global__ void __launch_bounds__(256) fork_count_kernel(const int32_t* __restrict__ table, int rows, int max_pages,
                                                         int32_t* __restrict__ refs) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int chunk = (int)(i / max_pages), c = (int)(i - (int64_t)chunk * max_pages);
  const int r0 = chunk * kForkRows;
  if (r0 >= rows) return;
  int pg[kForkRows];
#pragma unroll
  for (int k = 0; k < kForkRows; ++k) pg[k] = r0 + k < rows ? table[(int64_t)(r0 + k) * max_pages + c] : -1;
  int cur = -1, n = 0;
#pragma unroll
  for (int k = 0; k < kForkRows; ++k) {
    if (pg[k] != cur) {
      if (cur >= 0) atomicAdd(&refs[cur], n);
      cur = pg[k];
      n = 0;
    }
    ++n;
  }
  if (cur >= 0) atomicAdd(&refs[cur], n);
}

void page_fork(const PageForkArgs& a, hipStream_t s) {
  if (a.n_pages <= kForkSmallPages && (int64_t)a.new_rows * a.max_pages <= kForkSmallEntries) {
    SR_LAUNCH(fork_small_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
    SR_CHECK_LAUNCH();
    return;
  }
  const int64_t n = std::max<int64_t>((int64_t)a.new_rows * a.max_pages, a.n_pages);
  SR_LAUNCH(fork_table_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), 0, s, a);
  SR_CHECK_LAUNCH();
  if (a.new_rows == 0) return;
  const int64_t m = (int64_t)((a.new_rows + kForkRows - 1) / kForkRows) * a.max_pages;
  SR_LAUNCH(fork_count_kernel, dim3((unsigned)((m + 255) / 256)), dim3(256), 0, s, a.table_out, a.new_rows, a.max_pages,
            a.refs_out);
  SR_CHECK_LAUNCH();
}

// ----------------------------------------------------------------- reserve
// What the plan leaves for the second launch, per row: the column of its first
// new entry, their number, where they start in the list of free pages, its length
// and the tokens to add; and the pages to copy.  (info says whether it stands.)
struct ReservePlan {
  int32_t *start, *need, *first, *len, *add;   // [rows]
  int32_t *src, *at, *part;                    // [rows] pairs: page, index into free, filled slots
  int32_t* free;                             // [n_pages]
};
constexpr int kReserveArrays = 8;
__host__ __device__ inline ReservePlan reserve_plan(int32_t* scratch, int rows) {
  ReservePlan p;
  p.start = scratch;
  p.need = scratch + rows;
  p.first = scratch + 2 * rows;
  p.len = scratch + 3 * rows;
  p.add = scratch + 4 * rows;
  p.src = scratch + 5 * rows;
  p.at = scratch + 6 * rows;
  p.part = scratch + 7 * rows;
  p.free = scratch + kReserveArrays * rows;
  return p;
}

// A hash table in LDS counts, for every part-filled last page that more than
// one entry names, the rows that add tokens to it, and finds the lowest.
constexpr int kHashSize = 2 * kPageMaxRows;   // twice the rows: probing ends

// Two launches: the plan, bound by its chain of scans (12 us at 512 rows of 15
// entries), then the copies, bound by memory.  Work-group 0 plans; the others
// copy the table and the counts meanwhile (the second launch writes what changes).
__global__ void __launch_bounds__(kPlanThreads) reserve_plan_kernel(PageReserveArgs a) {
  const int np = a.p.n_pages, shift = a.p.shift, mp = a.max_pages, mask = (1 << shift) - 1;
  if (blockIdx.x > 0) {
    const int64_t tid = (int64_t)(blockIdx.x - 1) * kPlanThreads + threadIdx.x;
    const int64_t nthr = (int64_t)(gridDim.x - 1) * kPlanThreads;
    if (a.refs_out != a.refs)
      for (int64_t p = tid; p < np; p += nthr) a.refs_out[p] = a.refs[p];
    const int64_t n = (int64_t)a.rows * mp;
    for (int64_t i = tid; i < n; i += nthr) {
      const int r = (int)(i / mp), c = (int)(i - (int64_t)r * mp);
      const int old = a.table[i];
      const bool keep = is_page(old, np) && c < pages_of(clamp_len(a.lens[r], mp, shift), shift);
      if (!keep || a.table_out != a.table) a.table_out[i] = keep ? old : -1;
    }
    return;
  }
  __shared__ int hkey[kHashSize], hcount[kHashSize], hlow[kHashSize], hslot[kPageMaxRows];
  __shared__ uint64_t wsum[kPlanWaves];
  __shared__ int wides;
  constexpr int STEPS = 16;
  int v[STEPS];   // counts of the first pages, on their way while the rows are looked at
  auto load_counts = [&](int base) {
    const int p0 = base + (threadIdx.x >> 6) * 64 * STEPS + (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) v[i] = p0 + 64 * i < np ? a.refs[p0 + 64 * i] : 1;
  };
  load_counts(0);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // (a hash table for the rows there are: at least twice as many slots)
  const int bits = imax(6, 33 - __clz(imax(1, a.rows - 1)));
  for (int i = tid; i < 1 << bits; i += kPlanThreads) {
    hkey[i] = -1;
    hcount[i] = 0;
    hlow[i] = INT_MAX;
  }
  if (tid == 0) wides = 0;
  __syncthreads();
  const ReservePlan pl = reserve_plan(a.scratch, a.rows);
  struct Row {
    int len, add, last, refs;   // tokens, granted at best, part-filled last page (-1: none, or lost) and its count
    bool wide, lost;            // past the table; the part-filled last page's entry names no page
  };
  auto row = [&](int r) {
    Row w;
    w.len = clamp_len(a.lens[r], mp, shift);
    w.add = imax(0, a.n_add ? a.n_add[r] : a.n_add_all);
    const int room = (mp << shift) - w.len;
    w.wide = w.add > room;
    w.add = imin(w.add, room);
    w.last = -1;
    w.refs = 0;
    w.lost = false;
    if (w.add > 0 && (w.len & mask) != 0) {
      w.last = a.table[(int64_t)r * mp + pages_of(w.len, shift) - 1];
      w.lost = !is_page(w.last, np);
      if (w.lost) w.last = -1;
      else w.refs = a.refs[w.last];
    }
    return w;
  };
  Row first_row;   // of this thread's rows, the only one below 1024 rows
  for (int r = tid; r < a.rows; r += kPlanThreads) {
    const Row w = row(r);
    if (r == tid) first_row = w;
    if (w.wide) atomicAdd(&wides, 1);
    hslot[r] = -1;
    if (w.refs < 2) continue;
    int h = (int)(((uint32_t)w.last * 2654435761u) >> (32 - bits));
    for (;; h = (h + 1) & ((1 << bits) - 1)) {
      const int was = atomicCAS(&hkey[h], -1, w.last);
      if (was == -1 || was == w.last) break;
    }
    hslot[r] = h;
    atomicAdd(&hcount[h], 1);
    atomicMin(&hlow[h], r);
  }
  __syncthreads();
  int total = 0, copies = 0;
  for (int base = 0; base < a.rows; base += kPlanThreads) {
    const int r = base + tid;
    int2 need = make_int2(0, 0);
    Row w{0, 0, -1, 0, false, false};
    bool copy = false;
    if (r < a.rows) {
      w = base == 0 ? first_row : row(r);
      const int h = hslot[r];
      copy = h >= 0 && !(hcount[h] == w.refs && hlow[h] == r);
      need.x = pages_of(w.len + w.add, shift) - pages_of(w.len, shift) + (copy || w.lost ? 1 : 0);
      need.y = copy ? 1 : 0;
    }
    int2 sum;
    const int2 before = plan_scan2(need, wsum, &sum);
    if (r < a.rows) {
      pl.start[r] = pages_of(w.len, shift) - (copy || w.lost ? 1 : 0);
      pl.need[r] = need.x;
      pl.first[r] = total + before.x;
      pl.len[r] = w.len;
      pl.add[r] = w.add;
      if (copy) {
        const int pair = copies + before.y;
        pl.src[pair] = w.last;
        pl.at[pair] = total + before.x;
        pl.part[pair] = w.len & mask;
      }
    }
    total += sum.x;
    copies += sum.y;
  }
  // The lowest free pages, 64 KB of counts at a time: a wave takes 1024
  // consecutive ones.
  int found = 0;
  for (int base = 0; base < np && found < total; base += kPlanThreads * STEPS) {
    const int p0 = base + wave * 64 * STEPS + lane;
    uint64_t bits[STEPS];
    int n = 0;
    if (base > 0) load_counts(base);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      bits[i] = __ballot(v[i] == 0);
      n += __popcll(bits[i]);
    }
    int2 tot;
    int at = found + __shfl(plan_scan2(make_int2(lane == 0 ? n : 0, 0), wsum, &tot).x, 0, 64);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int rank = at + __popcll(bits[i] & ((1ull << lane) - 1));
      if (v[i] == 0 && rank < total) pl.free[rank] = p0 + 64 * i;
      at += __popcll(bits[i]);
    }
    found += tot.x;
  }
  const int missing = imax(0, total - found);
  const bool ok = missing == 0 && wides == 0;
  if (tid == 0) {
    a.info[0] = missing;
    a.info[1] = wides;
    a.info[2] = ok ? total : 0;
    a.info[3] = ok ? copies : 0;
  }
}

// The new entries, lengths and counts (a wave per row), then the copies (a
// wave per page, block and head: one run of filled slots).
__global__ void __launch_bounds__(256) reserve_apply_kernel(PageReserveArgs a) {
  const ReservePlan pl = reserve_plan(a.scratch, a.rows);
  const int lane = threadIdx.x & 63;
  const int w0 = blockIdx.x * 4 + (threadIdx.x >> 6), nw = gridDim.x * 4;
  const bool ok = a.info[0] == 0 && a.info[1] == 0;
  for (int r = w0; r < a.rows; r += nw) {
    const int need = ok ? pl.need[r] : 0, first = pl.first[r], start = pl.start[r];
    for (int k = lane; k < need; k += 64) {
      const int pg = pl.free[first + k];
      a.table_out[(int64_t)r * a.max_pages + start + k] = pg;
      a.refs_out[pg] = 1;
    }
    if (lane == 0) {
      const int got = ok ? pl.add[r] : 0;
      a.granted[r] = got;
      a.lens_out[r] = pl.len[r] + got;
    }
  }
  const int copies = a.info[3];
  for (int i = w0 * 64 + lane; i < copies; i += nw * 64) atomicSub(&a.refs_out[pl.src[i]], 1);
  const int row16 = a.p.row_bytes >> 4, hkv = a.p.hkv;
  const int64_t units = (int64_t)copies * 2 * a.p.n_layers * hkv;
  const int64_t run = ((int64_t)a.p.row_bytes << a.p.shift);   // bytes of a head's slots in a page
  for (int64_t u = w0; u < units; u += nw) {
    const int h = (int)(u % hkv);
    const int64_t pb = u / hkv;
    const int blk = (int)(pb % (2 * a.p.n_layers)), i = (int)(pb / (2 * a.p.n_layers));
    char* base = (char*)a.p.pool + blk * a.p.block_bytes;
    const uint4* src = reinterpret_cast<const uint4*>(base + ((int64_t)pl.src[i] * hkv + h) * run);
    uint4* dst = reinterpret_cast<uint4*>(base + ((int64_t)pl.free[pl.at[i]] * hkv + h) * run);
    const int n = pl.part[i] * row16;
    for (int k = lane; k < n; k += 64) dst[k] = src[k];
  }
}

size_t page_reserve_scratch(int rows, int max_pages, int n_pages) {
  (void)max_pages;
  return (size_t)kReserveArrays * rows + n_pages;
}

void page_reserve(const PageReserveArgs& a, hipStream_t s) {
  const int64_t n = std::max<int64_t>((int64_t)a.rows * a.max_pages, a.p.n_pages);
  const unsigned copiers = (unsigned)std::min<int64_t>((n + kPlanThreads - 1) / kPlanThreads, 512);
  SR_LAUNCH(reserve_plan_kernel, dim3(1 + copiers), dim3(kPlanThreads), 0, s, a);
  SR_CHECK_LAUNCH();
  const int64_t units = (int64_t)a.rows * 2 * a.p.n_layers * a.p.hkv;
  SR_LAUNCH(reserve_apply_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>((units + 3) / 4, 8192))),
            dim3(256), 0, s, a);
  SR_CHECK_LAUNCH();
}

// ----------------------------------------------------------------- compact
// scratch: the free pages below the live count, the live ones from it on (both
// ascending), the counts of the latter, and the new number of every page.
struct CompactPlan {
  int32_t *hole, *tail, *count, *to;
};
__host__ __device__ inline CompactPlan compact_plan(int32_t* scratch, int n_pages) {
  return {scratch, scratch + n_pages, scratch + 2 * (int64_t)n_pages, scratch + 3 * (int64_t)n_pages};
}

__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(PageCompactArgs a) {
  __shared__ int wsum[kPlanWaves];
  const int np = a.p.n_pages;
  const CompactPlan pl = compact_plan(a.scratch, np);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int STEPS = 16;
  int mine = 0, live;
  for (int p = tid; p < np; p += kPlanThreads) mine += a.refs[p] > 0 ? 1 : 0;
  plan_scan(mine, wsum, &live);
  int before = 0;   // live pages below base
  for (int base = 0; base < np; base += kPlanThreads * STEPS) {
    const int p0 = base + wave * 64 * STEPS + lane;
    uint64_t bits[STEPS];
    int v[STEPS], n = 0, tot;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) v[i] = p0 + 64 * i < np ? a.refs[p0 + 64 * i] : 0;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      bits[i] = __ballot(v[i] > 0);
      n += __popcll(bits[i]);
    }
    int at = before + __shfl(plan_scan(lane == 0 ? n : 0, wsum, &tot), 0, 64);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int p = p0 + 64 * i, below = at + __popcll(bits[i] & ((1ull << lane) - 1));   // live pages below p
      if (p < np) {
        pl.to[p] = p;
        if (p < live && v[i] <= 0) pl.hole[p - below] = p;
        if (p >= live && v[i] > 0) {
          // live pages below `live` = live - holes; this one's rank among the rest
          pl.tail[below] = p;
          pl.count[below] = v[i];
        }
      }
      at += __popcll(bits[i]);
    }
    before += tot;
  }
  // tail was filled from index (live pages below `live`); the holes number as
  // many as the live pages from `live` on
  int low = 0, stay;
  for (int p = tid; p < live; p += kPlanThreads) low += a.refs[p] > 0 ? 1 : 0;
  plan_scan(low, wsum, &stay);
  const int moved = live - stay;
  __syncthreads();
  for (int p = tid; p < np; p += kPlanThreads) {
    const int v = a.refs[p];
    if (p >= live) a.refs_out[p] = 0;
    else if (v > 0 && a.refs_out != a.refs) a.refs_out[p] = v;
  }
  __syncthreads();
  for (int k = tid; k < moved; k += kPlanThreads) {
    const int from = pl.tail[stay + k], to = pl.hole[k];
    pl.to[from] = to;
    a.refs_out[to] = pl.count[stay + k];
  }
  if (tid == 0) {
    a.info[0] = live;
    a.info[1] = moved;
    a.info[2] = 0;
    a.info[3] = 0;
  }
}

__global__ void __launch_bounds__(256) compact_move_kernel(PageCompactArgs a) {
  const CompactPlan pl = compact_plan(a.scratch, a.p.n_pages);
  const int64_t tid = (int64_t)blockIdx.x * 256 + threadIdx.x, nthr = (int64_t)gridDim.x * 256;
  const int live = a.info[0], moved = a.info[1], stay = live - moved;
  const int64_t n = (int64_t)a.rows * a.max_pages;
  for (int64_t i = tid; i < n; i += nthr) {
    const int r = (int)(i / a.max_pages), c = (int)(i - (int64_t)r * a.max_pages);
    const int pg = a.table[i];
    const bool keep = is_page(pg, a.p.n_pages) && c < pages_of(clamp_len(a.lens[r], a.max_pages, a.p.shift), a.p.shift);
    a.table_out[i] = keep ? pl.to[pg] : -1;
  }
  // a work-group moves 16 KB of a page at a time
  const int64_t page16 = (((int64_t)a.p.hkv * a.p.row_bytes) << a.p.shift) >> 4;
  const int nch = (int)((page16 + 1023) / 1024);
  const int64_t units = (int64_t)moved * 2 * a.p.n_layers * nch;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int c = (int)(u % nch);
    const int64_t kb = u / nch;
    const int blk = (int)(kb % (2 * a.p.n_layers)), k = (int)(kb / (2 * a.p.n_layers));
    char* base = (char*)a.p.pool + blk * a.p.block_bytes;
    const uint4* src = reinterpret_cast<const uint4*>(base) + pl.tail[stay + k] * page16;
    uint4* dst = reinterpret_cast<uint4*>(base) + pl.hole[k] * page16;
    const int64_t o = (int64_t)c * 1024 + threadIdx.x;
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = src[o + 256 * i < page16 ? o + 256 * i : page16 - 1];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (o + 256 * i < page16) dst[o + 256 * i] = v[i];
  }
}

size_t page_compact_scratch(int n_pages) { return (size_t)4 * n_pages; }

void page_compact(const PageCompactArgs& a, hipStream_t s) {
  SR_LAUNCH(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  SR_CHECK_LAUNCH();
  SR_LAUNCH(compact_move_kernel, dim3(8192), dim3(256), 0, s, a);
  SR_CHECK_LAUNCH();
}

// ------------------------------------------------------------------ append
// A work-group takes one token; a thread takes units of 8 dimensions: four
// rotated pairs, or 8 dimensions that pass.  (x, y) -> (x cos - y sin, y cos + x
// sin); angles, sines and cosines in 64 bits (an fp32 angle is off by up to
// 0.006 rad near position 65536), once per pair and token, through LDS for all heads.  Bound
// by memory: 24 prompts of up to 2011 tokens, 32 query and 8 KV heads of 64, 146
// us for 724 MB, 4.9 TB/s.
template <typename T, int HD>
__global__ void __launch_bounds__(256) append_kernel(PageAppendArgs a) {
  constexpr int UPH = HD / 8;   // units of a head
  __shared__ float cs[HD / 2], sn[HD / 2];
  const int row = blockIdx.x / a.lr, t = blockIdx.x - row * a.lr;
  const int len = clamp_len(a.lens[row], a.max_pages, a.shift);
  const int n = clamp_new(a.n_new ? a.n_new[row] : a.lr, a.lr, len);
  if (t >= n) return;
  const int pos = len - n + t, pairs = a.rot >> 1;
  for (int i = threadIdx.x; i < pairs; i += 256) {
    double s, c;
    sincos((double)pos * a.freqs[i], &s, &c);
    cs[i] = (float)c;
    sn[i] = (float)s;
  }
  __syncthreads();
  const int pg = a.table[(int64_t)row * a.max_pages + (pos >> a.shift)];
  const int heads = a.hq + 2 * a.hkv;
  const float* src = a.qkv + (int64_t)blockIdx.x * heads * HD;
  float* qd = a.q + (int64_t)blockIdx.x * a.hq * HD;
  for (int u = threadIdx.x; u < heads * UPH; u += 256) {
    const int h = u / UPH, w = u % UPH;
    const bool rotates = 4 * w < pairs && h < a.hq + a.hkv;
    // the unit's two runs of four dimensions
    const int d0 = rotates && !a.interleaved ? 4 * w : 8 * w;
    const int d1 = rotates && !a.interleaved ? pairs + 4 * w : 8 * w + 4;
    const float4 x = *reinterpret_cast<const float4*>(src + h * HD + d0);
    const float4 y = *reinterpret_cast<const float4*>(src + h * HD + d1);
    float v0[4] = {x.x, x.y, x.z, x.w}, v1[4] = {y.x, y.y, y.z, y.w};
    if (rotates) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float c0 = cs[4 * w + e], s0 = sn[4 * w + e], c1 = cs[4 * w + 2 + e], s1 = sn[4 * w + 2 + e];
          const float p = v0[2 * e], q = v0[2 * e + 1], r = v1[2 * e], z = v1[2 * e + 1];
          v0[2 * e] = p * c0 - q * s0;
          v0[2 * e + 1] = q * c0 + p * s0;
          v1[2 * e] = r * c1 - z * s1;
          v1[2 * e + 1] = z * c1 + r * s1;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float c = cs[4 * w + e], s = sn[4 * w + e], p = v0[e], q = v1[e];
          v0[e] = p * c - q * s;
          v1[e] = q * c + p * s;
        }
      }
    }
    if (h < a.hq) {
      *reinterpret_cast<float4*>(qd + h * HD + d0) = make_float4(v0[0], v0[1], v0[2], v0[3]);
      *reinterpret_cast<float4*>(qd + h * HD + d1) = make_float4(v1[0], v1[1], v1[2], v1[3]);
    } else if (is_page(pg, a.n_pages)) {
      const bool key = h < a.hq + a.hkv;
      T* dst = (T*)(key ? a.kpool : a.vpool) +
               page_offset(pg, a.hkv, key ? h - a.hq : h - a.hq - a.hkv, a.shift, pos, HD);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dst[d0 + e] = from_f32<T>(v0[e]);
        dst[d1 + e] = from_f32<T>(v1[e]);
      }
    }
  }
}

template <typename T>
static void append_by_hd(const PageAppendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.rows * a.lr));
  switch (a.hd) {
    case 32: SR_LAUNCH((append_kernel<T, 32>), grid, dim3(256), 0, s, a); break;
    case 64: SR_LAUNCH((append_kernel<T, 64>), grid, dim3(256), 0, s, a); break;
    default: SR_LAUNCH((append_kernel<T, 128>), grid, dim3(256), 0, s, a); break;
  }
  SR_CHECK_LAUNCH();
}

void page_append(const PageAppendArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.lr <= 0) return;
  if (a.dtype == SR_BF16) append_by_hd<bf16_t>(a, s);
  else append_by_hd<float>(a, s);
}

}  // namespace sr
