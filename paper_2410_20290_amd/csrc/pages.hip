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
constexpr int kPlanRows = kPageMaxRows / kPlanThreads;   // rows of a thread of the plan kernel

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

// -------------------------------------------------------------------- fork
// One thread per entry of the new table; the counts start at 0.
__global__ void __launch_bounds__(256) fork_table_kernel(PageForkArgs a) {
  const int64_t tid = (int64_t)blockIdx.x * 256 + threadIdx.x, nthr = (int64_t)gridDim.x * 256;
  for (int64_t p = tid; p < a.n_pages; p += nthr) a.refs_out[p] = 0;
  const int64_t n = (int64_t)a.new_rows * a.max_pages;
  for (int64_t i = tid; i < n; i += nthr) {
    const int j = (int)(i / a.max_pages), c = (int)(i - (int64_t)j * a.max_pages);
    const int par = a.parent[j];
    int pg = -1, len = 0;
    if ((uint32_t)par < (uint32_t)a.rows) {
      len = clamp_len(a.lens[par], a.max_pages, a.shift);
      if (c < pages_of(len, a.shift)) {
        pg = a.table[(int64_t)par * a.max_pages + c];
        // out of every later token's sight: the next one sits at position len
        const bool behind = ((c + 1) << a.shift) <= window_start(len, a.window) && (c << a.shift) >= a.sinks;
        if (!is_page(pg, a.n_pages) || behind) pg = -1;
      }
    }
    a.table_out[i] = pg;
    if (c == 0) a.lens_out[j] = len;
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
// new entry, their number, where they start in the list of free pages, and the
// new length; and the pages to copy.
struct ReservePlan {
  int32_t *start, *need, *first, *new_len;   // [rows]
  int32_t *src, *at, *part;                  // [rows] pairs: page, index into free, filled slots
  int32_t* free;                             // [n_pages]
};
constexpr int kReserveArrays = 7;
__host__ __device__ inline ReservePlan reserve_plan(int32_t* scratch, int rows) {
  ReservePlan p;
  p.start = scratch;
  p.need = scratch + rows;
  p.first = scratch + 2 * rows;
  p.new_len = scratch + 3 * rows;
  p.src = scratch + 4 * rows;
  p.at = scratch + 5 * rows;
  p.part = scratch + 6 * rows;
  p.free = scratch + kReserveArrays * rows;
  return p;
}

// A hash table in LDS counts, for every part-filled last page that more than
// one entry names, the rows that add tokens to it, and finds the lowest.
constexpr int kHashBits = 13, kHashSize = 1 << kHashBits;   // twice the rows: probing ends

// Work-group 0 plans; the others copy the table and the counts meanwhile (the
// second launch writes what changes).
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
  __shared__ int hkey[kHashSize], hcount[kHashSize], hlow[kHashSize];
  __shared__ int wsum[kPlanWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kHashSize; i += kPlanThreads) {
    hkey[i] = -1;
    hcount[i] = 0;
    hlow[i] = INT_MAX;
  }
  __syncthreads();
  const ReservePlan pl = reserve_plan(a.scratch, a.rows);
  int len[kPlanRows], add[kPlanRows], last[kPlanRows], slot[kPlanRows], refs[kPlanRows];
  bool lost[kPlanRows];   // the part-filled last page's entry names no page
  int wide = 0;
#pragma unroll
  for (int k = 0; k < kPlanRows; ++k) {
    const int r = tid * kPlanRows + k;
    len[k] = add[k] = 0;
    slot[k] = last[k] = -1;
    lost[k] = false;
    if (r >= a.rows) continue;
    len[k] = clamp_len(a.lens[r], mp, shift);
    add[k] = imax(0, a.n_add ? a.n_add[r] : a.n_add_all);
    if (add[k] > (mp << shift) - len[k]) {
      ++wide;
      add[k] = (mp << shift) - len[k];
    }
    if (add[k] == 0 || (len[k] & mask) == 0) continue;
    last[k] = a.table[(int64_t)r * mp + pages_of(len[k], shift) - 1];
    lost[k] = !is_page(last[k], np);
    refs[k] = lost[k] ? 0 : a.refs[last[k]];
    if (refs[k] < 2) continue;
    int h = (int)(((uint32_t)last[k] * 2654435761u) >> (32 - kHashBits));
    for (;; h = (h + 1) & (kHashSize - 1)) {
      const int was = atomicCAS(&hkey[h], -1, last[k]);
      if (was == -1 || was == last[k]) break;
    }
    slot[k] = h;
    atomicAdd(&hcount[h], 1);
    atomicMin(&hlow[h], r);
  }
  __syncthreads();
  int need[kPlanRows], nneed = 0, ncopy = 0;
  bool copy[kPlanRows];
#pragma unroll
  for (int k = 0; k < kPlanRows; ++k) {
    const int r = tid * kPlanRows + k;
    copy[k] = slot[k] >= 0 && !(hcount[slot[k]] == refs[k] && hlow[slot[k]] == r);
    need[k] = pages_of(len[k] + add[k], shift) - pages_of(len[k], shift) + (copy[k] || lost[k] ? 1 : 0);
    nneed += need[k];
    ncopy += copy[k] ? 1 : 0;
  }
  int total, copies, wides;
  int first = plan_scan(nneed, wsum, &total);
  int pair = plan_scan(ncopy, wsum, &copies);
  plan_scan(wide, wsum, &wides);
  // The lowest free pages, 64 KB of counts at a time: a wave takes 1024
  // consecutive ones.
  constexpr int STEPS = 16;
  int found = 0;
  for (int base = 0; base < np && found < total; base += kPlanThreads * STEPS) {
    const int p0 = base + wave * 64 * STEPS + lane;
    uint64_t bits[STEPS];
    int n = 0;
    int v[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) v[i] = p0 + 64 * i < np ? a.refs[p0 + 64 * i] : 1;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      bits[i] = __ballot(v[i] == 0);
      n += __popcll(bits[i]);
    }
    int tot;
    int at = found + __shfl(plan_scan(lane == 0 ? n : 0, wsum, &tot), 0, 64);
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int rank = at + __popcll(bits[i] & ((1ull << lane) - 1));
      if (v[i] == 0 && rank < total) pl.free[rank] = p0 + 64 * i;
      at += __popcll(bits[i]);
    }
    found += tot;
  }
  const int missing = imax(0, total - found);
  const bool ok = missing == 0 && wides == 0;
#pragma unroll
  for (int k = 0; k < kPlanRows; ++k) {
    const int r = tid * kPlanRows + k;
    if (r >= a.rows) continue;
    const int got = ok ? add[k] : 0;
    pl.start[r] = pages_of(len[k], shift) - (copy[k] || lost[k] ? 1 : 0);
    pl.need[r] = ok ? need[k] : 0;
    pl.first[r] = first;
    pl.new_len[r] = len[k] + got;
    a.granted[r] = got;
    if (copy[k]) {
      pl.src[pair] = last[k];
      pl.at[pair] = first;
      pl.part[pair] = len[k] & mask;
      ++pair;
    }
    first += need[k];
  }
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
  for (int r = w0; r < a.rows; r += nw) {
    const int need = pl.need[r], first = pl.first[r], start = pl.start[r];
    for (int k = lane; k < need; k += 64) {
      const int pg = pl.free[first + k];
      a.table_out[(int64_t)r * a.max_pages + start + k] = pg;
      a.refs_out[pg] = 1;
    }
    if (lane == 0) a.lens_out[r] = pl.new_len[r];
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
// rotated pairs, or 8 dimensions that pass.
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
