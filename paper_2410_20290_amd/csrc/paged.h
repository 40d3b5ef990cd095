// Index arithmetic of the paged candidate cache: which keys a query sees, in
// which order the attention kernels visit them, and which address every lane
// reads.  Plain functions of integers, so that the host can check every index
// they give (no HIP header is needed to compile them).
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define SR_HD __host__ __device__ __forceinline__
#else
#define SR_HD inline
#endif

namespace sr {

SR_HD int imin(int a, int b) { return a < b ? a : b; }
SR_HD int imax(int a, int b) { return a > b ? a : b; }

// Limits of the interface: positions stay below 2^24, table indices below 2^28
// and page ids below 2^20, so all of them are ints; element offsets into a
// pool are 64 bits.
constexpr int kPageMaxRows = 4096;
constexpr int kPageMaxPerRow = 65536;
constexpr int kPageMaxPages = 1 << 20;
constexpr int kMaxGroups = (1 << 24) - 1;   // work-groups of 256 in a launch: work-items are counted in 32 bits

// log2 of the page size, or -1 where it is none of 16 .. 256.
SR_HD int page_shift(int page_tokens) {
  for (int s = 4; s <= 8; ++s)
    if (page_tokens == 1 << s) return s;
  return -1;
}

// A row's tokens, and how many of them are the call's (the last ones).
SR_HD int clamp_len(int len, int max_pages, int shift) { return imax(0, imin(len, max_pages << shift)); }
SR_HD int clamp_new(int n_new, int lr, int len) { return imax(0, imin(n_new, imin(lr, len))); }

// The first key of the window of a query at position p (0 without a window).
SR_HD int window_start(int p, int window) { return window > 0 ? imax(0, p - window + 1) : 0; }

// Keys seen by some query of a unit of work: [0, sinks) and [lo, end), with
// sinks <= lo <= end, among keys from `from` on (a multiple of 32; those before
// are another pass's).  They are visited in blocks of 32 keys aligned to 32:
// block(0 .. count - 1) are the blocks that hold any, ascending.
struct KeyBlocks {
  int sinks, lo, end;
  int first, nsink, gap, count;

  SR_HD void set(int from, int sinks_, int lo_, int end_) {
    lo = lo_;
    end = end_;
    sinks = imin(sinks_, lo_);
    first = from >> 5;
    const int last = (imax(end, from) + 31) >> 5;
    nsink = imax(0, ((sinks + 31) >> 5) - first);
    const int w0 = imin(last, imax(lo, from) >> 5);
    gap = imax(0, w0 - (first + nsink));
    count = imax(0, last - first - gap);
    if (end <= from) count = imin(count, nsink);
  }
  SR_HD int key0(int i) const { return 32 * (first + i + (i >= nsink ? gap : 0)); }
  SR_HD bool has(int k) const { return k < end && (k < sinks || k >= lo); }
  // Whether the 16 keys from a on hold one of them.
  SR_HD bool any16(int a) const { return a < end && (a < sinks || a + 16 > lo); }
  // Whether all 32 keys from a on are among them.
  SR_HD bool all32(int a) const { return a + 32 <= end && (a >= lo || a + 32 <= sinks); }
  // Key j of the 16 from a on, of which any16(a), or where it is none of them
  // one that is: what a lane reads instead (its score is masked).
  SR_HD int safe(int a, int j) const {
    int k = imin(j, end - 1);
    if (k >= sinks && k < lo) k = lo < a + 16 ? lo : sinks - 1;
    return k;
  }
};

// Element offset of the slot of key a (of a page `pg`) in a layer's block of
// keys or values, for one KV head.
SR_HD int64_t page_offset(int pg, int n_kv_heads, int h, int shift, int a, int head_dim) {
  return ((((int64_t)pg * n_kv_heads + h) << shift) + (a & ((1 << shift) - 1))) * head_dim;
}

}  // namespace sr
