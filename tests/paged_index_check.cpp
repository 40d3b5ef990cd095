// Every index that csrc/paged.h gives, over small sizes, against what it should
// be: built and run on the host by test_ops_abi.py.
#include <cstdio>
#include <set>

#include "paged.h"

using namespace sr;

static int fail(const char* what, int a, int b, int c, int d) {
  std::printf("%s: %d %d %d %d\n", what, a, b, c, d);
  return 1;
}

int main() {
  // the blocks of a unit of work hold exactly its keys, ascending, and a lane
  // whose key is not among them reads one that is, in the same 16
  for (int from = 0; from <= 128; from += 32)
    for (int end = 0; end <= 170; ++end)
      for (int lo = 0; lo < imax(end, 1); lo += lo < 70 ? 1 : 7)
        for (int sinks = 0; sinks <= 110; sinks += sinks < 40 ? 1 : 9) {
          KeyBlocks b;
          b.set(from, sinks, lo, end);
          auto seen = [&](int j) { return j < end && (j < imin(sinks, lo) || j >= lo); };
          std::set<int> want, got;
          for (int j = from; j < end; ++j)
            if (seen(j)) want.insert(j >> 5);
          int prev = -1;
          for (int i = 0; i < b.count; ++i) {
            const int k = b.key0(i);
            if (k % 32 || k / 32 <= prev) return fail("order", from, sinks, lo, end);
            prev = k / 32;
            got.insert(prev);
            bool all = true;
            for (int j = k; j < k + 32; ++j) all = all && seen(j);
            if (b.all32(k) && !all) return fail("all32", from, sinks, lo, end);
            for (int a = k; a < k + 32; a += 16) {
              bool any = false;
              for (int j = a; j < a + 16; ++j) any = any || seen(j);
              if (any != b.any16(a)) return fail("any16", a, sinks, lo, end);
              if (!any) continue;
              for (int j = a; j < a + 16; ++j) {
                const int s = b.safe(a, j);
                if (s < a || s >= a + 16 || !seen(s) || (seen(j) && s != j)) return fail("safe", a, sinks, lo, end);
              }
            }
          }
          if (got != want) return fail("blocks", from, sinks, lo, end);
        }
  // lengths, new tokens and windows stay in range whatever the device holds
  const int odd[] = {INT32_MIN, -7, -1, 0, 1, 5, 31, 32, 1 << 20, INT32_MAX};
  for (int max_pages : {1, 7, kPageMaxPerRow})
    for (int shift = 4; shift <= 8; ++shift)
      for (int len : odd) {
        const int L = clamp_len(len, max_pages, shift);
        if (L < 0 || L > max_pages << shift) return fail("clamp_len", len, max_pages, shift, L);
        for (int n : odd)
          for (int lr : {0, 1, 9, 1 << 20}) {
            const int m = clamp_new(n, lr, L);
            if (m < 0 || m > lr || m > L) return fail("clamp_new", n, lr, L, m);
          }
        for (int w : {0, 1, 40, INT32_MAX}) {
          const int lo = window_start(L, w);
          if (lo < 0 || lo > L || (w > 0 && L - lo > w - 1) || (w == 0 && lo)) return fail("window", L, w, lo, 0);
        }
      }
  // slots of a page: inside the page, in 64 bits
  for (int shift = 4; shift <= 8; ++shift)
    for (int pg : {0, 1, kPageMaxPages - 1})
      for (int a = 0; a < 3 << shift; ++a) {
        const int64_t page = (int64_t)8 << shift, at = page_offset(pg, 8, 7, shift, a, 128);
        const int64_t want = (pg * page + ((int64_t)7 << shift) + a % (1 << shift)) * 128;
        if (at != want) return fail("page_offset", pg, shift, a, 0);
      }
  for (int p = -1; p <= 600; ++p) {
    const bool ok = p == 16 || p == 32 || p == 64 || p == 128 || p == 256;
    if ((page_shift(p) >= 0) != ok || (ok && 1 << page_shift(p) != p)) return fail("page_shift", p, 0, 0, 0);
  }
  std::puts("ok");
  return 0;
}
