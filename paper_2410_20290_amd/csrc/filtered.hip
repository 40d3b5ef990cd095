// Next tokens by temperature, top-k, top-p and min-p, from given random words.
//
// The entries of a row are ordered by value, then index; each weighs an integer
// (draw_weights.h).  top-k and top-p keep a prefix of that order, min-p those from
// a weight on, and the token is found by an inverse CDF in index order, all on
// 64-bit integers, so that no grouping of a sum can change a result.
//
// A work-group takes a row; its waves take tiles of 1024 entries.  After the
// maximum, entries are counted (top-k) or weighed (top-p) in bins of z = (l - max)
// / T, 92 to a unit of z: the bin that holds the border of the kept prefix follows
// from a scan of the bins.  Where the prefix up to that bin is short enough it is
// listed in LDS, sorted, cut and drawn from there; else only the border's bin is
// listed, sorted and cut, and another pass sums the kept weights tile by tile.
#include <algorithm>

#include "common.h"
#include "draw_weights.h"
#include "kernels.h"
#include "logit_rows.h"

#pragma clang fp contract(off)

namespace sr {

constexpr int kFltThreads = 1024;
constexpr int kFltWaves = kFltThreads / 64;
constexpr int kFltBins = 2048;     // the last one: entries of weight 0, never counted
constexpr int kFltList = 4096;     // listed entries
constexpr int kFltTiles = 256;     // of a row (262144 entries)

struct FilteredShared {
  uint64_t mass[kFltBins];   // later: the list's weights, then its draw
  uint64_t list[kFltList];
  uint64_t tile[kFltTiles];
  uint64_t wave[kFltWaves + 1];
  uint32_t count[kFltBins];
  int n, bin, kept;
  uint32_t before;
  uint64_t mass_before;
};

// A row's numbers.
struct RowDraw {
  float m, inv_t;
  bool greedy;
};

__device__ __forceinline__ float seen(float x) { return fmaxf(x, -INFINITY); }   // NaN counts as -inf
__device__ __forceinline__ uint64_t row_weight(float l, const RowDraw& r) {
  return l == r.m ? (uint64_t)1 << 32 : weight_of(l, r.m, r.inv_t);
}
// The bin of an entry: monotone in its value.
__device__ __forceinline__ int row_bin(float l, const RowDraw& r) {
  const float z = __fmul_rn(__fsub_rn(l, r.m), r.inv_t);
  const float d = fminf(__fmul_rn(z, -92.f), (float)(kFltBins - 1));   // (z <= -22.25: weight 0)
  return l == r.m ? 0 : (int)d;
}

// Inclusive sums over the work-group's threads, and their total.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* wsum, uint64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t u = shfl_up_u64(v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 63) wsum[wave] = v;
  __syncthreads();
  uint64_t base = 0, all = 0;
  for (int w = 0; w < kFltWaves; ++w) {
    if (w < wave) base += wsum[w];
    all += wsum[w];
  }
  *total = all;
  return base + v;
}

// Sorts the first n (up to kFltList) words, descending; n2 >= n a power of two.
__device__ void sort_words(uint64_t* w, int n2) {
  for (int k = 2; k <= n2; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int i = threadIdx.x; i < n2 / 2; i += kFltThreads) {
        const int a = (i / j) * 2 * j + (i % j), b = a + j;
        const uint64_t x = w[a], y = w[b];
        if ((x < y) == ((a & k) == 0)) {
          w[a] = y;
          w[b] = x;
        }
      }
      __syncthreads();
    }
}

__device__ __forceinline__ uint64_t scaled_word(uint64_t x, uint64_t total) {   // floor(x total / 2^32)
  return x * (total >> 32) + ((x * (total & 0xFFFFFFFFull)) >> 32);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kFltThreads) filtered_kernel(FilteredArgs a) {
  __shared__ FilteredShared sh;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* x = (const T*)a.logits + r * a.row_stride;
  const int vocab = a.vocab;
  const float T_ = a.temperature[r];
  RowDraw rd;
  rd.inv_t = (float)(1.0 / (double)T_);
  rd.greedy = !(T_ > 0.f) || !(rd.inv_t <= 3.402823466e38f);

  // f(values, base) for the wave's tiles, the next one's loads in flight
  auto pass = [&](auto&& f) {
    float v[16], nx[16];
    const int step = kFltWaves * kLpTile;
    int base = wave * kLpTile;
    if (base < vocab) Tile<T, VEC>::load(x, base, vocab, lane, v);
    for (; base < vocab; base += step) {
      if (base + step < vocab) Tile<T, VEC>::load(x, base + step, vocab, lane, nx);
      f(v, base);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = nx[e];
    }
  };
  auto index = [&](int base, int e) { return Tile<T, VEC>::index(base, e, lane); };

  // the best entry
  uint64_t best = 0;
  {
    float mt = -INFINITY;
    int at = 0;
    pass([&](const float(&v)[16], int base) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (v[e] > mt) {
          mt = v[e];
          at = index(base, e);
        }
    });
    best = entry_word(mt, at);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t u = shfl_xor_u64(best, o);
      best = u > best ? u : best;
    }
    if (lane == 0) sh.wave[wave] = best;
    __syncthreads();
    for (int w = 0; w < kFltWaves; ++w) best = sh.wave[w] > best ? sh.wave[w] : best;
    __syncthreads();
  }
  rd.m = word_value(best);
  auto answer = [&](int token, float lp, int kept) {   // (one thread)
    if (a.token) a.token[r] = token;
    if (a.logprob) a.logprob[r] = lp;
    if (a.kept) a.kept[r] = kept;
  };
  if (rd.m == -INFINITY) {
    if (tid == 0) answer(0, -INFINITY, 0);
    return;
  }
  if (rd.greedy) {
    if (tid == 0) answer(word_index(best), 0.f, 1);
    return;
  }
  const uint64_t word = a.random[r * a.random_stride];
  const int top_k = a.top_k[r];
  const float top_p = a.top_p[r], min_p = a.min_p[r];
  const bool by_p = top_p < 1.f;   // (false for NaN)
  const uint64_t part = by_p ? (uint64_t)((double)fmaxf(top_p, 0.f) * 4294967296.0) : 0;
  const uint64_t least = min_p > 0.f ? (uint64_t)((double)fminf(min_p, 1.f) * 4294967296.0) : 0;
  // the least weight of a prefix that holds top_p of `total`
  auto needed = [&](uint64_t total) {
    const uint64_t low = part * (total & 0xFFFFFFFFull);
    const uint64_t need = part * (total >> 32) + (low >> 32) + ((low & 0xFFFFFFFFull) ? 1 : 0);
    return need > 1 ? need : (uint64_t)1;
  };
  uint64_t border = 0;   // words below it are not kept

  // Fills the bins with counts (and weights) of the entries from `border` on.
  auto fill = [&](bool weigh) {
    for (int i = tid; i < kFltBins; i += kFltThreads) {
      sh.count[i] = 0;
      if (weigh) sh.mass[i] = 0;
    }
    __syncthreads();
    pass([&](const float(&v)[16], int base) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float l = seen(v[e]);
        const int b = row_bin(l, rd);
        if (b < kFltBins - 1 && entry_word(l, index(base, e)) >= border) {
          atomicAdd(&sh.count[b], 1u);
          if (weigh) atomicAdd((unsigned long long*)&sh.mass[b], (unsigned long long)row_weight(l, rd));
        }
      }
    });
    __syncthreads();
  };
  // The first bin up to which the counts (or weights) reach `target`, with what
  // lies before it; false where all together do not.
  auto find = [&](bool weigh, uint64_t target, uint64_t* total) {
    const int i = 2 * tid;
    const uint64_t v0 = weigh ? sh.mass[i] : sh.count[i], v1 = weigh ? sh.mass[i + 1] : sh.count[i + 1];
    const uint64_t inc = block_scan(v0 + v1, sh.wave, total), exc = inc - v0 - v1;
    if (exc < target && target <= inc) sh.bin = exc + v0 >= target ? i : i + 1;
    __syncthreads();
    if (*total < target) return false;
    // what lies before: counts and weights alike
    uint64_t all;
    const int b = sh.bin;
    const uint64_t ci = block_scan((i < b ? sh.count[i] : 0) + (i + 1 < b ? sh.count[i + 1] : 0), sh.wave, &all);
    (void)ci;
    if (tid == 0) sh.before = (uint32_t)all;
    if (weigh) {
      block_scan((i < b ? sh.mass[i] : 0) + (i + 1 < b ? sh.mass[i + 1] : 0), sh.wave, &all);
      if (tid == 0) sh.mass_before = all;
    }
    __syncthreads();
    return true;
  };
  // Lists the entries for which f holds (at most kFltList, as the caller knows),
  // sorted; returns their number.
  auto listed = [&](auto&& f) {
    if (tid == 0) sh.n = 0;
    __syncthreads();
    pass([&](const float(&v)[16], int base) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float l = seen(v[e]);
        const uint64_t w = entry_word(l, index(base, e));
        const bool in = index(base, e) < vocab && f(l, w);
        const uint64_t mask = __ballot(in);
        if (mask == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n, __popcll(mask));
        at = __builtin_amdgcn_readfirstlane(at) + __popcll(mask & ((1ull << lane) - 1));
        if (in && at < kFltList) sh.list[at] = w;
      }
    });
    __syncthreads();
    const int n = min(sh.n, kFltList);
    int n2 = 1;
    while (n2 < n) n2 <<= 1;
    for (int i = n + tid; i < n2; i += kFltThreads) sh.list[i] = 0;
    __syncthreads();
    sort_words(sh.list, n2);
    return n;
  };
  // The `rank`-th entry in order (from 1, by counts) or the first one up to which
  // the weights reach `rank`, among the entries of bin `b`: refined by digits of
  // their values until a list holds them, and by index among equals.
  auto border_in = [&](int b, uint64_t rank, bool weigh) -> uint64_t {
    uint32_t prefix = 0;   // upper bits of the values' keys that are settled
    int bits = 0;
    int n = (int)sh.count[b];
    __syncthreads();
    auto in_prefix = [&](uint64_t w) { return bits == 0 || (uint32_t)(w >> 32) >> (32 - bits) == prefix; };
    while (n > kFltList && bits < 32) {
      const int digit = min(11, 32 - bits);
      for (int i = tid; i < kFltBins; i += kFltThreads) {
        sh.count[i] = 0;
        sh.mass[i] = 0;
      }
      __syncthreads();
      pass([&](const float(&v)[16], int base) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float l = seen(v[e]);
          const uint64_t w = entry_word(l, index(base, e));
          if (row_bin(l, rd) == b && w >= border && in_prefix(w)) {
            // (descending: the largest digit first)
            const int d = (1 << digit) - 1 - (int)(((uint32_t)(w >> 32) >> (32 - bits - digit)) & ((1u << digit) - 1));
            atomicAdd(&sh.count[d], 1u);
            if (weigh) atomicAdd((unsigned long long*)&sh.mass[d], (unsigned long long)row_weight(l, rd));
          }
        }
      });
      __syncthreads();
      uint64_t total;
      find(weigh, rank, &total);
      rank -= weigh ? sh.mass_before : sh.before;
      n = (int)sh.count[sh.bin];
      prefix = (prefix << digit) | (uint32_t)((1 << digit) - 1 - sh.bin);
      bits += digit;
      __syncthreads();
    }
    if (n <= kFltList) {
      n = listed([&](float l, uint64_t w) { return row_bin(l, rd) == b && w >= border && in_prefix(w); });
      // four entries a thread
      uint64_t w4[4], sum = 0, total;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * tid + e;
        w4[e] = i >= n ? 0 : weigh ? row_weight(word_value(sh.list[i]), rd) : 1;
        sum += w4[e];
      }
      uint64_t run = block_scan(sum, sh.wave, &total) - sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (run < rank && rank <= run + w4[e]) sh.bin = 4 * tid + e;
        run += w4[e];
      }
      __syncthreads();
      const uint64_t found = sh.list[sh.bin];
      __syncthreads();
      return found;
    }
    // all equal: by index, of their common weight (at least 1: bin b is counted)
    const float l = word_value((uint64_t)prefix << 32);
    if (weigh) {
      const uint64_t w = row_weight(l, rd);
      rank = (rank + w - 1) / w;
    }
    if (tid < kFltTiles) sh.tile[tid] = 0;
    __syncthreads();
    auto tied = [&](float v, int i) {
      const uint64_t w = entry_word(seen(v), i);
      return i < vocab && (uint32_t)(w >> 32) == prefix && w >= border;
    };
    pass([&](const float(&v)[16], int base) {
      int c = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) c += __popcll(__ballot(tied(v[e], index(base, e))));
      if (lane == 0) sh.tile[base / kLpTile] = (uint64_t)c;
    });
    uint64_t total;
    __syncthreads();
    const uint64_t mine = tid < kFltTiles ? sh.tile[tid] : 0;
    uint64_t inc = block_scan(mine, sh.wave, &total);
    if (inc - mine < rank && rank <= inc) {
      sh.bin = tid;
      sh.mass_before = inc - mine;
    }
    __syncthreads();
    rank -= sh.mass_before;
    const int i = sh.bin * kLpTile + tid;   // an entry a thread
    const bool in = i < vocab && tied(to_f32<T>(x[min(i, vocab - 1)]), i);
    inc = block_scan(in ? 1 : 0, sh.wave, &total);
    if (in && inc == rank) sh.bin = i;
    __syncthreads();
    const uint64_t found = ((uint64_t)prefix << 32) | (uint32_t)~sh.bin;
    __syncthreads();
    return found;
  };

  // What the list of the leading bins holds, cut by the filters and drawn from.
  auto draw_from_list = [&](int last_bin, uint64_t keep, bool p_total_known, uint64_t p_total) {
    const int n = listed([&](float l, uint64_t) { return row_bin(l, rd) <= last_bin; });
    const int cut = (int)(keep < (uint64_t)n ? keep : (uint64_t)n);
    uint64_t w4[4], sum = 0, total;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      w4[e] = i < cut ? row_weight(word_value(sh.list[i]), rd) : 0;
      sum += w4[e];
    }
    uint64_t run = block_scan(sum, sh.wave, &total) - sum;
    if (by_p) {
      const uint64_t need = needed(p_total_known ? p_total : total);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint64_t w = w4[e];
        if (run >= need) w4[e] = 0;
        run += w;
      }
    }
    int kept = 0, n_pow = 1;
    sum = 0;
    while (n_pow < n) n_pow <<= 1;
    __syncthreads();
    // by index: words of (inverted index, weight), descending
    uint64_t i4[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * tid + e;
      if (w4[e] < least) w4[e] = 0;
      kept += w4[e] != 0;
      sum += w4[e];
      i4[e] = i < n ? ((uint64_t)(0x3FFFF - word_index(sh.list[i])) << 33) | w4[e] : 0;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (4 * tid + e < n_pow) sh.list[4 * tid + e] = i4[e];
    block_scan((uint64_t)kept, sh.wave, &total);
    kept = (int)total;
    block_scan(sum, sh.wave, &total);
    sort_words(sh.list, n_pow);
    const uint64_t t = scaled_word(word, total);
    sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      i4[e] = 4 * tid + e < n ? sh.list[4 * tid + e] : 0;
      sum += i4[e] & 0x1FFFFFFFFull;
    }
    uint64_t all;
    run = block_scan(sum, sh.wave, &all) - sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t w = i4[e] & 0x1FFFFFFFFull;
      if (run <= t && t < run + w)
        answer(0x3FFFF - (int)(i4[e] >> 33), (float)log((double)w / (double)total), kept);
      run += w;
    }
  };

  if (top_k >= 1 && top_k < vocab) {
    fill(false);
    uint64_t total;
    if (find(false, (uint64_t)top_k, &total)) {
      const int b = sh.bin;
      if (sh.before + sh.count[b] <= kFltList) {
        __syncthreads();
        draw_from_list(b, (uint64_t)top_k, false, 0);
        return;
      }
      const uint64_t rank = (uint64_t)top_k - sh.before;
      border = border_in(b, rank, false);
    }
  }
  if (by_p) {
    fill(true);
    uint64_t total;
    find(true, ~0ull, &total);
    const uint64_t need = needed(total);
    find(true, need, &total);
    const int b = sh.bin;
    if (border == 0 && sh.before + sh.count[b] <= kFltList) {
      __syncthreads();
      draw_from_list(b, ~0ull, true, total);
      return;
    }
    const uint64_t rank = need - sh.mass_before;
    border = border_in(b, rank, true);
  }

  // the kept weights tile by tile, then the tile, run and entry of the drawn point
  auto kept_weight = [&](float v, int i) -> uint64_t {
    const float l = seen(v);
    if (!(l > -INFINITY) || entry_word(l, i) < border) return 0;
    const uint64_t w = row_weight(l, rd);
    return w >= least ? w : 0;
  };
  if (tid < kFltTiles) sh.tile[tid] = 0;
  int kept = 0;
  __syncthreads();
  pass([&](const float(&v)[16], int base) {
    uint64_t w = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint64_t u = kept_weight(v[e], index(base, e));
      w += u;
      kept += u != 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) w += shfl_xor_u64(w, o);
    if (lane == 0) sh.tile[base / kLpTile] = w;
  });
  uint64_t total;
  block_scan((uint64_t)kept, sh.wave, &total);
  kept = (int)total;
  const uint64_t mine = tid < kFltTiles ? sh.tile[tid] : 0;
  uint64_t inc = block_scan(mine, sh.wave, &total);
  uint64_t t = scaled_word(word, total);
  if (inc - mine <= t && t < inc) {
    sh.bin = tid;
    sh.mass_before = inc - mine;
  }
  __syncthreads();
  t -= sh.mass_before;
  const int i = sh.bin * kLpTile + tid;   // an entry a thread
  const uint64_t w = i < vocab ? kept_weight(to_f32<T>(x[i]), i) : 0;
  uint64_t all;
  inc = block_scan(w, sh.wave, &all);
  if (inc - w <= t && t < inc) answer(i, (float)log((double)w / (double)total), kept);
}

size_t sample_filtered_scratch(int rows, int vocab) {
  (void)rows;
  (void)vocab;
  return 0;
}

template <typename T>
static void launch_filtered(const FilteredArgs& a, hipStream_t s) {
  const bool vec = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && (a.rows == 1 || a.row_stride * sizeof(T) % 16 == 0);
  if (vec) SR_LAUNCH((filtered_kernel<T, true>), dim3(a.rows), dim3(kFltThreads), 0, s, a);
  else SR_LAUNCH((filtered_kernel<T, false>), dim3(a.rows), dim3(kFltThreads), 0, s, a);
  SR_CHECK_LAUNCH();
}

void sample_filtered(const FilteredArgs& a, hipStream_t s) {
  if (a.rows <= 0) return;
  if (a.dtype == SR_BF16) launch_filtered<bf16_t>(a, s);
  else launch_filtered<float>(a, s);
}

}  // namespace sr
