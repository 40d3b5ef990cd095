// Next tokens by temperature, top-k, top-p and min-p, from given random words.
//
// The entries of a row are ordered by value, then index; each weighs an integer
// (draw_weights.h).  top-k and top-p keep a prefix of that order, min-p those from
// a weight on, and the token is found by an inverse CDF in index order, all on
// 64-bit integers, so that no grouping of a sum can change a result.
//
// Few entries matter to most draws, so a row is read twice: for its maximum, and to
// list its best entries (and weigh all of them where only top-p asks for the
// total).  Where "best" begins follows from the maxima of subsets of the row, 1024 by one
// work-group, 64 for every 4096 entries by the split readings: an entry that reaches the
// k-th largest of them is one of at least k.  Borders
// are then found in the list by counting and weighing its entries in 2048 bins.  Where
// the list is not enough (flat rows under top-p, a top-k above 1024, thousands of
// equals), the whole row goes into bins of z = (l - max) / T, 92 to a unit of z, then
// the border's bin is listed while what lies before it is weighed tile by tile.
//
// Measured with fp32 logits of 128256 entries: one row 18 us (its readings by 32
// work-groups; by one alone 50); 512 rows, of which one half keeps 50 and the rest follow
// other settings, 115 us.  The same rows (half of them flat) call after call: all with a
// top-k of 50 54 us, unfiltered 90 us, with a top-p of 0.9 182 us (263 MB, 48 us at the rate of
// a pure read: further readings, and the exponentials of 66 M entries).  256 flat rows of
// 32000 bf16 logits under a top-p of 0.95 57 to 60 us: maximum 6, whether a list can be
// enough 3, bins 15 (64-bit adds in LDS), the border's bin and the sums before it 12 (their
// exponentials), search 12, drawn entry 4 (timed one by one, with the gaps between them left
// out).
//
//   filtered_kernel         a work-group of 16 waves a row, from the logits to the token
//   filtered_maxima_kernel, few rows: the two readings by work-groups of four tiles
//   filtered_list_kernel    each, before filtered_kernel
#include <algorithm>
#include <cfloat>
#include <type_traits>

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
constexpr int kPLanes = 50;        // lanes of a wave whose maxima the list for top-p starts from
constexpr int kFltTiles = 256;     // of a row (262144 entries)
constexpr int kFltSplitWaves = 4;  // tiles of a work-group of the split readings
constexpr int kFltMaxima = 64 * kFltTiles / kFltSplitWaves;   // of a row, of the split readings
constexpr float kMasked = -3.38e38f;   // above the lowest values of fp32 and bf16, which mask entries

// Work-groups of a row of the split readings.
__host__ __device__ inline int split_chunks(int vocab) {
  return (vocab + kFltSplitWaves * kLpTile - 1) / (kFltSplitWaves * kLpTile);
}
// A row's scratch of the split readings.
struct FilteredRow {
  uint64_t total;            // weight of the row, or of what min-p keeps of it
  uint32_t n, kept;          // listed; kept by min-p
  uint64_t tile[kFltTiles];  // weights that min-p keeps, where nothing else filters
  uint64_t list[kFltList];
  float maxima[kFltMaxima];  // lane l of work-group c: of the entries that it reads
};

struct FilteredShared {
  uint64_t bins[kFltBins];   // counts or weights
  uint64_t list[kFltList];
  uint64_t tile[kFltTiles];
  uint64_t wave[kFltWaves], cand[128];
  uint64_t before, found, own;
  uint32_t wave32[kFltWaves];
  int n, c, bin;
};

// What all lanes hold alike, told to the compiler: it then stays in a scalar register.
__device__ __forceinline__ float uniform(float v) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}
__device__ __forceinline__ float seen(float x) { return fmaxf(x, -INFINITY); }   // NaN counts as -inf
// A row whose maximum is +inf is read as 0 there and -inf elsewhere.
template <int N>
__device__ __forceinline__ void read_infinite(float (&v)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = v[e] == INFINITY ? 0.f : -INFINITY;
}

// A row's settings.
struct RowDraw {
  float m, inv_t;
  bool greedy, by_k, by_p;
  int k;
  uint32_t least;   // least weight that min-p keeps (2^32 as 2^32 - 1, which no weight is)
  uint64_t part;

  __device__ __forceinline__ RowDraw(const FilteredArgs& a, int r) {
    const float t = a.temperature[r], p = a.top_p[r], mp = a.min_p[r];
    inv_t = (float)(1.0 / (double)t);
    greedy = !(t > 0.f) || !(inv_t <= 3.402823466e38f);
    if (greedy) inv_t = 1.f;
    k = a.top_k[r];
    by_k = k >= 1 && k < a.vocab;
    by_p = p < 1.f;   // (false for NaN)
    part = by_p ? (uint64_t)((double)fmaxf(p, 0.f) * 4294967296.0) : 0;
    least = mp > 0.f ? (uint32_t)fmin((double)fminf(mp, 1.f) * 4294967296.0, 4294967295.0) : 0;
  }
  // A weight, 2^32 as 2^32 - 1; and as it is.
  __device__ __forceinline__ uint32_t weight_word(float l) const { return weight32(l, m, inv_t); }
  __device__ __forceinline__ uint64_t weight(float l) const { return weight_of(l, m, inv_t); }
  // The sum of the weights of some entries of which keep(entry, weight word) holds (those
  // of 2^32, rare beside the maximum's own, are evaluated again; the empty asm keeps
  // that out of the straight line).
  template <int N, typename F>
  __device__ __forceinline__ uint64_t weights(const float (&v)[N], F&& keep) const {
    uint64_t w = 0;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint32_t u = weight_word(v[e]);
      const uint32_t k = keep(e, u) ? u : 0;
      w += k;
      top = max(top, k);
    }
    if (__builtin_expect(__any(top == 0xFFFFFFFFu), 0)) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float l = v[e];
        asm volatile("" : "+v"(l));
        const uint32_t u = weight_word(l);
        w += u == 0xFFFFFFFFu && keep(e, u) ? 1u : 0u;
      }
    }
    return w;
  }
  // Where an entry lies among the bins, as a number that grows as values fall.
  __device__ __forceinline__ float place(float l) const {
    const float z = __fmul_rn(__fsub_rn(l, m), inv_t);
    return fminf(__fmul_rn(z, -92.f), (float)(kFltBins - 1));   // (z <= -22.25: weight 0)
  }
  __device__ __forceinline__ int bin(float l) const { return (int)place(l); }
  // The least weight of a prefix that holds top_p of `total`.
  __device__ __forceinline__ uint64_t needed(uint64_t total) const {
    const uint64_t low = part * (total & 0xFFFFFFFFull);
    const uint64_t need = part * (total >> 32) + (low >> 32) + ((low & 0xFFFFFFFFull) ? 1 : 0);
    return need > 1 ? need : (uint64_t)1;
  }
};

__device__ __forceinline__ uint64_t scaled_word(uint64_t x, uint64_t total) {   // floor(x total / 2^32)
  return x * (total >> 32) + ((x * (total & 0xFFFFFFFFull)) >> 32);
}

// Inclusive sums over the lanes, by DPP: within rows of 16, then from row to row.
template <typename F>
__device__ __forceinline__ void wave_scan_steps(F&& step) {
  step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xF>{});   // row_shr 1, 2, 4, 8
  step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xF>{});
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});   // row_bcast 15, 31
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});
}
__device__ __forceinline__ uint32_t wave_scan32(uint32_t v) {
  wave_scan_steps([&](auto ctrl, auto rows) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  });
  return v;
}
__device__ __forceinline__ uint64_t wave_scan64(uint64_t v) {
  wave_scan_steps([&](auto ctrl, auto rows) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    v += (uint64_t)hi << 32 | lo;
  });
  return v;
}
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// The sum over the threads up to this one, and of all.
struct Scan {
  uint64_t upto, all;
};
__device__ __forceinline__ Scan block_scan(uint64_t v, FilteredShared& sh) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  v = wave_scan64(v);
  __syncthreads();   // (the last scan's sums are read)
  if (lane == 63) sh.wave[wave] = v;
  __syncthreads();
  const uint64_t w = wave_scan64(lane < kFltWaves ? sh.wave[lane] : 0);
  return {v + (wave > 0 ? lane_value(w, wave - 1) : 0), lane_value(w, 63)};
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  wave_scan_steps([&](auto ctrl, auto rows) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
  });
  return __builtin_amdgcn_readlane(v, 63);
}

// Sorts n2 (a power of two) words of the list, descending.
__device__ __forceinline__ void sort_words(uint64_t* w, int n2) {
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

__device__ __forceinline__ void clear_bins(FilteredShared& sh) {
  for (int i = threadIdx.x; i < kFltBins; i += kFltThreads) sh.bins[i] = 0;
  if (threadIdx.x == 0) sh.c = 0;
  __syncthreads();
}
__device__ __forceinline__ void add_to_bin(FilteredShared& sh, int b, uint64_t v) {
  atomicAdd((unsigned long long*)&sh.bins[b], (unsigned long long)v);
}
// The bins' sums over threads of two bins each.
__device__ __forceinline__ Scan scan_bins(FilteredShared& sh) {
  __syncthreads();
  return block_scan(sh.bins[2 * threadIdx.x] + sh.bins[2 * threadIdx.x + 1], sh);
}
// The first bin up to which they reach `target`, which they do: sh.bin, and what lies
// before it in sh.before.
__device__ __forceinline__ void find_bin(FilteredShared& sh, const Scan& s, uint64_t target) {
  const int i = 2 * threadIdx.x;
  const uint64_t exc = s.upto - sh.bins[i] - sh.bins[i + 1], mid = exc + sh.bins[i];
  if (exc < target && target <= s.upto) {
    sh.bin = mid < target ? i + 1 : i;
    sh.before = mid < target ? mid : exc;
  }
  __syncthreads();
}

// Borders and draws from a list of n entries: by top-k, by top-p, by index.  Each is
// the same search: entries of some size in 2048 bins, the bin that holds the sought
// point, and the entry among those of the bin.
struct ListCut {
  uint64_t border;      // words below it are not kept
  uint64_t found;       // the last search's entry (0: the list does not reach the point)
  uint64_t all, own;    // the last search's sum, and the found entry's part of it
  uint32_t kept;        // entries of it
};
enum { BY_K = 1, BY_P = 2, BY_INDEX = 4 };
// rank_k: the entries to keep; total: the weight that top-p goes by (0: of what is kept);
// rank_p: instead of it where not 0; bins over places [lo, lo + kFltBins / scale); least:
// the value that top-k's border has to reach (else nothing is found).
__device__ __forceinline__ ListCut cut_list(FilteredShared& sh, const RowDraw& rd, int n, int searches, uint64_t rank_k,
                                            uint64_t total, uint64_t rank_p, float lo, float scale, uint64_t word,
                                            float least = -FLT_MAX) {
  ListCut r{0, 0, 0, 0, 0};
  for (int which = BY_K; which <= BY_INDEX; which <<= 1) {   // (uniform; one body for the three)
    if (!(searches & which)) continue;
    clear_bins(sh);
    auto bin_of = [&](uint64_t w) {
      if (which == BY_INDEX) return word_index(w) >> 7;
      return min(kFltBins - 1, max(0, (int)((rd.place(word_value(w)) - lo) * scale)));
    };
    auto size_of = [&](uint64_t w) -> uint64_t {
      if (w < r.border) return 0;
      if (which == BY_K) return 1;
      const uint32_t u = rd.weight_word(word_value(w));
      if (which == BY_INDEX && u < rd.least) return 0;
      return (uint64_t)u + (u == 0xFFFFFFFFu ? 1 : 0);
    };
    uint32_t kept = 0;
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kFltThreads) {
      const uint64_t w = sh.list[i], u = size_of(w);
      if (u == 0) continue;
      ++kept;
      add_to_bin(sh, bin_of(w), u);
    }
    kept = wave_scan32(kept);   // (of the wave, in its last lane)
    if ((threadIdx.x & 63) == 63) sh.wave32[threadIdx.x >> 6] = kept;
    const Scan s = scan_bins(sh);
    r.all = s.all;
    r.kept = __builtin_amdgcn_readlane(wave_scan32((threadIdx.x & 63) < kFltWaves ? sh.wave32[threadIdx.x & 63] : 0), 63);
    uint64_t rank = which == BY_K ? rank_k : which == BY_INDEX ? scaled_word(word, s.all) + 1
                                                               : rank_p ? rank_p : rd.needed(total ? total : s.all);
    if (s.all < rank) {   // (uniform)
      r.found = 0;
      return r;
    }
    find_bin(sh, s, rank);
    const int bin = sh.bin;
    rank -= sh.before;
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kFltThreads) {
      const uint64_t w = sh.list[i];
      if (bin_of(w) != bin || size_of(w) == 0) continue;
      const int at = atomicAdd(&sh.c, 1);
      if (at < 128) sh.cand[at] = w;
    }
    __syncthreads();
    const int c = sh.c;
    if (c <= 128) {   // (always, by index)
      if ((int)threadIdx.x < c) {
        // larger words first; by index: larger inverted indices
        const uint64_t mask = which == BY_INDEX ? 0xFFFFFFFFull : ~0ull;
        const uint64_t mine = sh.cand[threadIdx.x], own = size_of(mine);
        uint64_t before = 0;
#pragma unroll 1
        for (int j = 0; j < c; ++j) {
          const uint64_t w = sh.cand[j];
          if ((w & mask) > (mine & mask)) before += size_of(w);
        }
        if (before < rank && rank <= before + own) {
          sh.found = mine;
          sh.own = own;
        }
      }
      __syncthreads();
    } else {   // many alike: in order
      int n2 = 1;
      while (n2 < n) n2 <<= 1;
      for (int i = n + threadIdx.x; i < n2; i += kFltThreads) sh.list[i] = 0;
      __syncthreads();
      sort_words(sh.list, n2);
      uint64_t sum = 0;
#pragma unroll 1
      for (int e = 0; e < 4; ++e) {   // (the bin's entries lie together)
        const int i = 4 * threadIdx.x + e;
        if (i < n && bin_of(sh.list[i]) == bin) sum += size_of(sh.list[i]);
      }
      uint64_t run = block_scan(sum, sh).upto - sum;
#pragma unroll 1
      for (int e = 0; e < 4; ++e) {
        const int i = 4 * threadIdx.x + e;
        const uint64_t u = i < n && bin_of(sh.list[i]) == bin ? size_of(sh.list[i]) : 0;
        if (run < rank && rank <= run + u) sh.found = sh.list[i];
        run += u;
      }
      __syncthreads();
    }
    r.found = sh.found;
    r.own = sh.own;
    if (which != BY_INDEX) r.border = r.found;
    if (which == BY_K && word_value(r.border) < least) {   // (uniform)
      r.found = 0;
      return r;
    }
  }
  return r;
}

// SPLIT: the row's maxima and list come from the split readings.
template <typename T, bool VEC, bool SPLIT>
__global__ void __launch_bounds__(kFltThreads, 8) filtered_kernel(FilteredArgs a) {
  __shared__ FilteredShared sh;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* x = (const T*)a.logits + r * a.row_stride;
  const int vocab = a.vocab;
  RowDraw rd(a, r);
  const FilteredRow* given = SPLIT ? (const FilteredRow*)a.scratch + r : nullptr;
  bool infinite = false;

  // f(values, base) for the wave's tiles, the next one's loads in flight
  auto pass = [&](auto&& f) {
    float v[16], nx[16];
    const int step = kFltWaves * kLpTile;
    int base = wave * kLpTile;
    if (base < vocab) Tile<T, VEC>::load(x, base, vocab, lane, v);
    for (; base < vocab; base += step) {
      if (base + step < vocab) Tile<T, VEC>::load(x, base + step, vocab, lane, nx);
      if (infinite) read_infinite(v);
      f(v, base);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = nx[e];
    }
  };
  // f(four neighbouring values, the first's index), the next ones' loads in flight: for
  // the passes of rows that no list decides, where fetching the code of a tile's 16
  // entries takes longer than running it (flat rows under a top-p of 0.95, 16 entries at a
  // time -> 4: 256 of 32000 bf16 values 66 -> 57.5 us, 512 of 128256 290 -> 222 us; whole tiles a
  // wave, so that a tile is summed once, a further 8 %).
  auto pass4 = [&](auto&& f) {
    auto load = [&](int i, float (&v)[4]) {
      if (VEC && i + 4 <= vocab) {
        if constexpr (sizeof(T) == 4) {
          const float4 q = *reinterpret_cast<const float4*>(x + i);
          v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        } else {
          const uint2 q = *reinterpret_cast<const uint2*>(x + i);
          v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xFFFF0000u);
          v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = i + e < vocab ? to_f32<T>(x[i + e]) : __uint_as_float(0x7FC00000u);
      }
      if (infinite) read_infinite(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = seen(v[e]);
    };
    // quarters of the wave's tiles, one after the other
    auto at = [&](int j) { return (wave + kFltWaves * (j >> 2)) * kLpTile + 256 * (j & 3) + 4 * lane; };
    float v[4], n1[4], n2[4];
    load(at(0), v);
    load(at(1), n1);
    const int tiles = (vocab + kLpTile - 1) / kLpTile, count = 4 * ((tiles - wave + kFltWaves - 1) / kFltWaves);
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
      load(at(j + 2), n2);
      f(v, at(j));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = n1[e];
        n1[e] = n2[e];
      }
    }
  };
  auto entry_at = [&](int i) {
    const float l = seen(to_f32<T>(x[i]));
    return !infinite ? l : l == INFINITY ? 0.f : -INFINITY;
  };
  auto index = [&](int base, int e) { return Tile<T, VEC>::index(base, e, lane); };
  auto answer = [&](int token, float lp, int kept) {   // (one thread)
    if (a.token) a.token[r] = token;
    if (a.logprob) a.logprob[r] = lp;
    if (a.kept) a.kept[r] = kept;
  };

  // Lists those of a tile that `wanted` holds for: one reservation a wave, its lanes' entries
  // one lane after the other.
  auto list_those = [&](const float(&v)[16], int base, auto&& wanted) {
    uint32_t in = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) in |= (uint32_t)wanted(v[e]) << e;
    if (!__any(in != 0)) return;
    const uint32_t mine = __popc(in), upto = wave_scan32(mine);
    int at = 0;
    if (lane == 63) at = atomicAdd(&sh.n, (int)upto);
    at = __builtin_amdgcn_readlane(at, 63) + (int)(upto - mine);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (in >> e & 1) {
        if (at < kFltList) sh.list[at] = entry_word(v[e], index(base, e));
        ++at;
      }
  };
  // A key that `want` of the wave's lanes reach with theirs (its upper 16 bits).
  auto reached = [&](uint32_t key, int want) {
    uint32_t t = 0;
#pragma unroll 1
    for (int b = 31; b >= 16; --b) {
      const uint32_t c = t | (1u << b);
      if (__popcll(__ballot(key >= c)) >= want) t = c;
    }
    return t;
  };
  auto key_of = [&](float l) { return (uint32_t)(entry_word(seen(l), 0) >> 32); };
  // (bits below -inf's read as a NaN)
  auto value_of = [&](uint32_t key) {
    const float f = word_value((uint64_t)key << 32);
    return f > -FLT_MAX ? f : -FLT_MAX;
  };

  // The maximum.  Under a top-k of a long row, every wave also lists what reaches a bound
  // that it takes from its first tile (from its later ones while they hold hardly more than
  // masks): if the k-th of the listed reaches the highest of these bounds, the list holds
  // the first k.  Else at least k entries reach that k-th, and the waves whose bounds are
  // above it list what lies between (logits that fall with the index, 512 x 128256, top-k
  // 50: 72 us, 62 where they do not; by bins 149).  Without k listed, or with too many, a
  // value that at least k entries reach is the least of the waves' k / waves-th largest
  // lanes' maxima (of those that have a whole tile), and another pass lists them (so it does
  // for top-p alone).
  const int whole = min(kFltWaves, vocab / kLpTile);
  const bool by_list = (rd.by_k && (rd.k <= 64 * whole || vocab <= kFltList)) || (!rd.by_k && rd.by_p);
  const bool at_once = !SPLIT && rd.by_k && !rd.greedy && rd.k <= kFltThreads && vocab >= 2 * kFltWaves * kLpTile;
  float from = -FLT_MAX, highest = -FLT_MAX;
  float own = kMasked;   // the wave's bound, and the tile from which on it holds
  int since = 0;
  if (tid == 0) sh.n = 0;
  __syncthreads();
  {
    float mt = -INFINITY;
    uint32_t bound = ~0u, first = 0;
    if constexpr (SPLIT) {
      for (int i = tid; i < split_chunks(vocab) * 64; i += kFltThreads) mt = fmaxf(mt, given->maxima[i]);
    } else {
      pass([&](const float(&v)[16], int base) {
#pragma unroll
        for (int e = 0; e < 16; ++e) mt = fmaxf(mt, v[e]);
        if (at_once) {
          if (own == kMasked) {   // (uniform)
            first = reached(key_of(mt), min(64, 8 + (int)(2 * (int64_t)rd.k * kLpTile / vocab)));
            own = uniform(fmaxf(value_of(first), kMasked));
            since = base;
          }
          list_those(v, base, [&](float l) { return l >= own; });
        }
      });
      if (wave < whole) bound = reached(key_of(mt), rd.by_k ? (rd.k + whole - 1) / whole : kPLanes);
    }
    const uint32_t best = wave_max_u32(key_of(mt));
    if (lane == 0) {
      sh.wave[wave] = (uint64_t)best << 32 | (uint32_t)~bound;
      if constexpr (!SPLIT) sh.wave32[wave] = first;
    }
    __syncthreads();
    const uint64_t w = lane < kFltWaves ? sh.wave[lane] : 0;
    rd.m = word_value((uint64_t)wave_max_u32((uint32_t)(w >> 32)) << 32);
    if (vocab > kFltList) from = uniform(value_of(~wave_max_u32((uint32_t)w)));
    if constexpr (!SPLIT) highest = uniform(value_of(wave_max_u32(lane < kFltWaves ? sh.wave32[lane] : 0)));
  }
  if (rd.m == -INFINITY) {
    if (tid == 0) answer(0, -INFINITY, 0);
    return;
  }
  if (rd.m == INFINITY) {
    infinite = true;
    rd.m = 0.f;
    from = from == INFINITY ? 0.f : -FLT_MAX;
  }
  if (rd.greedy) {
    int at = 0x7FFFFFFF;
    if (SPLIT && given->n <= kFltList) {
      for (int i = tid; i < (int)given->n; i += kFltThreads)
        if (word_value(given->list[i]) == rd.m) at = min(at, word_index(given->list[i]));
    } else {
      pass([&](const float(&v)[16], int base) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (v[e] == rd.m) at = min(at, index(base, e));
      });
    }
    __syncthreads();
    const uint32_t best = wave_max_u32(~(uint32_t)at);
    if (lane == 0) sh.wave32[wave] = best;
    __syncthreads();
    const uint32_t all = wave_max_u32(lane < kFltWaves ? sh.wave32[lane] : 0);
    if (tid == 0) answer((int)~all, 0.f, 1);
    return;
  }
  const uint64_t word = a.random[r * a.random_stride];
  auto draw = [&](const ListCut& c) {
    if (tid == 0) answer(word_index(c.found), (float)log((double)c.own / (double)c.all), (int)c.kept);
  };

  // Under top-p alone, whether what reaches `from` is likely to hold top_p: its share of
  // the waves' first tiles.
  bool flat = false;
  if (!SPLIT && by_list && !rd.by_k && vocab > kFltList) {
    float v[16];
    uint64_t sums = 0;   // of weights cut to 2^12: what reaches `from` above, all of them below
    if (wave * kLpTile < vocab) {
      Tile<T, VEC>::load(x, wave * kLpTile, vocab, lane, v);
      if (infinite) read_infinite(v);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t u = rd.weight_word(v[e]) >> 20;
        sums += (v[e] >= from ? (uint64_t)u << 32 : 0) + u;
      }
    }
    sums = block_scan(sums, sh).all;
    flat = (float)(uint32_t)(sums >> 32) < 0.9f * (float)(uint32_t)sums * a.top_p[r];
  }

  // The list of the best, where it can be enough: that of the first pass, or ...
  float lo = from, hi = INFINITY;   // (another pass lists from lo on, below hi, ...)
  bool again = true;                // (... from the start, not what the first one left out)
  if (at_once && !infinite) {
    const int n = sh.n;
    if (n <= kFltList && n >= rd.k) {
      const ListCut c = cut_list(sh, rd, n, BY_K | (rd.by_p ? BY_P : 0) | BY_INDEX, (uint64_t)rd.k, 0, 0, 0.f, 1.f, word, highest);
      if (c.found) {
        draw(c);
        return;
      }
      lo = fmaxf(lo, uniform(word_value(c.border)));
      hi = own;
      again = false;
    }
  }
  // ... of another one.  (For a top-k near the number of lanes that would take in too many:
  // 6800 to 8800 entries for 1000 of 128256 in no order, 2300 to 3300 for 896.)
  if (by_list && !flat && (!at_once || infinite || rd.k <= kFltThreads * 7 / 8)) {
    int n;
    uint64_t total = 0;
    float end = (float)(kFltBins - 1);
    if constexpr (SPLIT) {
      n = (int)given->n;
      total = given->total;
      end = 0.f;
      if (n <= kFltList)
        for (int i = tid; i < n; i += kFltThreads) {
          sh.list[i] = given->list[i];
          end = fmaxf(end, rd.place(word_value(sh.list[i])));
        }
    } else {
      const bool weigh = !rd.by_k;
      __syncthreads();
      if (again) {
        end = rd.place(from);
        since = 0;
        if (tid == 0) sh.n = 0;
        __syncthreads();
      }
      if (lo < hi)
        pass([&](const float(&v)[16], int base) {
          if (weigh) total += rd.weights(v, [](int, uint32_t) { return true; });
          if (base >= since) list_those(v, base, [&](float l) { return (l >= lo) & (l < hi); });
        });
      total = block_scan(total, sh).all;   // (and every entry is listed)
      n = sh.n;
    }
    if constexpr (SPLIT) {
      // (places are not negative: their bits order them)
      const uint32_t best = wave_max_u32(__float_as_uint(end));
      if (lane == 0) sh.wave32[wave] = best;
      __syncthreads();
      end = __uint_as_float(wave_max_u32(lane < kFltWaves ? sh.wave32[lane] : 0));
      __syncthreads();
    }
    if (n <= kFltList) {
      const int searches = (rd.by_k && n > rd.k ? BY_K : 0) | (rd.by_p ? BY_P : 0) | BY_INDEX;
      const ListCut c = cut_list(sh, rd, n, searches, (uint64_t)rd.k, rd.by_k ? 0 : total, 0, 0.f, (float)kFltBins / (end + 1.f), word);
      if (c.found) {
        draw(c);
        return;
      }
    }
    __syncthreads();
  }

  // The whole row: top-k's border, then top-p's among what that keeps.
  uint64_t border = 0;   // words below it are not kept
  uint64_t kept = 0;
  bool summed = false;   // sh.tile and kept are those of the kept entries
  for (int which = BY_K; which <= BY_P; which <<= 1) {   // (uniform)
    const bool by_mass = which == BY_P;
    if (by_mass ? !rd.by_p : !rd.by_k) continue;
    // entries of bin `b` (any bin: -1) and of the values whose upper `bits` are `prefix`
    int b = -1, bits = 0;
    uint32_t prefix = 0;
    uint64_t rank = 0;
    auto asked = [&](float l, uint64_t w) {
      return w >= border && (b < 0 ? rd.bin(l) < kFltBins - 1 : rd.bin(l) == b) &&
             (bits == 0 || (uint32_t)(w >> 32) >> (32 - bits) == prefix);
    };
    bool some = true;
    uint64_t found = 0;
    while (true) {   // by bins, then by digits of the values (the largest first), until a list holds them
      const int digit = min(11, 32 - bits);
      clear_bins(sh);
      if (tid < kFltTiles) sh.tile[tid] = 0;
      pass4([&](const float(&v)[4], int i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l = v[e];
          const uint64_t w = entry_word(l, i + e);
          if (!asked(l, w)) continue;
          const int to = b < 0 ? rd.bin(l)
                               : (1 << digit) - 1 - (int)(((uint32_t)(w >> 32) >> (32 - bits - digit)) & ((1u << digit) - 1));
          add_to_bin(sh, to, by_mass ? rd.weight(l) : 1);
        }
      });
      const Scan s = scan_bins(sh);
      if (b < 0) {
        rank = by_mass ? rd.needed(s.all) : (uint64_t)rd.k;
        some = s.all >= rank;
        if (!some) break;   // (fewer than top_k have weights)
      }
      find_bin(sh, s, rank);
      rank -= sh.before;
      if (b < 0) {
        b = sh.bin;
      } else {
        prefix = (prefix << digit) | (uint32_t)((1 << digit) - 1 - sh.bin);
        bits += digit;
      }
      if (tid == 0) sh.n = 0;
      // with the last border, what lies before its bin is summed on the way
      const bool last = bits == 0 && (by_mass || !rd.by_p);
      kept = 0;
      __syncthreads();
      const float near = (float)b, far = (float)(b + 1);
      uint64_t sum = 0;   // of this lane, in its tile
      pass4([&](const float(&v)[4], int i) {
        uint32_t in = 0, before = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l = v[e], p = rd.place(l);
          const bool here = (p >= near) & (p < far) & (i + e < vocab);
          const bool out = (bits != 0 || border != 0) && !asked(l, entry_word(l, i + e));
          in |= (uint32_t)(here && !out) << e;
          before |= (uint32_t)(p < near) << e;
        }
        if (last) {
          if (__any(before != 0)) {
            uint32_t mine = 0;
            sum += rd.weights(v, [&](int e, uint32_t u) {
              const bool in = (before >> e & 1) && u >= rd.least;
              mine |= (uint32_t)(in && u != 0) << e;
              return in;
            });
            kept += __popc(mine);
          }
          if ((i & 1023) >= 768) {   // (uniform: the tile's last quarter)
            const uint64_t w = wave_scan64(sum);
            if (lane == 63) sh.tile[i / kLpTile] = w;
            sum = 0;
          }
        }
        if (!__any(in != 0)) return;
        const uint32_t mine = __popc(in), upto = wave_scan32(mine);
        int at = 0;
        if (lane == 63) at = atomicAdd(&sh.n, (int)upto);
        at = __builtin_amdgcn_readlane(at, 63) + (int)(upto - mine);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (in >> e & 1) {
            if (at < kFltList) sh.list[at] = entry_word(v[e], i + e);
            ++at;
          }
      });
      __syncthreads();
      const int n = sh.n;
      if (n <= kFltList) {
        found = cut_list(sh, rd, n, which, rank, 0, rank, (float)b, (float)kFltBins, word).found;
        summed = last;
        if (summed)
          for (int i = tid; i < n; i += kFltThreads) {
            const uint64_t w = sh.list[i];
            const float l = word_value(w);
            if (w < found || rd.weight_word(l) < max(rd.least, 1u)) continue;
            atomicAdd((unsigned long long*)&sh.tile[word_index(w) / kLpTile], (unsigned long long)rd.weight(l));
            ++kept;
          }
        break;
      }
      if (bits == 32) break;
      __syncthreads();
    }
    if (!some) continue;
    if (found == 0) {
      // all equal: by index, of their common weight (at least 1: bin b is counted)
      if (by_mass) {
        const uint64_t w = rd.weight(word_value((uint64_t)prefix << 32));
        rank = (rank + w - 1) / w;
      }
      if (tid < kFltTiles) sh.tile[tid] = 0;
      __syncthreads();
      auto tied = [&](float l, int i) {
        const uint64_t w = entry_word(l, i);
        return (uint32_t)(w >> 32) == prefix && w >= border;
      };
      pass4([&](const float(&v)[4], int i) {
        int c = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) c += __popcll(__ballot(i + e < vocab && tied(v[e], i + e)));
        if (lane == 0 && c > 0) atomicAdd((unsigned long long*)&sh.tile[i / kLpTile], (unsigned long long)c);
      });
      __syncthreads();
      const uint64_t mine = tid < kFltTiles ? sh.tile[tid] : 0;
      uint64_t upto = block_scan(mine, sh).upto;
      if (upto - mine < rank && rank <= upto) {
        sh.bin = tid;
        sh.before = upto - mine;
      }
      __syncthreads();
      rank -= sh.before;
      const int i = sh.bin * kLpTile + tid;   // an entry a thread
      const bool in = i < vocab && tied(entry_at(min(i, vocab - 1)), i);
      upto = block_scan(in ? 1 : 0, sh).upto;
      if (in && upto == rank) sh.bin = i;
      __syncthreads();
      found = ((uint64_t)prefix << 32) | (uint32_t)~sh.bin;
      __syncthreads();
    }
    border = found;
  }

  // the kept weights tile by tile, then the tile and entry of the drawn point
  const float value = border ? word_value(border) : -FLT_MAX;   // the border's, or the lowest
  const int at_most = border ? word_index(border) : 0x7FFFFFFF;
  auto is_kept = [&](float l, int i, uint32_t u) {
    return ((l > value) | ((l == value) & (i <= at_most))) & (u >= rd.least);
  };
  if (!summed) {
    kept = 0;
    __syncthreads();
    if (tid < kFltTiles) sh.tile[tid] = 0;
    __syncthreads();
    if (SPLIT && !rd.by_k && !rd.by_p) {
      if (tid < (vocab + kLpTile - 1) / kLpTile) sh.tile[tid] = given->tile[tid];
      kept = tid == 0 ? given->kept : 0;
    } else {
      const bool count = a.kept != nullptr;
      pass([&](const float(&v)[16], int base) {
        uint64_t w;
        if (border == 0 && rd.least == 0 && !count) {   // (uniform: every entry)
          w = rd.weights(v, [](int, uint32_t) { return true; });
        } else {
          uint32_t mine = 0;
          w = rd.weights(v, [&](int e, uint32_t u) {
            const bool in = is_kept(v[e], index(base, e), u);
            mine |= (uint32_t)(in && u != 0) << e;
            return in;
          });
          kept += __popc(mine);
        }
        w = wave_scan64(w);
        if (lane == 63) sh.tile[base / kLpTile] = w;
      });
    }
  }
  kept = block_scan(kept, sh).all;   // (and the tiles are written)
  const uint64_t mine = tid < kFltTiles ? sh.tile[tid] : 0;
  const Scan s = block_scan(mine, sh);
  uint64_t t = scaled_word(word, s.all);
  if (s.upto - mine <= t && t < s.upto) {
    sh.bin = tid;
    sh.before = s.upto - mine;
  }
  __syncthreads();
  t -= sh.before;
  const int i = sh.bin * kLpTile + tid;   // an entry a thread
  uint64_t w = 0;
  if (i < vocab) {
    const float l = entry_at(i);
    w = is_kept(l, i, rd.weight_word(l)) ? rd.weight(l) : 0;
  }
  const uint64_t upto = block_scan(w, sh).upto;
  if (upto - w <= t && t < upto) answer(i, (float)log((double)w / (double)s.all), (int)kept);
}

// ------------------------------------------------------------- split readings
// Work-group = (four tiles of a row, row).
template <typename T, bool VEC>
__global__ void __launch_bounds__(64 * kFltSplitWaves) filtered_maxima_kernel(FilteredArgs a, int chunks) {
  __shared__ float m4[kFltSplitWaves][64];
  const int r = blockIdx.x / chunks, c = blockIdx.x - r * chunks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  FilteredRow* row = (FilteredRow*)a.scratch + r;
  const int base = (c * kFltSplitWaves + wave) * kLpTile;
  float m = -INFINITY;
  if (base < a.vocab) {
    float v[16];
    Tile<T, VEC>::load((const T*)a.logits + r * a.row_stride, base, a.vocab, lane, v);
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, v[e]);
  }
  m4[wave][lane] = m;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kFltSplitWaves; ++w) m = fmaxf(m, m4[w][lane]);
  row->maxima[64 * c + lane] = m;
  if (c == 0 && lane == 0) {
    row->total = 0;
    row->n = 0;
    row->kept = 0;
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(64 * kFltSplitWaves) filtered_list_kernel(FilteredArgs a, int chunks) {
  constexpr int N = 64 * kFltSplitWaves, PER = kFltBins / N;
  __shared__ uint32_t count[kFltBins];
  __shared__ float wmax[kFltSplitWaves];
  __shared__ uint32_t wsum[kFltSplitWaves];
  __shared__ int last_bin;
  const int r = blockIdx.x / chunks, c = blockIdx.x - r * chunks, tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  FilteredRow* row = (FilteredRow*)a.scratch + r;
  const int base = (c * kFltSplitWaves + wave) * kLpTile;
  float v[16];
  if (base < a.vocab) Tile<T, VEC>::load((const T*)a.logits + r * a.row_stride, base, a.vocab, lane, v);
  RowDraw rd(a, r);
  float mx[kFltMaxima / N], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kFltMaxima / N; ++i) {
    const int at = tid + N * i;
    mx[i] = at < 64 * chunks ? row->maxima[at] : -INFINITY;
    m = fmaxf(m, mx[i]);
  }
  for (int i = tid; i < kFltBins; i += N) count[i] = 0;
  if (tid == 0) last_bin = kFltBins - 2;
  m = wave_max(m);
  if (lane == 0) wmax[wave] = m;
  __syncthreads();
  m = wmax[0];
#pragma unroll
  for (int w = 1; w < kFltSplitWaves; ++w) m = fmaxf(m, wmax[w]);
  rd.m = seen(m);
  if (rd.m == -INFINITY) return;
  if (rd.m == INFINITY) {
    rd.m = 0.f;
#pragma unroll
    for (int i = 0; i < kFltMaxima / N; ++i) mx[i] = mx[i] == INFINITY ? 0.f : -INFINITY;
    read_infinite(v);
  }
  const bool whole = !rd.greedy && !rd.by_k && !rd.by_p;   // nothing but min-p filters
  if (!whole && a.vocab > kFltList) {
#pragma unroll
    for (int i = 0; i < kFltMaxima / N; ++i) {
      const int b = rd.bin(seen(mx[i]));
      if (b < kFltBins - 1) atomicAdd(&count[b], 1u);
    }
    __syncthreads();
    uint32_t own[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      own[i] = count[PER * tid + i];
      sum += own[i];
    }
    uint32_t inc = wave_scan32(sum);
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    for (int w = 0; w < wave; ++w) inc += wsum[w];
    const uint32_t want = rd.greedy ? 1 : rd.by_k ? (uint32_t)rd.k : kFltThreads / 2;
    uint32_t run = inc - sum;
    if (run < want && want <= inc) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (run < want && want <= run + own[i]) last_bin = PER * tid + i;
        run += own[i];
      }
    }
    __syncthreads();
  }
  if (base >= a.vocab) return;
  const float end = (float)(last_bin + 1);
  uint64_t total = 0;
  uint32_t in = 0, kept = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float l = seen(v[e]);
    if (!whole && rd.place(l) < end) in |= 1u << e;
    if (whole || !rd.by_k) {
      const uint64_t w = whole && rd.weight_word(l) < rd.least ? 0 : rd.weight(l);
      total += w;
      kept += w != 0;
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    total += shfl_xor_u64(total, o);
    kept += __shfl_xor(kept, o, 64);
  }
  if (lane == 0) {
    if (whole) {
      row->tile[base / kLpTile] = total;
      atomicAdd(&row->kept, kept);
    } else if (!rd.by_k) {
      atomicAdd((unsigned long long*)&row->total, (unsigned long long)total);
    }
  }
  if (__any(in != 0)) {
    // one reservation a wave: its lanes' entries one lane after the other
    const uint32_t mine = __popc(in), inc = wave_scan32(mine);
    uint32_t at = 0;
    if (lane == 63) at = atomicAdd(&row->n, inc);
    at = __shfl(at, 63, 64) + inc - mine;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (in >> e & 1) {
        if (at < kFltList) row->list[at] = entry_word(seen(v[e]), Tile<T, VEC>::index(base, e, lane));
        ++at;
      }
  }
}

// The split readings are made where the rows alone would leave CUs idle.
static bool split_rows(int rows, int vocab) { return rows <= 128 && vocab > 2 * kFltWaves * kLpTile; }

size_t sample_filtered_scratch(int rows, int vocab) {
  return split_rows(rows, vocab) ? (size_t)rows * (sizeof(FilteredRow) / 4) : 0;
}

template <typename T, bool VEC>
static void launch_filtered(const FilteredArgs& a, hipStream_t s) {
  const dim3 grid(a.rows), block(kFltThreads);
  if (split_rows(a.rows, a.vocab)) {
    const int chunks = split_chunks(a.vocab);
    const dim3 g2((unsigned)(a.rows * chunks)), b2(64 * kFltSplitWaves);
    SR_LAUNCH((filtered_maxima_kernel<T, VEC>), g2, b2, 0, s, a, chunks);
    SR_CHECK_LAUNCH();
    SR_LAUNCH((filtered_list_kernel<T, VEC>), g2, b2, 0, s, a, chunks);
    SR_CHECK_LAUNCH();
    SR_LAUNCH((filtered_kernel<T, VEC, true>), grid, block, 0, s, a);
  } else {
    SR_LAUNCH((filtered_kernel<T, VEC, false>), grid, block, 0, s, a);
  }
  SR_CHECK_LAUNCH();
}

template <typename T>
static void by_alignment(const FilteredArgs& a, hipStream_t s) {
  const bool vec = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && (a.rows == 1 || a.row_stride * sizeof(T) % 16 == 0);
  if (vec) launch_filtered<T, true>(a, s);
  else launch_filtered<T, false>(a, s);
}

void sample_filtered(const FilteredArgs& a, hipStream_t s) {
  if (a.rows <= 0) return;
  if (a.dtype == SR_BF16) by_alignment<bf16_t>(a, s);
  else by_alignment<float>(a, s);
}

}  // namespace sr
