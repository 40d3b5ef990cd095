// Log-probabilities of given tokens with the entropy of their distribution and
// its most likely tokens: softmax(logits / temperature) of every row.
//   ln p_i = z_i - ln S,  z_i = (x_i - max) / T,  S = sum e^z
//   H = ln S - (sum e^z z) / S
// One pass over the logits: every lane keeps the running maximum of its
// entries and the two sums relative to it, and every wave the most likely
// entries so far.  An entry travels as one word, its value's order-preserving
// bits above its inverted index, so that "larger" is "more likely, then lower
// index" and no order of merging can change a result.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "logit_rows.h"

namespace sr {

constexpr int kLpWaves = 4;
constexpr int kLpTop = 32;        // most alternatives
constexpr int kLpList = 128;      // entries of a wave's list of candidates
constexpr int kLpMaxChunks = 64;  // of a row: one per lane of the joining wave

// Logits of a row: NaN counts as -inf.
__device__ __forceinline__ float seen_logit(float x) { return fmaxf(x, -INFINITY); }
// (x - m) / T with the limits of a maximum of +inf, and of no maximum.
__device__ __forceinline__ float scaled(float x, float m, float inv_t) {
  return x == m ? 0.f : x == -INFINITY ? -INFINITY : (x - m) * inv_t;
}

// max, S and sum e^z z log2 e of a set of entries.
struct Sums {
  float m, s, t;
};
// The sums `a` and `b` of two sets as those of their union (k = log2 e / T).
__device__ __forceinline__ Sums join(Sums a, Sums b, float k) {
  const float m = fmaxf(a.m, b.m);
  auto part = [&](Sums x, float& s, float& t) {
    if (x.m == -INFINITY) return;
    const float d = x.m == m ? 0.f : fmaxf((x.m - m) * k, -200.f);
    const float c = __builtin_amdgcn_exp2f(d);
    s += x.s * c;
    t += (x.t + d * x.s) * c;
  };
  Sums r{m, 0.f, 0.f};
  part(a, r.s, r.t);
  part(b, r.s, r.t);
  return r;
}

// The best `keep` of a wave's n <= kLpList listed words, sorted, to the front of
// the list; returns their number.  Lane l ranks words l and l + 64 by counting
// the larger ones (words are distinct), eight at a time.  The list has room for
// eight more.
__device__ int list_sort(uint64_t* list, int n, int keep) {
  const int lane = threadIdx.x & 63;
  if (lane < 8) list[n + lane] = 0;   // (larger than nothing)
  const uint64_t a = lane < n ? list[lane] : 0, b = lane + 64 < n ? list[lane + 64] : 0;
  int ra = 0, rb = 0;
  for (int i = 0; i < n; i += 8) {
    uint64_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = list[i + j];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      ra += w[j] > a ? 1 : 0;
      rb += w[j] > b ? 1 : 0;
    }
  }
  __builtin_amdgcn_wave_barrier();   // (every lane has read before one writes: a wave's LDS operations are in order)
  if (lane < n && ra < keep) list[ra] = a;
  if (lane + 64 < n && rb < keep) list[rb] = b;
  __builtin_amdgcn_wave_barrier();
  return min(n, keep);
}

// The largest of the wave's values, by DPP: within rows of 16 lanes, then from
// row to row; lane 63 ends up with it.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  auto step = [&](auto ctrl) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false));
  };
  step(std::integral_constant<int, 0x111>{});   // row_shr 1, 2, 4, 8
  step(std::integral_constant<int, 0x112>{});
  step(std::integral_constant<int, 0x114>{});
  step(std::integral_constant<int, 0x118>{});
  step(std::integral_constant<int, 0x142>{});   // row_bcast 15, 31
  step(std::integral_constant<int, 0x143>{});
  return __builtin_amdgcn_readlane(v, 63);
}

// Partial results of a chunk: max, S, t, and `top` sorted words.
__host__ __device__ inline int64_t chunk_floats(int top) { return 4 + 2 * (int64_t)top; }

// A row's given token and its logit, read ahead of the sums.
struct Given {
  int tok;
  float x;
};
template <typename T>
__device__ __forceinline__ Given given(const LogprobArgs& a, int r) {
  Given g{-1, 0.f};
  if (a.logprob) {
    g.tok = a.tokens[r];
    if ((uint32_t)g.tok < (uint32_t)a.vocab)
      g.x = seen_logit(to_f32<T>(((const T*)a.logits + r * a.row_stride)[g.tok]));
  }
  return g;
}
// What a row's sums and best words give.
__device__ __forceinline__ void write_row(const LogprobArgs& a, int r, Given g, Sums s, float inv_t) {
  const bool none = s.m == -INFINITY;
  const float ls = none ? 0.f : logf(s.s);
  if (a.logprob) {
    float lp = __uint_as_float(0x7FC00000u);
    if (g.tok == -1) lp = 0.f;
    else if ((uint32_t)g.tok < (uint32_t)a.vocab) lp = none ? -INFINITY : scaled(g.x, s.m, inv_t) - ls;
    a.logprob[r] = lp;
  }
  if (a.entropy) a.entropy[r] = none ? 0.f : ls - 0.6931471805599453f * (s.t / s.s);
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, int r, int i, uint64_t w, Sums s, float inv_t) {
  const bool none = s.m == -INFINITY;
  if (a.top_ids) a.top_ids[(int64_t)r * a.top + i] = word_index(w);
  if (a.top_logprobs)
    a.top_logprobs[(int64_t)r * a.top + i] = none ? -INFINITY : scaled(word_value(w), s.m, inv_t) - logf(s.s);
}

// Work-group = (chunk of a row, row); wave w takes every fourth tile, the next
// one's loads in flight under this one's sums.
template <typename T, bool VEC, bool TOP>
__global__ void __launch_bounds__(64 * kLpWaves)
logprob_kernel(LogprobArgs a, int chunks, int chunk_len, float k, float inv_t) {
  __shared__ uint64_t lists[kLpWaves][kLpList + 8];
  __shared__ Sums wsums[kLpWaves];
  __shared__ int wcount[kLpWaves];
  const int r = blockIdx.x / chunks, chunk = blockIdx.x - r * chunks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* x = (const T*)a.logits + r * a.row_stride;
  const int c0 = chunk * chunk_len, c1 = min(a.vocab, c0 + chunk_len);
  uint64_t* list = lists[wave];
  int n = 0;                      // listed words (uniform in the wave)
  uint64_t floor_word = 0;        // words below it are not among the best
  float floor_value = -INFINITY;  // nor are values below it
  auto raise = [&](uint64_t w) {
    if (w <= floor_word) return;
    floor_word = w;
    const float f = word_value(w);
    floor_value = f == f ? f : -INFINITY;   // (bits below -inf's read as a NaN)
  };
  bool first = true;
  Sums s{-INFINITY, 0.f, 0.f};
  float v[16], nx[16];
  const int t0 = c0 + wave * kLpTile, step = kLpWaves * kLpTile;
  if (t0 < c1) Tile<T, VEC>::load(x, t0, c1, lane, v);
  for (int base = t0; base < c1; base += step) {
    if (base + step < c1) Tile<T, VEC>::load(x, base + step, c1, lane, nx);
    float mt = fmaxf(v[0], v[1]);
#pragma unroll
    for (int e = 2; e < 16; ++e) mt = fmaxf(mt, v[e]);
    mt = seen_logit(mt);
    if (mt > s.m) {
      const float d = fmaxf((s.m - mt) * k, -200.f), c = __builtin_amdgcn_exp2f(d);
      s.t = (s.t + d * s.s) * c;
      s.s *= c;
      s.m = mt;
    }
    if (__builtin_expect(__any(s.m == INFINITY), 0)) {   // the entries of +inf count 1 each
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float z = v[e] == s.m ? 0.f : fmaxf((v[e] - s.m) * k, -200.f);
        const float p = __builtin_amdgcn_exp2f(z);
        s.s += p;
        s.t = __builtin_fmaf(p, z, s.t);
      }
    } else {
      // -inf and NaN: (x - m) k is -inf or NaN, the larger of it and -200 is
      // -200, and 2^-200 is 0 in fp32
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float z = fmaxf((v[e] - s.m) * k, -200.f);
        const float p = __builtin_amdgcn_exp2f(z);
        s.s += p;
        s.t = __builtin_fmaf(p, z, s.t);
      }
    }
    if constexpr (TOP) {
      if (first) {
        // The top-th largest of the lanes' maxima bounds the wave's top-th best
        // entry from below: found bit by bit (at least 32 lanes have entries
        // wherever there are that many; else the bound stays 0).
        first = false;
        const uint32_t key = (uint32_t)(entry_word(mt, 0) >> 32);
        uint32_t t = 0;   // (its upper 16 bits are enough)
#pragma unroll
        for (int b = 31; b >= 16; --b) {
          const uint32_t c = t | (1u << b);
          if (__popcll(__ballot(key >= c)) >= a.top) t = c;
        }
        raise((uint64_t)t << 32);
      }
      if (__any(mt >= floor_value)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          uint64_t in = __ballot(seen_logit(v[e]) >= floor_value);   // (as values: ties are decided below)
          if (in == 0) continue;
          const int i = Tile<T, VEC>::index(base, e, lane);
          const uint64_t w = entry_word(seen_logit(v[e]), i);
          if (n + __popcll(in) > kLpList) {
            n = list_sort(list, n, a.top);
            if (n == a.top) raise(list[n - 1]);
          }
          in = __ballot(i < c1 && w >= floor_word);
          if (i < c1 && w >= floor_word) list[n + __popcll(in & ((1ull << lane) - 1))] = w;
          n += __popcll(in);
        }
        if (n >= a.top + 16) {   // (a higher floor saves the next tiles' candidates)
          n = list_sort(list, n, a.top);
          raise(list[n - 1]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = nx[e];
  }
  // the wave's lanes, then the work-group's waves
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    s = join(s, Sums{__shfl_xor(s.m, o, 64), __shfl_xor(s.s, o, 64), __shfl_xor(s.t, o, 64)}, k);
  if (TOP) n = list_sort(list, n, a.top);
  if (lane == 0) {
    wsums[wave] = s;
    wcount[wave] = n;
  }
  __syncthreads();
  if (wave != 0) return;
  s = wsums[0];
  for (int w = 1; w < kLpWaves; ++w) s = join(s, wsums[w], k);
  if (TOP) {
    // the waves' lists, at most kLpWaves * kLpTop = kLpList words, into one
    for (int w = 1; w < kLpWaves; ++w) {
      const int m = wcount[w];
      if (lane < m) list[n + lane] = lists[w][lane];
      n += m;
    }
    __builtin_amdgcn_wave_barrier();
    n = list_sort(list, n, a.top);
  }
  if (chunks == 1) {
    if (lane == 0) write_row(a, r, given<T>(a, r), s, inv_t);
    if (TOP && lane < n) write_top(a, r, lane, list[lane], s, inv_t);
    return;
  }
  float* p = a.scratch + ((int64_t)r * chunks + chunk) * chunk_floats(a.top);
  if (lane == 0) {
    p[0] = s.m;
    p[1] = s.s;
    p[2] = s.t;
    p[3] = __int_as_float(n);
  }
  if (TOP && lane < n) {
    p[4 + 2 * lane] = __uint_as_float((uint32_t)list[lane]);
    p[5 + 2 * lane] = __uint_as_float((uint32_t)(list[lane] >> 32));
  }
}

// A wave joins a row's chunks, lane c holding chunk c: the sums by a butterfly
// and the alternatives by taking the best of the chunks' next words each time
// (ranking the words that can be among them took 13.4 us a call instead of 14.9
// on 128256 entries with top 20, but 9.0 instead of 8.1 with top 1 and 16.6
// instead of 14.5 on 32000 with top 20).
template <typename T>
__global__ void __launch_bounds__(64) logprob_join_kernel(LogprobArgs a, int chunks, float k, float inv_t) {
  __shared__ uint64_t words[kLpMaxChunks * kLpTop];
  const int r = blockIdx.x, lane = threadIdx.x;
  const int64_t stride = chunk_floats(a.top);
  const float* row = a.scratch + (int64_t)r * chunks * stride;
  const Given g = given<T>(a, r);
#pragma unroll 8
  for (int i = lane; i < chunks * a.top; i += 64) {   // (those past a chunk's number are never taken)
    const int c = i / a.top;
    const float* w = row + c * stride + 4 + 2 * (i - c * a.top);
    words[i] = ((uint64_t)__float_as_uint(w[1]) << 32) | __float_as_uint(w[0]);
  }
  Sums s{-INFINITY, 0.f, 0.f};
  int n = 0;
  if (lane < chunks) {
    const float* p = row + lane * stride;
    s = Sums{p[0], p[1], p[2]};
    n = __float_as_int(p[3]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    s = join(s, Sums{__shfl_xor(s.m, o, 64), __shfl_xor(s.s, o, 64), __shfl_xor(s.t, o, 64)}, k);
  if (lane == 0) write_row(a, r, g, s, inv_t);
  if (a.top == 0) return;
  __syncthreads();
  int at = 0;
  uint64_t head = n > 0 ? words[lane * a.top] : 0, mine = 0;
  for (int i = 0; i < a.top; ++i) {
    const uint32_t hi = wave_max_u32((uint32_t)(head >> 32));
    const uint32_t lo = wave_max_u32((uint32_t)(head >> 32) == hi ? (uint32_t)head : 0);
    const uint64_t best = (uint64_t)hi << 32 | lo;
    if (lane == i) mine = best;
    if (head == best) {   // (one lane: words are distinct, and top <= vocab of them exist)
      ++at;
      head = at < n ? words[lane * a.top + at] : 0;
    }
  }
  if (lane < a.top) write_top(a, r, lane, mine, s, inv_t);
}

// Chunks of a row: of whole rounds of the waves' tiles, enough for about
// kLpTarget work-groups (512 rows of 128256 with 5 alternatives 65.5 us with
// twice as many, 61.5 with these, with 32 alternatives 96 and 82: every chunk
// finds its alternatives anew).
constexpr int kLpTarget = 1024;
static int logprob_chunk_len(int rows, int vocab) {
  const int round = kLpWaves * kLpTile;
  const int rounds = (vocab + round - 1) / round;
  const int want = std::min({rounds, kLpMaxChunks, std::max(1, kLpTarget / rows)});
  return (rounds + want - 1) / want * round;
}
static int logprob_chunks(int rows, int vocab) {
  const int len = logprob_chunk_len(rows, vocab);
  return (vocab + len - 1) / len;
}

size_t token_logprobs_scratch(int rows, int vocab, int top) {
  const int chunks = logprob_chunks(rows, vocab);
  return chunks > 1 ? (size_t)rows * chunks * chunk_floats(top) : 0;
}

template <typename T>
static void launch_logprobs(const LogprobArgs& a, hipStream_t s) {
  const float k = (float)(1.4426950408889634 / (double)a.temperature);
  const float inv_t = (float)(1.0 / (double)a.temperature);
  const int len = logprob_chunk_len(a.rows, a.vocab), chunks = logprob_chunks(a.rows, a.vocab);
  const bool vec = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && (a.rows == 1 || a.row_stride * sizeof(T) % 16 == 0);
  const bool top = a.top > 0 && (a.top_ids || a.top_logprobs);
  const dim3 grid((unsigned)(a.rows * chunks)), block(64 * kLpWaves);
  if (vec) {
    if (top) SR_LAUNCH((logprob_kernel<T, true, true>), grid, block, 0, s, a, chunks, len, k, inv_t);
    else SR_LAUNCH((logprob_kernel<T, true, false>), grid, block, 0, s, a, chunks, len, k, inv_t);
  } else {
    if (top) SR_LAUNCH((logprob_kernel<T, false, true>), grid, block, 0, s, a, chunks, len, k, inv_t);
    else SR_LAUNCH((logprob_kernel<T, false, false>), grid, block, 0, s, a, chunks, len, k, inv_t);
  }
  SR_CHECK_LAUNCH();
  if (chunks == 1) return;
  SR_LAUNCH(logprob_join_kernel<T>, dim3(a.rows), dim3(64), 0, s, a, chunks, k, inv_t);
  SR_CHECK_LAUNCH();
}

void token_logprobs(const LogprobArgs& args, hipStream_t s) {
  if (args.rows <= 0) return;
  LogprobArgs a = args;
  if (!a.top_ids && !a.top_logprobs) a.top = 0;
  if (a.dtype == SR_BF16) launch_logprobs<bf16_t>(a, s);
  else launch_logprobs<float>(a, s);
}

}  // namespace sr
