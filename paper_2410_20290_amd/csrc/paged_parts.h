// What the attention kernels over pages share: a row's state, the partial slots
// of split work and their joining, and the keys that rows have in common.
#pragma once

#include <algorithm>

#include "attn_tiles.h"
#include "common.h"
#include "kernels.h"
#include "paged.h"

namespace sr {

// A row's length, the call's tokens in it, and the first of their positions.
struct RowState {
  int len, n, p0;
};
__device__ __forceinline__ RowState row_state(const PagedAttnArgs& a, int row) {
  RowState r;
  r.len = clamp_len(a.lens[row], a.max_pages, a.shift);
  r.n = clamp_new(a.n_new ? a.n_new[row] : a.lr, a.lr, r.len);
  r.p0 = r.len - r.n;
  return r;
}

// Partial slots: all unnormalised outputs [tokens][hq][slots][hd], then (max,
// sum) [tokens][hq][slots][2].
struct Partials {
  float* part;
  int64_t th;   // tokens * hq
  int slots;
  __device__ __forceinline__ float* o(int64_t token_head, int slot, int hd) const {
    return part + (token_head * slots + slot) * hd;
  }
  __device__ __forceinline__ float* ml(int64_t token_head, int slot, int hd) const {
    return part + th * slots * hd + (token_head * slots + slot) * 2;
  }
};

// The leading keys of every row that the tile kernel attends for all rows at
// once: those in pages that the row has in common with row 0, before every
// query of the row, a multiple of 32 up to `shared`; none once the window of the
// row's first query has left key 0 (so a key that the pass reads is seen by some
// query).  A wave per row.
static __global__ void __launch_bounds__(256) paged_common_kernel(PagedAttnArgs a, int32_t* __restrict__ common) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= a.rows) return;
  const RowState rs = row_state(a, row);
  const int len0 = clamp_len(a.lens[0], a.max_pages, a.shift);
  int c = rs.n > 0 && window_start(rs.p0, a.window) == 0 ? imin(imin(a.shared, rs.p0), len0) : 0;
  const int32_t* mine = a.table + (int64_t)row * a.max_pages;
  const int pages = (c + (1 << a.shift) - 1) >> a.shift;
  for (int p = 0; p < pages; p += 64) {
    const int q = p + lane;
    const uint64_t other = __ballot(q < pages && mine[q] != a.table[q]);
    if (other) {
      c = imin(c, (p + (int)__builtin_ctzll(other)) << a.shift);
      break;
    }
  }
  if (lane == 0) common[row] = c & ~31;
}

// A wave joins the slots of one (token, query head): lane s weighs slots s and s
// + 64, then every lane sums its dimensions over the slots, eight loads at a time
// (one row of 8000 keys 16.1 us, one load at a time 19.6).
template <typename T, int HD>
static __global__ void __launch_bounds__(256) paged_merge_kernel(PagedAttnArgs a, int slots) {
  const int64_t th = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const Partials pt{a.part, (int64_t)a.rows * a.lr * a.hq, slots};
  if (th >= pt.th) return;
  const int token = (int)(th / a.hq), row = token / a.lr;
  if (token - row * a.lr >= row_state(a, row).n) return;
  const int lane = threadIdx.x & 63;
  const float2* ml = reinterpret_cast<const float2*>(pt.ml(th, 0, HD));
  const float2 none = make_float2(-INFINITY, 0.f);
  const float2 x = lane < slots ? ml[lane] : none, y = lane + 64 < slots ? ml[lane + 64] : none;
  const float M = wave_max(fmaxf(x.x, y.x));
  const float ref = M == -INFINITY ? 0.f : M;
  const float wx = __builtin_amdgcn_exp2f(x.x - ref), wy = __builtin_amdgcn_exp2f(y.x - ref);
  const float L = wave_sum(x.y * wx + y.y * wy);
  constexpr int N = HD < 64 ? 1 : HD / 64;   // dimensions of a lane
  float A[N] = {};
  // (every lane stays on, those without dimensions too: they hold weights)
  const bool mine = N * lane < HD;
  const float* o = pt.o(th, 0, HD) + (mine ? N * lane : 0);
  constexpr int U = 8;   // slots on their way together
  for (int s0 = 0; s0 < slots; s0 += U) {
    float v[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < N; ++e) v[u][e] = o[(int64_t)imin(s0 + u, slots - 1) * HD + e];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u;
      const float w = __shfl(s < 64 ? wx : wy, s & 63, 64);
      if (s < slots)
#pragma unroll
        for (int e = 0; e < N; ++e) A[e] += w * v[u][e];
    }
  }
  if (!mine) return;
#pragma unroll
  for (int e = 0; e < N; ++e) ((T*)a.out)[th * HD + N * lane + e] = from_f32<T>(L == 0.f ? 0.f : A[e] / L);
}

// Keys that a row's queries see at most, as far as the host knows.
static inline int64_t planned_keys(const PagedAttnArgs& a) {
  int64_t keys = std::min<int64_t>(a.max_len, (int64_t)a.max_pages << a.shift);
  if (a.window > 0) keys = std::min<int64_t>(keys, (int64_t)a.window + a.lr + a.sinks);
  return keys;
}

template <typename T, int HD>
static void launch_merge(const PagedAttnArgs& a, int slots, hipStream_t s) {
  const int64_t th = (int64_t)a.rows * a.lr * a.hq;
  SR_LAUNCH((paged_merge_kernel<T, HD>), dim3((unsigned)((th + 3) / 4)), dim3(256), 0, s, a, slots);
  SR_CHECK_LAUNCH();
}

}  // namespace sr
