// Attention over the paged candidate cache: causal, with a sliding window and
// sink tokens, rows of their own lengths.
//
//   paged_vector_kernel  (fp32, head_dim 32): one token and a few query heads
//                        of a KV head per work-group, vector ALU
//   paged_merge_kernel   joins the partials of a token's work-groups
//
// Online softmax in base 2 (queries carry log2 e / sqrt(head_dim)).  A pass
// leaves, for every token and query head, the unnormalised output, the running
// maximum and the sum in one of the `slots` partial slots, or the output itself
// where there is one slot.
#include <algorithm>
#include <climits>

#include "common.h"
#include "kernels.h"
#include "paged.h"

namespace sr {

constexpr float kLog2e = 1.4426950408889634f;

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

// ------------------------------------------------------------ vector ALU
// Work-group = (split of the visible keys, GC query heads of one KV head,
// token).  HD / 4 lanes share a key (four dimensions each), so a work-group
// has 1024 / HD groups of lanes, each with a softmax state of its own; a group
// has U keys in flight.  The groups are joined through LDS.
template <typename T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4<float>(const float* p) {
  return *reinterpret_cast<const float4*>(p);
}
template <>
__device__ __forceinline__ float4 load4<bf16_t>(const bf16_t* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xFFFF0000u));
}

template <typename T, int HD, int GC>
__global__ void __launch_bounds__(256) paged_vector_kernel(PagedAttnArgs a, int splits, float qscale) {
  constexpr int LPK = HD / 4, NG = 256 / LPK, U = 4;
  __shared__ float sm[NG][GC][HD + 2];
  const int split = blockIdx.x % splits, token = blockIdx.x / splits;
  const int row = token / a.lr, t = token - row * a.lr;
  const RowState rs = row_state(a, row);
  if (t >= rs.n) return;
  const int qh0 = blockIdx.y * GC, h = qh0 / (a.hq / a.hkv);
  const int p = rs.p0 + t, lo = window_start(p, a.window), sinks = imin(a.sinks, lo);
  const int seen = sinks + p + 1 - lo;                 // visible keys, in order
  const int per = (seen + splits - 1) / splits;
  const int v1 = imin(seen, (split + 1) * per);
  const int grp = threadIdx.x / LPK, d = 4 * (threadIdx.x % LPK);
  const T* kpool = (const T*)a.kpool;
  const T* vpool = (const T*)a.vpool;
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  float4 q[GC];
#pragma unroll
  for (int g = 0; g < GC; ++g) {
    q[g] = *reinterpret_cast<const float4*>(a.q + ((int64_t)token * a.hq + qh0 + g) * HD + d);
    q[g].x *= qscale; q[g].y *= qscale; q[g].z *= qscale; q[g].w *= qscale;
  }
  float m[GC], l[GC], acc[GC][4];
#pragma unroll
  for (int g = 0; g < GC; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[g][e] = 0.f;
  }
  for (int v0 = split * per; v0 < v1; v0 += NG * U) {   // (uniform in the work-group)
    int64_t off[U];
    bool ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + u * NG + grp, vc = imin(v, v1 - 1);
      const int j = vc < sinks ? vc : vc - sinks + lo;
      const int pg = tab[j >> a.shift];
      ok[u] = v < v1 && (uint32_t)pg < (uint32_t)a.n_pages;
      off[u] = page_offset(ok[u] ? pg : 0, a.hkv, h, a.shift, j, HD) + d;
    }
    float4 k[U], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = load4<T>(kpool + off[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load4<T>(vpool + off[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (!ok[u]) x[u] = make_float4(0.f, 0.f, 0.f, 0.f);   // (what lies there may be no number)
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      float s[U], mn = m[g];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        s[u] = q[g].x * k[u].x + q[g].y * k[u].y + q[g].z * k[u].z + q[g].w * k[u].w;
#pragma unroll
        for (int o = LPK / 2; o > 0; o >>= 1) s[u] += __shfl_xor(s[u], o, 64);
        if (!ok[u]) s[u] = -INFINITY;
        mn = fmaxf(mn, s[u]);
      }
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float corr = exp2f(m[g] - ref);   // (0 while nothing was seen)
      m[g] = mn;
      l[g] *= corr;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[g][e] *= corr;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = exp2f(s[u] - ref);
        l[g] += w;
        acc[g][0] += w * x[u].x; acc[g][1] += w * x[u].y; acc[g][2] += w * x[u].z; acc[g][3] += w * x[u].w;
      }
    }
  }
#pragma unroll
  for (int g = 0; g < GC; ++g) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sm[grp][g][d + e] = acc[g][e];
    if (d == 0) {
      sm[grp][g][HD] = m[g];
      sm[grp][g][HD + 1] = l[g];
    }
  }
  __syncthreads();
  const Partials pt{a.part, (int64_t)a.rows * a.lr * a.hq, splits};
  for (int i = threadIdx.x; i < GC * HD; i += 256) {
    const int g = i / HD, dd = i % HD;
    float M = -INFINITY;
    for (int k = 0; k < NG; ++k) M = fmaxf(M, sm[k][g][HD]);
    float L = 0.f, A = 0.f;
    if (M != -INFINITY)
      for (int k = 0; k < NG; ++k) {
        const float c = exp2f(sm[k][g][HD] - M);
        L += sm[k][g][HD + 1] * c;
        A += sm[k][g][dd] * c;
      }
    const int64_t th = (int64_t)token * a.hq + qh0 + g;
    if (splits == 1) {
      ((T*)a.out)[th * HD + dd] = from_f32<T>(L > 0.f ? A / L : 0.f);
    } else {
      pt.o(th, split, HD)[dd] = A;
      if (dd == 0) {
        pt.ml(th, split, HD)[0] = M;
        pt.ml(th, split, HD)[1] = L;
      }
    }
  }
}

// ----------------------------------------------------------------- merge
// A wave joins the slots of one (token, query head).
template <typename T, int HD>
__global__ void __launch_bounds__(256) paged_merge_kernel(PagedAttnArgs a, int slots) {
  const int64_t th = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const Partials pt{a.part, (int64_t)a.rows * a.lr * a.hq, slots};
  if (th >= pt.th) return;
  const int token = (int)(th / a.hq), row = token / a.lr;
  if (token - row * a.lr >= row_state(a, row).n) return;
  const int lane = threadIdx.x & 63;
  const float* ml = pt.ml(th, 0, HD);
  float M = -INFINITY;
  for (int s = 0; s < slots; ++s) M = fmaxf(M, ml[2 * s]);
  for (int d = lane; d < HD; d += 64) {
    float L = 0.f, A = 0.f;
    if (M != -INFINITY)
      for (int s = 0; s < slots; ++s) {
        const float c = exp2f(ml[2 * s] - M);
        L += ml[2 * s + 1] * c;
        A += pt.o(th, s, HD)[d] * c;
      }
    ((T*)a.out)[th * HD + d] = from_f32<T>(L > 0.f ? A / L : 0.f);
  }
}

// ------------------------------------------------------------------ plan
struct PagedPlan {
  int slots;
};

// Query heads of a work-group of the vector kernel.
static int vector_heads(int g) { return g % 4 == 0 ? 4 : g % 2 == 0 ? 2 : 1; }

static PagedPlan paged_plan(const PagedAttnArgs& a) {
  PagedPlan p;
  const int64_t cap = (int64_t)a.max_pages << a.shift;
  int64_t keys = std::min<int64_t>(a.max_len, cap);
  if (a.window > 0) keys = std::min<int64_t>(keys, (int64_t)a.window + a.sinks);
  const int64_t groups = (int64_t)a.rows * a.lr * (a.hq / vector_heads(a.hq / a.hkv));
  p.slots = (int)std::max<int64_t>(1, std::min<int64_t>({1024 / groups, keys / 256, 64}));
  return p;
}

size_t paged_attn_scratch(const PagedAttnArgs& a) {
  if (a.rows <= 0 || a.lr <= 0) return 0;
  const PagedPlan p = paged_plan(a);
  return p.slots > 1 ? (size_t)a.rows * a.lr * a.hq * p.slots * (a.hd + 2) : 0;
}

template <typename T, int HD>
static void launch_merge(const PagedAttnArgs& a, int slots, hipStream_t s) {
  const int64_t th = (int64_t)a.rows * a.lr * a.hq;
  SR_LAUNCH((paged_merge_kernel<T, HD>), dim3((unsigned)((th + 3) / 4)), dim3(256), 0, s, a, slots);
  SR_CHECK_LAUNCH();
}

template <typename T, int HD>
static void launch_vector(const PagedAttnArgs& a, hipStream_t s) {
  const PagedPlan p = paged_plan(a);
  const float qscale = kLog2e / sqrtf((float)HD);
  const int gc = vector_heads(a.hq / a.hkv);
  const dim3 grid((unsigned)((int64_t)a.rows * a.lr * p.slots), a.hq / gc);
  switch (gc) {
    case 4: SR_LAUNCH((paged_vector_kernel<T, HD, 4>), grid, dim3(256), 0, s, a, p.slots, qscale); break;
    case 2: SR_LAUNCH((paged_vector_kernel<T, HD, 2>), grid, dim3(256), 0, s, a, p.slots, qscale); break;
    default: SR_LAUNCH((paged_vector_kernel<T, HD, 1>), grid, dim3(256), 0, s, a, p.slots, qscale); break;
  }
  SR_CHECK_LAUNCH();
  if (p.slots > 1) launch_merge<T, HD>(a, p.slots, s);
}

template <typename T>
static void vector_by_hd(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.hd) {
    case 32: launch_vector<T, 32>(a, s); break;
    case 64: launch_vector<T, 64>(a, s); break;
    default: launch_vector<T, 128>(a, s); break;
  }
}

void paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.lr <= 0) return;
  if (a.dtype == SR_BF16) vector_by_hd<bf16_t>(a, s);
  else vector_by_hd<float>(a, s);
}

}  // namespace sr
