// Attention over the paged candidate cache: causal, with a sliding window and
// sink tokens, rows of their own lengths.
//
//   paged_wave_kernel    (bf16, up to 16 query columns a row and KV head: single
//                        tokens, short drafts): the waves split a row's keys
//   paged_tile_kernel    (bf16): 128 query columns a work-group, keys staged in
//                        LDS for all of them: prompts, and the part of the rows
//                        that lies in the pages of row 0, once for all rows
//   paged_vector_kernel  (fp32, and bf16 with head_dim 32): up to eight query
//                        columns of a row and KV head per work-group, of one token
//                        or several, vector ALU
//   paged_merge_kernel   joins the partials of a token's work-groups
//
// Online softmax in base 2 (queries carry log2 e / sqrt(head_dim)).  A pass
// leaves, for every token and query head, the unnormalised output, the running
// maximum and the sum in one of the `slots` partial slots, or the output itself
// where there is one slot.  A score that is NaN never raises a maximum and always
// enters the sum, so "nothing seen" is a sum equal to 0, not one that fails to be
// above it, and a maximum of -inf says nothing about the sum.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "paged_parts.h"

namespace sr {

// ------------------------------------------------------------ vector ALU
// Work-group = (split of the visible keys, GC query columns of one row, KV head);
// column x is token x / G, query head x % G as below.  HD / 4 lanes share a key
// (four dimensions each), so a work-group has 1024 / HD groups of lanes, each
// with a softmax state of its own per column; a group has U keys in flight, each
// read once for all its columns.  The groups are joined through LDS.
// Bound by instructions: 4 FMAs, log2(HD / 4) DPP adds and an exponential per key
// and column and lane (fp32 prompts of 2000 tokens 160 us with a column of its own
// for every group, 87 with up to eight; four of them, 4 heads of 32, 233 us for 4.1
// GFLOP, 18 TFLOP/s).
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

// The sum over aligned groups of LPK lanes, in every lane of a group: DPP moves
// within rows of 16 (quads by xor 1 and 2, then mirrored halves, which by then
// hold equal sums), a cross-lane move beyond.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int LPK>
__device__ __forceinline__ float lanes_sum(float v) {
  v = dpp_add<0xB1>(v);                         // quad_perm [1,0,3,2]
  v = dpp_add<0x4E>(v);                         // quad_perm [2,3,0,1]
  v = dpp_add<0x141>(v);                        // row_half_mirror
  if constexpr (LPK >= 16) v = dpp_add<0x140>(v);   // row_mirror
  if constexpr (LPK == 32) v += __shfl_xor(v, 16, 64);
  static_assert(LPK == 8 || LPK == 16 || LPK == 32, "lanes of a key");
  return v;
}

template <typename T, int HD, int GC>
__global__ void __launch_bounds__(256, 2) paged_vector_kernel(PagedAttnArgs a, int splits, float qscale) {
  constexpr int LPK = HD / 4, NG = 256 / LPK, U = 4;
  __shared__ float sm[NG][GC][HD + 2];
  const int g = a.hq / a.hkv, tiles = (a.lr * g + GC - 1) / GC;
  const int split = blockIdx.x % splits, tile = blockIdx.x / splits, h = blockIdx.y;
  const int row = tile / tiles, x0 = (tile - row * tiles) * GC;
  const RowState rs = row_state(a, row);
  const int X = rs.n * g;                        // the row's columns
  if (x0 >= X) return;
  const int grp = threadIdx.x / LPK, d = 4 * (threadIdx.x % LPK);
  const T* kpool = (const T*)a.kpool;
  const T* vpool = (const T*)a.vpool;
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  const int first = rs.p0 + x0 / g, last = rs.p0 + imin(x0 + GC, X) / g - (imin(x0 + GC, X) % g == 0 ? 1 : 0);
  // keys that some column sees: [0, sinks) and [lo, last], in this order
  const int lo = window_start(first, a.window), sinks = imin(a.sinks, lo), all_lo = window_start(last, a.window);
  const int seen = sinks + last + 1 - lo;
  const int per = (seen + splits - 1) / splits;
  const int v1 = imin(seen, (split + 1) * per);
  float4 q[GC];
  int end[GC], from[GC];                         // column c sees keys below end[c] from from[c] on, and the sinks
  float m[GC], l[GC], acc[GC][4];
#pragma unroll
  for (int c = 0; c < GC; ++c) {
    const int x = imin(x0 + c, X - 1), t = x / g;
    end[c] = rs.p0 + t + 1;
    from[c] = window_start(rs.p0 + t, a.window);
    q[c] = *reinterpret_cast<const float4*>(a.q + (((int64_t)row * a.lr + t) * a.hq + h * g + (x - t * g)) * HD + d);
    q[c].x *= qscale; q[c].y *= qscale; q[c].z *= qscale; q[c].w *= qscale;
    m[c] = -INFINITY;
    l[c] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[c][e] = 0.f;
  }
  for (int v0 = split * per; v0 < v1; v0 += NG * U) {   // (uniform in the work-group)
    int64_t off[U];
    int key[U];
    bool ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int v = v0 + u * NG + grp, vc = imin(v, v1 - 1);
      key[u] = vc < sinks ? vc : vc - sinks + lo;
      const int pg = tab[key[u] >> a.shift];
      ok[u] = v < v1 && (uint32_t)pg < (uint32_t)a.n_pages;
      off[u] = page_offset(ok[u] ? pg : 0, a.hkv, h, a.shift, key[u], HD) + d;
    }
    // some column does not see some of the keys
    const int vlast = imin(v0 + NG * U, v1) - 1;
    const bool edge = (vlast < sinks ? vlast : vlast - sinks + lo) > first || (v0 - sinks + lo < all_lo && v0 >= sinks) ||
                      (vlast >= sinks && v0 < sinks && lo < all_lo);
    float4 k[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = load4<T>(kpool + off[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) y[u] = load4<T>(vpool + off[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (!ok[u]) y[u] = make_float4(0.f, 0.f, 0.f, 0.f);   // (what lies there may be no number)
#pragma unroll
    for (int c = 0; c < GC; ++c) {
      float s[U], mn = m[c];
#pragma unroll
      for (int u = 0; u < U; ++u)
        s[u] = lanes_sum<LPK>(q[c].x * k[u].x + q[c].y * k[u].y + q[c].z * k[u].z + q[c].w * k[u].w);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        bool sees = ok[u];
        if (edge) sees = sees & (key[u] < end[c]) & ((key[u] >= from[c]) | (key[u] < a.sinks));
        if (!sees) s[u] = -INFINITY;
        mn = fmaxf(mn, s[u]);
      }
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float corr = __builtin_amdgcn_exp2f(m[c] - ref);   // (0 while nothing was seen)
      m[c] = mn;
      l[c] *= corr;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[c][e] *= corr;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = __builtin_amdgcn_exp2f(s[u] - ref);
        l[c] += w;
        acc[c][0] += w * y[u].x; acc[c][1] += w * y[u].y; acc[c][2] += w * y[u].z; acc[c][3] += w * y[u].w;
      }
    }
  }
#pragma unroll
  for (int c = 0; c < GC; ++c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sm[grp][c][d + e] = acc[c][e];
    if (d == 0) {
      sm[grp][c][HD] = m[c];
      sm[grp][c][HD + 1] = l[c];
    }
  }
  __syncthreads();
  const Partials pt{a.part, (int64_t)a.rows * a.lr * a.hq, splits};
  for (int i = threadIdx.x; i < GC * HD; i += 256) {
    const int c = i / HD, dd = i % HD, x = x0 + c;
    if (x >= X) break;
    float M = -INFINITY;
#pragma unroll 8
    for (int k = 0; k < NG; ++k) M = fmaxf(M, sm[k][c][HD]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f, A = 0.f;
#pragma unroll 8
    for (int k = 0; k < NG; ++k) {
      const float w = __builtin_amdgcn_exp2f(sm[k][c][HD] - ref);
      L += sm[k][c][HD + 1] * w;
      A += sm[k][c][dd] * w;
    }
    const int64_t th = ((int64_t)row * a.lr + x / g) * a.hq + h * g + x % g;
    if (splits == 1) {
      ((T*)a.out)[th * HD + dd] = from_f32<T>(L == 0.f ? 0.f : A / L);
    } else {
      pt.o(th, split, HD)[dd] = A;
      if (dd == 0) {
        pt.ml(th, split, HD)[0] = M;
        pt.ml(th, split, HD)[1] = L;
      }
    }
  }
}

// ------------------------------------------------------- waves split keys
// What the 16 keys of an entry that names no page, or that nobody sees, are
// read from: their scores are masked, and 0 times a finite value stays 0.
static __device__ __attribute__((aligned(16))) bf16_t zero_keys[16 * 128];

// bf16, head_dim 64 or 128, at most 16 query columns: column x is token x / G of
// the row's, query head x % G of the KV head's G, so the columns' queries and
// outputs are contiguous.  The queries are rounded to bf16 and so is what that
// leaves of them, and the two scores are added, so that they keep 16 bits (the
// output is then 0.0019 to 0.0020 off in the 2-norm instead of 0.0028 to 0.0030, of
// which 0.0017 are its own rounding).  TWICE: up to eight columns are there twice,
// 0 .. 7 the first part and 8 .. 15 the second, at no product more; more columns
// take a second product (64 rows of 300 to 900 keys, 8 KV heads of 128, 12 columns:
// 36.8 us with it and 36.7 without).  Work-group = (split, KV head, row), NW
// waves; every wave takes an even share of the 32-key blocks that hold visible
// keys and waits on no other until the merge.
//   S^T = K Q^T   (v_mfma_f32_16x16x32_bf16): the A operand, 16 keys x 32 dims,
//         comes from memory straight into registers.
//   O^T += V^T P^T: a V block goes memory -> LDS (the wave's own double buffer)
//         and its A operand comes from two transpose reads; the contraction
//         visits the keys in the order the lane holds their probabilities.
// The next block's keys and values are in flight while one is computed.  A
// block's 16-key halves lie in one page each; lane i holds the page numbers of
// block i of a run of 64, so a block's addresses cost two lane reads.  The keys
// below common[row] are another pass's.  Lanes whose key nobody sees read a visible
// key of the half instead (KeyBlocks::safe), and past the end of the half for its
// value, which gives zeros (0 times the infinity of a neighbour would be NaN).
// Bound by memory: each key and value byte is read once (8 KV heads of 128: 3 rows
// of 20011 to 40007 keys 369 MB in 79 us, 4.7 TB/s; 512 tails of 63 to 380 keys 464
// MB in 105 us, 4.4 TB/s; 64 rows in a window of 1024, 8 heads of 64, 135 MB in 25
// us, 5.4 TB/s).  head_dim 64 keeps four waves a SIMD (512 rows of 100 to 600 keys
// 75.7 us; as the compiler chooses, three, 77.5).
template <int HD, int NW, bool TWICE>
__global__ void __launch_bounds__(64 * NW, HD == 64 ? 4 : 1)
paged_wave_kernel(PagedAttnArgs a, const int32_t* __restrict__ common, int splits, int pre, int slots, float qscale) {
  constexpr int KS = HD / 32, DT = HD / 16, CPK = HD / 8, VB = 32 * HD;
  constexpr int KPD = 64 / CPK, NV = 32 / KPD;     // keys per V copy, copies of a block
  constexpr int INFLIGHT = 2 * KS + NV;            // memory operations of a block
  __shared__ __attribute__((aligned(1024))) bf16_t lds[NW * 2 * VB];
  const int split = blockIdx.x, h = blockIdx.y, row = blockIdx.z;
  const RowState rs = row_state(a, row);
  if (rs.n == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fg = lane >> 4;
  const int g = a.hq / a.hkv;
  const int x = TWICE ? fr & 7 : fr, t = x / g;    // this lane's column
  const bool live = t < rs.n;
  const int end_c = rs.p0 + (live ? t : 0) + 1, lo_c = window_start(end_c - 1, a.window);
  const int lo_last = window_start(rs.len - 1, a.window);
  KeyBlocks kb;
  kb.set(common ? common[row] : 0, a.sinks, window_start(rs.p0, a.window), rs.len);
  const int shares = splits * NW, me = split * NW + wave;
  const int i0 = (int)((int64_t)kb.count * me / shares), i1 = (int)((int64_t)kb.count * (me + 1) / shares);
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  bf16_t* vbuf = lds + wave * 2 * VB;

  // The pages of blocks [base, base + 64) of this wave, -1 for none.
  int base = i0, d0 = -1, d1 = -1;
  auto look_up = [&] {
    d0 = d1 = -1;
    if (base + lane < i1) {
      const int k0 = kb.key0(base + lane);
      const int p0 = kb.any16(k0) ? tab[k0 >> a.shift] : -1;
      const int p1 = kb.any16(k0 + 16) ? tab[(k0 + 16) >> a.shift] : -1;
      d0 = (uint32_t)p0 < (uint32_t)a.n_pages ? p0 : -1;
      d1 = (uint32_t)p1 < (uint32_t)a.n_pages ? p1 : -1;
    }
  };
  auto at = [&](const void* pool, int page, int key) -> const bf16_t* {
    return page < 0 ? zero_keys : (const bf16_t*)pool + page_offset(page, a.hkv, h, a.shift, key, HD);
  };
  auto halves = [&](int b, int (&pg)[2]) {
    pg[0] = __builtin_amdgcn_readlane(d0, b);
    pg[1] = __builtin_amdgcn_readlane(d1, b);
  };
  auto load_block = [&](int b, uint4 (&kr)[2][KS], int buf) {
    int pg[2];
    halves(b, pg);
    const int k0 = kb.key0(base + b);
    const bool whole = kb.all32(k0);
    int j[2] = {fr, fr};
    if (!whole) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (pg[u] >= 0) j[u] = kb.safe(k0 + 16 * u, k0 + 16 * u + fr) - (k0 + 16 * u);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bf16_t* src = at(a.kpool, pg[u], k0 + 16 * u);
#pragma unroll
      for (int st = 0; st < KS; ++st)
        kr[u][st] = *reinterpret_cast<const uint4*>(src + (j[u] * HD + 8 * fg + 32 * st));
    }
    constexpr int HALF = 16 * HD * 2;   // bytes
    const BufRsrc rv[2] = {buf_rsrc(at(a.vpool, pg[0], k0), HALF), buf_rsrc(at(a.vpool, pg[1], k0 + 16), HALF)};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int u = i * KPD / 16, kk = i * KPD + lane / CPK;   // half, key of the block
      uint32_t off = (uint32_t)(((kk - 16 * u) * HD + 8 * vslot<CPK>(kk, lane % CPK)) * 2);
      if (!whole && !kb.has(k0 + kk)) off = HALF;
      dma16(rv[u], off, 0, vbuf + buf * VB + i * 512);
    }
  };

  // The first block's loads go out before the queries are read.
  uint4 ka[2][KS], kc[2][KS];
  look_up();
  if (i0 < i1) load_block(0, ka, 0);

  // Q^T fragments (B operand): lane holds Q[column fr][32 s + 8 fg .. + 8]
  bf16x8 qf[KS], ql[TWICE ? 1 : KS];
  {
    const float* qr = a.q + (((int64_t)row * a.lr + (live ? t : 0)) * a.hq + h * g + (live ? x - t * g : 0)) * HD;
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      const float4 x = *reinterpret_cast<const float4*>(qr + 32 * st + 8 * fg);
      const float4 y = *reinterpret_cast<const float4*>(qr + 32 * st + 8 * fg + 4);
      const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float full = v[e] * qscale;
        const __bf16 top = (__bf16)full;
        const __bf16 left = (__bf16)(full - (float)top);
        qf[st][e] = TWICE && fr >= 8 ? left : top;
        if constexpr (!TWICE) ql[st][e] = left;
      }
    }
  }

  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  // transpose-read addresses: lane names 4 dims (dt 16 + 4 (fr & 3) ..) of key
  // 4 fg + (fr >> 2), and of the key 16 on (16 rows on, same slots)
  uint32_t vaddr[DT];
  {
    const int kr0 = 4 * fg + (fr >> 2);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      vaddr[dt] = lds_addr(vbuf + kr0 * HD + 8 * vslot<CPK>(kr0, 2 * dt + ((fr & 3) >> 1)) + 4 * (fr & 1));
  }
  auto compute = [&](int b, const uint4 (&kr)[2][KS], auto bufc) {
    f32x4 st[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      st[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s2 = 0; s2 < KS; ++s2) {
        st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[u][s2]), qf[s2], st[u], 0, 0, 0);
        if constexpr (!TWICE)
          st[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[u][s2]), ql[s2], st[u], 0, 0, 0);
      }
    }
    const int k0 = kb.key0(base + b);
    int pg[2];
    halves(b, pg);
    float sv[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sv[i] = st[0][i];
      sv[4 + i] = st[1][i];
    }
    if constexpr (TWICE) {   // the other of lanes fr and fr ^ 8 (a rotation by 8 of 16)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        sv[i] += __builtin_bit_cast(
            float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, sv[i]), 0x128, 0xF, 0xF, true));
    }
    // (uniform) some column does not see some key of the block
    if (k0 + 32 > rs.p0 + 1 || (k0 < lo_last && k0 + 32 > a.sinks) || pg[0] < 0 || pg[1] < 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = k0 + 4 * fg + (i & 3) + 16 * (i >> 2);
        const bool sees = j < end_c && (j >= lo_c || j < a.sinks) && pg[i >> 2] >= 0;
        if (!sees) sv[i] = -INFINITY;
      }
    }
    float mt = sv[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mt = fmaxf(mt, sv[i]);
    mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
    mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
    // rescaled only when some column's maximum grows; the exact maximum, so that
    // the largest probability, 1, loses nothing in bf16
    if (__any(mt > m)) {
      const float mn = fmaxf(m, mt);
      const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= corr;
      m = mn;
    }
    const float mr = m == -INFINITY ? 0.f : m;   // (a column without a key so far)
    bf16x8 pf;
    float ps = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float pv = __builtin_amdgcn_exp2f(sv[i] - mr);
      ps += pv;
      pf[i] = (__bf16)pv;
    }
    l += ps;
    constexpr int BUF = decltype(bufc)::value;
#pragma unroll
    for (int e0 = 0; e0 < DT; e0 += 4) {
      const uint32_t va[4] = {vaddr[e0], vaddr[e0 + 1], vaddr[e0 + 2], vaddr[e0 + 3]};
      i16x4 lo[4], hi[4];
      lds_read_tr16_pairs<4, BUF * VB * 2, (BUF * VB + 16 * HD) * 2>(va, lo, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        o[e0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tr16_pair(lo[i], hi[i]), pf, o[e0 + i], 0, 0, 0);
    }
  };

  // One block ahead.  Every fetch in the loop is unconditional, so the
  // compiler's own waits count the younger block's loads as in flight.
  const std::integral_constant<int, 0> buf0{};
  const std::integral_constant<int, 1> buf1{};
  const std::integral_constant<int, INFLIGHT> next{};
  auto compute_after = [&](auto left, int b, const uint4 (&kr)[2][KS], auto bufc) {
    __builtin_amdgcn_sched_barrier(0);   // (the fetch before it stays before it)
    vm_wait<decltype(left)::value>();
    compute(b, kr, bufc);
    __builtin_amdgcn_sched_barrier(0);
  };
  while (base < i1) {
    const int nb = imin(64, i1 - base);
    int b = 0;
    for (; b + 2 < nb; b += 2) {
      load_block(b + 1, kc, 1);
      compute_after(next, b, ka, buf0);
      load_block(b + 2, ka, 0);
      compute_after(next, b + 1, kc, buf1);
    }
    if (b + 1 < nb) {
      load_block(b + 1, kc, 1);
      compute_after(next, b, ka, buf0);
      compute_after(buf0, b + 1, kc, buf1);
    } else {
      compute_after(buf0, b, ka, buf0);
    }
    base += 64;
    if (base < i1) {   // (a run of 64 blocks drains: one round trip in 2048 keys)
      look_up();
      load_block(0, ka, 0);
    }
  }

  // join the waves: per column the unnormalised output, (max, sum) behind it
  constexpr int ROW = HD + 4;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();
  float* sm = reinterpret_cast<float*>(lds);   // [NW][16][ROW]
  float* w = sm + (wave * 16 + fr) * ROW;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(w + dt * 16 + 4 * fg) = o[dt];
  if (fg == 0) {
    w[HD] = m;
    w[HD + 1] = l;
  }
  __syncthreads();
  // A thread takes eight dimensions of a column.  With one split the shared keys'
  // slots are joined here too (up to FOLD at a time) and the output is written.
  constexpr int FOLD = 4;
  const Partials pt{a.part, (int64_t)a.rows * a.lr * a.hq, slots};
  for (int i = threadIdx.x; i < rs.n * g * CPK; i += 64 * NW) {
    const int c = i / CPK, d = 8 * (i % CPK);      // column
    const int64_t th = ((int64_t)row * a.lr + c / g) * a.hq + h * g + c % g;
    float M = -INFINITY, L = 0.f, A[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m1, float l1, const float* o8) {
      if (l1 == 0.f) return;   // nothing seen
      const float mn = fmaxf(M, m1), ca = __builtin_amdgcn_exp2f(M - mn), cb = __builtin_amdgcn_exp2f(m1 - mn);
      M = mn;
      L = L * ca + l1 * cb;
#pragma unroll
      for (int e = 0; e < 8; ++e) A[e] = A[e] * ca + o8[e] * cb;
    };
    if (splits == 1) {
      for (int k0 = 0; k0 < pre; k0 += FOLD) {
        float2 ml[FOLD];
        float4 v[FOLD][2];
#pragma unroll
        for (int k = 0; k < FOLD; ++k) {
          const int slot = imin(k0 + k, pre - 1);
          ml[k] = *reinterpret_cast<const float2*>(pt.ml(th, slot, HD));
          const float4* src = reinterpret_cast<const float4*>(pt.o(th, slot, HD) + d);
          v[k][0] = src[0];
          v[k][1] = src[1];
        }
#pragma unroll
        for (int k = 0; k < FOLD; ++k) {
          const float o8[8] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w, v[k][1].x, v[k][1].y, v[k][1].z, v[k][1].w};
          if (k0 + k < pre) add(ml[k].x, ml[k].y, o8);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      const float* ws = sm + (k * 16 + c) * ROW;
      const f32x4 u = *reinterpret_cast<const f32x4*>(ws + d), v = *reinterpret_cast<const f32x4*>(ws + d + 4);
      const float o8[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
      add(ws[HD], ws[HD + 1], o8);
    }
    if (splits == 1) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      bf16x8 r;
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = (__bf16)(A[e] * inv);
      *reinterpret_cast<bf16x8*>((bf16_t*)a.out + th * HD + d) = r;
    } else {
      float4* dst = reinterpret_cast<float4*>(pt.o(th, pre + split, HD) + d);
      dst[0] = make_float4(A[0], A[1], A[2], A[3]);
      dst[1] = make_float4(A[4], A[5], A[6], A[7]);
      if (d == 0) *reinterpret_cast<float2*>(pt.ml(th, pre + split, HD)) = make_float2(M, L);
    }
  }
}

// -------------------------------------------------------- query tiles
// bf16 flash attention with v_mfma_f32_32x32x16_bf16, head_dim 64 or 128, 128
// query columns a work-group, 32 a wave; column x is token x / G, query head x %
// G of the KV head's G, so four query heads of eight tokens share a wave, and
// the work-group's tokens are as few as they can be (their causal and window
// edges cost the fewest masked keys).
//   PRE = false: the tokens of one row, over all its keys.
//   PRE = true:  the tokens of all rows, over row 0's leading keys; a column
//                sees those its row has in common (`common`).
//   S^T = K Q^T   (keys x columns): lane l holds, of every 32 keys, the 16 with
//                 (key / 4) % 2 = l / 32 for column l % 32.
//   O^T += V^T P^T: the contraction visits a 16-key chunk in the order the lane
//                 holds it, so the B operand is the lane's own probabilities;
//                 the A operand comes from V by two LDS transpose reads.
// The 32-key blocks that hold a visible key go memory -> LDS by direct copies,
// three stages deep, one barrier a block; 16-byte chunks sit XOR-swizzled in the
// LDS rows.  Lane i keeps the addresses and mask flags of block i of a run of
// 64; blocks that every query sees whole skip the mask; the output is rescaled
// only when a maximum has moved by more than kStale.  Three work-groups a CU (48
// KB of LDS, at most 168 registers; PRE: two, which is all that it starts, see
// kTileTarget): one's exponentials and waits run under another's matrix
// instructions.  On 7777 tokens, 32 query and 8 KV heads of 128, in a window of
// 4096 with 4 sinks (384 GFLOP over visible keys): 390 to 413 us, 930 to 990 TFLOP/s
// (463 us in an uninterrupted run); earlier forms of this kernel with 64 columns a
// wave took 645 us (its registers move through the accumulation file), with 256
// columns a work-group 426, with one barrier per two blocks 420.  There the matrix
// cores are busy for 48 % and the vector ALU for 52 % of the time, at the 1.8 GHz
// that the part holds under both.  With several splits a work-group takes an even
// share of the blocks.
// Queries and probabilities are rounded to bf16 for the products: outputs are
// 0.0030 to 0.0033 off in the 2-norm, of which 0.0017 are their own rounding.  The
// queries' low part takes 8 matrix instructions on a block's 16 at head_dim 128,
// and 32 more registers, which three work-groups a CU do not leave (the prompt of
// 7777 531 us with it, 61 chunks of up to 381 258 and 193).  PRE has them
// and adds it, as the wave kernel does for the rest of the same rows: 0.0022 to
// 0.0023 instead of 0.0031 to 0.0033 (512 rows on 2048 shared keys, 8 KV heads of
// 128, 151.5 us instead of 147.8; 8 heads of 64, 1024 shared, 106.7 instead of 106.8).
constexpr int kTileStages = 3;
constexpr float kStale = 8.f;
constexpr int kTileCols = 128;

template <int HD, bool PRE>
__global__ void __launch_bounds__(256, PRE ? 2 : 3)
paged_tile_kernel(PagedAttnArgs a, const int32_t* __restrict__ common, int splits, int slots, float qscale) {
  constexpr int KT = 32, NW = 4;
  constexpr int KS = HD / 16, DT = HD / 32, CPK = HD / 8;
  constexpr int TILE = KT * HD;                // bf16 elements of a K (or V) block
  constexpr int RPI = 64 / CPK;                // keys per copy instruction (1 KB)
  constexpr int DPW = KT / RPI / NW;           // copies per wave of a K (or V) block
  constexpr int HALF = 16 * HD * 2;            // bytes of 16 keys
  constexpr int CPW = 2 * DPW;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[kTileStages * 2 * TILE];
  __shared__ int bounds[NW][2];
  // a 1-D grid dealt round-robin to the 8 XCDs: each takes consecutive logical
  // blocks, the query tiles of one (row, KV head, split) fastest, the last and
  // longest first, so that those reading the same keys share one L2; the KV heads
  // slowest, so that every XCD has its part of all rows, long and short ones, and
  // one copy of the pages that rows share (8 KV heads of 128, 7 rows of up to 1000
  // new tokens 110 us, with the rows slowest 161; 61 of up to 381 226 and 231)
  const int g = a.hq / a.hkv;
  const int X = (PRE ? a.rows * a.lr : a.lr) * g;                 // columns
  const int ngq = (X + kTileCols - 1) / kTileCols, total = ngq * splits * a.hkv * (PRE ? 1 : a.rows);
  const int per_xcd = (total + 7) / 8;
  const int pid = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (pid >= total) return;
  const int qg = ngq - 1 - pid % ngq;
  const int split = pid / ngq % splits;
  const int nrow = PRE ? 1 : a.rows;
  const int row = pid / (ngq * splits) % nrow;
  const int h = pid / (ngq * splits * nrow);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int x0 = qg * kTileCols, xw = x0 + 32 * wave;             // first column, of the wave too
  const int token0 = PRE ? 0 : row * a.lr;
  const RowState rs = row_state(a, row);
  if (!PRE && x0 >= rs.n * g) return;

  // This lane's column sees keys [0, sinks) and [lo, end); the wave's columns
  // all see a key below `all_end` at or past `all_lo`, none one at or past
  // wend.  Columns that are no query (live = false) see everything: their
  // results are dropped.
  bool live;
  int lo_c = 0, end_c = INT_MAX;
  {
    const int x = xw + fr, tok = x / g;
    if (PRE) {
      live = x < X;
      const int r = live ? tok / a.lr : 0, t = tok - r * a.lr;
      const RowState cs = row_state(a, r);
      live = live && t < cs.n;
      if (live) {
        end_c = common[r];
        lo_c = imin(end_c, window_start(cs.p0 + t, a.window));
      }
    } else {
      live = x < rs.n * g;
      if (live) {
        end_c = rs.p0 + tok + 1;
        lo_c = window_start(end_c - 1, a.window);
      }
    }
  }
  int all_end, all_lo, wend, wlo;   // over the wave's columns: min end, max lo, max end, min lo
  if (PRE) {
    all_end = end_c;
    all_lo = lo_c;
    wend = live ? end_c : 0;
    wlo = live ? lo_c : INT_MAX;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      all_end = imin(all_end, __shfl_xor(all_end, o, 64));
      all_lo = imax(all_lo, __shfl_xor(all_lo, o, 64));
      wend = imax(wend, __shfl_xor(wend, o, 64));
      wlo = imin(wlo, __shfl_xor(wlo, o, 64));
    }
    all_end = __builtin_amdgcn_readfirstlane(all_end);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    wend = __builtin_amdgcn_readfirstlane(wend);
    wlo = __builtin_amdgcn_readfirstlane(wlo);
  } else {
    const int last = imin(xw + 31, rs.n * g - 1);
    const bool any = xw < rs.n * g;
    all_end = rs.p0 + xw / g + 1;
    wend = any ? rs.p0 + last / g + 1 : 0;
    all_lo = any ? window_start(wend - 1, a.window) : 0;
    wlo = window_start(all_end - 1, a.window);
  }
  KeyBlocks kb;
  if (PRE) {
    if (lane == 0) {
      bounds[wave][0] = wlo;
      bounds[wave][1] = wend;
    }
    __syncthreads();
    const int end = imax(imax(bounds[0][1], bounds[1][1]), imax(bounds[2][1], bounds[3][1]));
    const int lo = imin(imin(bounds[0][0], bounds[1][0]), imin(bounds[2][0], bounds[3][0]));
    kb.set(0, a.sinks, __builtin_amdgcn_readfirstlane(imin(lo, end)), __builtin_amdgcn_readfirstlane(end));
  } else {
    const int last = imin(x0 + kTileCols - 1, rs.n * g - 1);
    kb.set(0, a.sinks, window_start(rs.p0 + x0 / g, a.window), rs.p0 + last / g + 1);
  }
  const int i0 = (int)((int64_t)kb.count * split / splits), i1 = (int)((int64_t)kb.count * (split + 1) / splits);
  const int ntile = i1 - i0;

  // Where blocks [64 c, 64 c + 64) of this split lie: lane i holds, for block 64
  // c + i, the addresses of its halves' keys and values (of zeros where no page
  // holds them) and its flags, so that issuing a block's copies costs a few lane
  // reads: scalar instructions in a row cost a wave 5-8 cycles each.
  enum {
    GONE0 = 1, GONE1 = 2,   // no page holds the half
    EDGE = 4,               // some column of the wave does not see every key
    PAST = 8,               // no column of the wave sees a key
    PARTLY = 16             // no column of the work-group sees some key
  };
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  uint32_t flags = 0;
  uint2 at[2][2];           // [keys, values][half]
  int entry[2];             // what the table says of block first + lane's halves
  auto read_table = [&](int first) {
    const int k0 = kb.key0(i0 + first + lane);
#pragma unroll
    for (int u = 0; u < 2; ++u)
      entry[u] = first + lane < ntile && kb.any16(k0 + 16 * u) ? tab[(k0 + 16 * u) >> a.shift] : -1;
  };
  auto look_up = [&](int first) {
    const int k0 = kb.key0(i0 + first + lane);
    flags = kb.all32(k0) ? 0 : PARTLY;
    if (k0 + 32 > all_end || (k0 < all_lo && k0 + 32 > a.sinks)) flags |= EDGE;
    if (k0 >= wend) flags |= PAST;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k = k0 + 16 * u;
      const int page = (uint32_t)entry[u] < (uint32_t)a.n_pages ? entry[u] : -1;
      const int64_t off = page < 0 ? 0 : page_offset(page, a.hkv, h, a.shift, k, HD);
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const bf16_t* pool = page < 0 ? zero_keys : (const bf16_t*)(v ? a.vpool : a.kpool);
        const uint64_t addr = reinterpret_cast<uintptr_t>(pool + off);
        at[v][u] = make_uint2((uint32_t)addr, (uint32_t)(addr >> 32));
      }
      if (page < 0) flags |= EDGE | (u ? GONE1 : GONE0);
    }
  };
  // The table first, so that the first keys do not wait behind the queries.
  read_table(0);
  __builtin_amdgcn_sched_barrier(0);

  // The wave's 32 queries, 16 bytes per lane along whole rows (clamped rows;
  // results of columns that are no query are dropped)
  constexpr int LPR = HD / 4, RPQ = 64 / LPR, NQ = 32 / RPQ;   // lanes per query, queries per load, loads
  float4 qv[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    const int x = imin(xw + RPQ * i + lane / LPR, X - 1), tok = x / g;
    qv[i] = reinterpret_cast<const float4*>(
        a.q + ((int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g)) * HD)[lane % LPR];
  }
  __builtin_amdgcn_sched_barrier(0);

  // Copies: instruction i of a wave moves keys RPI (wave + NW i) .. of the
  // block; lane l writes slot l % CPK of key l / CPK and fetches the chunk
  // stored there, from a buffer resource at its 16-key half (no vector
  // arithmetic where every key is seen).  Keys and values that nobody sees are read
  // past the end of the half, as zeros, or from zeros where no page holds them.
  auto vswz = [](int k) { return HD == 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2; };
  uint32_t kcopy[DPW], vcopy[DPW];   // byte offsets in the half
#pragma unroll
  for (int i = 0; i < DPW; ++i) {
    const int r = RPI * (wave + NW * i) + lane / CPK, sl = lane % CPK;
    kcopy[i] = (uint32_t)((r & 15) * HD + 8 * (sl ^ (r & (CPK - 1)))) * 2;
    vcopy[i] = (uint32_t)((r & 15) * HD + 8 * (sl ^ vswz(r))) * 2;
  }
  uint32_t ring = 0;   // four flags for each stage
  auto issue = [&](int tile, int buf) {
    if ((tile & 63) == 0) {
      if (tile > 0) read_table(tile);
      look_up(tile);
    }
    const int from = tile & 63;
    bf16_t* kd = lds + buf * 2 * TILE;
    const uint32_t f = __builtin_amdgcn_readlane(flags, from);
    ring = (ring & ~(15u << (4 * buf))) | (f & 15u) << (4 * buf);
    auto source = [&](const uint2& v) {
      const uint32_t lo = __builtin_amdgcn_readlane(v.x, from), hi = __builtin_amdgcn_readlane(v.y, from);
      return buf_rsrc(reinterpret_cast<const void*>((uint64_t)hi << 32 | lo), HALF);
    };
    uint32_t ko[DPW], vo[DPW];
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      ko[i] = kcopy[i];
      vo[i] = vcopy[i];
    }
    if (f & PARTLY) {
#pragma unroll
      for (int i = 0; i < DPW; ++i) {
        if (kb.has(kb.key0(i0 + tile) + RPI * (wave + NW * i) + lane / CPK)) continue;
        ko[i] = vo[i] = HALF;
      }
    }
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      const int r0 = RPI * (wave + NW * i);
      // (128 dims: the waves' copies i lie in half i; 64: a wave has one copy)
      const int u = DPW == 2 ? i : r0 >> 4;
      const uint2 ks = DPW == 2 ? at[0][i] : u ? at[0][1] : at[0][0], vs = DPW == 2 ? at[1][i] : u ? at[1][1] : at[1][0];
      dma16(source(ks), ko[i], 0, kd + r0 * HD);
      dma16(source(vs), vo[i], 0, kd + TILE + r0 * HD);
    }
  };
  auto wait_barrier = [](auto n) {
    constexpr int N = decltype(n)::value;
    if constexpr (N == 0) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if constexpr (N == 2) asm volatile("s_waitcnt vmcnt(2) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else if constexpr (N == 4) asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    else static_assert(N < 0, "add this wait count");
  };

  // LDS element offsets: the K fragment of key fr (chunk 2 s + fh), and the
  // four dims dt 32 + 16 (l / 16 % 2) + 4 (l % 4) .. of V key 4 fh + l % 16 / 4
  bf16x8 qf[KS], ql[PRE ? KS : 1];   // the queries in bf16, what that leaves of them
  // byte offset in a stage of chunk fh of K row fr (chunk 2 s + fh: this ^ 32 s)
  const uint32_t kbase = (uint32_t)(fr * HD + 8 * (fh ^ (fr & (CPK - 1)))) * 2;
  // LDS address in the first V block of dims 16 (l / 16 % 2) + 4 (l % 4) .. of key
  // 4 fh + l % 16 / 4 (dims 32 dt on: this ^ 64 dt)
  uint32_t vbase;
  {
    const int vk = 4 * fh + ((lane & 15) >> 2);
    vbase = lds_addr(lds + TILE + vk * HD + 8 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ vswz(vk)) + 4 * (lane & 1));
  }

  f32x16 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  // from the lowest finite score: while a column has seen only -inf its
  // probabilities are exp2(-inf) = 0, where -inf - -inf would be NaN; for columns
  // that are no query from +inf, which no score of theirs passes, so that they
  // never rescale the others (and what lies there changes no rounding)
  float m = live ? -FLT_MAX : INFINITY, l = 0.f;

  auto zero = [](f32x16& sc) {
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
  };
  // The greatest score of each column.
  auto peak = [](const f32x16& sc) {
    float mt = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mt = fmaxf(mt, sc[e]);
    return fmaxf(mt, other_half(mt));
  };
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  auto frag = [&](const bf16_t* base, int s) {
    return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(base) + (kbase ^ (32u * s)));
  };
  auto step = [&](auto stage, int tile, uint32_t f) {
    constexpr int ST = decltype(stage)::value;
    constexpr int VB = ST * 2 * TILE * 2;   // bytes from vbase
    f32x16 sc;
    zero(sc);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bf16x8 k = frag(lds + ST * 2 * TILE, s);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[s], sc, 0, 0, 0);
      if constexpr (PRE) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, ql[s], sc, 0, 0, 0);
    }
    if (f & EDGE) {                            // (uniform)
      asm volatile("");                        // (a branch, not selects on every block)
      // bit j: this lane's key j of the block (of the 32 from 4 fh on) is seen
      const int k4 = kb.key0(i0 + tile) + 4 * fh;
      auto below = [](int n) { return n >= 32 ? ~0u : (1u << imax(n, 0)) - 1u; };
      uint32_t seen = below(end_c - k4) & (~below(lo_c - k4) | below(a.sinks - k4));
      if (f & GONE0) seen &= 0xFFFF0000u;
      if (f & GONE1) seen &= 0x0000FFFFu;
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = (int)(seen << (31 - 8 * (e >> 2) - (e & 3))) < 0 ? sc[e] : -INFINITY;
    }
    const float mt = peak(sc);
    // Probabilities are relative to a maximum up to 2^kStale out of date: a
    // rescaling of the accumulators costs as much as half a block's
    // exponentials, and a wave's 32 columns would need one in most blocks.
    if (__any(mt > m + kStale)) {
      const float mn = fmaxf(m, mt);
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= corr;
      m = mn;
    }
    uint32_t va[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) va[dt] = vbase ^ (64u * dt);
    bf16x8 pf[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[c][e] = (__bf16)__builtin_amdgcn_exp2f(sc[8 * c + e] - m);
      // (of the rounded ones, as the product has them)
#pragma unroll
      for (int e = 0; e < 8; e += 2) l = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[c][e], pf[c][e + 1]}, ones, l, false);
    }
    i16x4 lo[DT], hi[DT];
    lds_read_tr16_pairs<DT, VB, VB + 8 * HD * 2>(va, lo, hi);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr16_pair(lo[dt], hi[dt]), pf[0], o[dt], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    lds_read_tr16_pairs<DT, VB + 16 * HD * 2, VB + 24 * HD * 2>(va, lo, hi);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr16_pair(lo[dt], hi[dt]), pf[1], o[dt], 0, 0, 0);
  };
  bf16_t* const slice = lds + wave * 32 * HD;
  if (ntile > 0) {
    issue(0, 0);
    // (through the wave's own slice: its LDS operations are in order)
    bf16_t* qs = slice + 2 * TILE;
    auto stage_queries = [&](auto part, auto& out) {
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const int r = RPQ * i + lane / LPR, c4 = lane % LPR;
        const bf16x4 v = {part(qv[i].x), part(qv[i].y), part(qv[i].z), part(qv[i].w)};
        *reinterpret_cast<bf16x4*>(qs + r * HD + 8 * ((c4 >> 1) ^ (r & (CPK - 1))) + 4 * (c4 & 1)) = v;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) out[s] = frag(qs, s);
    };
    stage_queries([&](float v) { return (__bf16)(v * qscale); }, qf);
    if constexpr (PRE)
      stage_queries([&](float v) { return (__bf16)(v * qscale - (float)(__bf16)(v * qscale)); }, ql);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // every wave's queries read
    if (ntile > 1) issue(1, 1);
    auto one = [&](auto stage, int tile) {
      constexpr int ST = decltype(stage)::value;
      if (tile + 1 < ntile) wait_barrier(std::integral_constant<int, CPW>{});
      else wait_barrier(std::integral_constant<int, 0>{});
      if (tile + 2 < ntile) issue(tile + 2, (ST + 2) % kTileStages);
      const uint32_t f = ring >> (4 * ST);
      if (!(f & PAST)) step(stage, tile, f);
    };
    for (int tile = 0; tile < ntile; tile += 3) {
      one(std::integral_constant<int, 0>{}, tile);
      if (tile + 1 < ntile) one(std::integral_constant<int, 1>{}, tile + 1);
      if (tile + 2 < ntile) one(std::integral_constant<int, 2>{}, tile + 2);
    }
  }
  l += other_half(l);
  if (PRE || slots > 1) {
    if (!live) return;
    const Partials pt{a.part, (int64_t)a.rows * a.lr * a.hq, slots};
    const int x = xw + fr, tok = x / g;
    const int64_t th = (int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g);
    float* po = pt.o(th, split, HD);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(po + 32 * dt + 8 * q4 + 4 * fh) =
            make_float4(o[dt][4 * q4], o[dt][4 * q4 + 1], o[dt][4 * q4 + 2], o[dt][4 * q4 + 3]);
    if (fh == 0) {
      float* ml = pt.ml(th, split, HD);
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  wait_barrier(std::integral_constant<int, 0>{});   // every wave is done with the blocks
  // The outputs pass through the wave's slice of LDS (chunks placed like K's),
  // so that a query's leave as one contiguous run.
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const bf16x4 v = {(__bf16)(o[dt][4 * q4] * inv), (__bf16)(o[dt][4 * q4 + 1] * inv),
                        (__bf16)(o[dt][4 * q4 + 2] * inv), (__bf16)(o[dt][4 * q4 + 3] * inv)};
      *reinterpret_cast<bf16x4*>(slice + fr * HD + 8 * ((4 * dt + q4) ^ (fr & (CPK - 1))) + 4 * fh) = v;
    }
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = RPI * i + lane / CPK, c = lane % CPK, x = xw + r, tok = x / g;
    const uint4 v = *reinterpret_cast<const uint4*>(slice + r * HD + 8 * (c ^ (r & (CPK - 1))));
    if (x >= rs.n * g) continue;
    *reinterpret_cast<uint4*>((bf16_t*)a.out + ((int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g)) * HD + 8 * c) = v;
  }
}

// ------------------------------------------------------------------ plan
enum PagedKind { PAGED_VECTOR, PAGED_WAVE, PAGED_TILE };
struct PagedPlan {
  PagedKind kind;
  int nw;       // PAGED_WAVE: waves of a work-group
  int splits;   // work-groups that share a row's keys
  int pre;      // PAGED_WAVE: splits of the shared keys' own pass (0: none)
  // Partial slots: the shared keys' first, then the row's own splits (none where
  // one work-group takes them all: it writes the output).
  int slots() const { return pre + (splits > 1 ? splits : 0); }
};

// Query columns of a work-group of the vector kernel, for rows of `cols` of them.
static int vector_cols(int cols) { return cols >= 8 ? 8 : cols >= 4 ? 4 : cols >= 2 ? 2 : 1; }
static int64_t vector_groups(const PagedAttnArgs& a) {
  const int cols = a.lr * (a.hq / a.hkv), gc = vector_cols(cols);
  return (int64_t)a.rows * a.hkv * ((cols + gc - 1) / gc);
}

// Work-groups of the tile kernel that the split aims at: two a CU (with three, 4
// to 32 prompts of 300 to 512 tokens take the same to 1 %; 512 rows on 2048 shared
// keys 152 us, with three 167, with one 163).
constexpr int kTileTarget = 512;
constexpr int kMaxSplits = 64;

// Splits of `blocks` 32-key blocks over work-groups of the tile kernel of which
// `groups` take all keys, at least eight blocks each.
static int tile_splits(int64_t groups, int64_t blocks) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({kTileTarget / groups, blocks / 8, kMaxSplits}));
}

// Waves that fill the chip (8 KV heads of 128: 64 rows on 300 keys 17.5 us, with
// half as many 18.0 and with twice as many 26.1; 8 on 8000 46.4, 49.6 and 49.6).
constexpr int kWaveTarget = 2048;
// The shared keys get a pass of their own where the rows would otherwise read them
// from the caches for at least so many bytes (at ~15 TB/s, 20 us: what the two
// launches and the joining cost).  8 KV heads of 128, tails of up to 60 keys: 64
// rows on 1024 shared keys 28.6 us without and 29.5 with (268 MB), 96 on 1024 38.3
// and 30.5 (403 MB), 128 on 1024 47 and 32 (537 MB), 512 on 256 58 and 51; beside
// tails of 63 to 380 keys 300 on 256 80.0 and 85.7 (315 MB); 8 heads of 64: 256 rows
// on 512 27.6 and 26.4 (268 MB).
constexpr int64_t kShareBytes = 300 << 20;

static PagedPlan paged_plan(const PagedAttnArgs& a) {
  PagedPlan p{PAGED_VECTOR, 1, 1, 0};
  const int g = a.hq / a.hkv;
  int64_t keys = planned_keys(a);
  if (a.dtype == SR_BF16 && a.hd >= 64 && a.lr * g <= 16) {
    p.kind = PAGED_WAVE;
    const bool far = a.window > 0 && a.max_len > a.window;   // (windows have left key 0)
    const int64_t shared = far ? 0 : std::min<int64_t>(a.shared, keys - a.lr);
    if (shared > 0 && (int64_t)a.rows * shared * a.hkv * a.hd * 4 >= kShareBytes) {
      const int64_t tiles = ((int64_t)a.rows * a.lr * g + kTileCols - 1) / kTileCols;
      p.pre = tile_splits(tiles * a.hkv, shared / 32);
      keys -= shared;
    }
    const int64_t pairs = (int64_t)a.rows * a.hkv, blocks = (keys + 31) / 32;
    int64_t want = std::max<int64_t>(1, std::min<int64_t>(kWaveTarget / pairs, blocks / 2));
    if (want > 8 && pairs * 8 >= 1024) want = 8;
    p.nw = want >= 8 ? 8 : want >= 4 ? 4 : want >= 2 ? 2 : 1;
    p.splits = (int)std::min<int64_t>(kMaxSplits, (want + p.nw - 1) / p.nw);
  } else if (a.dtype == SR_BF16 && a.hd >= 64) {
    p.kind = PAGED_TILE;
    const int64_t tiles = ((int64_t)a.lr * g + kTileCols - 1) / kTileCols;
    p.splits = tile_splits(tiles * a.hkv * a.rows, keys / 32);
  } else {
    const int64_t groups = vector_groups(a);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({1024 / groups, keys / 256, kMaxSplits}));
  }
  return p;
}

// Scratch: the partial slots, then common[rows].
static size_t partial_floats(const PagedAttnArgs& a, const PagedPlan& p) {
  return (size_t)a.rows * a.lr * a.hq * p.slots() * (a.hd + 2);
}
size_t paged_attn_scratch(const PagedAttnArgs& a) {
  if (a.rows <= 0 || a.lr <= 0) return 0;
  const PagedPlan p = paged_plan(a);
  return partial_floats(a, p) + (p.pre ? a.rows : 0);
}

template <typename T, int HD>
static void launch_vector(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  const float qscale = kLog2e / sqrtf((float)HD);
  const int64_t blocks = vector_groups(a) / a.hkv * p.splits;
  SR_REQUIRE(blocks <= kMaxGroups, SR_ERR_UNSUPPORTED, "attention grid too large");
  const dim3 grid((unsigned)blocks, a.hkv);
#define SR_VECTOR(GC) SR_LAUNCH((paged_vector_kernel<T, HD, GC>), grid, dim3(256), 0, s, a, p.splits, qscale)
  switch (vector_cols(a.lr * (a.hq / a.hkv))) {
    case 8: SR_VECTOR(8); break;
    case 4: SR_VECTOR(4); break;
    case 2: SR_VECTOR(2); break;
    default: SR_VECTOR(1); break;
  }
#undef SR_VECTOR
  SR_CHECK_LAUNCH();
  if (p.splits > 1) launch_merge<T, HD>(a, p.splits, s);
}

template <int HD, bool PRE>
static void launch_tile(const PagedAttnArgs& a, const int32_t* common, int splits, int slots, hipStream_t s) {
  const float qscale = kLog2e / sqrtf((float)HD);
  const int64_t cols = (int64_t)(PRE ? a.rows : 1) * a.lr * (a.hq / a.hkv);
  const int64_t total = (cols + kTileCols - 1) / kTileCols * splits * a.hkv * (PRE ? 1 : a.rows);
  SR_REQUIRE(total <= kMaxGroups - 8, SR_ERR_UNSUPPORTED, "attention grid too large");
  SR_LAUNCH((paged_tile_kernel<HD, PRE>), dim3((unsigned)(8 * ((total + 7) / 8))), dim3(256), 0, s, a, common, splits,
            slots, qscale);
  SR_CHECK_LAUNCH();
}

template <int HD>
static void launch_wave(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  const float qscale = kLog2e / sqrtf((float)HD);
  int32_t* common = nullptr;
  if (p.pre) {
    common = reinterpret_cast<int32_t*>(a.part + partial_floats(a, p));
    SR_LAUNCH(paged_common_kernel, dim3((a.rows + 3) / 4), dim3(256), 0, s, a, common);
    SR_CHECK_LAUNCH();
    launch_tile<HD, true>(a, common, p.pre, p.slots(), s);
  }
  const dim3 grid(p.splits, a.hkv, a.rows);
#define SR_PAGED_WAVE2(NW, TWICE)                                                                                 \
  SR_LAUNCH((paged_wave_kernel<HD, NW, TWICE>), grid, dim3(64 * NW), 0, s, a, (const int32_t*)common, p.splits, p.pre, \
            p.slots(), qscale)
#define SR_PAGED_WAVE(NW)                                       \
  do {                                                          \
    if (a.lr * (a.hq / a.hkv) <= 8) SR_PAGED_WAVE2(NW, true);   \
    else SR_PAGED_WAVE2(NW, false);                             \
  } while (0)
  switch (p.nw) {
    case 8: SR_PAGED_WAVE(8); break;
    case 4: SR_PAGED_WAVE(4); break;
    case 2: SR_PAGED_WAVE(2); break;
    default: SR_PAGED_WAVE(1); break;
  }
#undef SR_PAGED_WAVE
#undef SR_PAGED_WAVE2
  SR_CHECK_LAUNCH();
  if (p.splits > 1) launch_merge<bf16_t, HD>(a, p.slots(), s);
}

template <int HD>
static void matrix_cores(const PagedAttnArgs& a, const PagedPlan& p, hipStream_t s) {
  if (p.kind == PAGED_WAVE) {
    launch_wave<HD>(a, p, s);
    return;
  }
  launch_tile<HD, false>(a, nullptr, p.splits, p.slots(), s);
  if (p.splits > 1) launch_merge<bf16_t, HD>(a, p.slots(), s);
}

void paged_attn(const PagedAttnArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.lr <= 0) return;
  const PagedPlan p = paged_plan(a);
  if (p.kind != PAGED_VECTOR) {
    if (a.hd == 128) matrix_cores<128>(a, p, s);
    else matrix_cores<64>(a, p, s);
    return;
  }
  if (a.dtype == SR_BF16) {   // (head_dim 32: the others take the matrix cores)
    launch_vector<bf16_t, 32>(a, p, s);
    return;
  }
  switch (a.hd) {
    case 32: launch_vector<float, 32>(a, p, s); break;
    case 64: launch_vector<float, 64>(a, p, s); break;
    default: launch_vector<float, 128>(a, p, s); break;
  }
}

}  // namespace sr
