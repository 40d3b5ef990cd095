// Causal attention over pages of 4 bits, with a sliding window and sink tokens,
// rows of their own lengths, on the matrix cores.
//
//   fp4_wave_kernel   up to 16 query columns a row and KV head (single tokens, short
//                     drafts): the waves split a row's keys
//   fp4_tile_kernel   128 query columns a work-group, keys staged in LDS for all of
//                     them: prompts, and the part of the rows that lies in the pages
//                     of row 0, once for all rows
//   paged_merge_kernel joins the partials of a token's work-groups
//
// Two codes and their scale become two bf16 in one instruction, exactly
// (v_cvt_scalef32_pk_bf16_fp4), so the products see the cache's own values, and what
// is rounded is the queries and the probabilities.  They enter as parts of 8 bits each:
// what a rounding to bf16 leaves is the next part, and the products add up.  Outputs in
// fp32 take three parts of either, all 24 bits; in bf16 two of a query and, where a second
// one costs no product (up to 8 columns, fp4_wave_kernel), two of a probability, else one;
// prompts in bf16 multiply the codes themselves with queries in parts of 6 bits
// (fp4_tile_kernel).
// Online softmax in base 2 (queries carry log2 e / sqrt(head_dim)).  A score that is
// NaN never raises a maximum and always enters the sum, so "nothing seen" is a sum
// equal to 0 and a maximum of -inf says nothing about the sum.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "common.h"
#include "fp4.h"
#include "kernels.h"
#include "paged_parts.h"
#include "specrej_serving.h"

namespace sr {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

constexpr float kStale = 8.f;

// The parts of x: bf16(x), bf16 of what that leaves, and so on.
template <int P>
__device__ __forceinline__ void in_parts(float x, __bf16 (&p)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    p[i] = (__bf16)x;
    x -= (float)p[i];
  }
}

// The sum over the lanes that hold a column's parts, the same bits in each of them
// (rotations by 8, then 4 of 16 lanes: every addition is of the same pair in both of
// its lanes), or their probabilities' parts would not fit together.
template <int CTRL>
__device__ __forceinline__ float rotated(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int SPREAD>
__device__ __forceinline__ float parts_sum(float v) {
  if constexpr (SPREAD > 1) v += rotated<0x128>(v);
  if constexpr (SPREAD == 4) v += rotated<0x124>(v);
  return v;
}

// N 4-byte words from an address aligned to them.
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// The slot of chunk c (8 dimensions) of key k in a wave's LDS copy of values: keys
// four apart meet in a transpose read.
template <int CPK>
__device__ __forceinline__ int wslot(int k, int c) {
  if constexpr (CPK == 4) return c ^ (((k >> 2) & 1) << 1);
  else return vslot<CPK>(k, c);
}

// What all lanes hold alike, told to the compiler, which else keeps what comes of a
// division or a load in vector registers, and loops over it by masks.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ RowState uniform(const RowState& r) { return {uniform(r.len), uniform(r.n), uniform(r.p0)}; }

// ------------------------------------------------------- waves split keys
// Query columns of a work-group and where their parts go: with up to 8 (4) columns each
// is there SPREAD = 2 (4) times, and the matrix columns hold a part each of its query and
// of its probabilities, at no product more; else every part takes products of its own (of
// probabilities in bf16 there is one then).  Probabilities in two parts against one: 5
// rows of 30-60k keys 60 us for 60, outputs 0.0017 (their own rounding) off in the 2-norm
// for 0.0022; 512 rows on 1024 shared keys 71.6 us for 70.9.
template <bool F32, int SPREAD>
struct Fp4Parts {
  static constexpr int COLS = 16 / SPREAD;
  static constexpr int SETS = SPREAD > 1 ? 1 : F32 ? 3 : 2;   // products of a score
  static constexpr int PSETS = !F32 || SPREAD > 1 ? 1 : 3;    // of a value
};
// Part `part` of P parts of x, 0 beyond them.
template <int SPREAD, int P>
__device__ __forceinline__ __bf16 my_part(float x, int part) {
  __bf16 p[P];
  in_parts<P>(x, p);
  __bf16 r = p[0];
#pragma unroll
  for (int i = 1; i < SPREAD; ++i) r = part == i ? (i < P ? p[i < P ? i : 0] : (__bf16)0.f) : r;
  return r;
}

// At most 16 query columns: column x is token x / G of the row's, query head x % G of
// the KV head's G.  Work-group = (split, KV head, row), NW waves; every wave takes an
// even share of the 32-key blocks that hold visible keys and waits on no other until
// the merge.
//   S^T = K Q^T   (v_mfma_f32_16x16x32_bf16): a lane takes HD / 4 neighbouring
//         dimensions of a key, one load of codes and one scale, and converts them
//         in its registers; the contraction visits dimensions in that order.
//   O^T += V^T P^T (v_mfma_f32_16x16x32_bf16): a V block is converted on its way into
//         LDS (the wave's own) and its A operand comes from two transpose reads; the
//         contraction visits the keys in the order the lane holds their probabilities.
// A block's registers take over the next block as soon as they are read.  A block's
// 16-key halves lie in one page each; lane i holds the places and flags of block i of a
// run of 64.  The keys below common[row] are another pass's.  Keys that nobody sees are
// read where they lie (their scores are masked) and their values as zeros; a half
// without a page is read from page 0.
// Memory bounds long rows: 5 of 30-60k keys, 8 heads of 128 dimensions, 245 MB in 45 us
// (5.4 TB/s; a kernel that only reads reaches 5.5 to 6), the merge 5.4 us behind it.  512
// rows' own 41 to 460 keys 37 us (every wave has its own start and merge).
template <int HD, int NW, bool F32, int SPREAD>
__global__ void __launch_bounds__(64 * NW, HD == 128 && SPREAD == 1 ? 3 : 4)
fp4_wave_kernel(PagedAttnArgs a, const int32_t* __restrict__ common, int splits, int pre, int slots, float qscale) {
  typedef Fp4Parts<F32, SPREAD> PT;
  constexpr int COLS = PT::COLS, SETS = PT::SETS, PSETS = PT::PSETS;
  constexpr int KS = HD / 32, DT = HD / 16, CPK = HD / 8, VB = 32 * HD;
  // values: lanes of a key, loads of a block, words of a load
  constexpr int LPV = HD == 128 ? 4 : 2, NV = HD == 128 ? 2 : 1, WV = HD == 32 ? 2 : 4;
  constexpr int ROW = HD + 4;                       // floats of a column in the merge
  constexpr int BYTES = NW * 16 * ROW * 4 > NW * VB * 2 ? NW * 16 * ROW * 4 : NW * VB * 2;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[BYTES / 2];
  const int split = blockIdx.x, h = blockIdx.y, row = blockIdx.z;
  const RowState rs = uniform(row_state(a, row));
  if (rs.n == 0) return;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 15, fg = lane >> 4;
  const int g = a.hq / a.hkv;
  const int col = fr % COLS, part = fr / COLS;      // this lane's column, and which part of it
  const int t = col / g;
  const bool live = t < rs.n;
  const int end_c = rs.p0 + (live ? t : 0) + 1, lo_c = window_start(end_c - 1, a.window);
  const int lo_last = window_start(rs.len - 1, a.window);
  KeyBlocks kb;
  kb.set(common ? uniform(common[row]) : 0, a.sinks, window_start(rs.p0, a.window), rs.len);
  // (counts below 2^19, at most 256 shares)
  const int shares = splits * NW, me = split * NW + wave;
  const int i0 = uniform((uint32_t)(kb.count * me) / (uint32_t)shares);
  const int i1 = uniform((uint32_t)(kb.count * (me + 1)) / (uint32_t)shares);
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  const int mask = (1 << a.shift) - 1;
  bf16_t* vbuf = lds + wave * VB;

  // Blocks [base, base + 64) of this wave: lane i holds block base + i's places (the
  // pages' blocks of the KV head, in units of 16 bytes) and flags.
  enum {
    GONE0 = 1, GONE1 = 2,   // no page holds the half
    EDGE = 4,               // some column does not see some key
    PARTLY = 8              // nobody sees some key
  };
  int base = i0;
  uint32_t flags = 0;
  uint32_t place[2];   // (16 bytes of a layer's block: below 2^32 of them, 64 GB a layer, as the entry point checks)
  auto look_up = [&] {
    flags = EDGE | PARTLY | GONE0 | GONE1;
    place[0] = place[1] = 0;
    if (base + lane < i1) {
      const int k0 = kb.key0(base + lane);
      const int p0 = kb.any16(k0) ? tab[k0 >> a.shift] : -1;
      const int p1 = kb.any16(k0 + 16) ? tab[(k0 + 16) >> a.shift] : -1;
      const bool ok0 = (uint32_t)p0 < (uint32_t)a.n_pages, ok1 = (uint32_t)p1 < (uint32_t)a.n_pages;
      flags = (ok0 ? 0 : GONE0) | (ok1 ? 0 : GONE1);
      if (flags || !kb.all32(k0)) flags |= PARTLY;
      if (flags || k0 + 32 > rs.p0 + 1 || (k0 < lo_last && k0 + 32 > a.sinks)) flags |= EDGE;
      if (ok0) place[0] = (uint32_t)(fp4_block(p0, a.hkv, h, a.shift, HD) >> 4);
      if (ok1) place[1] = (uint32_t)(fp4_block(p1, a.hkv, h, a.shift, HD) >> 4);
    }
  };
  struct Block {
    uint32_t k[2][KS], v[NV][WV];
    uint8_t ks[2], vs[NV];
  } x;
  const uint32_t kcodes = fr * (HD / 2) + fg * (HD / 8), kscale = fr * KS + fg * (HD / 4) / 32;
  // (the place of a half of block b, and its first slot)
  auto half_at = [&](int b, int u) { return (uint64_t)(uint32_t)__builtin_amdgcn_readlane(place[u], b) << 4; };
  auto half_slot = [&](int b, int u) { return (kb.key0(base + b) + 16 * u) & mask; };
  auto load_keys = [&](int b) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t* src = (const uint8_t*)a.kpool + half_at(b, u);
      const int slot = half_slot(b, u);
      load_words<KS>(src + fp4_codes(slot, HD) + kcodes, x.k[u]);
      x.ks[u] = (src + fp4_scales(slot, a.shift, HD))[kscale];
    }
  };
  auto load_values = [&](int b) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int kk = i * (64 / LPV) + lane / LPV, c = lane % LPV;
      uint64_t from = half_at(b, NV == 2 ? i : 0);
      int s = half_slot(b, NV == 2 ? i : 0);
      if (NV == 1) {
        const uint64_t from1 = half_at(b, 1);
        const int s1 = half_slot(b, 1);
        if (lane >= 32) {
          from = from1;
          s = s1;
        }
      }
      const uint8_t* src = (const uint8_t*)a.vpool + from;
      load_words<WV>(src + fp4_codes(s, HD) + ((kk & 15) * (HD / 2) + c * 4 * WV), x.v[i]);
      x.vs[i] = (src + fp4_scales(s, a.shift, HD))[(kk & 15) * KS + c * WV / 4];
    }
  };

  // The first block's loads go out before the queries are read.
  auto start = [&] {
    look_up();
    load_keys(0);
    load_values(0);
  };
  if (i0 < i1) start();

  // Q^T fragments (B operand): lane holds Q[its column][HD / 4 fg + 8 s .. + 8]
  bf16x8 qf[SETS][KS];
  {
    const float* qr = a.q + (((int64_t)row * a.lr + (live ? t : 0)) * a.hq + h * g + (live ? col - t * g : 0)) * HD;
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      const float4 x4 = *reinterpret_cast<const float4*>(qr + HD / 4 * fg + 8 * st);
      const float4 y4 = *reinterpret_cast<const float4*>(qr + HD / 4 * fg + 8 * st + 4);
      const float v[8] = {x4.x, x4.y, x4.z, x4.w, y4.x, y4.y, y4.z, y4.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (SPREAD > 1) {
          qf[0][st][e] = my_part<SPREAD, F32 ? 3 : 2>(v[e] * qscale, part);
        } else {
          __bf16 p[SETS];
          in_parts<SETS>(v[e] * qscale, p);
#pragma unroll
          for (int i = 0; i < SETS; ++i) qf[i][st][e] = p[i];
        }
      }
    }
  }

  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  // from the lowest finite score: while a column has seen only -inf its
  // probabilities are exp2(-inf) = 0, where -inf - -inf would be NaN
  float m = -FLT_MAX, l = 0.f;
  // transpose-read addresses: lane names 4 dims (dt 16 + 4 (fr & 3) ..) of key
  // 4 fg + (fr >> 2), and of the key 16 on (16 rows on, same slots)
  // (slots differ from dt to dt by an exclusive or: they stay within aligned rows)
  uint32_t vaddr;
  {
    const int kr0 = 4 * fg + (fr >> 2);
    vaddr = lds_addr(vbuf + kr0 * HD + 8 * wslot<CPK>(kr0, (fr & 3) >> 1) + 4 * (fr & 1));
  }
  // Block b; its registers take over the next block's as soon as they are read.
  auto compute = [&](int b, bool more) {
    const int k0 = kb.key0(base + b);
    const uint32_t f = __builtin_amdgcn_readlane(flags, b);
    float sv[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      f32x4 st = f32x4{0.f, 0.f, 0.f, 0.f};
      const float scale = fp4_scale(x.ks[u]);
#pragma unroll
      for (int s2 = 0; s2 < KS; ++s2) {
        const bf16x8 k = fp4_to_bf16(x.k[u][s2], scale);
#pragma unroll
        for (int i = 0; i < SETS; ++i) st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[i][s2], st, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sv[4 * u + i] = parts_sum<SPREAD>(st[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_keys(b + 1);
    __builtin_amdgcn_sched_barrier(0);
    // values into LDS, zeros for those that nobody sees
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int kk = i * (64 / LPV) + lane / LPV, c = lane % LPV;
      if (f & PARTLY) {
        asm volatile("");   // (a branch)
        if (!kb.has(k0 + kk) || (f & (kk < 16 ? GONE0 : GONE1))) {
#pragma unroll
          for (int w = 0; w < WV; ++w) x.v[i][w] = 0;
          x.vs[i] = 127;
        }
      }
      const float scale = fp4_scale(x.vs[i]);
      char* dst = reinterpret_cast<char*>(vbuf + kk * HD);
      const uint32_t first = 16u * wslot<CPK>(kk, c * WV);
#pragma unroll
      for (int w = 0; w < WV; ++w) *reinterpret_cast<bf16x8*>(dst + (first ^ (16u * w))) = fp4_to_bf16(x.v[i][w], scale);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_values(b + 1);
    __builtin_amdgcn_sched_barrier(0);
    if (f & EDGE) {   // (uniform)
      asm volatile("");
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = k0 + 4 * fg + (i & 3) + 16 * (i >> 2);
        const bool sees = (j < end_c) & ((j >= lo_c) | (j < a.sinks)) & !(f & (i < 4 ? GONE0 : GONE1));
        if (!sees) sv[i] = -INFINITY;
      }
    }
    // Probabilities are relative to a maximum up to 2^kStale out of date; the lanes
    // of a column share it.
    float mt = sv[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mt = fmaxf(mt, sv[i]);
    if (__any(mt > m + kStale)) {
      mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
      mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
      const float mn = fmaxf(m, mt);
      const float corr = __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= corr;
      m = mn;
    }
    bf16x8 pf[PSETS];
    float ps = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float pv = __builtin_amdgcn_exp2f(sv[i] - m);
      ps += pv;
      if constexpr (SPREAD > 1) {
        const float first = __uint_as_float(__float_as_uint(pv) & 0xFFFF0000u);   // (cut, for one instruction)
        if constexpr (F32) pf[0][i] = my_part<SPREAD, 3>(pv, part);
        else pf[0][i] = (__bf16)(part == 0 ? first : pv - first);
      } else {
        __bf16 p[PSETS];
        in_parts<PSETS>(pv, p);
#pragma unroll
        for (int j = 0; j < PSETS; ++j) pf[j][i] = p[j];
      }
    }
    l += ps;
    constexpr int N = DT < 4 ? DT : 4;
#pragma unroll
    for (int e0 = 0; e0 < DT; e0 += N) {
      uint32_t va[N];
#pragma unroll
      for (int i = 0; i < N; ++i) va[i] = vaddr ^ (32u * (e0 + i));
      i16x4 lo[N], hi[N];
      lds_read_tr16_pairs<N, 0, 16 * HD * 2>(va, lo, hi);
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < PSETS; ++j)
          o[e0 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tr16_pair(lo[i], hi[i]), pf[j], o[e0 + i], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  while (base < i1) {
    const int nb = imin(64, i1 - base);
    for (int b = 0; b < nb; ++b) compute(b, b + 1 < nb);
    base += 64;
    if (base < i1) start();   // (a run of 64 blocks drains: one round trip in 2048 keys)
  }

  // join the waves: per column the unnormalised output, (max, sum) behind it
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if constexpr (F32 && SPREAD > 1) {   // the outputs of the probabilities' parts
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[dt][e] = parts_sum<SPREAD>(o[dt][e]);
  }
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
      float o8[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
      if constexpr (!F32 && SPREAD > 1) {   // (the outputs of the probabilities' second parts)
        const f32x4 u2 = *reinterpret_cast<const f32x4*>(ws + COLS * ROW + d), v2 = *reinterpret_cast<const f32x4*>(ws + COLS * ROW + d + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o8[e] += u2[e];
          o8[4 + e] += v2[e];
        }
      }
      add(ws[HD], ws[HD + 1], o8);
    }
    if (splits == 1) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      if constexpr (F32) {
        float4* dst = reinterpret_cast<float4*>((float*)a.out + th * HD + d);
        dst[0] = make_float4(A[0] * inv, A[1] * inv, A[2] * inv, A[3] * inv);
        dst[1] = make_float4(A[4] * inv, A[5] * inv, A[6] * inv, A[7] * inv);
      } else {
        bf16x8 r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (__bf16)(A[e] * inv);
        *reinterpret_cast<bf16x8*>((bf16_t*)a.out + th * HD + d) = r;
      }
    } else {
      float4* dst = reinterpret_cast<float4*>(pt.o(th, pre + split, HD) + d);
      dst[0] = make_float4(A[0], A[1], A[2], A[3]);
      dst[1] = make_float4(A[4], A[5], A[6], A[7]);
      if (d == 0) *reinterpret_cast<float2*>(pt.ml(th, pre + split, HD)) = make_float2(M, L);
    }
  }
}

// -------------------------------------------------------- query tiles
// v_mfma_f32_32x32x16_bf16, 128 query columns a work-group, 32 a wave; column x is
// token x / G, query head x % G of the KV head's G.
//   PRE = false: the tokens of one row, over all its keys.
//   PRE = true:  the tokens of all rows, over row 0's leading keys; a column
//                sees those its row has in common (`common`).
//   S^T = K Q^T   (keys x columns): lane l holds, of every 32 keys, the 16 with
//                 (key / 4) % 2 = l / 32 for column l % 32.
//   O^T += V^T P^T: the contraction visits a 16-key chunk in the order the lane
//                 holds it, so the B operand is the lane's own probabilities;
//                 the A operand comes from V by two LDS transpose reads.
// The 32-key blocks that hold a visible key pass through registers, two blocks
// ahead, and are converted on their way into one of two LDS stages (every thread 8 or
// 16 dimensions of a key and of a value, rows XOR-swizzled in chunks of 16 bytes); one
// barrier a block.
//   CODES (bf16 outputs of prompts): keys are not converted.  S^T is v_mfma_scale_f32_
//                 32x32x64 on their codes and scale bytes, times queries in three parts of
//                 6 bits (e2m3), each with a scale for 32 dimensions: at most 1 / 15360
//                 of the largest of these is left.  The products are exact, and a sum of
//                 64 of them with scales of any size is off by 2^-21 of the largest at
//                 most (measured).  Scores from queries in one bf16 took 5 % longer at
//                 head_dim 128 and 10 % less at 64, and were half as precise; in two 66
//                 and 11 % longer.
//                 The maximum is taken off by one more product, not by vector work
//                 (200 tokens on 60k keys 229 -> 209 us).
// 6011 tokens, hd 128: 304 to 318 us (930 to 975 TFLOP/s); 53 chunks of up to 333 tokens, hd
// 64: 129 to 134 us.  What bounds it: a block of 32 x 32 scores is 256 clocks of exponentials
// and some 250 of other vector work a wave, beside 480 (hd 128) or 256 of matrix work, and
// the waves of a SIMD hardly overlap them (matrix instructions busy 41 and 31 % of the
// clocks, vector ones 43 and 66 %).  The next block's scores beneath this one's exponentials, or
// two blocks a barrier: the same time.  Lane i keeps the place and the mask flags of block i of a
// run of 64.
// The output is rescaled only when a maximum has moved by more than
// kStale.
constexpr int kTileCols = 128;

template <int HD, bool PRE, bool F32>
__global__ void __launch_bounds__(256, HD == 128 || PRE || F32 ? 2 : 4)
fp4_tile_kernel(PagedAttnArgs a, const int32_t* __restrict__ common, int splits, int slots, float qscale) {
  constexpr int KT = 32, NW = 4;
  constexpr int KS = HD / 16, DT = HD / 32, CPK = HD / 8;
  constexpr bool CODES = !F32 && !PRE;         // scores from the codes themselves
  constexpr int PP = F32 ? 3 : 1, QP = PRE && !F32 ? 2 : 3;   // parts of a probability, of a query
  constexpr int GS = HD / 32, LJ = (HD + 63) / 64;   // groups of a key, products over these
  constexpr int TILE = KT * HD;                // bf16 elements of a K (or V) block
  constexpr int TPK = HD == 32 ? 4 : 8;        // threads that bring a key
  constexpr int WPT = CPK / TPK;               // chunks (words of codes) of each
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2 * 2 * TILE];
  __shared__ __attribute__((aligned(16))) uint8_t raw[2][CODES ? KT * 16 * GS : 16], raw_scale[2][CODES ? KT * 4 : 4];
  __shared__ int bounds[NW][2];
  // a 1-D grid dealt round-robin to the 8 XCDs: each takes consecutive logical
  // blocks, the query tiles of one (row, KV head, split) fastest, the last and
  // longest first, so that those reading the same keys share one L2; the KV heads
  // slowest, so that every XCD has its part of all rows, long and short ones, and
  // one copy of the pages that rows share
  const int g = a.hq / a.hkv;
  const int X = (PRE ? a.rows * a.lr : a.lr) * g;                 // columns
  const int ngq = (X + kTileCols - 1) / kTileCols, total = ngq * splits * a.hkv * (PRE ? 1 : a.rows);
  const int per_xcd = (total + 7) / 8;
  const int pid = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (pid >= total) return;
  const int nrow = PRE ? 1 : a.rows;
  const int qg = uniform(ngq - 1 - pid % ngq), split = uniform(pid / ngq % splits);
  const int row = uniform(pid / (ngq * splits) % nrow), h = uniform(pid / (ngq * splits * nrow));
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int x0 = qg * kTileCols, xw = x0 + 32 * wave;             // first column, of the wave too
  const int token0 = PRE ? 0 : row * a.lr;
  const RowState rs = uniform(row_state(a, row));
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
    all_end = rs.p0 + uniform(xw / g) + 1;
    wend = any ? rs.p0 + uniform(last / g) + 1 : 0;
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
    kb.set(0, a.sinks, uniform(imin(lo, end)), uniform(end));
  } else {
    const int last = imin(x0 + kTileCols - 1, rs.n * g - 1);
    kb.set(0, a.sinks, window_start(rs.p0 + uniform(x0 / g), a.window), rs.p0 + uniform(last / g) + 1);
  }
  // (counts below 2^19, at most 64 splits)
  const int i0 = uniform((uint32_t)(kb.count * split) / (uint32_t)splits);
  const int i1 = uniform((uint32_t)(kb.count * (split + 1)) / (uint32_t)splits);
  const int ntile = i1 - i0;

  // Blocks [64 c, 64 c + 64) of this split: lane i holds the flags of block 64 c + i and
  // the byte offset of the half's slots that this wave brings.
  enum {
    GONE0 = 1, GONE1 = 2,   // no page holds the half
    EDGE = 4,               // some column of the wave does not see every key
    PAST = 8,               // no column of the wave sees a key
    PARTLY = 16             // no column of the work-group sees some key
  };
  const int key = threadIdx.x / TPK, chunk = threadIdx.x % TPK * WPT;   // what this thread brings
  const bool brings = key < KT;
  const int half = wave * (64 / TPK) >> 4 & 1;                          // (uniform) of the block
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  const int mask = (1 << a.shift) - 1;
  uint32_t flags = 0;
  uint2 at = make_uint2(0, 0);   // the page's block of the KV head
  int entry[2];                  // what the table says of block first + lane's halves
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
      const int page = (uint32_t)entry[u] < (uint32_t)a.n_pages ? entry[u] : -1;
      if (page < 0) flags |= EDGE | PARTLY | (u ? GONE1 : GONE0);
      if (u == half) {
        const int64_t off = fp4_block(imax(page, 0), a.hkv, h, a.shift, HD);   // (page 0 where there is none)
        at = make_uint2((uint32_t)off, (uint32_t)(off >> 32));
      }
    }
  };
  // The table first, so that the first keys do not wait behind the queries.
  read_table(0);
  __builtin_amdgcn_sched_barrier(0);

  // The wave's 32 queries (clamped rows; results of columns that are no query are
  // dropped).  For CODES a lane takes dimensions 64 j + 32 fh .. of its column (32
  // dimensions: the lower half), else 16 bytes along whole rows.
  constexpr int LPR = HD / 4, RPQ = 64 / LPR, NQ = 32 / RPQ;   // lanes per query, queries per load, loads
  float4 qv[CODES ? 8 * LJ : NQ];
  if constexpr (CODES) {
    const int x = imin(xw + fr, X - 1), tok = x / g;
    const float4* src = reinterpret_cast<const float4*>(a.q + ((int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g)) * HD);
#pragma unroll
    for (int i = 0; i < 8 * LJ; ++i) qv[i] = src[i % 8 + (HD == 32 ? 0 : 16 * (i / 8) + 8 * fh)];
  } else {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int x = imin(xw + RPQ * i + lane / LPR, X - 1), tok = x / g;
      qv[i] = reinterpret_cast<const float4*>(
          a.q + ((int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g)) * HD)[lane % LPR];
    }
  }
  __builtin_amdgcn_sched_barrier(0);

  struct Codes {
    uint32_t k[WPT], v[WPT], f;
    uint8_t ks, vs;
  };
  auto load = [&](int tile, Codes& c) {
    if ((tile & 63) == 0) {
      if (tile > 0) read_table(tile);
      look_up(tile);
    }
    const int from = tile & 63;
    c.f = __builtin_amdgcn_readlane(flags, from);
    const int64_t off =
        (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(at.y, from) << 32 | (uint32_t)__builtin_amdgcn_readlane(at.x, from));
    const int slot = (kb.key0(i0 + tile) + 16 * half) & mask;
    if (HD == 32 && !brings) return;
    const int codes = fp4_codes(slot, HD), scales = fp4_scales(slot, a.shift, HD);
    const uint32_t own = (key & 15) * (HD / 2) + chunk * 4, owns = (key & 15) * (HD / 32) + chunk / 4;
    load_words<WPT>((const uint8_t*)a.kpool + off + codes + own, c.k);
    load_words<WPT>((const uint8_t*)a.vpool + off + codes + own, c.v);
    c.ks = ((const uint8_t*)a.kpool + off + scales)[owns];
    c.vs = ((const uint8_t*)a.vpool + off + scales)[owns];
  };
  // 16 bytes of codes of key k in a stage: 16 lanes' reads meet in no bank
  auto raw_slot = [](int k, int group) { return k * GS + (group ^ (HD == 128 ? (k >> 2) & 3 : HD == 64 ? (k >> 3) & 1 : 0)); };
  auto vswz = [](int k) { return HD == 128 ? (k & 3) << 2 : HD == 64 ? ((k >> 1) & 1) << 2 : 0; };
  auto stage = [&](int tile, Codes& c, int buf) {
    if (HD == 32 && !brings) return;
    if ((c.f & PARTLY) && (!kb.has(kb.key0(i0 + tile) + key) || (c.f & (half ? GONE1 : GONE0)))) {
#pragma unroll
      for (int w = 0; w < WPT; ++w) c.v[w] = 0;
      c.vs = 127;
    }
    bf16_t* kd = lds + buf * 2 * TILE + key * HD;
    const float ks = fp4_scale(c.ks), vs = fp4_scale(c.vs);
#pragma unroll
    for (int w = 0; w < WPT; ++w) {
      if constexpr (!CODES) *reinterpret_cast<bf16x8*>(kd + 8 * ((chunk + w) ^ (key & (CPK - 1)))) = fp4_to_bf16(c.k[w], ks);
      *reinterpret_cast<bf16x8*>(kd + TILE + 8 * ((chunk + w) ^ vswz(key))) = fp4_to_bf16(c.v[w], vs);
    }
    if constexpr (CODES) {
      uint32_t* dst = reinterpret_cast<uint32_t*>(raw[buf] + 16 * raw_slot(key, chunk / 4)) + chunk % 4;
#pragma unroll
      for (int w = 0; w < WPT; ++w) dst[w] = c.k[w];
      if (chunk % 4 == 0) raw_scale[buf][4 * key + chunk / 4] = c.ks;
    }
  };

  // the queries' parts: of 6 bits, groups of 32 dimensions with a scale byte (part p's of
  // product j: byte 2 p + j of the two words), or bf16
  u32x6 q6[CODES ? QP : 1][LJ];
  uint32_t q6_scale[2] = {0, 0};
  bf16x8 qf[CODES ? 1 : QP][KS];
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
  // never rescale the others
  // CODES: scores come out of the products less the maximum so far (0 at first), which
  // enters as three bf16 parts (all 24 bits) times ones; `limit` is what they may reach
  // until it moves: anything finite before a column's first score
  float m = CODES ? 0.f : live ? -FLT_MAX : INFINITY, l = 0.f;
  float limit = live ? -FLT_MAX : INFINITY;
  bf16x8 less = {}, ones3 = {};
  ones3[0] = ones3[1] = ones3[2] = (__bf16)(fh == 0 ? 1.f : 0.f);

  auto frag = [&](const bf16_t* base, int s) {
    return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(base) + (kbase ^ (32u * s)));
  };
  auto step = [&](auto bufc, int tile, uint32_t f) {
    constexpr int ST = decltype(bufc)::value;
    constexpr int VB = ST * 2 * TILE * 2;   // bytes from vbase
    f32x16 sc;
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = 0.f;
    if constexpr (CODES) {
      // key fr's codes, and the scale bytes from the lane's first group on (32 dimensions:
      // the queries are 0 in the other half, where the codes stand in for themselves)
      const uint32_t ks = *reinterpret_cast<const uint32_t*>(raw_scale[ST] + 4 * fr) >> (HD == 32 ? 0 : 8 * fh);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones3, less, sc, 0, 0, 0);
      i32x8 k[LJ];
#pragma unroll
      for (int j = 0; j < LJ; ++j) {
        const uint4 v = *reinterpret_cast<const uint4*>(raw[ST] + 16 * raw_slot(fr, HD == 32 ? 0 : 2 * j + fh));
        k[j] = i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
      }
      auto part = [&](auto p) {
        constexpr int P = decltype(p)::value;
        auto q = [&](int j) {
          const u32x6 w = q6[P][j];
          return i32x8{(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0};
        };
        sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k[0], q(0), sc, 4, 2, 0, ks, 2 * (P & 1), q6_scale[P / 2]);
        if constexpr (LJ == 2)
          sc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k[LJ - 1], q(LJ - 1), sc, 4, 2, 2, ks, 2 * (P & 1) + 1, q6_scale[P / 2]);
      };
      part(std::integral_constant<int, 2>{});   // (the least first)
      part(std::integral_constant<int, 1>{});
      part(std::integral_constant<int, 0>{});
    } else {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bf16x8 k = frag(lds + ST * 2 * TILE, s);
#pragma unroll
        for (int i = 0; i < QP; ++i) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[i][s], sc, 0, 0, 0);
      }
    }
    if (f & EDGE) {                            // (uniform)
      asm volatile("");                        // (a branch, not selects on every block)
      // bit j: this lane's key j of the block (of the 32 from 4 fh on) is seen
      const int k4 = kb.key0(i0 + tile) + 4 * fh;
      auto below = [](int n) { return n >= 32 ? ~0u : (1u << imax(n, 0)) - 1u; };
      uint32_t see = below(end_c - k4) & (~below(lo_c - k4) | below(a.sinks - k4));
      if (f & GONE0) see &= 0xFFFF0000u;
      if (f & GONE1) see &= 0x0000FFFFu;
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e] = (int)(see << (31 - 8 * (e >> 2) - (e & 3))) < 0 ? sc[e] : -INFINITY;
    }
    float mt = sc[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mt = fmaxf(mt, sc[e]);
    mt = fmaxf(mt, other_half(mt));
    if (CODES ? __any(mt > limit) : __any(mt > m + kStale)) {
      const bool moves = mt > limit;
      const float mn = CODES ? (moves ? m + mt : m) : fmaxf(m, mt);
      const float corr = CODES && limit != kStale ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= corr;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] *= corr;
      if constexpr (CODES) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] -= mn - m;
        __bf16 p[3];
        in_parts<3>(fh == 0 ? -mn : 0.f, p);
        less[0] = p[0]; less[1] = p[1]; less[2] = p[2];
        if (moves) limit = kStale;
      }
      m = mn;
    }
    uint32_t va[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) va[dt] = vbase ^ (64u * dt);
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
    bf16x8 pf[2][PP];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float pv = __builtin_amdgcn_exp2f(CODES ? sc[8 * c + e] : sc[8 * c + e] - m);
        __bf16 p[PP];
        in_parts<PP>(pv, p);
#pragma unroll
        for (int j = 0; j < PP; ++j) pf[c][j][e] = p[j];
        if constexpr (F32) l += pv;
      }
      if constexpr (!F32) {   // (of the rounded ones, as the product has them)
#pragma unroll
        for (int e = 0; e < 8; e += 2) l = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[c][0][e], pf[c][0][e + 1]}, ones, l, false);
      }
    }
    i16x4 lo[DT], hi[DT];
    lds_read_tr16_pairs<DT, VB, VB + 8 * HD * 2>(va, lo, hi);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < PP; ++j)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr16_pair(lo[dt], hi[dt]), pf[0][j], o[dt], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    lds_read_tr16_pairs<DT, VB + 16 * HD * 2, VB + 24 * HD * 2>(va, lo, hi);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < PP; ++j)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr16_pair(lo[dt], hi[dt]), pf[1][j], o[dt], 0, 0, 0);
  };
  bf16_t* const slice = lds + wave * 32 * HD;
  if (ntile > 0) {
    Codes c0, c1;
    load(0, c0);
    if (ntile > 1) load(1, c1);
    if constexpr (CODES) {
#pragma unroll
      for (int j = 0; j < LJ; ++j) {
        float x[32], top = 0.f;
        bool fine = true;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 v = qv[8 * j + i];
          x[4 * i] = v.x * qscale; x[4 * i + 1] = v.y * qscale; x[4 * i + 2] = v.z * qscale; x[4 * i + 3] = v.w * qscale;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          if (HD == 32 && fh) x[e] = 0.f;
          fine &= fabsf(x[e]) <= FLT_MAX;
          top = fmaxf(top, fabsf(x[e]));
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          // the least scale with the largest at most 7.5 of it, the type's end
          const int byte = imax(1, (int)((__float_as_uint(top) + 0xFFFFFu) >> 23) - 2);
          const float scale = __uint_as_float((uint32_t)byte << 23);
          f32x16 even, odd;   // (whose results alternate)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            even[e] = x[2 * e];
            odd[e] = x[2 * e + 1];
          }
          q6[p][j] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, scale);
          // It writes while it still reads, which the compiler does not know: the sources stay
          // alive until it is done, or the result may be put into them.  (At head_dim 32 the third
          // part went to the third register of `even`: scores of 250 were up to 0.1 off.)
          asm volatile("" : "+v"(q6[p][j]) : "v"(even), "v"(odd), "v"(scale));
          q6_scale[p / 2] |= (uint32_t)(fine ? byte : 255) << (8 * (2 * (p & 1) + j));   // (255: NaN)
          if (p + 1 == QP) break;
          f32x32 y = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q6[p][j], scale);
          asm volatile("" : "+v"(y) : "v"(q6[p][j]), "v"(scale));   // (likewise)
          top = 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            x[e] -= y[e];
            top = fmaxf(top, fabsf(x[e]));
          }
        }
      }
    } else {
      // (through the wave's own slice: its LDS operations are in order)
#pragma unroll
      for (int p = 0; p < QP; ++p) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
          const int r = RPQ * i + lane / LPR, c4 = lane % LPR;
          const float x[4] = {qv[i].x * qscale, qv[i].y * qscale, qv[i].z * qscale, qv[i].w * qscale};
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            __bf16 part[QP];
            in_parts<QP>(x[e], part);
            v[e] = part[p];
          }
          *reinterpret_cast<bf16x4*>(slice + r * HD + 8 * ((c4 >> 1) ^ (r & (CPK - 1))) + 4 * (c4 & 1)) = v;
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[p][s] = frag(slice, s);
      }
    }
    lds_barrier();   // every wave's queries read
    // Block t is staged, its registers take block t + 2, and behind the barrier all
    // waves compute it; who stages t + 1 next has passed this barrier, so nobody
    // reads the stage of t - 1 any more.
    auto one = [&](auto bufc, int tile, Codes& c) {
      constexpr int ST = decltype(bufc)::value;
      const uint32_t f = c.f;
      stage(tile, c, ST);
      if (tile + 2 < ntile) load(tile + 2, c);
      __builtin_amdgcn_sched_barrier(0);
      lds_barrier();
      if (!(f & PAST)) step(bufc, tile, f);
    };
    for (int tile = 0; tile < ntile; tile += 2) {
      one(std::integral_constant<int, 0>{}, tile, c0);
      if (tile + 1 < ntile) one(std::integral_constant<int, 1>{}, tile + 1, c1);
    }
  }
  l += other_half(l);
  if (PRE || slots > 1) {
    if (!live) return;
    if (CODES && limit != kStale) m = -FLT_MAX;   // (nothing seen: below every other part's)
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
  if constexpr (F32) {
    if (!live) return;
    const int x = xw + fr, tok = x / g;
    float* po = (float*)a.out + ((int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g)) * HD;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(po + 32 * dt + 8 * q4 + 4 * fh) =
            make_float4(o[dt][4 * q4] * inv, o[dt][4 * q4 + 1] * inv, o[dt][4 * q4 + 2] * inv, o[dt][4 * q4 + 3] * inv);
    return;
  }
  lds_barrier();   // every wave is done with the blocks
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
  constexpr int RPI = 64 / CPK;   // rows of a store
#pragma unroll
  for (int i = 0; i < 32 / RPI; ++i) {
    const int r = RPI * i + lane / CPK, c = lane % CPK, x = xw + r, tok = x / g;
    const uint4 v = *reinterpret_cast<const uint4*>(slice + r * HD + 8 * (c ^ (r & (CPK - 1))));
    if (x >= rs.n * g) continue;
    *reinterpret_cast<uint4*>((bf16_t*)a.out + ((int64_t)(token0 + tok) * a.hq + h * g + (x - tok * g)) * HD + 8 * c) = v;
  }
}

// ------------------------------------------------------------------ plan
struct Fp4Plan {
  bool tile;
  int nw;       // waves of a work-group (fp4_wave_kernel)
  int splits;   // work-groups that share a row's keys
  int pre;      // splits of the shared keys' own pass (0: none)
  int slots() const { return pre + (splits > 1 ? splits : 0); }
};

// How often fp4_wave_kernel has a column in its 16.
static int wave_spread(const PagedAttnArgs& a) {
  const int cols = a.lr * (a.hq / a.hkv), times = a.dtype == SR_BF16 ? 2 : 4;
  return cols * times <= 16 ? times : 1;
}

// Single tokens: as many waves as are resident at once (3 or 4 a SIMD, a wave having
// four blocks of keys at least), no more, since what does not fit waits for a whole
// round.  256 rows of 612 keys, hd 128: 2048 waves of several work-groups a row 36 us,
// 4096 31 us, 8192 35 us; 5 rows of 30-60k: 59.5, 60, 64 us; 200 rows of 700 in fp32,
// two blocks a wave: 16.5 us, four: 12.9 us.
constexpr int kSimds = 1024;
// Tiles: two work-groups a CU (20 tokens on 60k keys: one 65 us, two 51 us); for the
// shared keys one, since another split is another set of partials to write and read
// (512 rows, 1024 shared keys: two 73 us, one 71 us, half of the CUs 82 us).
constexpr int kTileTarget = 512, kPreTarget = 256;
// Bytes of the shared keys and values as often as rows read them, from which they get a
// pass of their own (1024 shared and 100-300 own keys of 8 heads of 128 dimensions: 128
// rows 34 us with it, 30 without, 192 rows 36 and 43, 512 rows 71 and 94; 512 rows with
// 256 shared 48 and 42, with 512 51 and 56).
constexpr int64_t kShareBytes = 190 << 20;
constexpr int kMaxSplits = 64;

static Fp4Plan fp4_plan(const PagedAttnArgs& a) {
  Fp4Plan p{false, 1, 1, 0};
  const int g = a.hq / a.hkv;
  int64_t keys = planned_keys(a);
  auto tile_splits = [&](int64_t groups, int64_t blocks, int target) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({target / groups, blocks / 8, kMaxSplits}));
  };
  if (a.lr * g <= 16) {
    const bool far = a.window > 0 && a.max_len > a.window;   // (windows have left key 0)
    const int64_t shared = far ? 0 : std::min<int64_t>(a.shared, keys - a.lr);
    if (shared > 0 && (int64_t)a.rows * shared * a.hkv * a.hd * 17 / 16 >= kShareBytes) {
      const int64_t tiles = ((int64_t)a.rows * a.lr * g + kTileCols - 1) / kTileCols;
      p.pre = tile_splits(tiles * a.hkv, shared / 32, kPreTarget);
      keys -= shared;
    }
    const int64_t pairs = (int64_t)a.rows * a.hkv, blocks = (keys + 31) / 32;
    const int resident = a.hd == 128 && wave_spread(a) == 1 ? 3 : 4;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(resident * kSimds / pairs, blocks / 4));
    p.nw = want >= 4 ? 4 : want >= 2 ? 2 : 1;
    p.splits = (int)std::min<int64_t>(kMaxSplits, want / p.nw);
  } else {
    p.tile = true;
    const int64_t tiles = ((int64_t)a.lr * g + kTileCols - 1) / kTileCols;
    p.splits = tile_splits(tiles * a.hkv * a.rows, keys / 32, kTileTarget);
  }
  return p;
}

// Scratch: the partial slots, then common[rows].
static size_t partial_floats(const PagedAttnArgs& a, const Fp4Plan& p) {
  return (size_t)a.rows * a.lr * a.hq * p.slots() * (a.hd + 2);
}
size_t paged_attn_fp4_scratch(const PagedAttnArgs& a) {
  if (a.rows <= 0 || a.lr <= 0) return 0;
  const Fp4Plan p = fp4_plan(a);
  return partial_floats(a, p) + (p.pre ? a.rows : 0);
}

template <int HD, bool PRE, bool F32>
static void launch_tile(const PagedAttnArgs& a, const int32_t* common, int splits, int slots, hipStream_t s) {
  const float qscale = kLog2e / sqrtf((float)HD);
  const int64_t cols = (int64_t)(PRE ? a.rows : 1) * a.lr * (a.hq / a.hkv);
  const int64_t total = (cols + kTileCols - 1) / kTileCols * splits * a.hkv * (PRE ? 1 : a.rows);
  SR_REQUIRE(total <= kMaxGroups - 8, SR_ERR_UNSUPPORTED, "attention grid too large");
  SR_LAUNCH((fp4_tile_kernel<HD, PRE, F32>), dim3((unsigned)(8 * ((total + 7) / 8))), dim3(256), 0, s, a, common,
            splits, slots, qscale);
  SR_CHECK_LAUNCH();
}

template <int HD, bool F32>
static void launch_fp4(const PagedAttnArgs& a, hipStream_t s) {
  typedef std::conditional_t<F32, float, bf16_t> T;
  const Fp4Plan p = fp4_plan(a);
  if (p.tile) {
    launch_tile<HD, false, F32>(a, nullptr, p.splits, p.slots(), s);
  } else {
    const float qscale = kLog2e / sqrtf((float)HD);
    int32_t* common = nullptr;
    if (p.pre) {
      common = reinterpret_cast<int32_t*>(a.part + partial_floats(a, p));
      SR_LAUNCH(paged_common_kernel, dim3((a.rows + 3) / 4), dim3(256), 0, s, a, common);
      SR_CHECK_LAUNCH();
      launch_tile<HD, true, F32>(a, common, p.pre, p.slots(), s);
    }
    const dim3 grid(p.splits, a.hkv, a.rows);
#define SR_FP4_WAVE2(NW, SPREAD)                                                                                    \
  SR_LAUNCH((fp4_wave_kernel<HD, NW, F32, SPREAD>), grid, dim3(64 * NW), 0, s, a, (const int32_t*)common, p.splits, \
            p.pre, p.slots(), qscale)
#define SR_FP4_WAVE(NW)                                         \
  do {                                                          \
    if (wave_spread(a) > 1) SR_FP4_WAVE2(NW, (F32 ? 4 : 2));    \
    else SR_FP4_WAVE2(NW, 1);                                   \
  } while (0)
    switch (p.nw) {
      case 4: SR_FP4_WAVE(4); break;
      case 2: SR_FP4_WAVE(2); break;
      default: SR_FP4_WAVE(1); break;
    }
#undef SR_FP4_WAVE
#undef SR_FP4_WAVE2
    SR_CHECK_LAUNCH();
  }
  if (p.splits > 1) launch_merge<T, HD>(a, p.slots(), s);
}

template <int HD>
static void by_type(const PagedAttnArgs& a, hipStream_t s) {
  if (a.dtype == SR_BF16) launch_fp4<HD, false>(a, s);
  else launch_fp4<HD, true>(a, s);
}

void paged_attn_fp4(const PagedAttnArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.lr <= 0) return;
  switch (a.hd) {
    case 32: by_type<32>(a, s); break;
    case 64: by_type<64>(a, s); break;
    default: by_type<128>(a, s); break;
  }
}

}  // namespace sr
