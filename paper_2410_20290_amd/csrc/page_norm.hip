// Head norms, rotation and append to a cache of fp32, bf16 or 4 bits; and the
// tokens of the pages read back.
#include <algorithm>

#include "common.h"
#include "fp4.h"
#include "kernels.h"
#include "paged.h"
#include "specrej_serving.h"

namespace sr {

__device__ __forceinline__ bool is_page(int pg, int n_pages) { return (uint32_t)pg < (uint32_t)n_pages; }

// A double as a cache element, rounded once: to bf16 by way of the fp32 below
// it whose last bit says that something was cut off.
template <typename T> __device__ __forceinline__ T round_once(double v);
template <> __device__ __forceinline__ float round_once<float>(double v) { return (float)v; }
template <> __device__ __forceinline__ bf16_t round_once<bf16_t>(double v) {
  const float f = __double2float_rz(v);
  return f32_to_bf16(__uint_as_float(__float_as_uint(f) | ((double)f != v ? 1u : 0u)));
}

// ------------------------------------------------------------------ append
// A work-group takes one token; a thread takes units of 8 dimensions of a head,
// HD / 8 neighbouring lanes a head: four rotated pairs, or 8 dimensions that pass.
// Everything in 64 bits, rounded once.  Memory bounds prompts: 19 ragged ones of up to 2333
// tokens, 48 heads of 64 dimensions, into 4 bits 133 to 136 us (with the read below 697 MB in
// 154, 4.5 TB/s, a copy reaches 4.9); one token a row is bound by loads that wait for each
// other (length, token count, frequencies, angles, projections).  128 threads where a token has up to 512 units, so that
// few idle in the last pass over it (those prompts, of 384 units: 256 threads 150 us), 256
// where it has more (512 tokens of 768 units: 9.6 us with 256, 13 with 128).
template <typename T, int HD>
__global__ void __launch_bounds__(256) append_norm_kernel(PageAppendNormArgs na) {
  constexpr int UPH = HD / 8, NG = HD / 32;   // units of a head, groups of 4-bit values
  constexpr bool FP4 = sizeof(T) == 1;
  const PageAppendArgs& a = na.a;
  __shared__ double cs[HD / 2], sn[HD / 2];
  const int row = blockIdx.x / a.lr, t = blockIdx.x - row * a.lr;
  const int len = clamp_len(a.lens[row], a.max_pages, a.shift);
  const int n = clamp_new(a.n_new ? a.n_new[row] : a.lr, a.lr, len);
  if (t >= n) return;
  const int pos = len - n + t, pairs = a.rot >> 1;
  for (int i = threadIdx.x; i < pairs; i += blockDim.x) sincos((double)pos * a.freqs[i], &sn[i], &cs[i]);
  __syncthreads();
  const int pg = a.table[(int64_t)row * a.max_pages + (pos >> a.shift)];
  const int heads = a.hq + 2 * a.hkv;
  const float* src = a.qkv + (int64_t)blockIdx.x * heads * HD;
  float* qd = a.q + (int64_t)blockIdx.x * a.hq * HD;
  for (int u = threadIdx.x; u < heads * UPH; u += blockDim.x) {   // (the lanes of a head stay together)
    const int h = u / UPH, w = u % UPH;
    const bool rotates = 4 * w < pairs && h < a.hq + a.hkv;
    // the unit's two runs of four dimensions
    const int d0 = rotates && !a.interleaved ? 4 * w : 8 * w;
    const int d1 = rotates && !a.interleaved ? pairs + 4 * w : 8 * w + 4;
    const float4 x = *reinterpret_cast<const float4*>(src + h * HD + d0);
    const float4 y = *reinterpret_cast<const float4*>(src + h * HD + d1);
    double v0[4] = {x.x, x.y, x.z, x.w}, v1[4] = {y.x, y.y, y.z, y.w};
    const float* gain = h < a.hq ? na.q_gain : h < a.hq + a.hkv ? na.k_gain : nullptr;
    if (gain) {
      double s = 0.0;
#pragma unroll
      for (int e = 0; e < 4; ++e) s += v0[e] * v0[e] + v1[e] * v1[e];
#pragma unroll
      for (int o = 1; o < UPH; o <<= 1) s += __shfl_xor(s, o, 64);
      const double r = 1.0 / sqrt(s / HD + na.eps);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v0[e] *= r * (double)gain[d0 + e];
        v1[e] *= r * (double)gain[d1 + e];
      }
    }
    if (rotates) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const double c0 = cs[4 * w + e], s0 = sn[4 * w + e], c1 = cs[4 * w + 2 + e], s1 = sn[4 * w + 2 + e];
          const double p = v0[2 * e], q = v0[2 * e + 1], r = v1[2 * e], z = v1[2 * e + 1];
          v0[2 * e] = p * c0 - q * s0;
          v0[2 * e + 1] = q * c0 + p * s0;
          v1[2 * e] = r * c1 - z * s1;
          v1[2 * e + 1] = z * c1 + r * s1;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double c = cs[4 * w + e], s = sn[4 * w + e], p = v0[e], q = v1[e];
          v0[e] = p * c - q * s;
          v1[e] = q * c + p * s;
        }
      }
    }
    if (h < a.hq) {
      *reinterpret_cast<float4*>(qd + h * HD + d0) = make_float4((float)v0[0], (float)v0[1], (float)v0[2], (float)v0[3]);
      *reinterpret_cast<float4*>(qd + h * HD + d1) = make_float4((float)v1[0], (float)v1[1], (float)v1[2], (float)v1[3]);
      continue;
    }
    const bool key = h < a.hq + a.hkv;
    void* pool = key ? a.kpool : a.vpool;
    const int kh = key ? h - a.hq : h - a.hq - a.hkv;
    if constexpr (FP4) {
      // the largest magnitude of every group, over the lanes of the head
      uint32_t m0 = 0, m1 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m0 = max(m0, fp4_mag(v0[e]));
        m1 = max(m1, fp4_mag(v1[e]));
      }
      int b0 = 0, b1 = 0, mine = 0;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        uint32_t m = max(d0 / 32 == g ? m0 : 0u, d1 / 32 == g ? m1 : 0u);
#pragma unroll
        for (int o = 1; o < UPH; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
        const int b = fp4_scale_byte(m);
        if (d0 / 32 == g) b0 = b;
        if (d1 / 32 == g) b1 = b;
        if (w == g) mine = b;
      }
      if (!is_page(pg, a.n_pages)) continue;
      const int slot = pos & ((1 << a.shift) - 1);
      uint8_t* blk = (uint8_t*)pool + fp4_block(pg, a.hkv, kh, a.shift, HD);
      uint32_t c0 = 0, c1 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c0 |= fp4_code(v0[e], b0) << (4 * e);
        c1 |= fp4_code(v1[e], b1) << (4 * e);
      }
      uint8_t* codes = blk + fp4_codes(slot, HD);
      *reinterpret_cast<uint16_t*>(codes + d0 / 2) = (uint16_t)c0;
      *reinterpret_cast<uint16_t*>(codes + d1 / 2) = (uint16_t)c1;
      if (w < NG) blk[fp4_scales(slot, a.shift, HD) + w] = (uint8_t)mine;
    } else {
      if (!is_page(pg, a.n_pages)) continue;
      T* dst = (T*)pool + page_offset(pg, a.hkv, kh, a.shift, pos, HD);
      typedef T t4 __attribute__((ext_vector_type(4)));   // (multiples of four: aligned)
      t4 x0, x1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x0[e] = round_once<T>(v0[e]);
        x1[e] = round_once<T>(v1[e]);
      }
      *reinterpret_cast<t4*>(dst + d0) = x0;
      *reinterpret_cast<t4*>(dst + d1) = x1;
    }
  }
}

template <typename T>
static void append_norm_by_hd(const PageAppendNormArgs& a, hipStream_t s) {
  const int units = (a.a.hq + 2 * a.a.hkv) * (a.a.hd / 8);
  const dim3 grid((unsigned)(a.a.rows * a.a.lr)), block(units <= 512 ? 128 : 256);
  switch (a.a.hd) {
    case 32: SR_LAUNCH((append_norm_kernel<T, 32>), grid, block, 0, s, a); break;
    case 64: SR_LAUNCH((append_norm_kernel<T, 64>), grid, block, 0, s, a); break;
    default: SR_LAUNCH((append_norm_kernel<T, 128>), grid, block, 0, s, a); break;
  }
  SR_CHECK_LAUNCH();
}

void page_append_norm(const PageAppendNormArgs& a, hipStream_t s) {
  if (a.a.rows <= 0 || a.a.lr <= 0) return;
  if (a.a.dtype == SR_FP4) append_norm_by_hd<uint8_t>(a, s);
  else if (a.a.dtype == SR_BF16) append_norm_by_hd<bf16_t>(a, s);
  else append_norm_by_hd<float>(a, s);
}

// -------------------------------------------------------------------- read
// A thread takes 8 dimensions of a key and of a value; a work-group whole tokens, as many
// as fill it.  Those prompts' 8 heads out of 4 bits: 21 us (3.5 TB/s) (work-groups of 256 units of keys
// or of values, each unit's token by a 64-bit division: 39).
constexpr int kReadThreads = 256;
template <typename C, typename T, int HD>
__device__ __forceinline__ void read_unit(const PageReadArgs& a, const void* pool, int pg, int h, int pos, int w, T* dst) {
  if constexpr (sizeof(C) == 1) {
    uint32_t c = 0;
    float scale = 1.f;
    if (is_page(pg, a.n_pages)) {
      const int slot = pos & ((1 << a.shift) - 1);
      const uint8_t* blk = (const uint8_t*)pool + fp4_block(pg, a.hkv, h, a.shift, HD);
      c = *reinterpret_cast<const uint32_t*>(blk + fp4_codes(slot, HD) + 4 * w);
      scale = fp4_scale(blk[fp4_scales(slot, a.shift, HD) + w / 4]);
    }
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<bf16x8*>(dst) = fp4_to_bf16(c, scale);
    } else {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fp4_value(c >> (4 * e), scale);
      reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (is_page(pg, a.n_pages)) {
      const C* src = (const C*)pool + page_offset(pg, a.hkv, h, a.shift, pos, HD) + 8 * w;
#pragma unroll
      for (int e = 0; e < 8; e += Vec16<C>::N) Vec16<C>::load(src + e, v + e);
    }
    if constexpr (sizeof(T) == 2) {
      uint32_t p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = f32_to_bf16(v[2 * e]) | ((uint32_t)f32_to_bf16(v[2 * e + 1]) << 16);
      *reinterpret_cast<uint4*>(dst) = make_uint4(p[0], p[1], p[2], p[3]);
    } else {
      reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
}

__host__ __device__ inline int read_tokens(int units) { return units < kReadThreads ? kReadThreads / units : 1; }   // of a work-group

template <typename C, typename T, int HD>
__global__ void __launch_bounds__(kReadThreads) read_kernel(PageReadArgs a) {
  constexpr int UPH = HD / 8;
  const int units = a.hkv * UPH, per = read_tokens(units);
  const int mine = per > 1 ? (int)threadIdx.x / units : 0;
  const int token = blockIdx.x * per + mine;
  if (mine >= per || token >= a.rows * a.lr) return;
  const int row = token / a.lr, t = token - row * a.lr;
  const int len = clamp_len(a.lens[row], a.max_pages, a.shift);
  const int n = clamp_new(a.n_new ? a.n_new[row] : a.lr, a.lr, len);
  if (t >= n) return;
  const int pos = len - n + t;
  const int pg = a.table[(int64_t)row * a.max_pages + (pos >> a.shift)];
  for (int u = threadIdx.x - mine * units; u < units; u += kReadThreads) {   // (once where it holds several tokens)
    const int h = u / UPH, w = u % UPH;
    const int64_t at = ((int64_t)token * units + u) * 8;
    if (a.k_out) read_unit<C, T, HD>(a, a.kpool, pg, h, pos, w, (T*)a.k_out + at);
    if (a.v_out) read_unit<C, T, HD>(a, a.vpool, pg, h, pos, w, (T*)a.v_out + at);
  }
}

template <typename C, typename T>
static void launch_read(const PageReadArgs& a, hipStream_t s) {
  const int per = read_tokens(a.hkv * (a.hd / 8));
  const dim3 grid((unsigned)((a.rows * a.lr + per - 1) / per)), block(kReadThreads);
  switch (a.hd) {
    case 32: SR_LAUNCH((read_kernel<C, T, 32>), grid, block, 0, s, a); break;
    case 64: SR_LAUNCH((read_kernel<C, T, 64>), grid, block, 0, s, a); break;
    default: SR_LAUNCH((read_kernel<C, T, 128>), grid, block, 0, s, a); break;
  }
  SR_CHECK_LAUNCH();
}

template <typename C>
static void read_by_type(const PageReadArgs& a, hipStream_t s) {
  if (a.dtype == SR_BF16) launch_read<C, bf16_t>(a, s);
  else launch_read<C, float>(a, s);
}

void page_read(const PageReadArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.lr <= 0) return;
  if (a.cache == SR_FP4) read_by_type<uint8_t>(a, s);
  else if (a.cache == SR_BF16) read_by_type<bf16_t>(a, s);
  else read_by_type<float>(a, s);
}

}  // namespace sr
