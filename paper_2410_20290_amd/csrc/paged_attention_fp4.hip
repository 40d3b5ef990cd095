// Causal attention over pages of 4 bits, with a sliding window and sink tokens.
#include "common.h"
#include "fp4.h"
#include "kernels.h"
#include "paged_parts.h"
#include "specrej_serving.h"

namespace sr {

// A wave takes one token and query head: a key a lane, then its values' dimensions.
template <typename T>
__global__ void __launch_bounds__(64) fp4_plain_kernel(PagedAttnArgs a, float qscale) {
  __shared__ float q[128];
  const int head = blockIdx.x % a.hq, token = blockIdx.x / a.hq, row = token / a.lr, t = token - row * a.lr;
  const RowState rs = row_state(a, row);
  if (t >= rs.n) return;
  const int lane = threadIdx.x, h = head / (a.hq / a.hkv), p = rs.p0 + t;
  const int64_t th = (int64_t)token * a.hq + head;
  for (int d = lane; d < a.hd; d += 64) q[d] = a.q[th * a.hd + d] * qscale;
  __syncthreads();
  const int lo = window_start(p, a.window), sinks = imin(a.sinks, lo), seen = sinks + p + 1 - lo;
  const int32_t* tab = a.table + (int64_t)row * a.max_pages;
  float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
  auto block = [&](const void* pool, int pg) { return (const uint8_t*)pool + fp4_block(pg, a.hkv, h, a.shift, a.hd); };
  auto key_of = [&](int v) { return v < sinks ? v : v - sinks + lo; };
  for (int v0 = 0; v0 < seen; v0 += 64) {
    const int key = key_of(imin(v0 + lane, seen - 1)), slot = key & ((1 << a.shift) - 1);
    const int pg = tab[key >> a.shift];
    const bool ok = v0 + lane < seen && (uint32_t)pg < (uint32_t)a.n_pages;
    float s = 0.f;
    if (ok) {
      const uint8_t* b = block(a.kpool, pg);
      for (int d = 0; d < a.hd; ++d)
        s += q[d] * fp4_value(b[fp4_codes(slot, a.hd) + d / 2] >> (4 * (d & 1)), fp4_scale(b[fp4_scales(slot, a.shift, a.hd) + d / 32]));
    }
    if (!ok) s = -INFINITY;
    const float mn = fmaxf(m, wave_max(fmaxf(s, -INFINITY))), ref = mn == -INFINITY ? 0.f : mn;
    const float corr = exp2f(m - ref), w = exp2f(s - ref);
    m = mn;
    l = l * corr + wave_sum(w);
    o[0] *= corr;
    o[1] *= corr;
    for (int k = 0; k < 64 && v0 + k < seen; ++k) {
      const float wk = __shfl(w, k, 64);
      const int kk = key_of(v0 + k), sl = kk & ((1 << a.shift) - 1), pk = tab[kk >> a.shift];
      if ((uint32_t)pk >= (uint32_t)a.n_pages) continue;
      const uint8_t* b = block(a.vpool, pk);
      for (int i = 0, d = lane; d < a.hd; ++i, d += 64)
        o[i] += wk * fp4_value(b[fp4_codes(sl, a.hd) + d / 2] >> (4 * (d & 1)), fp4_scale(b[fp4_scales(sl, a.shift, a.hd) + d / 32]));
    }
  }
  for (int i = 0, d = lane; d < a.hd; ++i, d += 64) ((T*)a.out)[th * a.hd + d] = from_f32<T>(l == 0.f ? 0.f : o[i] / l);
}

size_t paged_attn_fp4_scratch(const PagedAttnArgs&) { return 0; }

void paged_attn_fp4(const PagedAttnArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.lr <= 0) return;
  const float qscale = kLog2e / sqrtf((float)a.hd);
  const dim3 grid((unsigned)(a.rows * a.lr * a.hq));
  if (a.dtype == SR_BF16) SR_LAUNCH(fp4_plain_kernel<bf16_t>, grid, dim3(64), 0, s, a, qscale);
  else SR_LAUNCH(fp4_plain_kernel<float>, grid, dim3(64), 0, s, a, qscale);
  SR_CHECK_LAUNCH();
}

}  // namespace sr
