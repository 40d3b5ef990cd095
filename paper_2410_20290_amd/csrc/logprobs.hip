// Log-probabilities of given tokens with the entropy of their distribution and
// its most likely tokens: softmax(logits / temperature) of every row.
//   ln p_i = z_i - ln S, z_i = (x_i - max) / T, S = sum e^z
//   H = ln S - (sum e^z z) / S
#include <climits>

#include "common.h"
#include "kernels.h"

namespace sr {

// NaN counts as -inf.
__device__ __forceinline__ float seen_logit(float x) { return x == x ? x : -INFINITY; }
// (x - m) / T with the limits of a maximum of +inf, and of no maximum.
__device__ __forceinline__ float scaled(float x, float m, float inv_t) {
  return x == m ? 0.f : x == -INFINITY ? -INFINITY : (x - m) * inv_t;
}

template <typename T>
__global__ void __launch_bounds__(256) logprob_row_kernel(LogprobArgs a, float inv_t) {
  __shared__ float rv[4], rs[4], rt[4];
  __shared__ int ri[4];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* x = (const T*)a.logits + r * a.row_stride;
  float m = -INFINITY;
  for (int i = tid; i < a.vocab; i += 256) m = fmaxf(m, seen_logit(to_f32<T>(x[i])));
  m = wave_max(m);
  if (lane == 0) rv[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(rv[0], rv[1]), fmaxf(rv[2], rv[3]));
  float s = 0.f, t = 0.f;
  if (m != -INFINITY)
    for (int i = tid; i < a.vocab; i += 256) {
      const float z = scaled(seen_logit(to_f32<T>(x[i])), m, inv_t);
      const float e = expf(z);
      s += e;
      if (e > 0.f) t += e * z;
    }
  s = wave_sum(s);
  t = wave_sum(t);
  if (lane == 0) {
    rs[wave] = s;
    rt[wave] = t;
  }
  __syncthreads();
  s = (rs[0] + rs[1]) + (rs[2] + rs[3]);
  t = (rt[0] + rt[1]) + (rt[2] + rt[3]);
  const bool none = m == -INFINITY;
  const float ls = none ? 0.f : logf(s);
  if (tid == 0) {
    if (a.logprob) {
      const int tok = a.tokens[r];
      float lp = __uint_as_float(0x7FC00000u);
      if (tok == -1) lp = 0.f;
      else if ((uint32_t)tok < (uint32_t)a.vocab)
        lp = none ? -INFINITY : scaled(seen_logit(to_f32<T>(x[tok])), m, inv_t) - ls;
      a.logprob[r] = lp;
    }
    if (a.entropy) a.entropy[r] = none ? 0.f : ls - t / s;
  }
  // the next entry in (value descending, index ascending) order, each time
  float pv = INFINITY;
  int pi = -1;
  for (int k = 0; k < a.top; ++k) {
    float bv = -INFINITY;
    int bi = INT_MAX;
    for (int i = tid; i < a.vocab; i += 256) {
      const float v = seen_logit(to_f32<T>(x[i]));
      const bool after = v < pv || (v == pv && i > pi);
      if (after && (v > bv || (v == bv && i < bi))) { bv = v; bi = i; }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float ov = __shfl_xor(bv, o, 64);
      const int oi = __shfl_xor(bi, o, 64);
      if (ov > bv || (ov == bv && oi < bi)) { bv = ov; bi = oi; }
    }
    __syncthreads();
    if (lane == 0) { rv[wave] = bv; ri[wave] = bi; }
    __syncthreads();
    bv = rv[0];
    bi = ri[0];
    for (int w = 1; w < 4; ++w)
      if (rv[w] > bv || (rv[w] == bv && ri[w] < bi)) { bv = rv[w]; bi = ri[w]; }
    pv = bv;
    pi = bi;
    if (tid == 0) {
      if (a.top_ids) a.top_ids[(int64_t)r * a.top + k] = bi;
      if (a.top_logprobs) a.top_logprobs[(int64_t)r * a.top + k] = none ? -INFINITY : scaled(bv, m, inv_t) - ls;
    }
  }
}

size_t token_logprobs_scratch(int rows, int vocab, int top) {
  (void)rows; (void)vocab; (void)top;
  return 0;
}

void token_logprobs(const LogprobArgs& a, hipStream_t s) {
  if (a.rows <= 0) return;
  const float inv_t = (float)(1.0 / (double)a.temperature);
  if (a.dtype == SR_BF16) SR_LAUNCH(logprob_row_kernel<bf16_t>, dim3(a.rows), dim3(256), 0, s, a, inv_t);
  else SR_LAUNCH(logprob_row_kernel<float>, dim3(a.rows), dim3(256), 0, s, a, inv_t);
  SR_CHECK_LAUNCH();
}

}  // namespace sr
