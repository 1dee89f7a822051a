// Log-probabilities of given tokens with the entropy and the best alternatives of their rows, and the gradient of both
// with respect to the logits.
//   m = max_j x_j,  L = log sum_j e^(x_j - m),  lp_j = x_j - m - L,  p_j = e^(lp_j)
//   logp = lp_token,   H = -sum_j p_j lp_j = L - sum_j (x_j - m) e^(x_j - m) / sum_j e^(x_j - m)
//   d logits_j = g ([j == token] - p_j) - h p_j (lp_j + H),    g = dL/dlogp, h = dL/dH
// A logit of -inf bans its token: p = 0 and no part in any sum.  A row with nothing but banned tokens has logp = -inf, H = 0 and
// gradient 0; NaN or +inf in a row make its results NaN.
#include "kernels.h"

namespace {

constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ bool better(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// One block per row: maximum, sums, then one turn over the row for every alternative.
template <bool BF16>
__global__ __launch_bounds__(256) void token_logprobs_kernel(const TokenLogprobs a) {
  __shared__ float red[4];
  __shared__ float sv[4];
  __shared__ int si[4];
  for (size_t r = blockIdx.x; r < (size_t)a.n; r += gridDim.x) {
    const size_t at = r * a.ld;
    float m = LOWEST;
    for (int j = threadIdx.x; j < a.vocab; j += 256) m = fmaxf(m, ld_io<BF16>(a.logits, at + j));
    m = block_max<256>(m, red);
    float s = 0.f, u = 0.f;
    for (int j = threadIdx.x; j < a.vocab; j += 256) {
      const float t = ld_io<BF16>(a.logits, at + j) - m, e = __builtin_amdgcn_exp2f(t * LOG2E);
      s += e;
      u += e * fmaxf(t, -1e4f);
    }
    s = block_sum<256>(s, red);
    u = block_sum<256>(u, red);
    const bool empty = s == 0.f, bad = s != s;
    const float L = empty ? 0.f : logf(s);
    if (threadIdx.x == 0) {
      if (a.row_stats) {
        a.row_stats[2 * r] = bad ? NAN : empty ? -INFINITY : m;
        a.row_stats[2 * r + 1] = bad ? NAN : L;
      }
      if (a.entropy) a.entropy[r] = empty ? 0.f : L - u / s;
      if (a.logp) {
        const int t = a.token_ids[r];
        a.logp[r] = t >= 0 && t < a.vocab ? (bad ? NAN : empty ? -INFINITY : ld_io<BF16>(a.logits, at + t) - m - L) : 0.f;
      }
    }
    float pv = INFINITY;
    int pi = -1;
    for (int k = 0; k < a.top_k; ++k) {
      float bv = -INFINITY;
      int bi = 0x7fffffff;
      for (int j = threadIdx.x; j < a.vocab && !bad; j += 256) {
        const float x = ld_io<BF16>(a.logits, at + j);
        if (x > -INFINITY && better(pv, pi, x, j) && better(x, j, bv, bi)) { bv = x; bi = j; }
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const float ov = __shfl_xor(bv, o, 64);
        const int oi = __shfl_xor(bi, o, 64);
        if (better(ov, oi, bv, bi)) { bv = ov; bi = oi; }
      }
      __syncthreads();
      if ((threadIdx.x & 63) == 0) { sv[threadIdx.x >> 6] = bv; si[threadIdx.x >> 6] = bi; }
      __syncthreads();
      pv = sv[0]; pi = si[0];
      for (int w = 1; w < 4; ++w)
        if (better(sv[w], si[w], pv, pi)) { pv = sv[w]; pi = si[w]; }
      const bool none = pi == 0x7fffffff;
      if (threadIdx.x == 0) {
        a.top_ids[r * a.top_k + k] = none ? -1 : pi;
        if (a.top_logp) a.top_logp[r * a.top_k + k] = bad ? NAN : none ? -INFINITY : pv - m - L;
      }
    }
  }
}

template <bool BF16, bool OUT_BF16>
__global__ __launch_bounds__(256) void token_logprobs_grad_kernel(const TokenLogprobsGrad a) {
  for (size_t r = blockIdx.x; r < (size_t)a.n; r += gridDim.x) {
    const int tok = a.d_logp ? a.token_ids[r] : -1;
    const float g = tok >= 0 && tok < a.vocab ? a.d_logp[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f;
    const float m = a.row_stats[2 * r], L = a.row_stats[2 * r + 1], H = a.d_entropy ? a.entropy[r] : 0.f;
    const bool zero = m == -INFINITY || (g == 0.f && h == 0.f);
    for (int j = threadIdx.x; j < a.vocab; j += 256) {
      float o = 0.f;
      if (!zero) {
        const float lp = ld_io<BF16>(a.logits, r * a.ld + j) - m - L, p = __builtin_amdgcn_exp2f(lp * LOG2E);
        o = (j == tok ? g : 0.f) - g * p - h * p * (fmaxf(lp, -1e4f) + H);
      }
      st_io<OUT_BF16>(a.d_logits, r * a.ld_d + j, o);
    }
  }
}

}  // namespace

size_t token_logprobs_scratch_bytes(int, int, int) { return 0; }

hipError_t launch_token_logprobs(const TokenLogprobs &a, bool bf16, void *, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  const dim3 grid(a.n < (1 << 20) ? a.n : 1 << 20);
  if (bf16) hipLaunchKernelGGL(token_logprobs_kernel<true>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(token_logprobs_kernel<false>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_token_logprobs_grad(const TokenLogprobsGrad &a, bool bf16, bool out_bf16, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  auto *k = bf16 ? (out_bf16 ? token_logprobs_grad_kernel<true, true> : token_logprobs_grad_kernel<true, false>)
                 : (out_bf16 ? token_logprobs_grad_kernel<false, true> : token_logprobs_grad_kernel<false, false>);
  hipLaunchKernelGGL(k, dim3(a.n < (1 << 20) ? a.n : 1 << 20), dim3(256), 0, st, a);
  return hipGetLastError();
}
