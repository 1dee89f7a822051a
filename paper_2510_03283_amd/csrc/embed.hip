// Embedding rows of token ids, scaled, and the gradient of the table they come from.
//   forward   out[r, :] = io(scale * E[id_r, :])
//   backward  dE[v, :] (+)= scale * sum over the rows r with id_r = v, in order of r, of dx[r, :]
// A token id outside [0, vocab) is padding: its row of out is zero and its row of dx is not read.
#include "kernels.h"

namespace {

// One block per row.
template <bool BF16>
__global__ __launch_bounds__(256) void embed_rows_kernel(const void *__restrict__ table, const int32_t *__restrict__ ids, int n, int vocab, int d,
                                                         float scale, void *__restrict__ out) {
  for (size_t r = blockIdx.x; r < (size_t)n; r += gridDim.x) {
    const int id = ids[r];
    const bool there = id >= 0 && id < vocab;
    for (int k = threadIdx.x; k < d; k += 256) st_io<BF16>(out, r * d + k, there ? scale * ld_io<BF16>(table, (size_t)id * d + k) : 0.f);
  }
}

// One block per row of the table, which looks through all ids.
__global__ __launch_bounds__(256) void embed_grad_kernel(const int32_t *__restrict__ ids, int n, int vocab, int d, const float *__restrict__ dx,
                                                         float scale, float *__restrict__ d_table, int accumulate) {
  __shared__ unsigned long long hits[4];
  for (int v = blockIdx.x; v < vocab; v += gridDim.x) {
    for (int k0 = 0; k0 < d; k0 += 256) {
      const int k = k0 + threadIdx.x;
      float s = 0.f;
      bool any = false;
      for (long long r0 = 0; r0 < n; r0 += 256) {
        const unsigned long long b = __ballot(r0 + threadIdx.x < n && ids[r0 + threadIdx.x] == v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) hits[threadIdx.x >> 6] = b;
        __syncthreads();
        for (int w = 0; w < 4; ++w)
          for (unsigned long long m = hits[w]; m; m &= m - 1) {
            any = true;
            if (k < d) s += dx[(size_t)(r0 + 64 * w + __builtin_ctzll(m)) * d + k];
          }
      }
      if (k < d && (any || !accumulate)) d_table[(size_t)v * d + k] = scale * s + (accumulate ? d_table[(size_t)v * d + k] : 0.f);
    }
  }
}

}  // namespace

hipError_t launch_embed_rows(const void *table, bool bf16, const int32_t *ids, int n, int vocab, int d, float scale, void *out, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const dim3 grid(n < (1 << 20) ? n : 1 << 20);
  if (bf16) hipLaunchKernelGGL((embed_rows_kernel<true>), grid, dim3(256), 0, st, table, ids, n, vocab, d, scale, out);
  else hipLaunchKernelGGL((embed_rows_kernel<false>), grid, dim3(256), 0, st, table, ids, n, vocab, d, scale, out);
  return hipGetLastError();
}

size_t embed_grad_scratch_bytes(int, int, int) { return 0; }

hipError_t launch_embed_grad(const int32_t *ids, int n, int vocab, int d, const float *dx, float scale, float *d_table, bool accumulate, void *,
                             hipStream_t st) {
  if (n <= 0 && accumulate) return hipSuccess;
  hipLaunchKernelGGL(embed_grad_kernel, dim3(vocab < (1 << 20) ? vocab : 1 << 20), dim3(256), 0, st, ids, n, vocab, d, dx, scale, d_table, accumulate ? 1 : 0);
  return hipGetLastError();
}
