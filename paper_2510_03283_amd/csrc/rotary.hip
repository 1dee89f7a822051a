// Rotary positions of the heads of a batch of rows: pair (a, b) -> m (a cos - b sin, b cos + a sin) with the angle
// positions[r] * inv_freq[i] in 64 bits.  The pairs are (i, i + rot / 2) or (2 i, 2 i + 1) of the first rot columns of a head.  Each row is
// read and written once, so the bytes bound it; the (cos, sin) of a row are formed once for all its heads.
#include "kernels.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int THREADS = 256;

template <bool BF16, int V>
struct Vec {
  typedef std::conditional_t<BF16, bf16_t, float> elem;
  struct alignas(V * sizeof(elem)) type { elem e[V]; };
};

// V pairs an item, as two accesses of V elements.  A block takes `rows` rows: first their (cos, sin) into LDS, then its items, V pairs or V copied columns each.
// items_mul = ceil(2^32 / items of a head).
template <bool BF16, int V, bool INTER>
__global__ __launch_bounds__(THREADS) void rotary_kernel(Rotary a, int rows, int head_items, uint32_t items_mul) {
  typedef typename Vec<BF16, V>::type vec;
  typedef typename Vec<BF16, V>::elem elem;
  extern __shared__ float2 cs[];                     // [rows][rot / 2]
  const int half = a.rot >> 1, r0 = blockIdx.x * rows, nr = min(rows, a.n - r0);
  for (int i = threadIdx.x; i < nr * half; i += THREADS) {
    const int r = i / half, p = i - r * half;
    double s, c;
    rope_sincos((double)a.positions[r0 + r] * a.inv_freq[p], s, c);
    cs[i] = make_float2((float)(a.magnitude * c), (float)(a.magnitude * (a.inverse ? -s : s)));
  }
  __syncthreads();
  const int row_items = a.n_heads * head_items, pair_items = half / V;
  for (int r = 0; r < nr; ++r) {
    const elem *x = (const elem *)a.x + (size_t)(r0 + r) * a.ld_x;
    elem *out = (elem *)a.out + (size_t)(r0 + r) * a.ld_out;
    for (int it = blockIdx.y * THREADS + threadIdx.x; it < row_items; it += gridDim.y * THREADS) {
      const int head = head_items == 1 ? it : (int)__umulhi((uint32_t)it, items_mul), w = it - head * head_items;
      const size_t h0 = (size_t)head * a.hd;
      if (w >= pair_items) {                         // a column behind the turned part
        const size_t o = h0 + a.rot + (size_t)(w - pair_items) * V;
        *(vec *)(out + o) = *(const vec *)(x + o);
        continue;
      }
      const int p = w * V;
      const size_t o0 = h0 + (INTER ? 2 * p : p), o1 = INTER ? o0 + V : o0 + half;
      const vec u = *(const vec *)(x + o0), v = *(const vec *)(x + o1);
      float f[2 * V], g[2 * V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        f[e] = BF16 ? bf2f(u.e[e]) : (float)u.e[e];
        f[V + e] = BF16 ? bf2f(v.e[e]) : (float)v.e[e];
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 t = cs[r * half + p + e];
        const int ia = INTER ? 2 * e : e, ib = INTER ? 2 * e + 1 : V + e;
        g[ia] = f[ia] * t.x - f[ib] * t.y;
        g[ib] = f[ib] * t.x + f[ia] * t.y;
      }
      vec y, z;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if constexpr (BF16) { y.e[e] = f2bf(g[e]); z.e[e] = f2bf(g[V + e]); }
        else { y.e[e] = g[e]; z.e[e] = g[V + e]; }
      }
      *(vec *)(out + o0) = y;
      *(vec *)(out + o1) = z;
    }
  }
}

template <bool BF16, int V>
void launch(const Rotary &a, hipStream_t st) {
  const int half = a.rot / 2, copied = a.x == a.out ? 0 : (a.hd - a.rot) / V, head_items = half / V + copied;
  const long long items = (long long)a.n_heads * head_items;
  const int rows = std::max(1, std::min(THREADS / half, a.n / 1024));
  const uint32_t mul = (uint32_t)(((1ull << 32) + head_items - 1) / head_items);
  const dim3 grid(cdiv(a.n, rows), (unsigned)std::min<long long>(16, std::max<long long>(1, items / (4 * THREADS))));
  const size_t lds = (size_t)rows * half * sizeof(float2);
  if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<BF16, V, true>), grid, dim3(THREADS), lds, st, a, rows, head_items, mul);
  else hipLaunchKernelGGL((rotary_kernel<BF16, V, false>), grid, dim3(THREADS), lds, st, a, rows, head_items, mul);
}

}  // namespace

hipError_t launch_rotary(const Rotary &a, bool bf16, hipStream_t st) {
  if (a.n <= 0 || a.n_heads <= 0) return hipSuccess;
  // The widest access (at most 16 bytes) that the pairs' halves, the rest of a head, the strides and the pointers are multiples of.
  const int es = bf16 ? 2 : 4;
  int v = 16 / es;
  while (v > 1 && ((a.rot / 2) % v || (a.hd - a.rot) % v || a.ld_x % v || a.ld_out % v || ((uintptr_t)a.x | (uintptr_t)a.out) % (v * es))) v >>= 1;
  if (bf16) v == 8 ? launch<true, 8>(a, st) : v == 4 ? launch<true, 4>(a, st) : v == 2 ? launch<true, 2>(a, st) : launch<true, 1>(a, st);
  else v == 4 ? launch<false, 4>(a, st) : v == 2 ? launch<false, 2>(a, st) : launch<false, 1>(a, st);
  return hipGetLastError();
}
