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

// The quotient of x below n by d, which the host gives as ceil(2^32 / d): exact, because n * d is at most 2^32.  0 where n is no more than d.
struct Divisor {
  uint32_t d, mul;
};
__device__ __forceinline__ uint32_t operator/(uint32_t x, Divisor v) { return v.d == 1 ? x : __umulhi(x, v.mul); }

// V pairs an item, as two accesses of V elements.  A block takes `rows` rows: first their (cos, sin) into LDS, then the items of all of them, V pairs or 2 V copied columns each.
template <bool BF16, int V, bool INTER>
__global__ __launch_bounds__(THREADS) void rotary_kernel(Rotary a, int rows, Divisor head_items, Divisor row_items) {
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
  const int pair_items = half / V;
  for (uint32_t it = blockIdx.y * THREADS + threadIdx.x; it < nr * row_items.d; it += gridDim.y * THREADS) {
    const uint32_t r = it / row_items, in_row = it - r * row_items.d, head = in_row / head_items;
    const int w = (int)(in_row - head * head_items.d);
    const elem *x = (const elem *)a.x + (size_t)(r0 + r) * a.ld_x;
    elem *out = (elem *)a.out + (size_t)(r0 + r) * a.ld_out;
    const size_t h0 = (size_t)head * a.hd;
    // columns behind the turned part take the same way with their values as they are (a branch of their own would wait for its loads before the others')
    const bool turned = w < pair_items;
    const int p = turned ? w * V : 0, rest = a.rot + (w - pair_items) * 2 * V;
    const size_t o0 = h0 + (turned ? (INTER ? 2 * p : p) : rest), o1 = INTER || !turned ? o0 + V : o0 + half;
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
      if constexpr (BF16) { y.e[e] = turned ? (bf16_t)cvt_pk_bf16(g[e], 0.f) : u.e[e]; z.e[e] = turned ? (bf16_t)cvt_pk_bf16(g[V + e], 0.f) : v.e[e]; }
      else { y.e[e] = turned ? g[e] : u.e[e]; z.e[e] = turned ? g[V + e] : v.e[e]; }
    }
    *(vec *)(out + o0) = y;
    *(vec *)(out + o1) = z;
  }
}

Divisor divisor(int64_t n, int d) { return {(uint32_t)d, n <= d ? 0 : (uint32_t)(((1ull << 32) + d - 1) / d)}; }

// Rows of a block: as many as a quarter of its threads form the angles of at once and as give each thread two items, as long as there are 1024 blocks, and within 16 KB of
// angles.  (66576 rows of 64 heads of 128, 64 columns turned: at four times as many 449 us, now 402, 5.4 TB/s; 12289 x 40 x 128 in fp32 100 and 92.)
template <bool BF16, int V>
void launch(const Rotary &a, hipStream_t st) {
  const int half = a.rot / 2, copied = a.x == a.out ? 0 : (a.hd - a.rot) / (2 * V), head_items = half / V + copied, items = a.n_heads * head_items;
  const int exact = (int)std::min((1ll << 32) / ((long long)items * items), 2048ll);           // rows that `divisor` holds for
  const int rows = std::max(1, std::min({std::max(THREADS / half / 4, cdiv(2 * THREADS, items)), a.n / 1024, 2048 / half, exact}));
  const unsigned across = (unsigned)std::min(16, std::max(1, items / (4 * THREADS)));
  const size_t lds = (size_t)rows * half * sizeof(float2);
  // (a grid has less than 2^32 threads in a direction: more rows go in several launches)
  const int most = (int)std::min<long long>(INT32_MAX, (long long)rows << 23);
  for (int r0 = 0; r0 < a.n; r0 += std::min(most, a.n - r0)) {
    Rotary b = a;
    const size_t es = BF16 ? 2 : 4;
    b.x = (const char *)a.x + (size_t)r0 * a.ld_x * es;
    b.out = (char *)a.out + (size_t)r0 * a.ld_out * es;
    b.positions = a.positions + r0;
    b.n = std::min(most, a.n - r0);
    const dim3 grid(cdiv(b.n, rows), across);
    if (a.interleaved) hipLaunchKernelGGL((rotary_kernel<BF16, V, true>), grid, dim3(THREADS), lds, st, b, rows, divisor(items, head_items), divisor((int64_t)rows * items, items));
    else hipLaunchKernelGGL((rotary_kernel<BF16, V, false>), grid, dim3(THREADS), lds, st, b, rows, divisor(items, head_items), divisor((int64_t)rows * items, items));
  }
}

}  // namespace

hipError_t launch_rotary(const Rotary &a, bool bf16, hipStream_t st) {
  if (a.n <= 0 || a.n_heads <= 0) return hipSuccess;
  // The widest access (at most 16 bytes) that the pairs' halves, the rest of a head, the strides and the pointers are multiples of.
  const int es = bf16 ? 2 : 4;
  int v = 16 / es;
  while (v > 1 && ((a.rot / 2) % v || (a.hd - a.rot) % (2 * v) || a.ld_x % v || a.ld_out % v || ((uintptr_t)a.x | (uintptr_t)a.out) % (v * es))) v >>= 1;
  if (bf16) v == 8 ? launch<true, 8>(a, st) : v == 4 ? launch<true, 4>(a, st) : v == 2 ? launch<true, 2>(a, st) : launch<true, 1>(a, st);
  else v == 4 ? launch<false, 4>(a, st) : v == 2 ? launch<false, 2>(a, st) : launch<false, 1>(a, st);
  return hipGetLastError();
}
