// Paged cache in 4 bits: rows are rounded and scattered by slot, and read back.  A thread takes eight values (four bytes of codes), four lanes share a
// group of 32 and its scale.  Bound by the bytes of the rows in their own type: 16384 rows of 8 heads of 128 in bf16 are put in in 20 us (4.3 TB/s) and read back in
// 18 (4.7).  The rows that come in are read past the caches' order of use: they are not read again, and what is written then stays there (23.5 us without).  64 rows
// of 32 heads: 3.4 and 2.9 us, three loads one after the other.
#include "kernels.h"
#include "kv4.h"

namespace {

constexpr int THREADS = 256;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

__device__ __forceinline__ uint32_t token_index(const Kv4Cache &c, long long slot, int head) {
  return (((uint32_t)(slot >> c.bshift) * c.Hkv + head) << c.bshift) + (uint32_t)(slot & ((1 << c.bshift) - 1));
}

// Row and place in it of a thread: the 64-bit quotient is the block's, once; a thread's is of small numbers.
__device__ __forceinline__ void place_of(int parts, long long &r, int &p) {
  const long long first = (long long)blockIdx.x * THREADS, r0 = first / parts;
  const uint32_t x = (uint32_t)(first - r0 * parts) + threadIdx.x, q = x / (uint32_t)parts;
  r = r0 + q;
  p = (int)(x - q * parts);
}

template <bool BF16>
struct Eight {                                       // eight values as they are stored
  u32x4_t w[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ Eight<BF16> load8(const void *from, size_t i) {
  const u32x4_t *at = (const u32x4_t *)((const char *)from + i * (BF16 ? 2 : 4));
  Eight<BF16> u;
#pragma unroll
  for (int k = 0; k < (BF16 ? 1 : 2); ++k) u.w[k] = __builtin_nontemporal_load(at + k);
  return u;
}
template <bool BF16>
__device__ __forceinline__ void unpack(const Eight<BF16> &u, float x[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (BF16) x[i] = __uint_as_float(i % 2 ? u.w[0][i / 2] & 0xffff0000u : u.w[0][i / 2] << 16);
    else x[i] = __uint_as_float(u.w[i / 4][i % 4]);
  }
}

// parts = Hkv * hd / 8 threads a row, each for its eight of K and of V.  The rows are asked for before it is known whether their slots are any.
template <bool BF16, int HD>
__global__ __launch_bounds__(THREADS) void kv4_append_kernel(Kv4Cache c, const void *kn, long long ld_k, const void *vn, long long ld_v,
                                                             const int32_t *__restrict__ slots, int slot_heads, const int32_t *__restrict__ positions, int n) {
  constexpr int TPH = HD / 8;                        // threads a head
  long long r;
  int p;
  place_of(c.Hkv * TPH, r, p);
  const int head = p / TPH, e = p % TPH;
  if (r >= n) return;                                // (whole heads leave: the lanes of a group stay together)
  const long long slot = slots[(size_t)r * slot_heads + (slot_heads > 1 ? head : 0)];
  const int position = c.position ? positions[r] : 0;
  const Eight<BF16> in[2] = {load8<BF16>(kn, (size_t)r * ld_k + (size_t)p * 8), load8<BF16>(vn, (size_t)r * ld_v + (size_t)p * 8)};
  const bool ok = slot >= 0 && slot < (long long)c.num_blocks << c.bshift;
  const uint32_t t = ok ? token_index(c, slot, head) : 0u;
#pragma unroll
  for (int values = 0; values < 2; ++values) {
    float x[8];
    unpack<BF16>(in[values], x);
    uint32_t top = 0;                                // magnitudes compare as their bits, infinities and NaN above all others
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    const uint32_t b = kv4::scale_byte(top);
    const uint32_t code = b == kv4::NAN_SCALE ? 0u : kv4::encode8(x, kv4::scale_value(b));
    // the scale bytes of a head, gathered in its first lane
    uint32_t sc = b << (8 * (e >> 2));
    sc |= (uint32_t)__shfl_xor((int)sc, 4, 64);
    if constexpr (HD == 128) sc |= (uint32_t)__shfl_xor((int)sc, 8, 64);
    if (ok) {
      ((uint32_t *)(values ? c.v : c.k))[(size_t)t * TPH + e] = code;
      if (e == 0) {
        if constexpr (HD == 128) ((uint32_t *)(values ? c.v_scale : c.k_scale))[t] = sc;
        else ((uint16_t *)(values ? c.v_scale : c.k_scale))[t] = (uint16_t)sc;
      }
    }
  }
  if (ok && e == 0) {
    if (c.weight) c.weight[t] = 0.f;
    if (c.position) c.position[t] = position;
  }
}

template <bool BF16, int HD>
__global__ __launch_bounds__(THREADS) void kv4_gather_kernel(Kv4Cache c, const int32_t *__restrict__ slots, int slot_heads, int n, void *ko, void *vo) {
  constexpr int TPH = HD / 8;
  const int parts = c.Hkv * TPH;
  long long r;
  int p;
  place_of(parts, r, p);
  const int head = p / TPH, e = p % TPH;
  if (r >= n) return;
  const long long slot = slots[(size_t)r * slot_heads + (slot_heads > 1 ? head : 0)];
  const bool ok = slot >= 0 && slot < (long long)c.num_blocks << c.bshift;       // another slot yields zeros, never a wild read
  const uint32_t t = ok ? token_index(c, slot, head) : 0;
  const size_t at = (size_t)t * TPH + e, scale_at = (size_t)t * (HD / 32) + (e >> 2), o = (size_t)r * parts + p;
  const uint32_t codes[2] = {((const uint32_t *)c.k)[at], ((const uint32_t *)c.v)[at]};
  const float scales[2] = {kv4::scale_value(c.k_scale[scale_at]), kv4::scale_value(c.v_scale[scale_at])};
#pragma unroll
  for (int values = 0; values < 2; ++values) {
    const uint32_t code = codes[values];
    const float scale = scales[values];
    if constexpr (BF16) {
      const uint4 u = __builtin_bit_cast(uint4, kv4::decode8(code, scale));
      ((uint4 *)(values ? vo : ko))[o] = ok ? u : make_uint4(0, 0, 0, 0);
    } else {
      const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
      const f32x2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
      float4 *dst = (float4 *)(values ? vo : ko) + 2 * o;
      dst[0] = ok ? make_float4(a[0], a[1], b[0], b[1]) : make_float4(0.f, 0.f, 0.f, 0.f);
      dst[1] = ok ? make_float4(d[0], d[1], f[0], f[1]) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
}

dim3 grid_of(const Kv4Cache &c, int n) { return dim3((unsigned)(((long long)n * c.Hkv * (c.hd / 8) + THREADS - 1) / THREADS)); }

}  // namespace

hipError_t launch_kv4_append(const Kv4Cache &c, const void *k_new, long long ld_k, const void *v_new, long long ld_v, bool bf16, const int32_t *slots,
                             int slot_heads, const int32_t *positions, int n, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid_of(c, n), dim3(THREADS), 0, st, c, k_new, ld_k, v_new, ld_v, slots, slot_heads, positions, n); };
  if (c.hd == 128) bf16 ? go(kv4_append_kernel<true, 128>) : go(kv4_append_kernel<false, 128>);
  else bf16 ? go(kv4_append_kernel<true, 64>) : go(kv4_append_kernel<false, 64>);
  return hipGetLastError();
}

hipError_t launch_kv4_gather(const Kv4Cache &c, const int32_t *slots, int slot_heads, int n, void *k_out, void *v_out, bool bf16, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid_of(c, n), dim3(THREADS), 0, st, c, slots, slot_heads, n, k_out, v_out); };
  if (c.hd == 128) bf16 ? go(kv4_gather_kernel<true, 128>) : go(kv4_gather_kernel<false, 128>);
  else bf16 ? go(kv4_gather_kernel<true, 64>) : go(kv4_gather_kernel<false, 64>);
  return hipGetLastError();
}
