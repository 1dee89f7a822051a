// Paged cache in 4 bits: rows are rounded and scattered by slot, and read back.  A thread takes eight values (four bytes of codes), four lanes share a
// group of 32 and its scale.  Bound by the bytes of the rows in their own type.
#include "kernels.h"
#include "kv4.h"

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ uint32_t token_index(const Kv4Cache &c, long long slot, int head) {
  return (((uint32_t)(slot >> c.bshift) * c.Hkv + head) << c.bshift) + (uint32_t)(slot & ((1 << c.bshift) - 1));
}

// grid (threads of all rows, 2): y = 0 keys, 1 values.  parts = Hkv * hd / 8 threads a row.
template <bool BF16, int HD>
__global__ __launch_bounds__(THREADS) void kv4_append_kernel(Kv4Cache c, const void *kn, long long ld_k, const void *vn, long long ld_v,
                                                             const int32_t *__restrict__ slots, int slot_heads, const int32_t *__restrict__ positions, int n) {
  constexpr int TPH = HD / 8;                        // threads a head
  const int parts = c.Hkv * TPH;
  const long long id = (long long)blockIdx.x * THREADS + threadIdx.x;
  const int r = (int)(id / parts), p = (int)(id - (long long)r * parts), head = p / TPH, e = p % TPH;
  const bool values = blockIdx.y;
  const long long slot = r < n ? slots[(size_t)r * slot_heads + (slot_heads > 1 ? head : 0)] : -1;
  const bool ok = slot >= 0 && slot < (long long)c.num_blocks << c.bshift;       // the lanes of a row stay together: the group's maximum is taken across four of them
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.f;
  if (ok) {
    const size_t o = (size_t)r * (values ? ld_v : ld_k) + (size_t)p * 8;
    if constexpr (BF16) {
      const uint4 u = *(const uint4 *)((const bf16_t *)(values ? vn : kn) + o);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
      const float4 a = *(const float4 *)((const float *)(values ? vn : kn) + o), b = *((const float4 *)((const float *)(values ? vn : kn) + o) + 1);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
  }
  uint32_t top = 0;                                  // magnitudes compare as their bits, infinities and NaN above all others
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
  if (!ok) return;
  const uint32_t t = token_index(c, slot, head);
  ((uint32_t *)(values ? c.v : c.k))[(size_t)t * TPH + e] = code;
  if (e == 0) {
    if constexpr (HD == 128) ((uint32_t *)(values ? c.v_scale : c.k_scale))[t] = sc;
    else ((uint16_t *)(values ? c.v_scale : c.k_scale))[t] = (uint16_t)sc;
    if (!values && c.weight) c.weight[t] = 0.f;
    if (!values && c.position) c.position[t] = positions[r];
  }
}

template <bool BF16, int HD>
__global__ __launch_bounds__(THREADS) void kv4_gather_kernel(Kv4Cache c, const int32_t *__restrict__ slots, int slot_heads, int n, void *ko, void *vo) {
  constexpr int TPH = HD / 8;
  const int parts = c.Hkv * TPH;
  const long long id = (long long)blockIdx.x * THREADS + threadIdx.x;
  const int r = (int)(id / parts), p = (int)(id - (long long)r * parts), head = p / TPH, e = p % TPH;
  if (r >= n) return;
  const bool values = blockIdx.y;
  const long long slot = slots[(size_t)r * slot_heads + (slot_heads > 1 ? head : 0)];
  const bool ok = slot >= 0 && slot < (long long)c.num_blocks << c.bshift;       // another slot yields zeros, never a wild read
  const uint32_t t = ok ? token_index(c, slot, head) : 0;
  const uint32_t code = ((const uint32_t *)(values ? c.v : c.k))[(size_t)t * TPH + e];
  const float scale = kv4::scale_value((values ? c.v_scale : c.k_scale)[(size_t)t * (HD / 32) + (e >> 2)]);
  const size_t o = (size_t)r * parts + p;
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

dim3 grid_of(const Kv4Cache &c, int n) { return dim3((unsigned)(((long long)n * c.Hkv * (c.hd / 8) + THREADS - 1) / THREADS), 2); }

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
