// Embedding rows of token ids, scaled, and the gradient of the table they come from.
//   forward   out[r, :] = io(scale * E[id_r, :])
//   backward  dE[v, :] (+)= scale * sum over the rows r with id_r = v, in order of r, of dx[r, :]
// A token id outside [0, vocab) is padding: its row of out is zero and its row of dx is not read.
#include "kernels.h"

#include <algorithm>

namespace {

// ------------------------------------------------------------------ rows
// 2^lg threads per row, 16-byte accesses, up to four of them in flight a thread.
template <bool BF16>
__global__ __launch_bounds__(256) void embed_rows_kernel(const void *__restrict__ table, const int32_t *__restrict__ ids, int n, int vocab, int d,
                                                         float scale, void *__restrict__ out, int lg) {
  const int vecs = d / (BF16 ? 8 : 4), per = 1 << lg, lane = threadIdx.x & (per - 1), rows = 256 >> lg;
  for (size_t r = (size_t)blockIdx.x * rows + (threadIdx.x >> lg); r < (size_t)n; r += (size_t)gridDim.x * rows) {
    const int id = ids[r];
    const bool there = id >= 0 && id < vocab;
    const uint4 *src = (const uint4 *)table + (size_t)(there ? id : 0) * vecs;
    uint4 *dst = (uint4 *)out + r * vecs;
    for (int k0 = lane; k0 < vecs; k0 += 4 * per) {
      uint4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (there && k0 + i * per < vecs) x[i] = src[k0 + i * per];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (k0 + i * per >= vecs) break;
        uint4 y = make_uint4(0, 0, 0, 0);
        if (there) {
          uint32_t *w = (uint32_t *)&x[i], *o = (uint32_t *)&y;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (BF16) o[j] = cvt_pk_bf16(scale * __uint_as_float(w[j] << 16), scale * __uint_as_float(w[j] & 0xffff0000u));
            else o[j] = __float_as_uint(scale * __uint_as_float(w[j]));
          }
        }
        dst[k0 + i * per] = y;
      }
    }
  }
}

// ------------------------------------------------------------------ gradient of the table
// Three launches.
//  order  The rows sorted by token, rows of one token in their order: a block owns `keys` adjacent tokens, reads all ids, and counts
//         those below its range (where its part of the order begins) and each of its own; a second turn over the ids puts the
//         rows in place.  No block waits for another and no order depends on one.
//  sum    The sorted order is cut into windows of equal length, a wave per window and column strip, so that the work does not
//         depend on how often a token occurs.  A token whose rows all lie in the window is finished there; the sums of one that
//         began before the window or goes on behind it are set aside.  Further waves write the zeros of tokens that do not occur.
//  join   Per window: the token that goes on behind it, if it begins there, from the sums that were set aside, in window order.
constexpr int ORDER_WAVES = 16, MAX_KEYS = 512;
struct Placed {
  int row, token;
};

__global__ __launch_bounds__(64 * ORDER_WAVES) void embed_order_kernel(const int32_t *__restrict__ ids, int n, int vocab, int lg_keys, int *__restrict__ starts,
                                                                       Placed *__restrict__ order) {
  __shared__ int hist[ORDER_WAVES][MAX_KEYS];
  __shared__ int red[ORDER_WAVES], below_all;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, keys = 1 << lg_keys;
  const long long per = ((long long)n + 64 * ORDER_WAVES - 1) / (64 * ORDER_WAVES) * 64, i0 = per * wave, i1 = min((long long)n, i0 + per);
  for (long long v0 = (long long)blockIdx.x << lg_keys; v0 < vocab; v0 += (long long)gridDim.x << lg_keys) {
    const int first = (int)v0, last = (int)min((long long)vocab, v0 + keys);
    for (int i = threadIdx.x; i < ORDER_WAVES * keys; i += 64 * ORDER_WAVES) hist[i >> lg_keys][i & (keys - 1)] = 0;
    __syncthreads();
    int below = 0;
    for (long long i = i0 + lane; i < i1; i += 8 * 64) {
      int id[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) id[k] = i + 64 * k < i1 ? ids[i + 64 * k] : -1;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (id[k] >= 0 && id[k] < first) ++below;
        if (id[k] >= first && id[k] < last) atomicAdd(&hist[wave][id[k] - first], 1);
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
    if (lane == 0) red[wave] = below;
    __syncthreads();
    if (threadIdx.x == 0) {
      int t = 0;
      for (int w = 0; w < ORDER_WAVES; ++w) t += red[w];
      below_all = t;
    }
    // offsets of (token, wave): tokens in order, waves in order within a token
    int mine = 0;
    if (threadIdx.x < keys)
      for (int w = 0; w < ORDER_WAVES; ++w) mine += hist[w][threadIdx.x];
    int sum = mine;                               // inclusive over the wave
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    __syncthreads();
    if (lane == 63) red[wave] = sum;
    __syncthreads();
    if (threadIdx.x < keys) {
      int at = below_all + sum - mine;
      for (int w = 0; w < wave; ++w) at += red[w];
      if (first + (int)threadIdx.x < last) starts[first + threadIdx.x] = at;
      if (first + (int)threadIdx.x == vocab - 1) starts[vocab] = at + mine;
      for (int w = 0; w < ORDER_WAVES; ++w) {
        const int c = hist[w][threadIdx.x];
        hist[w][threadIdx.x] = at;
        at += c;
      }
    }
    __syncthreads();
    for (long long i = i0; i < i1; i += 8 * 64) {
      int id[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) id[k] = i + 64 * k + lane < i1 ? ids[i + 64 * k + lane] : -1;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool in = id[k] >= first && id[k] < last;
        unsigned long long same = __ballot(in);
        if (!same) continue;
        const int key = id[k] - first;
        for (int b = 0; b < lg_keys; ++b) {
          const unsigned long long set = __ballot((key >> b) & 1);
          same &= (key >> b) & 1 ? set : ~set;
        }
        const int leader = in ? __builtin_ctzll(same) : lane;
        int at = 0;
        if (in && lane == leader) at = atomicAdd(&hist[wave][key], __popcll(same));      // only this wave's lanes, one turn after the other
        at = __shfl(at, leader, 64) + __popcll(same & ((1ull << lane) - 1));
        if (in) order[at] = Placed{(int)(i + 64 * k + lane), id[k]};
      }
    }
    __syncthreads();
  }
}

__device__ __forceinline__ float4 scaled(float4 a, float s) { return make_float4(s * a.x, s * a.y, s * a.z, s * a.w); }
__device__ __forceinline__ float4 added(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

constexpr int ZERO_ROWS = 8;          // rows of the table that a wave looks at for zeros

// A unit is (window, strip of 256 NV columns), or (ZERO_ROWS tokens, strip) behind the windows' units.
template <int NV, bool ACC>
__global__ __launch_bounds__(256) void embed_sum_kernel(const int *__restrict__ starts, const Placed *__restrict__ order, const float *__restrict__ dx, int vocab,
                                                        int d, float scale, float *__restrict__ d_table, float *__restrict__ aside, int window,
                                                        long long windows, int strips) {
  const int lane = threadIdx.x & 63;
  const long long units = (windows + (ACC ? 0 : (vocab + ZERO_ROWS - 1) / ZERO_ROWS)) * strips;
  for (long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); unit < units; unit += (long long)gridDim.x * 4) {
    const long long win = unit / strips;
    const int col0 = (int)(unit - win * strips) * 256 * NV + 4 * lane;
    if (!ACC && win >= windows) {
      const int v0 = (int)(win - windows) * ZERO_ROWS;
      const int s = starts[min(v0 + lane, vocab)], e = starts[min(v0 + lane + 1, vocab)];
      const unsigned long long none = __ballot(lane < ZERO_ROWS && v0 + lane < vocab && s == e);
      for (int i = 0; i < ZERO_ROWS; ++i) {
        if (!((none >> i) & 1)) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (col0 + 256 * j < d) *(float4 *)(d_table + (size_t)(v0 + i) * d + col0 + 256 * j) = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      continue;
    }
    const int total = starts[vocab];
    const long long pos = win * window;
    if (pos >= total) continue;
    const int cnt = (int)min((long long)window, total - pos);
    const Placed mine = order[pos + min(lane, cnt - 1)];
    const int first = __shfl(mine.token, 0, 64), last = __shfl(mine.token, cnt - 1, 64);
    const bool from_before = starts[first] < pos, goes_on = starts[last + 1] > pos + cnt;
    const int next = __shfl_down(mine.token, 1, 64);
    const unsigned long long ends = __ballot(lane < cnt && (lane == cnt - 1 || next != mine.token));
    float4 acc[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < cnt; i += 4) {
      float4 x[4][NV], old[4][NV];
      int token[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = min(i + k, cnt - 1), row = __builtin_amdgcn_readlane(mine.row, at);
        token[k] = __builtin_amdgcn_readlane(mine.token, at);
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (col0 + 256 * j < d) x[k][j] = *(const float4 *)(dx + (size_t)row * d + col0 + 256 * j);
        if constexpr (ACC) {
          if ((ends >> at) & 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
              if (col0 + 256 * j < d) old[k][j] = *(const float4 *)(d_table + (size_t)token[k] * d + col0 + 256 * j);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i + k >= cnt) break;
#pragma unroll
        for (int j = 0; j < NV; ++j) acc[j] = added(acc[j], x[k][j]);
        if (!((ends >> (i + k)) & 1)) continue;
        const bool before = from_before && token[k] == first, behind = goes_on && token[k] == last;
        float *to = before || behind ? aside + (size_t)(2 * win + (before ? 0 : 1)) * d : d_table + (size_t)token[k] * d;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float4 o = acc[j];
          if (!(before || behind)) {
            o = scaled(o, scale);
            if constexpr (ACC) o = added(old[k][j], o);
          }
          if (col0 + 256 * j < d) *(float4 *)(to + col0 + 256 * j) = o;
          acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
    }
  }
}

// A block per (window, 1024 columns).
template <bool ACC>
__global__ __launch_bounds__(256) void embed_join_kernel(const int *__restrict__ starts, const Placed *__restrict__ order, int vocab, int d, float scale,
                                                         float *__restrict__ d_table, const float *__restrict__ aside, int window, long long windows, int strips) {
  const int total = starts[vocab];
  for (long long unit = blockIdx.x; unit < windows * strips; unit += gridDim.x) {
    const long long win = unit / strips, pos = win * window, end = pos + window;
    if (end >= total) continue;
    const int token = order[end - 1].token, s = starts[token], e = starts[token + 1];
    const int col = (int)(unit - win * strips) * 1024 + 4 * (int)threadIdx.x;
    if (e <= end || s < pos || col >= d) continue;
    const long long last = (e - 1) / window;
    float4 acc = *(const float4 *)(aside + (size_t)(2 * win + 1) * d + col), old = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (ACC) old = *(const float4 *)(d_table + (size_t)token * d + col);
    for (long long w = win + 1; w <= last; w += 8) {
      float4 x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = *(const float4 *)(aside + (size_t)(2 * min(w + k, last)) * d + col);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (w + k <= last) acc = added(acc, x[k]);
    }
    *(float4 *)(d_table + (size_t)token * d + col) = ACC ? added(old, scaled(acc, scale)) : scaled(acc, scale);
  }
}

struct GradPlan {
  int nv, strips, window, lg_keys;
  long long windows;
  size_t order_at, aside_at, bytes;
};
GradPlan plan_grad(int n, int vocab, int d) {
  GradPlan p;
  p.nv = d > 512 ? 4 : d > 256 ? 2 : 1;
  p.strips = (d + 256 * p.nv - 1) / (256 * p.nv);
  p.window = 64;
  while (p.window > 4 && (long long)((n + p.window - 1) / p.window) * p.strips < 4096) p.window >>= 1;
  p.windows = ((long long)n + p.window - 1) / p.window;
  p.lg_keys = vocab <= (1 << 15) ? 7 : vocab <= (1 << 16) ? 8 : 9;
  p.order_at = align_up(((size_t)vocab + 1) * sizeof(int), 256);
  p.aside_at = align_up(p.order_at + (size_t)n * sizeof(Placed), 256);
  // the windows of fewer rows may be shorter, and so more: never more than n / 4, nor, while they are shorter than 64, than 8192 units
  const long long most = std::max<long long>(((long long)n + 63) / 64, std::min<long long>(((long long)n + 3) / 4, 8192 / p.strips + 1));
  p.bytes = p.aside_at + (size_t)std::max(most, p.windows) * 2 * d * sizeof(float);
  return p;
}

}  // namespace

hipError_t launch_embed_rows(const void *table, bool bf16, const int32_t *ids, int n, int vocab, int d, float scale, void *out, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  const int vecs = d / (bf16 ? 8 : 4);
  int lg = 3;
  while (lg < 8 && (4 << lg) < vecs) ++lg;
  const int rows = 256 >> lg;
  const dim3 grid((unsigned)std::min<long long>(((long long)n + rows - 1) / rows, 1 << 22));
  if (bf16) hipLaunchKernelGGL((embed_rows_kernel<true>), grid, dim3(256), 0, st, table, ids, n, vocab, d, scale, out, lg);
  else hipLaunchKernelGGL((embed_rows_kernel<false>), grid, dim3(256), 0, st, table, ids, n, vocab, d, scale, out, lg);
  return hipGetLastError();
}

size_t embed_grad_scratch_bytes(int n, int vocab, int d) { return plan_grad(n, vocab, d).bytes; }

hipError_t launch_embed_grad(const int32_t *ids, int n, int vocab, int d, const float *dx, float scale, float *d_table, bool accumulate, void *scratch,
                             hipStream_t st) {
  if (n <= 0 && accumulate) return hipSuccess;
  const GradPlan p = plan_grad(n, vocab, d);
  int *starts = (int *)scratch;
  Placed *order = (Placed *)((char *)scratch + p.order_at);
  float *aside = (float *)((char *)scratch + p.aside_at);
  const int keys = 1 << p.lg_keys;
  hipLaunchKernelGGL(embed_order_kernel, dim3(std::min((vocab + keys - 1) / keys, 1 << 20)), dim3(64 * ORDER_WAVES), 0, st, ids, n, vocab, p.lg_keys, starts, order);
  const long long units = (p.windows + (accumulate ? 0 : (vocab + ZERO_ROWS - 1) / ZERO_ROWS)) * p.strips;
  const dim3 grid((unsigned)std::min<long long>((units + 3) / 4, 1 << 22));
  auto *sum = p.nv == 4 ? (accumulate ? embed_sum_kernel<4, true> : embed_sum_kernel<4, false>)
              : p.nv == 2 ? (accumulate ? embed_sum_kernel<2, true> : embed_sum_kernel<2, false>)
                          : (accumulate ? embed_sum_kernel<1, true> : embed_sum_kernel<1, false>);
  hipLaunchKernelGGL(sum, grid, dim3(256), 0, st, starts, order, dx, vocab, d, scale, d_table, aside, p.window, p.windows, p.strips);
  if (p.windows > 1) {
    const int strips = (d + 1023) / 1024;
    const dim3 joins((unsigned)std::min<long long>(p.windows * strips, 1 << 22));
    auto *join = accumulate ? embed_join_kernel<true> : embed_join_kernel<false>;
    hipLaunchKernelGGL(join, joins, dim3(256), 0, st, starts, order, vocab, d, scale, d_table, aside, p.window, p.windows, strips);
  }
  return hipGetLastError();
}
