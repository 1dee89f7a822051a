// Attention of rows of queries over the 4-bit paged cache of their request.
//
//   x_t = scale q . k_t,  p_t = exp(x_t - max x) / sum exp(x - max x),  out = sum_t p_t v_t       (t <= context + number of the row)
//
// A wave takes 16 rows (query rows x query heads of one kv head) and, 64 tokens a turn, forms the transposed products
//   S^T [token, row] = K Q^T   and   O^T [channel, row] += V^T P^T
// with 16x16x32 MFMAs, so that a row's maximum, sum and rescaling stay in one lane of each quarter of the wave and P needs no movement at all: lane
// (i, g) = (lane % 16, lane / 16) holds row i and, with the tokens of the four S^T tiles chosen as 16 (i / 4) + 4 j + i % 4, the probabilities of tokens 16 g .. 16 g + 15,
// which is the order in which a transposing LDS read hands out 16 tokens of a channel of V.  K: a lane's elements (32 of a 128-wide head, 16 of a 64-wide one)
// lie in one group, so its scale goes into the conversion to bf16.  V: the scale belongs to a token, which is the reduction index, so it goes into P, once
// for every 32 channels.  Both conversions are exact; P is rounded to bf16 (half a step, 2^-9 of each term) for bf16 rows and split into three
// terms (24 bits) for fp32 rows, as q is.  Sums, maxima and the output before its rounding are fp32.
#include "kernels.h"
#include "kv4.h"

#include <algorithm>

namespace {

typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr int WAVES = 4, ROWS = 16, TURN = 64;     // waves a block, rows a wave, tokens a turn of a wave
constexpr float LOG2E = 1.4426950408889634f;

// Where the rows of a block come from: request, kv head, rows m0 .. m1 - 1 of the n * group rows of the request at this kv head (row m = query m / group, head m % group).
struct Rows {
  int req, kvh, row0, n, ctx, m0, m1;
};
__device__ __forceinline__ Rows rows_of(const Kv4Attention &a, int req, int kvh, int tile) {
  Rows w;
  w.req = req;
  w.kvh = kvh;
  w.row0 = req;
  w.n = 1;
  if (a.q_offsets) {
    const int b = min(max(a.q_offsets[req], 0), a.n_rows), e = min(max(a.q_offsets[req + 1], 0), a.n_rows);
    w.row0 = b;
    w.n = min(max(e - b, 0), a.max_rows);
  }
  const int room = (int)min((long long)a.max_blocks << a.c.bshift, (long long)INT32_MAX);
  w.ctx = min(max(a.lens[(size_t)req * a.len_heads + (a.len_heads > 1 ? kvh : 0)], 0), a.max_context);
  w.ctx = min(w.ctx, room - w.n);                    // (below 0 where the table has no room: then some rows see nothing)
  w.m0 = tile * ROWS;
  w.m1 = min(w.m0 + ROWS, w.n * a.group);
  return w;
}

// Q as MFMA operand: lane (i, g) holds row i, elements g HD / 4 + 8 s .. + 7 of step s, in TERMS bf16 terms.
template <int HD, int TERMS>
__device__ __forceinline__ void load_q(const Kv4Attention &a, const Rows &w, int i, int g, bf16x8_t (&q)[TERMS][HD / 32]) {
  const int m = w.m0 + i;
  const bool ok = m < w.m1;
  const int mc = ok ? m : w.m0;
  const size_t o = (size_t)(w.row0 + mc / a.group) * a.ld_q + (size_t)(w.kvh * a.group + mc % a.group) * HD + g * (HD / 4);
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
    if constexpr (TERMS == 1) {
      q[0][s] = *(const bf16x8_t *)((const bf16_t *)a.q + o + 8 * s);
    } else {
      const float4 u = *(const float4 *)((const float *)a.q + o + 8 * s), v = *((const float4 *)((const float *)a.q + o + 8 * s) + 1);
      float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        uint32_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r[e] = cvt_pk_bf16(f[2 * e], f[2 * e + 1]);
          f[2 * e] -= __uint_as_float(r[e] << 16);
          f[2 * e + 1] -= __uint_as_float(r[e] & 0xffff0000u);
        }
        q[t][s] = __builtin_bit_cast(bf16x8_t, make_uint4(r[0], r[1], r[2], r[3]));
      }
    }
  }
}

// Index of a token of this request and head, and whether its block exists; else index 0, whose bytes are read and not used.
__device__ __forceinline__ uint32_t token_of(const Kv4Cache &c, const int32_t *table, int kvh, int t, int end, bool &ok) {
  ok = t < end;
  const int blk = ok ? table[t >> c.bshift] : -1;
  ok = blk >= 0 && (uint32_t)blk < c.num_blocks;
  return ok ? (((uint32_t)blk * c.Hkv + kvh) << c.bshift) + (t & ((1 << c.bshift) - 1)) : 0u;
}

// Codes of one lane for one S^T tile: HD / 4 elements.
template <int HD> struct KCodes { uint32_t w[HD / 32]; };
template <int HD>
__device__ __forceinline__ KCodes<HD> load_k(const Kv4Cache &c, uint32_t token, int g) {
  KCodes<HD> r;
  if constexpr (HD == 128) {
    const uint4 u = *(const uint4 *)(c.k + (size_t)token * 64 + g * 16);
    r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
  } else {
    const uint2 u = *(const uint2 *)(c.k + (size_t)token * 32 + g * 8);
    r.w[0] = u.x; r.w[1] = u.y;
  }
  return r;
}

template <int HD, int TERMS>
__global__ __launch_bounds__(64 * WAVES) void kv4_attention_kernel(Kv4Attention a, int tiles, int chunk, int nsplit, float *__restrict__ partial, float2 *__restrict__ stats) {
  constexpr int NS = HD / 32, NG = HD / 32, CT = HD / 16;      // MFMA steps along the head, scale groups, channel tiles
  constexpr int VB = HD / 2, VROW = VB + 16;                   // bytes of a token of V; padded in LDS, so that 16 tokens' reads of one channel tile meet 16 different banks
  constexpr int CPT = VB / 16;                                 // 16-byte chunks of a token of V
  constexpr int OROW = HD + 4;
  constexpr int SM = WAVES * TURN * VROW > WAVES * ROWS * (OROW + 2) * 4 ? WAVES * TURN * VROW : WAVES * ROWS * (OROW + 2) * 4;
  __shared__ __align__(16) unsigned char sm[SM];
  const int kvh = blockIdx.x / tiles, tile = blockIdx.x - kvh * tiles, split = blockIdx.y;
  const Rows w = rows_of(a, blockIdx.z, kvh, tile);
  if (w.m0 >= w.m1) return;
  const int end = w.ctx + (w.m1 - 1) / a.group + 1;            // tokens that the last row sees
  const int c0 = split * chunk, c1 = min(end, c0 + chunk);
  if (c0 >= end && split > 0) return;                          // (the first one writes the rows that see nothing)
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, g = lane >> 4;
  const int32_t *table = a.tables + (size_t)w.req * a.max_blocks;
  const int limit = w.ctx + min(w.m0 + i, w.m1 - 1) / a.group + 1;       // tokens that this lane's row sees
  const int all = w.ctx + w.m0 / a.group + 1;                  // tokens that every row sees
  const float sc = a.scale * LOG2E;

  bf16x8_t q[TERMS][NS];
  load_q<HD, TERMS>(a, w, i, g, q);
  f32x4_t o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  unsigned char *vs = sm + wave * TURN * VROW;

  for (int t0 = c0 + wave * TURN; t0 < c1; t0 += WAVES * TURN) {
    // K and its scales; S^T
    f32x4_t s[4];
    bool whole = t0 + TURN <= min(all, c1);
    uint64_t there[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bool ok;
      const uint32_t tok = token_of(a.c, table, kvh, t0 + 16 * (i >> 2) + 4 * j + (i & 3), c1, ok);
      there[j] = __ballot(ok);
      whole = whole && there[j] == ~0ull;
      const KCodes<HD> k = load_k<HD>(a.c, tok, g);
      const float ks = kv4::scale_value(a.c.k_scale[(size_t)tok * NG + g * (HD / 4) / kv4::GROUP]);
      s[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8_t kf = kv4::decode8(k.w[st], ks);
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[t][st], s[j], 0, 0, 0);
      }
    }
    // V into LDS, token by token
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int u = 0; u < CPT; ++u) {
      const int ch = u * 64 + lane, t = ch / CPT, c = ch % CPT;
      bool ok;
      const uint32_t tok = token_of(a.c, table, kvh, t0 + t, c1, ok);
      *(uint4 *)(vs + t * VROW + c * 16) = *(const uint4 *)(a.c.v + (size_t)tok * VB + c * 16);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    // probabilities of tokens t0 + 16 g + 4 j + r
    float p[4][4], mx = m;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[j][r] = s[j][r] * sc;
        if (!whole) p[j][r] = t0 + 16 * g + 4 * j + r < limit && ((there[j] >> (4 * g + r)) & 1) ? p[j][r] : -INFINITY;
        mx = fmaxf(mx, p[j][r]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float base = mx == -INFINITY ? 0.f : mx, alpha = exp2f(m - base);      // (m = -inf: 0)
    m = mx;
    l *= alpha;
#pragma unroll
    for (int c = 0; c < CT; ++c) o[c] *= alpha;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[j][r] = exp2f(p[j][r] - base);
        l += p[j][r];
      }
    // V's scales of this lane's 16 tokens
    uint32_t vsc[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      bool ok;
      const uint32_t tok = token_of(a.c, table, kvh, t0 + 16 * g + t, c1, ok);
      if constexpr (HD == 128) vsc[t] = ((const uint32_t *)a.c.v_scale)[tok];
      else vsc[t] = ((const uint16_t *)a.c.v_scale)[tok];
    }
#pragma unroll
    for (int gr = 0; gr < NG; ++gr) {
      bf16x8_t pf[TERMS][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int t = 8 * h + e;
          const float x = p[t >> 2][t & 3];
          f[e] = x * kv4::scale_value((vsc[t] >> (8 * gr)) & 255u);
          if (!whole) f[e] = x == 0.f ? 0.f : f[e];            // a masked token adds nothing, whatever its scale is
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
          uint32_t r[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            r[e] = cvt_pk_bf16(f[2 * e], f[2 * e + 1]);
            if (t + 1 < TERMS) {
              f[2 * e] -= __uint_as_float(r[e] << 16);
              f[2 * e + 1] -= __uint_as_float(r[e] & 0xffff0000u);
            }
          }
          pf[t][h] = __builtin_bit_cast(bf16x8_t, make_uint4(r[0], r[1], r[2], r[3]));
        }
      }
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const int c = gr * 2 + cc;
        const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(vs + (16 * g + i) * VROW + c * 8));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8_t vf = kv4::decode8((uint32_t)v[h], 1.f);
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t][h], o[c], 0, 0, 0);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  // the waves' states -> one
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();
  float *so = (float *)sm, *sml = so + WAVES * ROWS * OROW;
#pragma unroll
  for (int c = 0; c < CT; ++c) *(f32x4_t *)(so + (wave * ROWS + i) * OROW + 16 * c + 4 * g) = o[c];
  if (g == 0) {
    sml[(wave * ROWS + i) * 2] = m;
    sml[(wave * ROWS + i) * 2 + 1] = l;
  }
  __syncthreads();
  for (int idx = tid; idx < ROWS * HD; idx += 64 * WAVES) {
    const int row = idx / HD, e = idx % HD, mr = w.m0 + row;
    if (mr >= w.m1) break;
    float mn = -INFINITY, ls = 0.f, as = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) mn = fmaxf(mn, sml[(k * ROWS + row) * 2]);
    const float base = mn == -INFINITY ? 0.f : mn;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const float f = exp2f(sml[(k * ROWS + row) * 2] - base);
      ls += sml[(k * ROWS + row) * 2 + 1] * f;
      as += so[(k * ROWS + row) * OROW + e] * f;
    }
    const size_t r = w.row0 + mr / a.group;
    const int head = kvh * a.group + mr % a.group, Hq = a.c.Hkv * a.group;
    const size_t at = ((size_t)w.req * a.max_rows + mr / a.group) * Hq + head;           // in the workspace
    if (nsplit == 1) {
      const float v = ls == 0.f ? 0.f : as / ls;
      if constexpr (TERMS == 1) ((bf16_t *)a.out)[r * a.ld_out + (size_t)head * HD + e] = f2bf(v);
      else ((float *)a.out)[r * a.ld_out + (size_t)head * HD + e] = v;
      if (e == 0) {
        if (a.lse) a.lse[r * Hq + head] = ls == 0.f ? -INFINITY : (mn + log2f(ls)) / LOG2E;
        if (stats) stats[at] = make_float2(base, ls);
      }
    } else {
      float *dst = partial + (at * nsplit + split) * (HD + 2);
      dst[e] = as;
      if (e == 0) { dst[HD] = mn; dst[HD + 1] = ls; }
    }
  }
}

// Joins the splits of a row and head, in order.
template <int HD, bool BF16>
__global__ __launch_bounds__(HD) void kv4_join_kernel(Kv4Attention a, int chunk, int nsplit, const float *__restrict__ partial, float2 *__restrict__ stats) {
  const int Hq = a.c.Hkv * a.group, head = blockIdx.x, e = threadIdx.x;
  const Rows w = rows_of(a, blockIdx.z, head / a.group, 0);
  const int k = blockIdx.y;
  if (k >= w.n) return;
  const size_t r = w.row0 + k, at = ((size_t)w.req * a.max_rows + k) * Hq + head;
  // the splits that the row's tile had: by the last row of its tile
  const int m = k * a.group + head % a.group, m1 = min((m / ROWS + 1) * ROWS, w.n * a.group);
  const int ns = max(1, min(nsplit, (w.ctx + (m1 - 1) / a.group + 1 + chunk - 1) / chunk));
  const float *src = partial + at * nsplit * (HD + 2);
  float mn = -INFINITY, ls = 0.f, as = 0.f;
  for (int s = 0; s < ns; ++s) mn = fmaxf(mn, src[s * (HD + 2) + HD]);
  const float base = mn == -INFINITY ? 0.f : mn;
  for (int s = 0; s < ns; ++s) {
    const float f = exp2f(src[s * (HD + 2) + HD] - base);
    ls += src[s * (HD + 2) + HD + 1] * f;
    as += src[s * (HD + 2) + e] * f;
  }
  const float v = ls == 0.f ? 0.f : as / ls;
  if constexpr (BF16) ((bf16_t *)a.out)[r * a.ld_out + (size_t)head * HD + e] = f2bf(v);
  else ((float *)a.out)[r * a.ld_out + (size_t)head * HD + e] = v;
  if (e == 0) {
    if (a.lse) a.lse[r * Hq + head] = ls == 0.f ? -INFINITY : (mn + log2f(ls)) / LOG2E;
    if (stats) stats[at] = make_float2(base, ls);
  }
}

// Adds every token's probabilities, summed over the rows of its request and the query heads of its kv head, to its weight.  A wave takes 64 tokens and goes over all
// rows, so a token of one request is added to once (blocks that requests share: once a request, by atomics).
template <int HD, int TERMS>
__global__ __launch_bounds__(64 * WAVES) void kv4_weight_kernel(Kv4Attention a, const float2 *__restrict__ stats) {
  constexpr int NS = HD / 32, NG = HD / 32;
  const int kvh = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  Rows w = rows_of(a, blockIdx.z, kvh, 0);
  const int end = w.ctx + w.n, t0 = (blockIdx.x * WAVES + wave) * TURN, Hq = a.c.Hkv * a.group;
  if (w.n == 0 || t0 >= end) return;
  const int32_t *table = a.tables + (size_t)w.req * a.max_blocks;
  const float sc = a.scale * LOG2E;
  bf16x8_t kf[4][NS];
  uint32_t tok[4];
  bool ok[4];
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    tok[j] = token_of(a.c, table, kvh, t0 + 16 * j + i, end, ok[j]);
    const KCodes<HD> k = load_k<HD>(a.c, tok[j], g);
    const float ks = kv4::scale_value(a.c.k_scale[(size_t)tok[j] * NG + g * (HD / 4) / kv4::GROUP]);
#pragma unroll
    for (int st = 0; st < NS; ++st) kf[j][st] = kv4::decode8(k.w[st], ks);
  }
  const int first = max(0, t0 - w.ctx);              // queries before it see none of these tokens
  for (w.m0 = first * a.group / ROWS * ROWS; w.m0 < w.n * a.group; w.m0 += ROWS) {
    w.m1 = min(w.m0 + ROWS, w.n * a.group);
    bf16x8_t q[TERMS][NS];
    load_q<HD, TERMS>(a, w, i, g, q);
    float2 ml[4];
    int limit[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int m = w.m0 + 4 * g + r, mc = min(m, w.m1 - 1);
      ml[r] = stats[((size_t)w.req * a.max_rows + mc / a.group) * Hq + kvh * a.group + mc % a.group];
      limit[r] = m < w.m1 ? w.ctx + mc / a.group + 1 : 0;
      ml[r].y = 1.f / ml[r].y;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t][st], kf[j][st], s, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[j] += ok[j] && t0 + 16 * j + i < limit[r] ? exp2f(s[r] * sc - ml[r].x) * ml[r].y : 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    sum[j] += __shfl_xor(sum[j], 16, 64);
    sum[j] += __shfl_xor(sum[j], 32, 64);
    if (g == j && ok[j]) unsafeAtomicAdd(a.c.weight + tok[j], sum[j]);
  }
}

// Tokens of a block: enough blocks to fill the chip, not below a turn of all its waves.
int chunk_tokens(int n_req, int tiles, int Hkv, int tokens) {
  int chunk = 4096;
  while (chunk > 256 && (long long)n_req * Hkv * tiles * cdiv(tokens, chunk) < 1024) chunk /= 2;
  return chunk;
}

}  // namespace

// Partial states of the splits and (base, sum) of every row and head.
size_t kv4_attention_scratch_bytes(int n_req, int max_rows, int max_context, int Hq, int Hkv, int hd) {
  const int tokens = max_context + max_rows, tiles = cdiv(max_rows * (Hq / Hkv), ROWS);
  const int nsplit = cdiv(tokens, chunk_tokens(n_req, tiles, Hkv, tokens));
  const size_t heads = (size_t)n_req * max_rows * Hq;
  return align_up(heads * sizeof(float2), 256) + (nsplit > 1 ? heads * nsplit * (hd + 2) * sizeof(float) : 0);
}

hipError_t launch_kv4_attention(const Kv4Attention &a, bool bf16, void *scratch, hipStream_t st) {
  if (a.n_req <= 0 || a.n_rows <= 0) return hipSuccess;
  const int Hkv = a.c.Hkv, Hq = Hkv * a.group, tokens = a.max_context + a.max_rows, tiles = cdiv(a.max_rows * a.group, ROWS);
  const int chunk = chunk_tokens(a.n_req, tiles, Hkv, tokens), nsplit = cdiv(tokens, chunk);
  float2 *stats = a.add_weight ? (float2 *)scratch : nullptr;
  float *partial = (float *)((char *)scratch + align_up((size_t)a.n_req * a.max_rows * Hq * sizeof(float2), 256));
  auto main = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(Hkv * tiles, nsplit, a.n_req), dim3(64 * WAVES), 0, st, a, tiles, chunk, nsplit, partial, stats); };
  auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(Hq, a.max_rows, a.n_req), dim3(a.c.hd), 0, st, a, chunk, nsplit, partial, stats); };
  auto weight = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(cdiv(tokens, TURN * WAVES), Hkv, a.n_req), dim3(64 * WAVES), 0, st, a, stats); };
  if (a.c.hd == 128) bf16 ? main(kv4_attention_kernel<128, 1>) : main(kv4_attention_kernel<128, 3>);
  else bf16 ? main(kv4_attention_kernel<64, 1>) : main(kv4_attention_kernel<64, 3>);
  if (nsplit > 1) {
    if (a.c.hd == 128) bf16 ? join(kv4_join_kernel<128, true>) : join(kv4_join_kernel<128, false>);
    else bf16 ? join(kv4_join_kernel<64, true>) : join(kv4_join_kernel<64, false>);
  }
  if (a.add_weight) {
    if (a.c.hd == 128) bf16 ? weight(kv4_weight_kernel<128, 1>) : weight(kv4_weight_kernel<128, 3>);
    else bf16 ? weight(kv4_weight_kernel<64, 1>) : weight(kv4_weight_kernel<64, 3>);
  }
  return hipGetLastError();
}
