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
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr int WAVES = 4, ROWS = 16, TURN = 64;     // waves a block, rows a wave, tokens a turn of a wave
constexpr float LOG2E = 1.4426950408889634f;

// Where the rows of a block come from: request, kv head, rows m0 .. m1 - 1 of the n * group rows of the request at this kv head (row m = query m / group, head m % group).
struct Rows {
  int req, kvh, row0, n, ctx, m0, m1;
};
template <int N>
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
  w.m0 = tile * N;
  w.m1 = min(w.m0 + N, w.n * a.group);
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

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

// Codes of one lane for one S^T tile: HD / 4 elements.  (The cache is read once and should not displace what else is in the caches: 521 -> 502 us for 128
// requests of 2048 - 8192 tokens.)
template <int HD> struct KCodes { uint32_t w[HD / 32]; };
template <int HD>
__device__ __forceinline__ KCodes<HD> load_k(const unsigned char *p) {
  KCodes<HD> r;
  if constexpr (HD == 128) {
    const u32x4_t u = __builtin_nontemporal_load((const u32x4_t *)p);
    r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
  } else {
    const u32x2_t u = __builtin_nontemporal_load((const u32x2_t *)p);
    r.w[0] = u.x; r.w[1] = u.y;
  }
  return r;
}

// What a lane holds of a turn's 64 tokens: codes and scale of token 16 j + i for S^T tile j, its 16-byte pieces of V (token by token), the scales of
// V of tokens 16 j + 4 g .. + 3, and which of tokens 16 j + 4 g + r exist.
template <int HD>
struct Turn {
  KCodes<HD> k[4];
  uint32_t ks[4];
  u32x4_t v[HD / 32];
  uint32_t vs[4][HD / 32];
  uint32_t there;                                    // bit 4 j + r
};

// Block ids of the four runs of 16 tokens of a turn (blocks of 16 tokens or more): lane l has that of run l % 4.
__device__ __forceinline__ int run_entry(const Kv4Cache &c, const int32_t *table, int t0, int end, int lane) {
  const int t = t0 + 16 * (lane & 3);
  return t < end ? table[t >> c.bshift] : -1;
}

template <int HD, bool RUNS>
__device__ __forceinline__ void load_turn(const Kv4Cache &c, const int32_t *table, int entry, int kvh, int t0, int end, int lane, Turn<HD> &u) {
  constexpr int NG = HD / 32, VB = HD / 2, CPT = VB / 16;
  const int i = lane & 15, g = lane >> 4;
  if constexpr (RUNS) {
    uint32_t base[4];                                // uniform
    u.there = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int blk = __builtin_amdgcn_readlane(entry, j);
      const bool ok = blk >= 0 && (uint32_t)blk < c.num_blocks;
      const uint32_t at = (((uint32_t)blk * c.Hkv + kvh) << c.bshift) + ((t0 + 16 * j) & ((1 << c.bshift) - 1));
      base[j] = ok ? at : 0u;
      u.there |= ok ? 15u << (4 * j) : 0u;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) u.k[j] = load_k<HD>(c.k + (size_t)base[j] * VB + (i * VB + g * (VB / 4)));
#pragma unroll
    for (int j = 0; j < 4; ++j) u.ks[j] = (c.k_scale + (size_t)base[j] * NG)[i * NG + g * (HD / 4) / kv4::GROUP];
#pragma unroll
    for (int p = 0; p < CPT; ++p) {
      if constexpr (HD == 128) u.v[p] = __builtin_nontemporal_load((const u32x4_t *)(c.v + (size_t)base[p] * VB + lane * 16));
      else {
        const uint32_t b0 = base[2 * p], b1 = base[2 * p + 1];   // (read before the choice: an index that differs between lanes would put the array into memory)
        u.v[p] = __builtin_nontemporal_load((const u32x4_t *)(c.v + (size_t)(lane < 32 ? b0 : b1) * VB + (lane & 31) * 16));
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned char *s = c.v_scale + (size_t)base[j] * NG + 4 * g * NG;
      if constexpr (HD == 128) {
        const uint4 w = *(const uint4 *)s;
        u.vs[j][0] = w.x; u.vs[j][1] = w.y; u.vs[j][2] = w.z; u.vs[j][3] = w.w;
      } else {
        const uint2 w = *(const uint2 *)s;
        u.vs[j][0] = w.x; u.vs[j][1] = w.y;
      }
    }
  } else {
    bool ok;
    u.there = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t tok = token_of(c, table, kvh, t0 + 16 * j + i, end, ok);
      const uint64_t all = __ballot(ok);               // (tile row 4 g + r is token 4 g + r of the run)
      u.there |= (uint32_t)((all >> (4 * g)) & 15) << (4 * j);
      u.k[j] = load_k<HD>(c.k + (size_t)tok * VB + g * (VB / 4));
      u.ks[j] = c.k_scale[(size_t)tok * NG + g * (HD / 4) / kv4::GROUP];
    }
#pragma unroll
    for (int p = 0; p < CPT; ++p) u.v[p] = *(const u32x4_t *)(c.v + (size_t)token_of(c, table, kvh, t0 + (p * 64 + lane) / CPT, end, ok) * VB + lane % CPT * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint32_t tok = token_of(c, table, kvh, t0 + 16 * j + 4 * g + r, end, ok);
        if constexpr (HD == 128) w[r] = ((const uint32_t *)c.v_scale)[tok];
        else w[r] = ((const uint16_t *)c.v_scale)[tok];
      }
      if constexpr (HD == 128) { u.vs[j][0] = w[0]; u.vs[j][1] = w[1]; u.vs[j][2] = w[2]; u.vs[j][3] = w[3]; }
      else { u.vs[j][0] = w[0] | w[1] << 16; u.vs[j][1] = w[2] | w[3] << 16; }
    }
  }
}
// Scale of group gr of the token of tile j, register r.
template <int HD>
__device__ __forceinline__ float v_scale_of(const Turn<HD> &u, int j, int r, int gr) {
  if constexpr (HD == 128) return kv4::scale_value((u.vs[j][r] >> (8 * gr)) & 255u);
  else return kv4::scale_value((u.vs[j][r >> 1] >> (16 * (r & 1) + 8 * gr)) & 255u);
}

// Eight probabilities as MFMA operand in TERMS bf16 terms.
template <int TERMS>
__device__ __forceinline__ void split8(float (&f)[8], bf16x8_t (&out)[TERMS]) {
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
    out[t] = __builtin_bit_cast(bf16x8_t, make_uint4(r[0], r[1], r[2], r[3]));
  }
}

// Where a call's workspace lies: partial sums [rows, splits, HD] and (maximum, sum) [rows, splits] of the splits, and log2 sum exp2 [rows] of rows that are done.
// A row is (request * max_rows + number of the row) * query heads + head.
struct States {
  float *acc;
  float2 *ml;
  float *lse2;
  int nsplit, chunk, tile_rows;      // splits; tokens a split; rows a tile of the first launch
};
__device__ __forceinline__ size_t row_id(const Kv4Attention &a, int req, int k, int head) { return ((size_t)req * a.max_rows + k) * (a.c.Hkv * a.group) + head; }
// Splits that the tile of row k of this head had, by the tile's last row.
__device__ __forceinline__ int splits_of(const Kv4Attention &a, const States &x, const Rows &w, int k, int head) {
  const int m = k * a.group + head % a.group, m1 = min((m / x.tile_rows + 1) * x.tile_rows, w.n * a.group);
  return max(1, min(x.nsplit, (w.ctx + (m1 - 1) / a.group + 1 + x.chunk - 1) / x.chunk));
}

// REP: copies of each row among the 16 columns of a tile.  P is scaled for every 32 channels anew, so few rows (16 / REP) are repeated, copy c scales for groups c, c + REP, ..,
// and of an output tile the columns of the copy that scaled for its group are the rows.
template <int HD, int TERMS, int REP, bool RUNS>
__global__ __launch_bounds__(64 * WAVES, TERMS == 1 && HD == 64 ? 4 : 2) void kv4_attention_kernel(Kv4Attention a, States x, int tiles) {
  constexpr int NS = HD / 32, NG = HD / 32, CT = HD / 16;      // MFMA steps along the head, scale groups, channel tiles
  constexpr int VB = HD / 2, VROW = VB + 16;                   // bytes of a token of V; padded in LDS, so that 16 tokens' reads of one channel tile meet 16 different banks
  constexpr int CPT = VB / 16;                                 // 16-byte pieces of a token of V
  constexpr int NR = ROWS / REP, OROW = HD + 4;
  constexpr int SM = WAVES * TURN * VROW > WAVES * NR * (OROW + 2) * 4 ? WAVES * TURN * VROW : WAVES * NR * (OROW + 2) * 4;
  __shared__ __align__(16) unsigned char sm[SM];
  const int kvh = blockIdx.x / tiles, tile = blockIdx.x - kvh * tiles, split = blockIdx.y;
  const Rows w = rows_of<NR>(a, blockIdx.z, kvh, tile);
  if (w.m0 >= w.m1) return;
  const int end = w.ctx + (w.m1 - 1) / a.group + 1;            // tokens that the last row sees
  const int c0 = split * x.chunk, c1 = min(end, c0 + x.chunk);
  if (c0 >= end && split > 0) return;                          // (the first one writes the rows that see nothing)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4, copy = i / NR;
  const int32_t *table = a.tables + (size_t)w.req * a.max_blocks;
  const int limit = w.ctx + min(w.m0 + i % NR, w.m1 - 1) / a.group + 1;  // tokens that this lane's row sees
  const int all = w.ctx + w.m0 / a.group + 1;                  // tokens that every row sees
  const float sc = a.scale * LOG2E;

  int t0 = c0 + wave * TURN;
  constexpr int STEP = WAVES * TURN;
  int entry = 0;
  if constexpr (RUNS) entry = run_entry(a.c, table, t0, c1, lane);
  bf16x8_t q[TERMS][NS];
  load_q<HD, TERMS>(a, w, i % NR, g, q);
  f32x4_t o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  unsigned char *vs = sm + wave * TURN * VROW;
  const unsigned char *vread = vs + (16 * (i >> 2) + 4 * g + (i & 3)) * VROW;          // the token whose 16 channels this lane brings to a transposing read
  unsigned char *vwrite = vs + lane / CPT * VROW + lane % CPT * 16;

  Turn<HD> u;
  if (t0 < c1) {
    load_turn<HD, RUNS>(a.c, table, entry, w.kvh, t0, c1, lane, u);
    if constexpr (RUNS) entry = run_entry(a.c, table, t0 + STEP, c1, lane);
  }
  for (; t0 < c1; t0 += STEP) {
#pragma unroll
    for (int p = 0; p < CPT; ++p) *(u32x4_t *)(vwrite + p * (64 / CPT) * VROW) = u.v[p];
    f32x4_t s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float ks = kv4::scale_value(u.ks[j]);
      s[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8_t kf = kv4::decode8(u.k[j].w[st], ks);
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[t][st], s[j], 0, 0, 0);
      }
    }
    const Turn<HD> n = u;                              // its scales of V and what exists of it
    if (t0 + STEP < c1) {                              // the next turn's loads fly while this one's probabilities and products are formed
      load_turn<HD, RUNS>(a.c, table, entry, w.kvh, t0 + STEP, c1, lane, u);
      if constexpr (RUNS) entry = run_entry(a.c, table, t0 + 2 * STEP, c1, lane);
    }
    // probabilities of tokens t0 + 16 j + 4 g + r
    const bool whole = t0 + TURN <= min(all, c1) && __all(n.there == 0xffffu);
    float mx = m;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[j][r] *= sc;
    if (!whole) {
      const int last = min(limit, c1) - t0 - 4 * g;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[j][r] = 16 * j + r < last && ((n.there >> (4 * j + r)) & 1) ? s[j][r] : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[j][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float base = mx == -INFINITY ? 0.f : mx;
    if (__any(mx != m)) {                              // (a row of NaN has -inf or its last finite maximum here, and stays NaN through its sum)
      const float alpha = __builtin_amdgcn_exp2f(m - base);      // (m = -inf: 0)
      m = mx;
      l *= alpha;
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c] *= alpha;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[j][r] = __builtin_amdgcn_exp2f(s[j][r] - base);
        l += s[j][r];
      }
#pragma unroll
    for (int pass = 0; pass < NG / REP; ++pass) {
      bf16x8_t pf[2][TERMS];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = 2 * h + (e >> 2), r = e & 3;
          f[e] = s[j][r] * v_scale_of<HD>(n, j, r, REP == 1 ? pass : pass * REP + copy);
        }
        if (!whole) {                                  // a masked token adds nothing, whatever its scale is
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = s[2 * h + (e >> 2)][e & 3] == 0.f ? 0.f : f[e];
        }
        split8<TERMS>(f, pf[h]);
      }
#pragma unroll
      for (int cc = 0; cc < 2 * REP; ++cc) {
        const int c = pass * 2 * REP + cc;
        const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(vread + c * 8));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8_t vf = kv4::decode8((uint32_t)v[h], 1.f);
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[h][t], o[c], 0, 0, 0);
        }
      }
    }
  }

  // the waves' states -> one
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();
  float *so = (float *)sm, *sml = so + WAVES * NR * OROW;
#pragma unroll
  for (int c = 0; c < CT; ++c)
    if (REP == 1 || c / 2 % REP == copy) *(f32x4_t *)(so + (wave * NR + i % NR) * OROW + 16 * c + 4 * g) = o[c];
  if (lane < NR) {
    sml[(wave * NR + i) * 2] = m;
    sml[(wave * NR + i) * 2 + 1] = l;
  }
  __syncthreads();
  for (int idx = tid; idx < NR * HD; idx += 64 * WAVES) {
    const int row = idx / HD, e = idx % HD, mr = w.m0 + row;
    if (mr >= w.m1) break;
    float mn = -INFINITY, ls = 0.f, as = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) mn = fmaxf(mn, sml[(k * NR + row) * 2]);
    const float base = mn == -INFINITY ? 0.f : mn;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      const float f = __builtin_amdgcn_exp2f(sml[(k * NR + row) * 2] - base);
      ls += sml[(k * NR + row) * 2 + 1] * f;
      as += so[(k * NR + row) * OROW + e] * f;
    }
    const size_t r = w.row0 + mr / a.group;
    const int head = kvh * a.group + mr % a.group, Hq = a.c.Hkv * a.group;
    const size_t at = row_id(a, w.req, mr / a.group, head);
    if (x.nsplit == 1) {
      const float v = ls == 0.f ? 0.f : as / ls;
      if constexpr (TERMS == 1) ((bf16_t *)a.out)[r * a.ld_out + (size_t)head * HD + e] = f2bf(v);
      else ((float *)a.out)[r * a.ld_out + (size_t)head * HD + e] = v;
      if (e == 0) {
        const float lse2 = ls == 0.f ? -INFINITY : mn + log2f(ls);
        if (a.lse) a.lse[r * Hq + head] = lse2 / LOG2E;
        if (a.add_weight) { x.ml[at] = make_float2(mn, ls); x.lse2[at] = lse2; }
      }
    } else {
      x.acc[(at * x.nsplit + split) * HD + e] = as;
      if (e == 0) x.ml[at * x.nsplit + split] = make_float2(mn, ls);
    }
  }
}

// Joins the splits of a row and head: `groups` teams of HD / 4 lanes (four channels each) take every groups-th split with a soft-max state of their own and are merged
// in order.  The time is the latency of the loads, so a team has those of IN_FLIGHT splits under way.
constexpr int IN_FLIGHT = 4;
template <int HD, bool BF16>
__device__ __forceinline__ void join_rows(const Kv4Attention &a, const States &x, int block, int groups, bool keep_lse2, float4 *so, float2 *sml) {
  constexpr int LANES = HD / 4;
  const int Hq = a.c.Hkv * a.group, team = threadIdx.x / LANES, e = threadIdx.x % LANES, grp = team % groups;
  const size_t at = (size_t)block * (64 * WAVES / LANES / groups) + team / groups, rows = (size_t)a.n_req * a.max_rows * Hq;
  const int head = (int)(at % Hq), k = (int)(at / Hq % a.max_rows), req = (int)(min(at, rows - 1) / Hq / a.max_rows);
  const Rows w = rows_of<1>(a, req, head / a.group, 0);
  const bool live = at < rows && k < w.n;
  const int ns = live ? splits_of(a, x, w, k, head) : 0;
  const float *acc = x.acc + at * x.nsplit * HD;
  const float2 *ml = x.ml + at * x.nsplit;
  float mn = -INFINITY, ls = 0.f;
  float4 as = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = grp; s0 < ns; s0 += IN_FLIGHT * groups) {
    float4 v[IN_FLIGHT];
    float2 y[IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) {
      const int s = min(s0 + u * groups, ns - 1);
      y[u] = ml[s];
      v[u] = ((const float4 *)(acc + (size_t)s * HD))[e];
    }
    float top = mn;
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) {
      if (s0 + u * groups >= ns) { y[u] = make_float2(-INFINITY, 0.f); v[u] = make_float4(0.f, 0.f, 0.f, 0.f); }
      top = fmaxf(top, y[u].x);
    }
    const float base = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(mn - base);
    mn = top;
    ls *= old;
    as.x *= old; as.y *= old; as.z *= old; as.w *= old;
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) {
      const float f = __builtin_amdgcn_exp2f(y[u].x - base);
      ls += y[u].y * f;
      as.x += v[u].x * f; as.y += v[u].y * f; as.z += v[u].z * f; as.w += v[u].w * f;
    }
  }
  if (groups > 1) {
    so[threadIdx.x] = as;
    if (e == 0) sml[team] = make_float2(mn, ls);
    __syncthreads();
    if (grp == 0) {
      for (int s = 1; s < groups; ++s) mn = fmaxf(mn, sml[team + s].x);
      const float base = mn == -INFINITY ? 0.f : mn;
      ls = 0.f;
      as = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < groups; ++s) {
        const float f = __builtin_amdgcn_exp2f(sml[team + s].x - base);
        const float4 v = so[threadIdx.x + s * LANES];
        ls += sml[team + s].y * f;
        as.x += v.x * f; as.y += v.y * f; as.z += v.z * f; as.w += v.w * f;
      }
    }
  }
  if (!live || grp) return;
  const float inv = ls == 0.f ? 0.f : 1.f / ls;
  const size_t r = w.row0 + k;
  const size_t to = r * a.ld_out + (size_t)head * HD + 4 * e;
  if constexpr (BF16) *(uint2 *)((bf16_t *)a.out + to) = make_uint2(cvt_pk_bf16(as.x * inv, as.y * inv), cvt_pk_bf16(as.z * inv, as.w * inv));
  else *(float4 *)((float *)a.out + to) = make_float4(as.x * inv, as.y * inv, as.z * inv, as.w * inv);
  if (e == 0) {
    const float lse2 = ls == 0.f ? -INFINITY : mn + log2f(ls);
    if (a.lse) a.lse[r * Hq + head] = lse2 / LOG2E;
    if (keep_lse2) x.lse2[at] = lse2;
  }
}

template <int HD, bool BF16>
__global__ __launch_bounds__(64 * WAVES) void kv4_join_kernel(Kv4Attention a, States x, int groups) {
  __shared__ float4 so[64 * WAVES];
  __shared__ float2 sml[64 * WAVES / (HD / 4)];
  join_rows<HD, BF16>(a, x, blockIdx.x, groups, a.add_weight, so, sml);
}

// Adds every token's probabilities, summed over the rows of its request and the query heads of its kv head, to its weight, from the product S = Q K^T formed again
// (lane (i, g) has token i of a tile of 16 and rows 4 g .. 4 g + 3) and the rows' log sums: 68 or 34 bytes of K a token again instead of 8 for every row.  A wave takes 64 tokens
// and all rows, so a request adds to a token once (blocks that requests share get one addition from each, by atomics).
// Here: requests of one tile of rows, whose log sums the block forms from the splits' states; the first `joins` blocks join the splits meanwhile.
template <int HD, int TERMS, bool RUNS>
__global__ __launch_bounds__(64 * WAVES) void kv4_weight_kernel(Kv4Attention a, States x, int joins, int groups, int pieces) {
  constexpr int NS = HD / 32;
  __shared__ float4 so[64 * WAVES];
  __shared__ float2 sml[64 * WAVES / (HD / 4)];
  __shared__ float slse[ROWS];
  if ((int)blockIdx.x < joins) {
    join_rows<HD, TERMS == 1>(a, x, blockIdx.x, groups, false, so, sml);
    return;
  }
  const int id = blockIdx.x - joins, kvh = id % a.c.Hkv, piece = id / a.c.Hkv % pieces, req = id / a.c.Hkv / pieces;
  const Rows w = rows_of<ROWS>(a, req, kvh, 0);
  const int end = w.ctx + w.n, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, g = lane >> 4;
  if (w.n == 0 || piece * WAVES * TURN >= end) return;
  const int t0 = (piece * WAVES + wave) * TURN;
  const int32_t *table = a.tables + (size_t)req * a.max_blocks;
  const float sc = a.scale * LOG2E;
  // keys
  KCodes<HD> k[4];
  uint32_t ks[4], tok[4], there = 0;
  if constexpr (RUNS) {
    const int entry = run_entry(a.c, table, t0, end, lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int blk = __builtin_amdgcn_readlane(entry, j);
      const bool ok = blk >= 0 && (uint32_t)blk < a.c.num_blocks;
      const uint32_t at = (((uint32_t)blk * a.c.Hkv + kvh) << a.c.bshift) + ((t0 + 16 * j) & ((1 << a.c.bshift) - 1)), base = ok ? at : 0u;
      there |= ok ? 1u << j : 0u;
      tok[j] = base + i;
      k[j] = load_k<HD>(a.c.k + (size_t)base * (HD / 2) + (i * (HD / 2) + g * (HD / 8)));
      ks[j] = (a.c.k_scale + (size_t)base * (HD / 32))[i * (HD / 32) + g * (HD / 4) / kv4::GROUP];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bool ok;
      tok[j] = token_of(a.c, table, kvh, t0 + 16 * j + i, end, ok);
      there |= ok ? 1u << j : 0u;
      k[j] = load_k<HD>(a.c.k + (size_t)tok[j] * (HD / 2) + g * (HD / 8));
      ks[j] = a.c.k_scale[(size_t)tok[j] * (HD / 32) + g * (HD / 4) / kv4::GROUP];
    }
  }
  bf16x8_t q[TERMS][NS];
  load_q<HD, TERMS>(a, w, i, g, q);
  // log sums of the rows: 16 threads a row
  {
    const int row = threadIdx.x / 16, mr = min(row, w.m1 - 1), kr = mr / a.group, head = kvh * a.group + mr % a.group;
    const float2 *ml = x.ml + row_id(a, req, kr, head) * x.nsplit;
    const int ns = splits_of(a, x, w, kr, head);
    float mn = -INFINITY, ls = 0.f;
    for (int s = threadIdx.x % 16; s < ns; s += 16) {
      const float2 y = ml[s];
      const float top = fmaxf(mn, y.x), base = top == -INFINITY ? 0.f : top;
      ls = ls * __builtin_amdgcn_exp2f(mn - base) + y.y * __builtin_amdgcn_exp2f(y.x - base);
      mn = top;
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const float m2 = __shfl_xor(mn, o, 64), l2 = __shfl_xor(ls, o, 64), top = fmaxf(mn, m2), base = top == -INFINITY ? 0.f : top;
      ls = ls * __builtin_amdgcn_exp2f(mn - base) + l2 * __builtin_amdgcn_exp2f(m2 - base);
      mn = top;
    }
    if (threadIdx.x % 16 == 0) slse[row] = mn + log2f(ls);
  }
  __syncthreads();
  float lse2[4];
  int last[4];                                       // tokens that the row sees
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int m = 4 * g + r;
    lse2[r] = slse[m];
    last[r] = m < w.m1 ? w.ctx + m / a.group + 1 : 0;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float scale = kv4::scale_value(ks[j]);
    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      const bf16x8_t kf = kv4::decode8(k[j].w[st], scale);
#pragma unroll
      for (int t = TERMS - 1; t >= 0; --t) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t][st], kf, s, 0, 0, 0);
    }
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += t0 + 16 * j + i < last[r] ? __builtin_amdgcn_exp2f(s[r] * sc - lse2[r]) : 0.f;
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (g == j && ((there >> j) & 1) && t0 + 16 * j + i < end) unsafeAtomicAdd(a.c.weight + tok[j], sum);
  }
}

// The same for more rows, whose log sums are there already.
template <int HD, int TERMS>
__global__ __launch_bounds__(64 * WAVES) void kv4_weight_rows_kernel(Kv4Attention a, States x) {
  constexpr int NS = HD / 32, NG = HD / 32;
  const int kvh = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  Rows w = rows_of<ROWS>(a, blockIdx.z, kvh, 0);
  const int end = w.ctx + w.n, t0 = (blockIdx.x * WAVES + wave) * TURN;
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
    const KCodes<HD> k = load_k<HD>(a.c.k + (size_t)tok[j] * (HD / 2) + g * (HD / 8));
    const float ks = kv4::scale_value(a.c.k_scale[(size_t)tok[j] * NG + g * (HD / 4) / kv4::GROUP]);
#pragma unroll
    for (int st = 0; st < NS; ++st) kf[j][st] = kv4::decode8(k.w[st], ks);
  }
  const int first = max(0, t0 - w.ctx);              // queries before it see none of these tokens
  for (w.m0 = first * a.group / ROWS * ROWS; w.m0 < w.n * a.group; w.m0 += ROWS) {
    w.m1 = min(w.m0 + ROWS, w.n * a.group);
    bf16x8_t q[TERMS][NS];
    load_q<HD, TERMS>(a, w, i, g, q);
    float lse2[4];
    int last[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int m = w.m0 + 4 * g + r, mc = min(m, w.m1 - 1);
      lse2[r] = x.lse2[row_id(a, w.req, mc / a.group, kvh * a.group + mc % a.group)];
      last[r] = m < w.m1 ? w.ctx + mc / a.group + 1 : 0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st)
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t][st], kf[j][st], s, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[j] += ok[j] && t0 + 16 * j + i < last[r] ? __builtin_amdgcn_exp2f(s[r] * sc - lse2[r]) : 0.f;
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
// Copies of a row in a tile: as many as rows and scale groups leave room for.
int copies(int rows, int hd) { return rows <= 4 && hd == 128 ? 4 : rows <= 8 ? 2 : 1; }

struct Plan {
  int rep, tiles, nsplit, chunk;
  size_t rows;
};
Plan plan_of(int n_req, int max_rows, int max_context, int Hq, int Hkv, int hd) {
  const int rows = max_rows * (Hq / Hkv), tokens = max_context + max_rows, rep = copies(rows, hd), tiles = cdiv(rows, ROWS / rep);
  const int chunk = chunk_tokens(n_req, tiles, Hkv, tokens);
  return {rep, tiles, cdiv(tokens, chunk), chunk, (size_t)n_req * max_rows * Hq};
}
// (acc is there for several splits only)
size_t ml_bytes(const Plan &p) { return align_up(p.rows * p.nsplit * sizeof(float2), 256); }
size_t lse_bytes(const Plan &p) { return align_up(p.rows * sizeof(float), 256); }

}  // namespace

size_t kv4_attention_scratch_bytes(int n_req, int max_rows, int max_context, int Hq, int Hkv, int hd) {
  const Plan p = plan_of(n_req, max_rows, max_context, Hq, Hkv, hd);
  return ml_bytes(p) + lse_bytes(p) + (p.nsplit > 1 ? p.rows * p.nsplit * hd * sizeof(float) : 0);
}

hipError_t launch_kv4_attention(const Kv4Attention &a, bool bf16, void *scratch, hipStream_t st) {
  if (a.n_req <= 0 || a.n_rows <= 0) return hipSuccess;
  const int Hkv = a.c.Hkv, hd = a.c.hd, tokens = a.max_context + a.max_rows;
  const Plan p = plan_of(a.n_req, a.max_rows, a.max_context, Hkv * a.group, Hkv, hd);
  const bool runs = a.c.bshift >= 4;
  char *at = (char *)scratch;
  const States x = {(float *)(at + ml_bytes(p) + lse_bytes(p)), (float2 *)at, (float *)(at + ml_bytes(p)), p.nsplit, p.chunk, ROWS / p.rep};
  auto main = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(Hkv * p.tiles, p.nsplit, a.n_req), dim3(64 * WAVES), 0, st, a, x, p.tiles); };
  // teams of a row and head: one up to the splits that it has under way at once, else four or all of a block
  const int teams = 64 * WAVES / (hd / 4), groups = p.nsplit <= IN_FLIGHT ? 1 : p.nsplit <= 4 * IN_FLIGHT ? 4 : teams;
  const int joins = p.nsplit > 1 ? (int)((p.rows * groups + teams - 1) / teams) : 0, pieces = cdiv(tokens, TURN * WAVES);
  const bool one_tile = a.max_rows * a.group <= ROWS;
  auto join = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(joins), dim3(64 * WAVES), 0, st, a, x, groups); };
  auto weight = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(joins + Hkv * pieces * a.n_req), dim3(64 * WAVES), 0, st, a, x, joins, groups, pieces); };
  auto weight_rows = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(pieces, Hkv, a.n_req), dim3(64 * WAVES), 0, st, a, x); };
  auto pick = [&](auto terms, auto in_runs) {
    constexpr int T = decltype(terms)::value;
    constexpr bool R = decltype(in_runs)::value;
    if (hd == 128) p.rep == 4 ? main(kv4_attention_kernel<128, T, 4, R>) : p.rep == 2 ? main(kv4_attention_kernel<128, T, 2, R>) : main(kv4_attention_kernel<128, T, 1, R>);
    else p.rep == 2 ? main(kv4_attention_kernel<64, T, 2, R>) : main(kv4_attention_kernel<64, T, 1, R>);
    if (a.add_weight && one_tile) hd == 128 ? weight(kv4_weight_kernel<128, T, R>) : weight(kv4_weight_kernel<64, T, R>);
    else if (joins) hd == 128 ? join(kv4_join_kernel<128, T == 1>) : join(kv4_join_kernel<64, T == 1>);
    if (a.add_weight && !one_tile) hd == 128 ? weight_rows(kv4_weight_rows_kernel<128, T>) : weight_rows(kv4_weight_rows_kernel<64, T>);
  };
  using std::integral_constant;
  if (bf16) runs ? pick(integral_constant<int, 1>{}, std::true_type{}) : pick(integral_constant<int, 1>{}, std::false_type{});
  else runs ? pick(integral_constant<int, 3>{}, std::true_type{}) : pick(integral_constant<int, 3>{}, std::false_type{});
  return hipGetLastError();
}
