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
// for every 32 channels.  Both conversions are exact; P enters as two bf16 terms for bf16 rows (16 bits: at most 2^-16 of each term) and as three
// (24 bits) for fp32 rows, as q does.  Sums, maxima and the output before its rounding are fp32.  (One term, 2^-8 of a probability, is faster - 477 us against 503 for the
// 128 requests below, 407 against 505 for 16 pieces of 256 rows behind 4000 tokens - but of values of either sign its error is three quarters of the output's own rounding,
// 2.1e-3 of the norm against 1.66e-3; two terms leave 1e-4 of difference to probabilities in fp32.)
//
// Few rows: the bytes of the cache bound it, so tokens are split over waves and blocks (128 requests of 2048 to 8192 tokens, 32 heads of 128: 503 us, 5.9 TB/s; one of 131001, 8 kv heads: 30 us
// and 4 for the join, 4.7 TB/s).  A short batch is a chain of loads, table - codes - products (32 requests of 256 to 2048 tokens, 8 kv heads of 64: 12 us).  Many rows: the instructions, below.
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
__device__ __forceinline__ int query_of(const Kv4Attention &a, int m) { return m >> a.gshift; }
__device__ __forceinline__ int head_of(const Kv4Attention &a, int kvh, int m) { return (kvh << a.gshift) + (m & (a.group - 1)); }
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

// bf16 terms of a probability for rows of so many terms.
constexpr int p_terms(int terms) { return terms == 1 ? 2 : terms; }
// Eight numbers as MFMA operand in TERMS bf16 terms: the upper 8 bits of each (cut off: rounded up, the largest numbers would be infinite), of what is left, ..; the last term
// is rounded to nearest.
template <int TERMS>
__device__ __forceinline__ void split8(float (&f)[8], bf16x8_t (&out)[TERMS]) {
#pragma unroll
  for (int t = 0; t < TERMS; ++t) {
    uint32_t r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (t + 1 < TERMS) {
        const uint32_t x = __float_as_uint(f[2 * e]), y = __float_as_uint(f[2 * e + 1]);
        r[e] = __builtin_amdgcn_perm(y, x, 0x07060302u);     // the upper halves of both
        f[2 * e] -= __uint_as_float(x & 0xffff0000u);
        f[2 * e + 1] -= __uint_as_float(y & 0xffff0000u);
      } else {
        r[e] = cvt_pk_bf16(f[2 * e], f[2 * e + 1]);
      }
    }
    out[t] = __builtin_bit_cast(bf16x8_t, make_uint4(r[0], r[1], r[2], r[3]));
  }
}

// Q as MFMA operand: lane (i, g) holds row m (the last one again behind it), elements g HD / 4 + 8 s .. + 7 of step s, in TERMS bf16 terms; negated
// where the scale is negative, so that the products' scale is not.
template <int HD, int TERMS>
__device__ __forceinline__ void load_q(const Kv4Attention &a, const Rows &w, int m, int g, bf16x8_t (&q)[TERMS][HD / 32]) {
  const int mc = min(m, w.m1 - 1);
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  const size_t o = (size_t)(w.row0 + query_of(a, mc)) * a.ld_q + (size_t)head_of(a, w.kvh, mc) * HD + g * (HD / 4);
#pragma unroll
  for (int s = 0; s < HD / 32; ++s) {
    if constexpr (TERMS == 1) {
      const uint4 u = *(const uint4 *)((const bf16_t *)a.q + o + 8 * s);
      q[0][s] = __builtin_bit_cast(bf16x8_t, make_uint4(u.x ^ flip, u.y ^ flip, u.z ^ flip, u.w ^ flip));
    } else {
      const float4 u = *(const float4 *)((const float *)a.q + o + 8 * s), v = *((const float4 *)((const float *)a.q + o + 8 * s) + 1);
      float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
      bf16x8_t y[TERMS];
      split8<TERMS>(f, y);
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        const uint4 r = __builtin_bit_cast(uint4, y[t]);
        q[t][s] = __builtin_bit_cast(bf16x8_t, make_uint4(r.x ^ flip, r.y ^ flip, r.z ^ flip, r.w ^ flip));
      }
    }
  }
}

// Scale of the products, as exponents of 2; the smallest number in place of 0, which would make -inf NaN.
__device__ __forceinline__ float score_scale(const Kv4Attention &a) { return fmaxf(fabsf(a.scale) * LOG2E, 1.4e-45f); }

// Index of a token of this request and head, and whether its block exists; else index 0, whose bytes are read and not used.
__device__ __forceinline__ uint32_t token_of(const Kv4Cache &c, const int32_t *table, int kvh, int t, int end, bool &ok) {
  ok = t < end;
  const int blk = ok ? table[t >> c.bshift] : -1;
  ok = blk >= 0 && (uint32_t)blk < c.num_blocks;
  return ok ? (((uint32_t)blk * c.Hkv + kvh) << c.bshift) + (t & ((1 << c.bshift) - 1)) : 0u;
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

// Codes of one lane for one S^T tile: HD / 4 elements.  (The cache is read once and should not displace what else is in the caches: 525 -> 489 us for 128
// requests of 2048 - 8192 tokens.)
template <int HD> struct KCodes { uint32_t w[HD / 32]; };
template <int HD, bool ONCE = true>
__device__ __forceinline__ KCodes<HD> load_k(const unsigned char *p) {
  KCodes<HD> r;
  if constexpr (HD == 128) {
    const u32x4_t u = ONCE ? __builtin_nontemporal_load((const u32x4_t *)p) : *(const u32x4_t *)p;
    r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
  } else {
    const u32x2_t u = ONCE ? __builtin_nontemporal_load((const u32x2_t *)p) : *(const u32x2_t *)p;
    r.w[0] = u.x; r.w[1] = u.y;
  }
  return r;
}

// Block ids of the four runs of 16 tokens of a turn (blocks of 16 tokens or more, RUNS below): lane l has that of run l % 4.
__device__ __forceinline__ int run_entry(const Kv4Cache &c, const int32_t *table, int t0, int end, int lane) {
  const int t = t0 + 16 * (lane & 3);
  return t < end ? table[t >> c.bshift] : -1;
}

// What a lane holds of the keys of a turn's 64 tokens: codes and scale of token 16 j + i for tile j, and where that token is: base + i (RUNS: base uniform).
template <int HD>
struct Keys {
  KCodes<HD> k[4];
  uint32_t ks[4], base[4];
};
// Returns which tokens exist: bit 16 j + i of the turn.
template <int HD, bool RUNS, bool ONCE>
__device__ __forceinline__ uint64_t load_keys(const Kv4Cache &c, const int32_t *table, int entry, int kvh, int t0, int end, int lane, Keys<HD> &u) {
  constexpr int NG = HD / 32, KB = HD / 2;
  const int i = lane & 15, g = lane >> 4;
  uint64_t there = 0;
  if constexpr (RUNS) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int blk = __builtin_amdgcn_readlane(entry, j);
      const bool ok = blk >= 0 && (uint32_t)blk < c.num_blocks;
      const uint32_t at = (((uint32_t)blk * c.Hkv + kvh) << c.bshift) + ((t0 + 16 * j) & ((1 << c.bshift) - 1));
      u.base[j] = ok ? at : 0u;
      there |= ok ? (uint64_t)0xffff << (16 * j) : 0ull;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) u.k[j] = load_k<HD, ONCE>(c.k + (size_t)u.base[j] * KB + (i * KB + g * (KB / 4)));
#pragma unroll
    for (int j = 0; j < 4; ++j) u.ks[j] = (c.k_scale + (size_t)u.base[j] * NG)[i * NG + g * (HD / 4) / kv4::GROUP];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bool ok;
      const uint32_t tok = token_of(c, table, kvh, t0 + 16 * j + i, end, ok);
      there |= (__ballot(ok) & 0xffff) << (16 * j);
      u.base[j] = tok - i;
      u.k[j] = load_k<HD, ONCE>(c.k + (size_t)tok * KB + g * (KB / 4));
      u.ks[j] = c.k_scale[(size_t)tok * NG + g * (HD / 4) / kv4::GROUP];
    }
  }
  return there;
}

// A turn of the first kernel: keys, and of the values a lane's 16-byte pieces (token by token) and the scales of tokens 16 j + 4 g .. + 3.
template <int HD>
struct Turn {
  Keys<HD> keys;
  u32x4_t v[HD / 32];
  uint32_t vs[4][HD / 32];
  uint64_t there;
};
template <int HD, bool RUNS>
__device__ __forceinline__ void load_turn(const Kv4Cache &c, const int32_t *table, int entry, int kvh, int t0, int end, int lane, Turn<HD> &u) {
  constexpr int NG = HD / 32, VB = HD / 2, CPT = VB / 16;
  const int g = lane >> 4;
  u.there = load_keys<HD, RUNS, true>(c, table, entry, kvh, t0, end, lane, u.keys);
  if constexpr (RUNS) {
    const uint32_t *base = u.keys.base;
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
// -inf in place of the products of this lane's row and tokens from `last` on (16 j + 4 g + r, counted from 4 g) or tokens that are not there.
__device__ __forceinline__ void mask_scores(f32x4_t (&s)[4], int last, uint64_t there, int g) {
  there >>= 4 * g;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) s[j][r] = 16 * j + r < last && ((there >> (16 * j + r)) & 1) ? s[j][r] : -INFINITY;
}
// Soft-max of a row, whose tokens are spread over four lanes: probabilities are 2^(sc s - top), and `top` follows the largest product only when one is more than `lag`
// above it.  lag = MANY_LAG, where many rows make the instructions count: most turns need neither an exchange between lanes nor a rescaling (a piece of 4096 rows, 32 heads
// and 8 kv heads of 128, behind 4096 tokens 680 -> 652 us).  The relative error of a probability does not depend on it.
constexpr float MANY_LAG = 8.f;
struct Softmax {
  float top = -INFINITY, minus = 0.f, l = 0.f;        // minus: -top, 0 as long as the row has seen nothing; l: this lane's part of the sum
};
// Whether some row of the wave has to follow, then the factor of everything summed so far (rows that need not have 1).
__device__ __forceinline__ bool lags(const f32x4_t (&s)[4], float sc, const Softmax &x, float lag, float &largest) {
  largest = s[0][0];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) largest = fmaxf(largest, s[j][r]);
  return __any(largest * sc - x.top > lag);            // (-inf above -inf: NaN, no)
}
__device__ __forceinline__ float follow(float largest, float sc, Softmax &x) {
  largest = fmaxf(largest, __shfl_xor(largest, 16, 64));
  largest = fmaxf(largest, __shfl_xor(largest, 32, 64));
  const float top = fmaxf(x.top, largest * sc), factor = top == x.top ? 1.f : __builtin_amdgcn_exp2f(x.top - top);
  x.top = top;
  x.minus = top == -INFINITY ? 0.f : -top;
  x.l *= factor;
  return factor;
}
// Scale of group gr of the token of tile j, register r.
template <int HD>
__device__ __forceinline__ float v_scale_of(const Turn<HD> &u, int j, int r, int gr) {
  if constexpr (HD == 128) return kv4::scale_value((u.vs[j][r] >> (8 * gr)) & 255u);
  else return kv4::scale_value((u.vs[j][r >> 1] >> (16 * (r & 1) + 8 * gr)) & 255u);
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
  const int m = k * a.group + (head & (a.group - 1)), m1 = min((m / x.tile_rows + 1) * x.tile_rows, w.n * a.group);
  return max(1, min(x.nsplit, (w.ctx + query_of(a, m1 - 1) + 1 + x.chunk - 1) / x.chunk));
}

// REP: copies of each row among the 16 columns of a tile.  P is scaled for every 32 channels anew, so few rows (16 / REP) are repeated, copy c scales for groups c, c + REP, ..,
// and of an output tile the columns of the copy that scaled for its group are the rows.
template <int HD, int TERMS, int REP, bool RUNS>
__global__ __launch_bounds__(64 * WAVES, TERMS == 1 && HD == 64 ? 4 : 2) void kv4_attention_kernel(Kv4Attention a, States x, int tiles) {
  constexpr int NS = HD / 32, NG = HD / 32, CT = HD / 16;      // MFMA steps along the head, scale groups, channel tiles
  constexpr int VB = HD / 2, VROW = VB + 16;                   // bytes of a token of V; padded in LDS, so that 16 tokens' reads of one channel tile meet 16 different banks
  constexpr int CPT = VB / 16;                                 // 16-byte pieces of a token of V
  constexpr int NR = ROWS / REP, OROW = HD + 4, PT = p_terms(TERMS);
  constexpr int SM = WAVES * TURN * VROW > WAVES * NR * (OROW + 2) * 4 ? WAVES * TURN * VROW : WAVES * NR * (OROW + 2) * 4;
  __shared__ __align__(16) unsigned char sm[SM];
  const int kvh = blockIdx.x / tiles, tile = blockIdx.x - kvh * tiles, split = blockIdx.y;
  const Rows w = rows_of<NR>(a, blockIdx.z, kvh, tile);
  if (w.m0 >= w.m1) return;
  const int end = w.ctx + query_of(a, w.m1 - 1) + 1;            // tokens that the last row sees
  const int c0 = split * x.chunk, c1 = split == x.nsplit - 1 ? end : min(end, c0 + x.chunk);      // (the last split takes a tail of up to a turn)
  if (c0 >= end && split > 0) return;                          // (the first one writes the rows that see nothing)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4, copy = i / NR;
  const int32_t *table = a.tables + (size_t)w.req * a.max_blocks;
  const int limit = w.ctx + query_of(a, min(w.m0 + i % NR, w.m1 - 1)) + 1;  // tokens that this lane's row sees
  const int all = w.ctx + query_of(a, w.m0) + 1;                  // tokens that every row sees
  const float sc = score_scale(a);

  int t0 = c0 + wave * TURN;
  constexpr int STEP = WAVES * TURN;
  int entry = 0;
  if constexpr (RUNS) entry = run_entry(a.c, table, t0, c1, lane);
  bf16x8_t q[TERMS][NS];
  load_q<HD, TERMS>(a, w, w.m0 + i % NR, g, q);
  f32x4_t o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  Softmax sx;
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
      const float ks = kv4::scale_value(u.keys.ks[j]);
      s[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        const bf16x8_t kf = kv4::decode8(u.keys.k[j].w[st], ks);
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
    const bool whole = t0 + TURN <= min(all, c1) && n.there == ~0ull;
    if (!whole) mask_scores(s, min(limit, c1) - t0 - 4 * g, n.there, g);
    float largest;
    if (lags(s, sc, sx, 0.f, largest)) {
      const float factor = follow(largest, sc, sx);
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c] *= factor;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[j][r] = __builtin_amdgcn_exp2f(fmaf(s[j][r], sc, sx.minus));
        sx.l += s[j][r];
      }
#pragma unroll
    for (int pass = 0; pass < NG / REP; ++pass) {
      bf16x8_t pf[2][PT];
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
        split8<PT>(f, pf[h]);
      }
#pragma unroll
      for (int cc = 0; cc < 2 * REP; ++cc) {
        const int c = pass * 2 * REP + cc;
        const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2 *)(vread + c * 8));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8_t vf = kv4::decode8((uint32_t)v[h], 1.f);
#pragma unroll
          for (int t = PT - 1; t >= 0; --t) o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[h][t], o[c], 0, 0, 0);
        }
      }
    }
  }

  // the waves' states -> one
  sx.l += __shfl_xor(sx.l, 16, 64);
  sx.l += __shfl_xor(sx.l, 32, 64);
  __syncthreads();
  float *so = (float *)sm, *sml = so + WAVES * NR * OROW;
#pragma unroll
  for (int c = 0; c < CT; ++c)
    if (REP == 1 || c / 2 % REP == copy) *(f32x4_t *)(so + (wave * NR + i % NR) * OROW + 16 * c + 4 * g) = o[c];
  if (lane < NR) {
    sml[(wave * NR + i) * 2] = sx.top;
    sml[(wave * NR + i) * 2 + 1] = sx.l;
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
    const size_t r = w.row0 + query_of(a, mr);
    const int head = head_of(a, kvh, mr), Hq = a.c.Hkv * a.group;
    const size_t at = row_id(a, w.req, query_of(a, mr), head);
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

// Many rows of a request: a block of 128 rows, 32 a wave, goes through the tokens together.  A thread takes a group of 32 of a token's key and value: the key's codes go to LDS as they are
// and are decoded by every wave (a quarter of the bytes that decoded ones would be read in), the value's are decoded with their scale first and lie there as bf16, token by token,
// so that P needs no scaling and a transposing read of 4 tokens x 16 channels hands out V^T.  A value group that is NaN counts as 0 there and is noted beside it: only the
// rows that see the token become NaN.  A turn's codes are asked for two turns ahead, put into LDS one ahead, their
// blocks looked up three ahead.  A piece of 4096 rows, 32 heads and 8 kv heads of 128, behind 4096 tokens takes 656 us, 0.63 PFLOP/s (0.94 with the second term of P): the matrix pipes are
// busy for 45 % of the cycles, vector instructions (exponentials, terms, maxima, decoding, the issue of the products) take 64 %.
constexpr int ROW_TILES = 2, BLOCK_ROWS = WAVES * ROW_TILES * ROWS, LEAST_TURNS = 4, NEAR = 2;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// The work of a kv head, the turns of all blocks of rows of all requests one after the other, is cut into equal shares, one a thread block, since lengths and rows are known on the device only and
// differ (a grid of requests, blocks of rows and equal splits of the longest context leaves the chip half idle: six requests of 134 to 238 rows at 2500 to 6700 tokens, 8 kv heads of 128, 209
// us and by shares 167; 64 of 5 to 60 rows at 500 to 6000 435 and 277).  A block of rows that is cut leaves states that
// kv4_rows_join_kernel joins; a cut NEAR turns or less from the rows' begin or end, the price of one, moves there.
// (With workers = 0 the thread blocks are the splits of the blocks of rows, as few rows have them.)
struct Shares {
  float *acc;                        // [Hkv, workers, 2, BLOCK_ROWS, HD] what a worker leaves of the rows that it began with in their middle and of those that it left before their end
  float2 *ml;                        // [Hkv, workers, 2, BLOCK_ROWS]
  float *lse2;
  int4 *start;                       // [Hkv, workers] request, block of rows, turn in it (0: nothing cut)
  int workers, nsplit, chunk;        // chunk: turns of a split
};
// Turns of the blocks of rows of a request.  (Rows that see nothing have some as well: they are written.)
struct Turns {
  int ctx, n, shift, tiles;          // 1 << shift: queries a block of rows
  __device__ __forceinline__ Turns(const Kv4Attention &a, const Rows &w) : ctx(max(w.ctx, 0)), n(w.n), shift(__builtin_ctz(BLOCK_ROWS) - a.gshift), tiles((w.n + (1 << shift) - 1) >> shift) {}
  __device__ __forceinline__ int of(int tile) const { return (ctx + min((tile + 1) << shift, n) + TURN - 1) / TURN; }
  // of blocks 0 .. m - 1; (ctx + 63 + (k + 1) 2^shift) / 64 for a whole block k.  (Below 2^31; what is subtracted on the way may wrap.)
  __device__ __forceinline__ uint32_t before(int m) const { return m == 0 ? 0u : m == tiles ? before_whole(m - 1) + (uint32_t)of(m - 1) : before_whole(m); }
  __device__ __forceinline__ uint32_t before_whole(uint32_t m) const {
    constexpr int TS = __builtin_ctz(TURN);
    if (shift >= TS) return m * ((uint32_t)(ctx + TURN - 1) >> TS) + (half_product(m) << (shift - TS));
    const uint32_t u = (uint32_t)(ctx + TURN - 1) >> shift;
    return quotients(u + m, TS - shift) - quotients(u, TS - shift);
  }
  static __device__ __forceinline__ uint32_t half_product(uint32_t m) { return m % 2 ? (m + 1) / 2 * m : m / 2 * (m + 1); }      // m (m + 1) / 2
  static __device__ __forceinline__ uint32_t quotients(uint32_t y, int s) {                                                       // sum of j >> s, j = 0 .. y
    const uint32_t q = (y + 1) >> s;
    return (half_product(q - 1) << s) + q * (y + 1 - (q << s));
  }
};

template <int HD>
__global__ __launch_bounds__(64 * WAVES, 2) void kv4_rows_kernel(Kv4Attention a, Shares x) {
  constexpr int NS = HD / 32, NG = HD / 32, CT = HD / 16, VROW = HD * 2, KROW = HD / 2, PT = p_terms(1);
  __shared__ __align__(16) unsigned char sv[2][TURN * VROW], sk[2][TURN * KROW], sks[2][TURN * NG];
  __shared__ int any[3];                               // by turn, as the next two: read in it, filled in the one before, cleared in the one before that
  __shared__ unsigned long long nan[3][NG], missing[3];
  __shared__ int sums[WAVES];
  __shared__ int4 cuts[2];                             // request, block of rows, turn in it, turns of all before
  const int kvh = blockIdx.x % a.c.Hkv, worker = blockIdx.x / a.c.Hkv;      // (the workers of a kv head on one XCD where there are 8 heads)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
  const float sc = score_scale(a);

  // Where this share begins and the next one does: each thread adds up some requests, the one in whose part a cut falls finds the request, wave k the k-th cut's block of rows.
  int left, req, tile, turn0 = 0;
  if (x.workers > 0) {
    const int per = (a.n_req + 64 * WAVES - 1) / (64 * WAVES), r0 = min(tid * per, a.n_req), r1 = min(r0 + per, a.n_req);
    int mine = 0;
    for (int r = r0; r < r1; ++r) {
      const Turns w(a, rows_of<BLOCK_ROWS>(a, r, kvh, 0));
      mine += (int)w.before(w.tiles);
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(upto, o, 64);
      if (lane >= o) upto += y;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) {
      if (k < wave) upto += sums[k];
      total += sums[k];
    }
    const int shares = min(x.workers, (total + LEAST_TURNS - 1) / LEAST_TURNS);
    auto cut_of = [&](int k) { return k < shares ? (int)((double)total * k / shares) : total; };      // (exact before it is cut off: a product below 2^53, a quotient by less than 2^10)
    for (int k = 0; k < 2; ++k) {
      const int at = cut_of(worker + k);
      if (at < upto - mine || at >= upto) continue;
      int rest = at - (upto - mine);
      for (int r = r0; r < r1; ++r) {
        const Turns w(a, rows_of<BLOCK_ROWS>(a, r, kvh, 0));
        const int here = (int)w.before(w.tiles);
        if (rest < here) {
          cuts[k] = make_int4(r, 0, rest, 0);
          break;
        }
        rest -= here;
      }
    }
    __syncthreads();
    if (wave < 2) {
      const int at = cut_of(worker + wave);
      int4 in = make_int4(0, 0, 0, total);
      if (at < total) {
        const int r = __builtin_amdgcn_readfirstlane(cuts[wave].x), rest = cuts[wave].z;
        const Turns w(a, rows_of<BLOCK_ROWS>(a, r, kvh, 0));
        int b = 0;
        for (int step = w.tiles > 64 ? 64 : 1;; step = 1) {
          const int m = b + (lane + 1) * step;
          b += step * __popcll(__ballot(m < w.tiles && (int)w.before(min(m, w.tiles)) <= rest));
          if (step == 1) break;
        }
        const int turn = rest - (int)w.before(b), behind = w.of(b) - turn, near = min(NEAR, total / (8 * shares));
        const int by = turn <= near ? -turn : behind <= near ? behind : 0;
        in = make_int4(r, by > 0 ? b + 1 : b, by ? 0 : turn, at + by);
      }
      if (lane == 0) cuts[wave] = in;
    }
    __syncthreads();
    const int4 in = cuts[0];
    left = __builtin_amdgcn_readfirstlane(cuts[1].w - in.w);
    req = __builtin_amdgcn_readfirstlane(in.x);
    tile = __builtin_amdgcn_readfirstlane(in.y);
    turn0 = __builtin_amdgcn_readfirstlane(in.z);
    if (tid == 0) x.start[kvh * x.workers + worker] = left > 0 ? in : make_int4(0, 0, 0, 0);
    if (left <= 0) return;
  } else {
    req = blockIdx.y;
    tile = gridDim.x / a.c.Hkv - 1 - worker;           // long ones first
    const Rows w = rows_of<BLOCK_ROWS>(a, req, kvh, tile);
    if (w.m0 >= w.m1) return;
    turn0 = blockIdx.z * x.chunk;
    left = min(x.chunk, Turns(a, w).of(tile) - turn0);
    if (left <= 0) return;
  }

  for (;; ++tile, turn0 = 0) {
  Rows w = rows_of<BLOCK_ROWS>(a, req, kvh, tile);
  while (w.m0 >= w.m1) {                               // behind the last rows of a request
    if (++req >= a.n_req) return;
    tile = 0;
    w = rows_of<BLOCK_ROWS>(a, req, kvh, 0);
  }
  const int turns = Turns(a, w).of(tile), turn1 = min(turns, turn0 + left);
  const bool cut = x.workers > 0 ? turn0 > 0 || turn1 < turns : x.nsplit > 1;
  const int c0 = turn0 * TURN, c1 = min(w.ctx + query_of(a, w.m1 - 1) + 1, turn1 * TURN);
  const int32_t *table = a.tables + (size_t)w.req * a.max_blocks;
  __syncthreads();                                     // nobody reads the rows before any more

  // thread (token tid / NG, group tid % NG) of a turn (64-wide heads: the first 128 threads)
  const int vt = tid / NG, vg = tid % NG;
  const bool loads = HD == 128 || tid < TURN * NG;
  struct Codes {
    u32x4_t k, v;
    uint32_t ks, vs;
    bool ok;
  };
  auto entry_of = [&](int t0) { return loads && t0 + vt < c1 ? table[(t0 + vt) >> a.c.bshift] : -1; };
  auto load = [&](int t0, int blk) {
    Codes n;
    n.ok = blk >= 0 && (uint32_t)blk < a.c.num_blocks;
    const uint32_t tok = n.ok ? (((uint32_t)blk * a.c.Hkv + kvh) << a.c.bshift) + ((t0 + vt) & ((1 << a.c.bshift) - 1)) : 0u;
    n.k = *(const u32x4_t *)(a.c.k + (size_t)tok * KROW + vg * 16);
    n.v = *(const u32x4_t *)(a.c.v + (size_t)tok * KROW + vg * 16);
    n.ks = a.c.k_scale[(size_t)tok * NG + vg];
    n.vs = a.c.v_scale[(size_t)tok * NG + vg];
    return n;
  };
  auto swizzle = [](int row) { return HD == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };      // 16 rows' reads of one channel tile meet every bank twice
  auto store = [&](const Codes &n, int buf, int turn) {
    if (!loads) return;
    *(u32x4_t *)(sk[buf] + vt * KROW + vg * 16) = n.k;
    sks[buf][vt * NG + vg] = (unsigned char)n.ks;
    const bool bad = n.ok && n.vs == kv4::NAN_SCALE, none = !n.ok || bad;
    if (none) {
      atomicOr(bad ? &nan[turn][vg] : &missing[turn], 1ull << vt);
      any[turn] = 1;
    }
    const float s = none ? 1.f : kv4::scale_value(n.vs);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *(bf16x8_t *)(sv[buf] + vt * VROW + (((4 * vg + e) ^ swizzle(vt)) << 4)) = kv4::decode8(none ? 0u : n.v[e], s);
  };

  const int first = entry_of(c0), second = entry_of(c0 + TURN);
  int entry = entry_of(c0 + 2 * TURN);                 // of the turn whose codes are asked for next
  const Codes now = load(c0, first);
  Codes codes = load(c0 + TURN, second);               // of the next turn
  const int mw = w.m0 + wave * ROW_TILES * ROWS;
  const int wave_end = mw < w.m1 ? w.ctx + query_of(a, min(mw + ROW_TILES * ROWS - 1, w.m1 - 1)) + 1 : 0;      // tokens that the wave's last row sees, and that all its rows see
  const int wave_all = w.ctx + query_of(a, min(mw, w.m1 - 1)) + 1;
  int limit[ROW_TILES];
  bf16x8_t q[ROW_TILES][1][NS];
  f32x4_t o[ROW_TILES][CT];
  Softmax sx[ROW_TILES];
#pragma unroll
  for (int b = 0; b < ROW_TILES; ++b) {
    const int row = mw + b * ROWS + i;
    limit[b] = w.ctx + query_of(a, min(row, w.m1 - 1)) + 1;
    load_q<HD, 1>(a, w, row, g, q[b]);
#pragma unroll
    for (int c = 0; c < CT; ++c) o[b][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  if (tid < 3 * NG) nan[tid / NG][tid % NG] = 0;
  if (tid < 3) { missing[tid] = 0; any[tid] = 0; }
  __syncthreads();
  if (c0 < c1) store(now, 0, 0);
  const int vrow = 4 * g + (i >> 2);
  int buf = 0, turn = 0;
  for (int t0 = c0; t0 < c1; t0 += TURN, buf ^= 1) {
    __syncthreads();                                   // this turn's keys and values are there, and the other buffer is free
    const int next = turn == 2 ? 0 : turn + 1, after = next == 2 ? 0 : next + 1;
    if (tid < NG) nan[after][tid] = 0;
    if (tid == 0) { missing[after] = 0; any[after] = 0; }
    if (t0 + TURN < c1) store(codes, buf ^ 1, next);
    if (t0 + 2 * TURN < c1) {
      codes = load(t0 + 2 * TURN, entry);
      entry = entry_of(t0 + 3 * TURN);
    }
    if (t0 < wave_end) {
      const int marked = any[turn];
      f32x4_t s[ROW_TILES][4];
      KCodes<HD> k[4];
      uint32_t ks[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ks[j] = sks[buf][(16 * j + i) * NG + g * (HD / 4) / kv4::GROUP];
        k[j] = load_k<HD, false>(sk[buf] + (16 * j + i) * KROW + g * (KROW / 4));
      }
      __builtin_amdgcn_sched_barrier(0);                 // (all keys read before the first product, as the values below)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int b = 0; b < ROW_TILES; ++b) s[b][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < NS; ++st) {
          const bf16x8_t kf = kv4::decode8(k[j].w[st], kv4::scale_value(ks[j]));
#pragma unroll
          for (int b = 0; b < ROW_TILES; ++b) s[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[b][0][st], s[b][j], 0, 0, 0);
        }
      }
      // lane (i, g) brings channels 4 (i % 4) .. + 3 of tile c from token 16 (2 h + n) + 4 g + i / 4 and gets channel i of tokens 4 g .. + 3 of the run
      auto read_v = [&](int c, bf16x8_t (&v)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          s16x4_t p[2];
#pragma unroll
          for (int n = 0; n < 2; ++n)
            p[n] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(sv[buf] + (16 * (2 * h + n) + vrow) * VROW + (((2 * c + ((i >> 1) & 1)) ^ swizzle(vrow)) << 4) + 8 * (i & 1)));
          v[h] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(p[0], p[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
      };
      bf16x8_t vf[2];
      read_v(0, vf);
      const bool whole = t0 + TURN <= min(wave_all, c1) && !marked;
      const uint64_t there = marked ? ~missing[turn] : ~0ull;
      bf16x8_t pf[ROW_TILES][2][PT];
#pragma unroll
      for (int b = 0; b < ROW_TILES; ++b) {
        if (!whole) mask_scores(s[b], min(limit[b], c1) - t0 - 4 * g, there, g);
        float largest;
        if (lags(s[b], sc, sx[b], MANY_LAG, largest)) {
          const float factor = follow(largest, sc, sx[b]);
#pragma unroll
          for (int c = 0; c < CT; ++c) o[b][c] *= factor;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            f[e] = __builtin_amdgcn_exp2f(fmaf(s[b][2 * h + (e >> 2)][e & 3], sc, sx[b].minus));
            sx[b].l += f[e];
          }
          split8<PT>(f, pf[b][h]);
        }
      }
      // operands of the next channel tile are read before the products of this one (left to itself, the compiler reads each where it is used and waits)
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        bf16x8_t vn[2];
        if (c + 1 < CT) read_v(c + 1, vn);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int t = PT - 1; t >= 0; --t)
#pragma unroll
            for (int b = 0; b < ROW_TILES; ++b) o[b][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[h], pf[b][h][t], o[b][c], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        vf[0] = vn[0];
        vf[1] = vn[1];
      }
      if (marked) {
#pragma unroll
        for (int gr = 0; gr < NG; ++gr) {
          const uint64_t bad = nan[turn][gr];
#pragma unroll
          for (int b = 0; b < ROW_TILES; ++b) {
            const int last = limit[b] - t0;            // the row sees tokens below it
            const uint64_t seen = last >= 64 ? bad : last > 0 ? bad & ((1ull << last) - 1) : 0ull;
            if (seen) { o[b][2 * gr] = f32x4_t{NAN, NAN, NAN, NAN}; o[b][2 * gr + 1] = o[b][2 * gr]; }
          }
        }
      }
    }
    turn = next;
  }

#pragma unroll
  for (int b = 0; b < ROW_TILES; ++b) {
    float l = sx[b].l;
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const int mr = mw + b * ROWS + i;
    if (mr >= w.m1) continue;
    const int k = query_of(a, mr), head = head_of(a, kvh, mr), Hq = a.c.Hkv * a.group;
    const size_t r = w.row0 + k, at = row_id(a, w.req, k, head);
    if (!cut) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16_t *to = (bf16_t *)a.out + r * a.ld_out + (size_t)head * HD + 4 * g;
#pragma unroll
      for (int c = 0; c < CT; ++c) *(uint2 *)(to + 16 * c) = make_uint2(cvt_pk_bf16(o[b][c][0] * inv, o[b][c][1] * inv), cvt_pk_bf16(o[b][c][2] * inv, o[b][c][3] * inv));
      if (g == 0) {
        const float lse2 = l == 0.f ? -INFINITY : sx[b].top + log2f(l);
        if (a.lse) a.lse[r * Hq + head] = lse2 / LOG2E;
        if (a.add_weight) x.lse2[at] = lse2;
      }
    } else {
      const size_t state = x.workers > 0 ? (((size_t)kvh * x.workers + worker) * 2 + (turn0 == 0)) * BLOCK_ROWS + (mr - w.m0) : at * x.nsplit + blockIdx.z;
      float *to = x.acc + state * HD + 4 * g;
#pragma unroll
      for (int c = 0; c < CT; ++c) *(f32x4_t *)(to + 16 * c) = o[b][c];
      if (g == 0) x.ml[state] = make_float2(sx[b].top, l);
    }
  }
  left -= turn1 - turn0;
  if (left <= 0) return;
  }
}

// Joins the splits of a row and head: `groups` teams of HD / 4 lanes (four channels each) take every groups-th split with a soft-max state of their own and are merged
// in order.  The time is the latency of the loads, so a team has those of IN_FLIGHT splits under way (4 us for 32 heads of 64 splits).
constexpr int IN_FLIGHT = 4;
// Merges states first, first + step, .. below n, of which s lies at place(s): channels 4 e .. + 3.
template <int HD, class Place>
__device__ __forceinline__ void merge(const float *acc, const float2 *ml, int first, int n, int step, int e, Place place, float &mn, float &ls, float4 &as) {
  mn = -INFINITY;
  ls = 0.f;
  as = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = first; s0 < n; s0 += IN_FLIGHT * step) {
    float4 v[IN_FLIGHT];
    float2 y[IN_FLIGHT];
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) {
      const size_t at = place(min(s0 + u * step, n - 1));
      y[u] = ml[at];
      v[u] = ((const float4 *)(acc + at * HD))[e];
    }
    float top = mn;
#pragma unroll
    for (int u = 0; u < IN_FLIGHT; ++u) {
      if (s0 + u * step >= n) { y[u] = make_float2(-INFINITY, 0.f); v[u] = make_float4(0.f, 0.f, 0.f, 0.f); }
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
}
// Writes channels 4 e .. + 3 of row r of the output and, by e = 0, its log sum; keep: where the weights read it, or null.
template <int HD, bool BF16>
__device__ __forceinline__ void put_joined(const Kv4Attention &a, size_t r, int head, int e, float mn, float ls, const float4 &as, float *keep) {
  const float inv = ls == 0.f ? 0.f : 1.f / ls;
  const size_t to = r * a.ld_out + (size_t)head * HD + 4 * e;
  if constexpr (BF16) *(uint2 *)((bf16_t *)a.out + to) = make_uint2(cvt_pk_bf16(as.x * inv, as.y * inv), cvt_pk_bf16(as.z * inv, as.w * inv));
  else *(float4 *)((float *)a.out + to) = make_float4(as.x * inv, as.y * inv, as.z * inv, as.w * inv);
  if (e == 0) {
    const float lse2 = ls == 0.f ? -INFINITY : mn + log2f(ls);
    if (a.lse) a.lse[r * (a.c.Hkv * a.group) + head] = lse2 / LOG2E;
    if (keep) *keep = lse2;
  }
}
template <int HD, bool BF16>
__device__ __forceinline__ void join_rows(const Kv4Attention &a, const States &x, int block, int groups, bool keep_lse2, float4 *so, float2 *sml) {
  constexpr int LANES = HD / 4;
  const int Hq = a.c.Hkv * a.group, team = threadIdx.x / LANES, e = threadIdx.x % LANES, grp = team % groups;
  const size_t at = (size_t)block * (64 * WAVES / LANES / groups) + team / groups, rows = (size_t)a.n_req * a.max_rows * Hq;
  const int head = (int)(at % Hq), k = (int)(at / Hq % a.max_rows), req = (int)(min(at, rows - 1) / Hq / a.max_rows);
  const Rows w = rows_of<1>(a, req, head >> a.gshift, 0);
  const bool live = at < rows && k < w.n;
  const int ns = live ? splits_of(a, x, w, k, head) : 0;
  float mn, ls;
  float4 as;
  merge<HD>(x.acc, x.ml, grp, ns, groups, e, [&](int s) { return at * x.nsplit + s; }, mn, ls, as);
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
  put_joined<HD, BF16>(a, (size_t)w.row0 + k, head, e, mn, ls, as, keep_lse2 ? x.lse2 + at : nullptr);
}

template <int HD, bool BF16>
__global__ __launch_bounds__(64 * WAVES) void kv4_join_kernel(Kv4Attention a, States x, int groups) {
  __shared__ float4 so[64 * WAVES];
  __shared__ float2 sml[64 * WAVES / (HD / 4)];
  join_rows<HD, BF16>(a, x, blockIdx.x, groups, a.add_weight, so, sml);
}

// Joins what the workers of a kv head left of the rows that they cut: block (worker, head, part of the rows) does so for the rows that the worker begins in the middle of, if it is the
// first to do so; the others of the same rows follow it.
template <int HD>
__global__ __launch_bounds__(64 * WAVES) void kv4_rows_join_kernel(Kv4Attention a, Shares x) {
  constexpr int LANES = HD / 4;
  const int worker = blockIdx.x + 1, kvh = blockIdx.y, e = threadIdx.x % LANES;
  const int4 *starts = x.start + kvh * x.workers, start = starts[worker];
  auto same = [&](const int4 &y) { return y.x == start.x && y.y == start.y && y.z > 0; };
  if (start.z == 0 || same(starts[worker - 1])) return;
  int n = 2;                         // with the worker before
  while (worker + n - 1 < x.workers && same(starts[worker + n - 1])) ++n;
  const Rows w = rows_of<BLOCK_ROWS>(a, start.x, kvh, start.y);
  const int row = blockIdx.z * (64 * WAVES / LANES) + threadIdx.x / LANES, m = w.m0 + row;
  if (m >= w.m1) return;
  const int k = query_of(a, m), head = head_of(a, kvh, m);
  const size_t before = (((size_t)kvh * x.workers + worker - 1) * 2 + 1) * BLOCK_ROWS + row;
  float mn, ls;
  float4 as;
  // the worker before left the second of its two, the others the first
  merge<HD>(x.acc, x.ml, 0, n, 1, e, [&](int s) { return s == 0 ? before : before + (size_t)(2 * s - 1) * BLOCK_ROWS; }, mn, ls, as);
  put_joined<HD, true>(a, (size_t)w.row0 + k, head, e, mn, ls, as, a.add_weight ? x.lse2 + row_id(a, w.req, k, head) : nullptr);
}

// Adds every token's probabilities, summed over the rows of its request and the query heads of its kv head, to its weight, from the product S = Q K^T formed again
// (lane (i, g) has token i of a tile of 16 and rows 4 g .. 4 g + 3) and the rows' log sums: 68 or 34 bytes of K a token again instead of 8 for every row.  A wave takes 64 tokens
// and all rows, so a request adds to a token once (blocks that requests share get one addition from each, by atomics).
// Here: requests of one tile of rows, whose log sums the block forms from the splits' states; the first `joins` blocks join the splits meanwhile.  (32 requests of 256 to 2048
// tokens, 8 kv heads of 64: 9.5 us, the chain table - codes - products - addition beside that of the log sums.)
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
  const float sc = score_scale(a);
  Keys<HD> u;
  int entry = 0;
  if constexpr (RUNS) entry = run_entry(a.c, table, t0, end, lane);
  const uint64_t there = load_keys<HD, RUNS, false>(a.c, table, entry, kvh, t0, end, lane, u);
  bf16x8_t q[TERMS][NS];
  load_q<HD, TERMS>(a, w, w.m0 + i, g, q);
  // log sums of the rows: 16 threads a row
  {
    const int row = threadIdx.x / 16, mr = min(row, w.m1 - 1), kr = query_of(a, mr), head = head_of(a, kvh, mr);
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
    if (threadIdx.x % 16 == 0) slse[row] = ls == 0.f ? INFINITY : mn + log2f(ls);      // (nothing is left of a row without a token, or all of whose products are -inf)
  }
  __syncthreads();
  float lse2[4];
  int last[4];                                       // tokens that the row sees
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int m = 4 * g + r;
    lse2[r] = slse[m];
    last[r] = m < w.m1 ? w.ctx + query_of(a, m) + 1 : 0;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float scale = kv4::scale_value(u.ks[j]);
    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      const bf16x8_t kf = kv4::decode8(u.k[j].w[st], scale);
#pragma unroll
      for (int t = TERMS - 1; t >= 0; --t) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t][st], kf, s, 0, 0, 0);
    }
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) sum += t0 + 16 * j + i < last[r] ? __builtin_amdgcn_exp2f(s[r] * sc - lse2[r]) : 0.f;
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (g == j && ((there >> (16 * j + i)) & 1) && t0 + 16 * j + i < end) unsafeAtomicAdd(a.c.weight + (u.base[j] + i), sum);
  }
}

// The same for more rows, whose log sums are there already.  A wave keeps the decoded keys of its 64 tokens; the rows come in stages of 64 (fp32: 16) through LDS,
// shared by the waves of a block, a stage ahead in registers.  (The ragged pieces above: 75 us; 45 of them products and exponentials, the rest stages that a block waits for and the
// last blocks alone.  Blocks in the order of requests first, heads next: 81 and 83.)
template <int HD, int TERMS>
__global__ __launch_bounds__(64 * WAVES, 2) void kv4_weight_rows_kernel(Kv4Attention a, States x) {
  constexpr int NS = HD / 32, NG = HD / 32, STAGE = TERMS == 1 ? 64 : 16, CPR = HD / 8;      // 16-byte pieces of a row in bf16
  constexpr int PER = STAGE * CPR / (64 * WAVES) ? STAGE * CPR / (64 * WAVES) : 1;            // pieces a thread brings
  __shared__ __align__(16) uint4 sq[2][TERMS][STAGE * CPR];
  __shared__ __align__(16) float slse[2][STAGE];
  const int kvh = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i = lane & 15, g = lane >> 4;
  const Rows w = rows_of<1>(a, blockIdx.z, kvh, 0);
  const int n_rows = w.n * a.group, end = w.ctx + w.n, b0 = blockIdx.x * WAVES * TURN, t0 = b0 + wave * TURN;
  if (n_rows == 0 || b0 >= end) return;
  const int32_t *table = a.tables + (size_t)w.req * a.max_blocks;
  const float sc = score_scale(a);
  auto swizzle = [](int row) { return HD == 128 ? row & 15 : (row >> 1) & 7; };      // the 16 rows of a read lie in different banks
  // pieces of the rows from m0 on: thread -> (row, piece); behind the last row the last one again, with a log sum that leaves nothing of it
  uint4 piece[TERMS][PER];
  float lse2 = INFINITY;
  auto load = [&](int m0) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int at = p * 64 * WAVES + tid, m = min(m0 + at / CPR, n_rows - 1);
      if (at >= STAGE * CPR) continue;
      const size_t o = (size_t)(w.row0 + query_of(a, m)) * a.ld_q + (size_t)head_of(a, kvh, m) * HD + at % CPR * 8;
      if constexpr (TERMS == 1) {
        piece[0][p] = *(const uint4 *)((const bf16_t *)a.q + o);
      } else {
        const float4 u = *(const float4 *)((const float *)a.q + o), v = *((const float4 *)((const float *)a.q + o) + 1);
        float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
        bf16x8_t y[TERMS];
        split8<TERMS>(f, y);
#pragma unroll
        for (int t = 0; t < TERMS; ++t) piece[t][p] = __builtin_bit_cast(uint4, y[t]);
      }
    }
    if (tid < STAGE) {
      const int m = m0 + tid, mc = min(m, n_rows - 1);
      lse2 = x.lse2[row_id(a, w.req, query_of(a, mc), head_of(a, kvh, mc))];
      if (m >= n_rows || lse2 == -INFINITY) lse2 = INFINITY;
    }
  };
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  auto store = [&](int buf) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int at = p * 64 * WAVES + tid;
      if (at >= STAGE * CPR) continue;
#pragma unroll
      for (int t = 0; t < TERMS; ++t) {
        const uint4 u = piece[t][p];
        sq[buf][t][at / CPR * CPR + (at % CPR ^ swizzle(at / CPR))] = make_uint4(u.x ^ flip, u.y ^ flip, u.z ^ flip, u.w ^ flip);
      }
    }
    if (tid < STAGE) slse[buf][tid] = lse2;
  };

  const int first = max(0, b0 - w.ctx) * a.group / ROWS * ROWS;      // rows before it see none of the block's tokens
  load(first);
  bf16x8_t kf[4][NS];
  uint32_t tok[4];
  bool ok[4];
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    tok[j] = token_of(a.c, table, kvh, t0 + 16 * j + i, end, ok[j]);
    const KCodes<HD> k = load_k<HD, false>(a.c.k + (size_t)tok[j] * (HD / 2) + g * (HD / 8));
    const float ks = kv4::scale_value(a.c.k_scale[(size_t)tok[j] * NG + g * (HD / 4) / kv4::GROUP]);
#pragma unroll
    for (int st = 0; st < NS; ++st) kf[j][st] = kv4::decode8(k.w[st], ks);
  }
  store(0);
  auto stage = [&](int m0, int buf, auto masked) {
#pragma unroll
    for (int r0 = 0; r0 < STAGE; r0 += ROWS) {         // (behind the last row: nothing is added)
      bf16x8_t q[TERMS][NS];
#pragma unroll
      for (int t = 0; t < TERMS; ++t)
#pragma unroll
        for (int st = 0; st < NS; ++st) q[t][st] = __builtin_bit_cast(bf16x8_t, sq[buf][t][(r0 + i) * CPR + ((g * (CPR / 4) + st) ^ swizzle(i))]);
      const f32x4_t ls = *(const f32x4_t *)(slse[buf] + r0 + 4 * g);
      f32x4_t s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t][st], kf[j][st], s[j], 0, 0, 0);
      }
      int last[4];                                     // this row sees the wave's tokens below it, counted from i
      if constexpr (masked) {
#pragma unroll
        for (int r = 0; r < 4; ++r) last[r] = w.ctx + query_of(a, m0 + r0 + 4 * g + r) + 1 - t0 - i;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[j][r], sc, -ls[r]));
          sum[j] += !masked || 16 * j < last[r] ? p : 0.f;      // (masked behind the exponential: a row whose log sum is NaN adds nothing where it does not look)
        }
    }
  };
  int buf = 0;
  for (int m0 = first; m0 < n_rows; m0 += STAGE, buf ^= 1) {
    __syncthreads();
    if (m0 + STAGE < n_rows) load(m0 + STAGE);
    // one branch for a stage, not for its tiles, so that the products of a tile run beside the exponentials of the one before
    if (t0 + TURN <= w.ctx + query_of(a, m0) + 1) stage(m0, buf, std::false_type{});
    else stage(m0, buf, std::true_type{});
    if (m0 + STAGE < n_rows) store(buf ^ 1);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    sum[j] += __shfl_xor(sum[j], 16, 64);
    sum[j] += __shfl_xor(sum[j], 32, 64);
    if (g == j && ok[j]) unsafeAtomicAdd(a.c.weight + tok[j], sum[j]);
  }
}

// Splits of `chunk` tokens.  Bounds are powers of two as a rule, and the rows' own tokens come on top: a tail of up to a turn is the last split's where that leaves one split (no join:
// 16 requests of 1024 tokens, 8 kv heads of 128, 14 us, and 17 with a split for the tail; 128 of 4096 122 and 162; 256 of 16384 749 and 797) or the chip is full; else a block of its
// own costs nothing (4 of 2048 17.4, and 19 in the last split).
int splits_for(long long blocks, int tokens, int chunk) {
  const int n = std::max(1, cdiv(tokens - TURN, chunk));
  return n == 1 || blocks * n >= 512 ? n : cdiv(tokens, chunk);
}
// Tokens of a block: 4096, less where that makes fewer blocks than two a CU, not below four turns of its waves (a second launch to join splits costs
// more than it saves below that).  us at 256 / 512 / 1024 / 2048 / 4096 tokens, one row a request, 4 query heads a kv head: 4 requests of 400 - 1000 tokens, 8 kv heads of 128
// 14.6 / 12.6 / 11.2 / 11.5 / 12.0; 16 of 1500 - 4000 23.1 / 23.9 / 21.4 / 22.3 / 30.0; 64 of 1500 - 4000 69 / 61 / 59 / 58 / 51; 1 of 60000 29.8 / 25.8 / 24.2 / 24.5 / 33.9.
// Requests of up to 16384 tokens are not split where there are six blocks a CU without that, since a block's first loads and its end are worth two turns: at 4096 and whole 256 of 4000 - 16000 640 and
// 546, 192 of them with 64-wide heads 314 and 278, 1024 2334 and 1862 (1024 blocks, 32 requests of 32 kv heads: 248 and 259; 300 of 1000 - 60000: 1784, and 2177 at 16384, where the last
// long ones are alone).  More than 65536 blocks are never wanted, nor more than 16384 where a request has several tiles (one piece of 4096 fp32 rows at 16000: 4800 and 4400), so that
// there are no more than 2^20 states of rows: 537 MB of sums and 8 of maxima and sums of exponentials.
int chunk_tokens(int n_req, int tiles, int Hkv, int tokens) {
  const long long blocks = (long long)n_req * Hkv * tiles;
  int chunk = blocks >= 1536 && splits_for(blocks, tokens, 16384) == 1 ? 16384 : 4096;
  while (chunk > 4 * WAVES * TURN && blocks * splits_for(blocks, tokens, chunk) < 512) chunk /= 2;
  while (chunk < tokens && blocks * splits_for(blocks, tokens, chunk) > (tiles > 1 ? 16384 : 65536)) chunk *= 2;
  return chunk;
}
// Rows of a kv head up to which the first kernel takes bf16 requests, tile by tile; us on it and on the kernel of many rows, 64 requests of 2000 tokens, 8 kv heads: 16 / 24 / 32 rows
// of 128-wide heads 48 and 84 / 87 and 80 / 85 and 80, 32 / 48 / 64 rows of 64-wide ones 47 and 64 / 66 and 85 / 89 and 84.
int few_rows(int hd) { return hd == 128 ? 16 : 48; }
// Splits of a block of rows: two thread blocks a CU, or splits of four turns.
int rows_chunk(int n_req, int tiles, int Hkv, int tokens) {
  const long long blocks = (long long)n_req * Hkv * tiles;
  const int nsplit = (int)std::max(1ll, std::min<long long>(cdiv(tokens, 4 * TURN), (512 + blocks - 1) / blocks));
  return cdiv(cdiv(tokens, nsplit), TURN) * TURN;
}
// Thread blocks of a kv head for shares, two a CU in all; 0: blocks of rows and their splits are the thread blocks, long ones first.  That is for many blocks of rows, for twice as many as run at once
// that come from long pieces, whose blocks are alike, and for short work, where finding the shares costs more than they give; few rows a request, of any lengths, need shares.  us by
// blocks and by shares, 8 kv heads of 128: a piece of 4096 rows behind 4096 tokens 659 and 702, three of 600 to 2000 rows 173 and 196; 96 requests of 5 to 60 rows at 500 to 6000 tokens 635
// and 477, 120 of them 727 and 522 (16 of 256 rows at 4000 each, 32 heads: 458 and 458); one of 64 rows at 2000 24 and 31, 64 of 8 rows at 300 to 700 30 and 41, 32 of 5 to 30 rows
// at 300 to 2000, 16 turns a share, 67 and 56, six of 37 to 256 rows at 1000 to 2000, 24 turns, 93 and 70.
constexpr int ENOUGH = 2000, ENOUGH_ALIKE = 1024, ALIKE = 16, SHORT = 14;
int workers_of(int n_req, int tiles, int Hkv, int tokens) {
  const long long blocks = (long long)n_req * tiles, turns = blocks * cdiv(tokens, TURN);
  const int workers = std::max(1, 512 / Hkv);
  return blocks * Hkv >= (tiles >= ALIKE ? ENOUGH_ALIKE : ENOUGH) || turns < (long long)SHORT * workers ? 0 : workers;
}
static_assert(ENOUGH * (((1ll << 26) + 65535) / TURN + 1) < INT32_MAX, "turns of a kv head");
// Copies of a row in a tile: as many as rows and scale groups leave room for.
int copies(int rows, int hd) { return rows <= 4 && hd == 128 ? 4 : rows <= 8 ? 2 : 1; }

struct Plan {
  bool many;                 // blocks of many rows, by `workers` a kv head where that is not 0
  int rep, tile_rows, tiles, nsplit, chunk, workers;
  size_t rows;
};
Plan plan_of(int n_req, int max_rows, int max_context, int Hq, int Hkv, int hd, bool bf16) {
  Plan p;
  const int rows = max_rows * (Hq / Hkv), tokens = max_context + max_rows;
  p.many = bf16 && rows > few_rows(hd);
  p.rep = copies(rows, hd);
  p.tile_rows = p.many ? BLOCK_ROWS : ROWS / p.rep;
  p.tiles = cdiv(rows, p.tile_rows);
  p.workers = p.many ? workers_of(n_req, p.tiles, Hkv, tokens) : 0;
  p.chunk = p.workers ? tokens : p.many ? rows_chunk(n_req, p.tiles, Hkv, tokens) : chunk_tokens(n_req, p.tiles, Hkv, tokens);
  p.nsplit = p.many ? cdiv(tokens, p.chunk) : splits_for((long long)n_req * Hkv * p.tiles, tokens, p.chunk);
  p.rows = (size_t)n_req * max_rows * Hq;
  return p;
}
// A workspace: log sums of all rows, states of the splits (acc for several only) or shares and what they leave.
struct Layout {
  size_t lse2, ml, start, acc, bytes;
};
Layout layout_of(const Plan &p, int Hkv, int hd) {
  Layout l;
  const size_t states = p.workers ? (size_t)Hkv * p.workers * 2 * BLOCK_ROWS : p.rows * p.nsplit;
  l.lse2 = 0;
  l.ml = align_up(p.rows * sizeof(float), 256);
  l.start = l.ml + align_up(states * sizeof(float2), 256);
  l.acc = l.start + (p.workers ? align_up((size_t)Hkv * p.workers * sizeof(int4), 256) : 0);
  l.bytes = l.acc + (p.workers || p.nsplit > 1 ? states * hd * sizeof(float) : 0);
  return l;
}

}  // namespace

size_t kv4_attention_scratch_bytes(int n_req, int max_rows, int max_context, int Hq, int Hkv, int hd, bool bf16) {
  return layout_of(plan_of(n_req, max_rows, max_context, Hq, Hkv, hd, bf16), Hkv, hd).bytes;
}

hipError_t launch_kv4_attention(const Kv4Attention &a, bool bf16, void *scratch, hipStream_t st) {
  if (a.n_req <= 0 || a.n_rows <= 0) return hipSuccess;
  const int Hkv = a.c.Hkv, hd = a.c.hd, tokens = a.max_context + a.max_rows;
  const Plan p = plan_of(a.n_req, a.max_rows, a.max_context, Hkv * a.group, Hkv, hd, bf16);
  const bool runs = a.c.bshift >= 4;
  char *at = (char *)scratch;
  const Layout l = layout_of(p, Hkv, hd);
  const States x = {(float *)(at + l.acc), (float2 *)(at + l.ml), (float *)(at + l.lse2), p.nsplit, p.chunk, p.tile_rows};
  const Shares shares = {(float *)(at + l.acc), (float2 *)(at + l.ml), (float *)(at + l.lse2), (int4 *)(at + l.start), p.workers, p.nsplit, cdiv(p.chunk, TURN)};
  auto main = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(Hkv * p.tiles, p.nsplit, a.n_req), dim3(64 * WAVES), 0, st, a, x, p.tiles); };
  auto many = [&](auto kernel, auto join) {
    hipLaunchKernelGGL(kernel, p.workers ? dim3(Hkv * p.workers) : dim3(Hkv * p.tiles, a.n_req, p.nsplit), dim3(64 * WAVES), 0, st, a, shares);
    if (p.workers > 1) hipLaunchKernelGGL(join, dim3(p.workers - 1, Hkv, BLOCK_ROWS * (hd / 4) / (64 * WAVES)), dim3(64 * WAVES), 0, st, a, shares);
  };
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
    if constexpr (T == 1) {
      if (p.many) hd == 128 ? many(kv4_rows_kernel<128>, kv4_rows_join_kernel<128>) : many(kv4_rows_kernel<64>, kv4_rows_join_kernel<64>);
    }
    if (p.many) {}
    else if (hd == 128) p.rep == 4 ? main(kv4_attention_kernel<128, T, 4, R>) : p.rep == 2 ? main(kv4_attention_kernel<128, T, 2, R>) : main(kv4_attention_kernel<128, T, 1, R>);
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
