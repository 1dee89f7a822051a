// Log-probabilities of given tokens with the entropy and the best alternatives of their rows, and the gradient of both
// with respect to the logits.
//   m = max_j x_j,  L = log sum_j e^(x_j - m),  lp_j = x_j - m - L,  p_j = e^(lp_j)
//   logp = lp_token,   H = -sum_j p_j lp_j = L - sum_j (x_j - m) e^(x_j - m) / sum_j e^(x_j - m)
//   d logits_j = g ([j == token] - p_j) - h p_j (lp_j + H),    g = dL/dlogp, h = dL/dH
// A logit of -inf bans its token: p = 0 and no part in any sum.  A row with nothing but banned tokens has logp = -inf, H = 0 and
// gradient 0; NaN or +inf in a row make its results NaN.
#include "kernels.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
// Differences of logits (in units of log 2: FAR2) below these have an exponential of 0; clamped, 0 times one is 0 and not NaN.
constexpr float FAR = -1e4f, FAR2 = -1.4e4f;
// Up to this magnitude of a row's maximum the rounding of its product with log2 e is a small part of an exponent (at most 0.06).
constexpr float BIG = 1e6f;

// 16 bytes of a row: 4 fp32 or 8 bf16 values.  Rows start at any element (odd vocabularies, padded heads).  A 16-byte access needs no more than
// its elements' alignment, but a wave's 1 KB then touches one cache line more and, at an odd bf16 element, takes longer; long rows (LEAD) are cut where
// their address is a multiple of a line's 128 bytes: their columns are counted from up to 63 places before the row, which are not read.
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
template <bool BF16>
struct Chunk {
  static constexpr int N = BF16 ? 8 : 4;
  typedef typename std::conditional<BF16, u32x4_a2, u32x4_a4>::type raw_t;
  raw_t raw;
  template <bool STREAM>
  __device__ __forceinline__ void load(const void *row, int col) {
    const raw_t *p = (const raw_t *)((const char *)row + (size_t)col * (BF16 ? 2 : 4));
    if constexpr (STREAM) raw = __builtin_nontemporal_load(p);
    else raw = *p;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (BF16) return __uint_as_float(i & 1 ? raw[i >> 1] & 0xffff0000u : raw[i >> 1] << 16);
    else return __uint_as_float(raw[i]);
  }
  // columns col .. col + N - 1, -inf before 0 (LEAD) and from `end` on
  template <bool LEAD>
  __device__ __forceinline__ void load_edge(const void *row, int col, int end) {
    if ((!LEAD || col >= 0) && col + N <= end) return load<false>(row, col);
    const auto there = [&](int c) { return LEAD ? (unsigned)c < (unsigned)end : c < end; };
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        const int c = col + 2 * i;
        const uint32_t lo = there(c) ? ((const bf16_t *)row)[c] : 0xff80u, hi = there(c + 1) ? ((const bf16_t *)row)[c + 1] : 0xff80u;
        w[i] = lo | hi << 16;
      } else {
        w[i] = there(col + i) ? ((const uint32_t *)row)[col + i] : 0xff800000u;
      }
    }
    raw = raw_t{w[0], w[1], w[2], w[3]};
  }
};

constexpr int LINE = 128;
template <bool BF16>
__device__ __forceinline__ int lead_of(const void *row) { return (int)((uintptr_t)row % LINE) / (BF16 ? 2 : 4); }

// The reference of a thread's terms: its maximum in units of log 2, ROUNDED - as a product that is never contracted into what uses it.
__device__ __forceinline__ float reference_of(float m) {
#pragma clang fp contract(off)
  return fmaxf(m, -BIG) * LOG2E;
}
// u - delta s, the product rounded as the sum's own terms are: a row with one allowed token has an entropy of exactly 0.
__device__ __forceinline__ float without(float u, float delta, float s) {
#pragma clang fp contract(off)
  return u - delta * s;
}
__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * LOG2E); }

// Reductions over a wave without LDS: quads, halves and rows of 16 lanes by DPP, the four rows through scalar registers.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
constexpr int QUAD_XOR_1 = 0xB1, QUAD_XOR_2 = 0x4E, HALF_MIRROR = 0x141, MIRROR = 0x140;
__device__ __forceinline__ float lane_of(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }
__device__ __forceinline__ float max_quad(float x) {
  x = fmaxf(x, dpp<QUAD_XOR_1>(x));
  return fmaxf(x, dpp<QUAD_XOR_2>(x));
}
__device__ __forceinline__ float max_row16(float x) {
  x = max_quad(x);
  x = fmaxf(x, dpp<HALF_MIRROR>(x));
  return fmaxf(x, dpp<MIRROR>(x));
}
__device__ __forceinline__ float max_all(float x) {
  x = max_row16(x);
  return fmaxf(fmaxf(lane_of(x, 0), lane_of(x, 16)), fmaxf(lane_of(x, 32), lane_of(x, 48)));
}
__device__ __forceinline__ float sum_all(float x) {
  x += dpp<QUAD_XOR_1>(x);
  x += dpp<QUAD_XOR_2>(x);
  x += dpp<HALF_MIRROR>(x);
  x += dpp<MIRROR>(x);
  return (lane_of(x, 0) + lane_of(x, 16)) + (lane_of(x, 32) + lane_of(x, 48));
}

// What a set of columns contributes: ones + rest = sum e^(x - m), u = sum (x - m) e^(x - m).  `ones` counts columns that hold the
// maximum (one of each thread that met it; others are in rest), so that the logarithm of a sum just above 1 keeps its digits.
struct State {
  float m, ones, rest, u;
};

// log(1 + y), y >= 0, to about 2 ulp also where it is small: 2 artanh(y / (2 + y)) up to y = 0.5, where the first term left out is 4e-9.
__device__ __forceinline__ float log_1p(float y) {
  const float t = y * __builtin_amdgcn_rcpf(2.f + y), z = t * t;
  const float small = 2.f * fmaf(t * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 9.f, 1.f / 7.f), 1.f / 5.f), 1.f / 3.f), t);
  return y <= 0.5f ? small : __builtin_amdgcn_logf(1.f + y) * LN2;
}

struct Row {
  float m, L;          // statistics as they are reported
  int empty, bad;
  __device__ __forceinline__ float logp(float x) const { return bad ? NAN : empty ? -INFINITY : x - m - L; }
};
__device__ __forceinline__ Row finish(const State &t, const TokenLogprobs &a, size_t r, bool given, float x_token, bool writes) {
  Row o;
  const float s = t.ones + t.rest;
  o.bad = s != s;
  o.empty = s == 0.f;
  o.m = o.bad ? NAN : o.empty ? -INFINITY : t.m;
  o.L = o.bad ? NAN : o.empty ? 0.f : log_1p((t.ones - 1.f) + t.rest);
  if (writes) {
    if (a.row_stats) {
      a.row_stats[2 * r] = o.m;
      a.row_stats[2 * r + 1] = o.L;
    }
    if (a.entropy) a.entropy[r] = o.bad ? NAN : o.empty ? 0.f : fmaxf(o.L - t.u * __builtin_amdgcn_rcpf(s), 0.f);
    if (a.logp) a.logp[r] = given ? o.logp(x_token) : 0.f;
  }
  return o;
}

constexpr int U = 4;                             // 16-byte accesses of a thread in a turn
constexpr int RANK_STEP = 8;

// A turn of a block of NT threads is NT * U consecutive 16-byte accesses; the four lanes of a quad hold U x 64 bytes of it, a group,
// whose maximum is kept: the alternatives are then found without a second pass over the row.  MAX_GROUPS maxima fit the LDS (131072
// fp32 columns of a part with 256 or 512 threads, 8192 with 64), and CAND candidates.
template <bool BF16, int NT>
struct Turn {
  static constexpr int N = Chunk<BF16>::N, COLS = NT * U * N, GROUPS = NT / 4, GROUP_COLS = 4 * U * N;
  static constexpr int WAVES = NT / 64, MAX_GROUPS = NT == 64 ? 128 : 2048, MAX_TURNS = MAX_GROUPS / GROUPS, CAND = NT == 64 ? 512 : 1024;
  static __device__ __forceinline__ int column(int turn, int u, int thread) { return turn * COLS + (u * NT + thread) * N; }
};

// A column that may be among the best, as one number that is larger for the better one: the logit's bits, made monotonic, over the
// complement of the column (equal logits: the lower column).  -0 counts as 0.
typedef unsigned long long Candidate;
__device__ __forceinline__ Candidate candidate(float v, int col) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return (Candidate)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~col;
}
__device__ __forceinline__ float value_of(Candidate c) {
  const uint32_t b = (uint32_t)(c >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int column_of(Candidate c) { return (int)~(uint32_t)c; }
template <int NT>
struct TopScratch {
  using T = Turn<false, NT>;
  alignas(16) Candidate c[T::CAND + RANK_STEP];
  float group[T::MAX_GROUPS];
  uint16_t list[T::MAX_GROUPS];
  alignas(16) float set[64];
  int n_list, n_cand, scan[T::WAVES];
  float tau;
  Row row;
};

// Appends the passing lanes' items to a list in LDS whose length is *n: one atomic a wave; the order of the items is not used.
template <typename T>
__device__ __forceinline__ void append(T *list, int most, int *n, bool pass, T item) {
  const unsigned long long b = __ballot(pass);
  if (!b) return;
  int at = 0;
  if ((threadIdx.x & 63) == 0) at = atomicAdd(n, __popcll(b));
  at = __builtin_amdgcn_readfirstlane(at) + __popcll(b & ((1ull << (threadIdx.x & 63)) - 1));
  if (pass && at < most) list[at] = item;
}

// The k-th largest of 64 values, at least the lowest finite one; k <= 64.
__device__ __forceinline__ float kth_of_64(const float *set, int k) {
  const float v = set[threadIdx.x & 63];
  int above = 0;
#pragma unroll
  for (int j = 0; j < 64; j += 32) {
    float4 w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *(const float4 *)(set + j + 4 * i);
#pragma unroll
    for (int i = 0; i < 8; ++i) above += (w[i].x > v) + (w[i].y > v) + (w[i].z > v) + (w[i].w > v);
  }
  return fmaxf(-max_all(above < k ? -v : -INFINITY), LOWEST);      // the least of those with fewer than k above them
}

// Leaves the columns whose value passes (strict ? > : >=) tau in S.c and returns their number, of which S.c holds CAND: lists the
// groups whose maximum passes, and reads those again, eight loads of a wave at a time.
template <bool BF16, int NT, bool LEAD>
__device__ __forceinline__ int collect(TopScratch<NT> &S, const void *row, int c0, int c1, int n_groups, float tau, bool strict) {
  using T = Turn<BF16, NT>;
  constexpr int WAVES = T::WAVES, CAND = T::CAND;
  constexpr int PER = T::GROUP_COLS / 64, AT_ONCE = 8 / PER;    // adjacent columns of a lane and group; groups
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int g0 = 0; g0 < n_groups; g0 += NT) {
    const int g = g0 + (int)threadIdx.x;
    const float v = g < n_groups ? S.group[g] : NAN;
    append(S.list, T::MAX_GROUPS, &S.n_list, strict ? v > tau : v >= tau, (uint16_t)g);
  }
  __syncthreads();
  const int n = S.n_list;
  const int in_group = T::column(0, lane / 16, 0) + lane % 16 * PER;       // a group: U runs of 64 bytes
  for (int i0 = wave; i0 < n; i0 += WAVES * AT_ONCE) {
    float x[AT_ONCE][PER];
    int first[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      if (i0 + k * WAVES >= n) break;
      const int g = __builtin_amdgcn_readfirstlane((int)S.list[i0 + k * WAVES]);
      first[k] = c0 + T::column(g / T::GROUPS, 0, 4 * (g % T::GROUPS));
#pragma unroll
      for (int e = 0; e < PER; ++e) x[k][e] = ld_io<BF16>(row, LEAD ? max(0, min(first[k] + in_group + e, c1 - 1)) : first[k] + min(in_group + e, c1 - 1 - first[k]));
    }
    unsigned long long pass[AT_ONCE][PER];
    int total = 0, at = 0;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      if (i0 + k * WAVES >= n) break;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        pass[k][e] = __ballot((!LEAD || first[k] + in_group + e >= 0) && in_group + e < c1 - first[k] && (strict ? x[k][e] > tau : x[k][e] >= tau));
        total += __popcll(pass[k][e]);
      }
    }
    if (!total) continue;
    if (lane == 0) at = atomicAdd(&S.n_cand, total);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      if (i0 + k * WAVES >= n) break;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int mine = at + __popcll(pass[k][e] & ((1ull << lane) - 1));
        if (((pass[k][e] >> lane) & 1) && mine < CAND) S.c[mine] = candidate(x[k][e], first[k] + in_group + e);
        at += __popcll(pass[k][e]);
      }
    }
  }
  __syncthreads();
  return S.n_cand;
}

// How many of list[0 .. n) are better than c.  RANK_STEP at a time: the list is read up to that many places behind its end.
__device__ __forceinline__ int rank_of(const Candidate *list, Candidate c, int n) {
  int r = 0;
  for (int j = 0; j < n; j += RANK_STEP)
#pragma unroll
    for (int e = 0; e < RANK_STEP; ++e) r += list[j + e] > c ? j + e < n : 0;
  return r;
}

// More than CAND columns reach tau (many equal logits: a mask of the lowest value; a row in ascending order): tau is raised to the
// k-th largest of NT columns above it until those above it fit, and if they are fewer than k, columns equal to tau fill up,
// from the lowest on.
template <bool BF16, int NT, bool LEAD>
__device__ __noinline__ int best_columns_crowded(TopScratch<NT> &S, const void *row, int c0, int c1, int n_groups, int k, float tau) {
  constexpr int WAVES = NT / 64, CAND = Turn<BF16, NT>::CAND;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int n;
  for (;;) {
    __syncthreads();
    if (threadIdx.x == 0) S.n_list = S.n_cand = 0;
    __syncthreads();
    n = collect<BF16, NT, LEAD>(S, row, c0, c1, n_groups, tau, true);
    if (n <= CAND) break;
    const Candidate c = S.c[threadIdx.x];
    if (rank_of(S.c, c, NT) == k - 1) S.tau = value_of(c);
    __syncthreads();
    tau = S.tau;
  }
  const int above = n;
  for (int c = c0; c < c1 && n < k; c += NT) {
    const int col = c + threadIdx.x;
    const bool tie = (unsigned)col < (unsigned)c1 && ld_io<BF16>(row, col) == tau;
    const unsigned long long b = __ballot(tie);
    __syncthreads();
    if (lane == 0) S.scan[wave] = __popcll(b);
    __syncthreads();
    int at = n + __popcll(b & ((1ull << lane) - 1));
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) at += S.scan[w];
      n += S.scan[w];
    }
    if (tie && at < k) S.c[at] = candidate(tau, col);
  }
  __syncthreads();
  return min(n, max(k, above));
}

// The k best of columns [c0, c1): leaves at least min(k, allowed columns) of them, the best among them, in S.c and returns their
// number.  m: this thread's maximum, -inf if it met none.
// tau, the k-th largest of 64 maxima of disjoint sets of columns (a lane's, a quad's or of eight lanes), has at least k columns at or above it, and about
// -64 log(1 - k / 64) where the values are spread by chance: 24 for k = 20, 44 for k = 32.  The groups whose maximum reaches tau, about as
// many, are read again, 256 bytes each.
// meanwhile: what the last wave does while the first looks for tau.
template <bool BF16, int NT, bool LEAD, typename F>
__device__ __forceinline__ int best_columns(TopScratch<NT> &S, const void *row, int c0, int c1, int turns, int k, float m, F meanwhile) {
  using T = Turn<BF16, NT>;
  constexpr int SET = NT / 64;                   // threads of a set
  const int n_groups = turns * T::GROUPS;
  if (SET > 1) m = max_quad(m);
  if (SET == 8) m = fmaxf(m, dpp<HALF_MIRROR>(m));
  if (threadIdx.x % SET == 0) S.set[threadIdx.x / SET] = m;
  if (threadIdx.x == 0) S.n_list = S.n_cand = 0;
  __syncthreads();
  if (threadIdx.x < 64) {
    const float t = kth_of_64(S.set, k);
    if (threadIdx.x == 0) S.tau = t;
  }
  if (threadIdx.x >= NT - 64) meanwhile();
  __syncthreads();
  const float tau = S.tau;
  const int n = collect<BF16, NT, LEAD>(S, row, c0, c1, n_groups, tau, false);
  return n <= T::CAND ? n : best_columns_crowded<BF16, NT, LEAD>(S, row, c0, c1, n_groups, k, tau);
}

// Floats of the partial results of one part when a row is shared by several blocks: State, then the part's alternatives, best first.
__host__ __device__ __forceinline__ size_t part_floats(int k) { return (size_t)(4 + 2 * k + 3) & ~(size_t)3; }

// A block per row, or per part of a row.  One pass over the logits with a running maximum in every thread.  The exponent of a term is one
// fma, x log2 e - m2, with m2 the product for the maximum rounded to fp32: every term carries the factor 2^delta,
// delta = m log2 e - m2, which is taken out at the end (it is the term of the maximum itself).
// 32768 x 32000 fp32: 600 us, 7.0 TB/s, HBM-bound.  2048 x 128011 bf16 with 8 alternatives: 91 us, 5.8 TB/s, bound by vector instructions (a logit takes about 9
// slots, four of them its exponential).  One row of 32000 with 5 alternatives: 7 us, a chain of four turns, three reductions and a second look at some groups.
// Waves a SIMD, where the compiler's own choice of registers is not best: us with 4 / 5 / 6, 16384 x 32000 bf16 with 8 alternatives 236 / 220 / 231, 2048 x 128064 96 / 96 / 102, but
// 16384 x 32000 fp32 331 / 355 / 349; 64 threads, 30000 x 2048 bf16 5 / 6 67.6 / 75.6.
constexpr int waves_wanted(bool bf16, bool top, int nt) { return nt == 64 || (nt == 256 && bf16 && top) ? 5 : 1; }
template <bool BF16, bool ENT, bool TOP, int NT, bool STREAM, bool LEAD>
__global__ __launch_bounds__(NT, waves_wanted(BF16, TOP, NT)) void token_logprobs_kernel(const TokenLogprobs a, int parts, int part_turns, float *__restrict__ scratch) {
  using T = Turn<BF16, NT>;
  constexpr int WAVES = T::WAVES;
  __shared__ float red[4][WAVES];
  __shared__ typename std::conditional<TOP, TopScratch<NT>, int>::type S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long w = blockIdx.x; w < (long long)a.n * parts; w += gridDim.x) {
    const long long r = parts == 1 ? w : w / parts;
    const int part = (int)(w - r * parts);
    const void *row = (const char *)a.logits + (size_t)r * a.ld * (BF16 ? 2 : 4);
    const int c0 = part * part_turns * T::COLS - (LEAD ? lead_of<BF16>(row) : 0), c1 = min(a.vocab, c0 + part_turns * T::COLS);
    const int turns = (c1 - c0 + T::COLS - 1) / T::COLS;
    const int tok = parts == 1 && a.logp ? a.token_ids[r] : -1;          // asked for ahead of the row, used behind it
    float m = -INFINITY, m2 = -BIG * LOG2E, s = 0.f, u = 0.f;
    Chunk<BF16> next[U];
    const auto ask = [&](int t) {
      if ((!LEAD || c0 + t * T::COLS >= 0) && c0 + (t + 1) * T::COLS <= c1) {
#pragma unroll
        for (int i = 0; i < U; ++i) next[i].template load<STREAM>(row, c0 + T::column(t, i, threadIdx.x));
      } else {
#pragma unroll
        for (int i = 0; i < U; ++i) next[i].template load_edge<LEAD>(row, c0 + T::column(t, i, threadIdx.x), c1);
      }
    };
    ask(0);
    for (int t = 0; t < turns; ++t) {
      Chunk<BF16> x[U];
#pragma unroll
      for (int i = 0; i < U; ++i) x[i] = next[i];
      if (t + 1 < turns) ask(t + 1);
      float g = -INFINITY;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < T::N; ++j) g = fmaxf(g, x[i].get(j));
      m = fmaxf(m, g);
      const float mn = reference_of(m), d = fmaxf(m2 - mn, FAR2), c = __builtin_amdgcn_exp2f(d);
      if constexpr (ENT) u = c * (u + s * d);
      s *= c;
      m2 = mn;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < T::N; ++j) {
          const float y = fmaf(x[i].get(j), LOG2E, -m2), e = __builtin_amdgcn_exp2f(y);
          s += e;
          if constexpr (ENT) u += e * fmaxf(y, FAR2);
        }
      if constexpr (TOP) {
        g = max_quad(g);
        if ((threadIdx.x & 3) == 0) S.group[t * T::GROUPS + (threadIdx.x >> 2)] = g;
      }
    }
    const bool given = tok >= 0 && tok < a.vocab;
    const float x_token = given ? ld_io<BF16>(row, tok) : 0.f;
    State st;
    st.m = max_all(m);
    if (lane == 0) red[3][wave] = st.m;
    __syncthreads();
    st.m = red[3][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) st.m = fmaxf(st.m, red[3][i]);
    // This thread's sums relative to its maximum, the maximum's own term (e0) left out: sum e^(x - m) = 1 + s.  A thread that met
    // nothing near the row's maximum has none.
    float top = m;
    bool one;
    if (fabsf(st.m) <= BIG || st.m == -INFINITY) {          // (-inf: nothing but banned tokens, no term is there)
      const float delta = fmaf(m, LOG2E, -m2), e0 = __builtin_amdgcn_exp2f(delta);
      one = s > 0.f && e0 > 1e-30f;
      const float inv = __builtin_amdgcn_rcpf(e0);
      if constexpr (ENT) u = one ? without(u, delta, s) * (LN2 * inv) : 0.f;
      s = one ? (s - e0) * inv : s;
    } else {                                     // a maximum of huge magnitude: again, with differences of the logits themselves
      top = st.m;
      s = u = 0.f;
      for (int t = 0; t < turns; ++t) {
        ask(t);
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
          for (int j = 0; j < T::N; ++j) {
            const float y = next[i].get(j) - top, e = exp_of(y);
            s += e;
            if constexpr (ENT) u += e * fmaxf(y, FAR);
          }
      }
      one = s >= 1.f;
      s = one ? s - 1.f : s;
    }
    {
      const float d = fmaxf(top - st.m, FAR), c = exp_of(d), all = one ? 1.f + s : s;
      const bool is_top = one && top == st.m;
      st.ones = sum_all(is_top ? 1.f : 0.f);
      st.rest = sum_all(is_top ? s : c * all);
      st.u = ENT ? sum_all(c * (u + all * d)) : 0.f;
      if (lane == 0) { red[0][wave] = st.ones; red[1][wave] = st.rest; red[2][wave] = st.u; }
      __syncthreads();
      st.ones = red[0][0]; st.rest = red[1][0]; st.u = red[2][0];
#pragma unroll
      for (int i = 1; i < WAVES; ++i) { st.ones += red[0][i]; st.rest += red[1][i]; st.u += red[2][i]; }
    }
    float *out = parts == 1 ? nullptr : scratch + (size_t)w * part_floats(a.top_k);
    const bool writer = threadIdx.x == NT - 64;
    Row o = {};
    const auto results = [&]() {
      if (parts == 1) o = finish(st, a, (size_t)r, given, x_token, writer);
      else if (writer) *(float4 *)out = make_float4(st.m, st.ones, st.rest, st.u);
    };
    if constexpr (!TOP) {
      if (threadIdx.x >= NT - 64) results();
    } else {
      const int k = a.top_k;
      const int n = best_columns<BF16, NT, LEAD>(S, row, c0, c1, turns, k, m, [&]() {
        results();
        if (writer) S.row = o;
      });
      o = S.row;
      for (int i = threadIdx.x; i < max(n, k); i += NT) {
        const bool there = i < n;                // (not: the places behind the last allowed column)
        const Candidate c = there ? S.c[i] : 0;
        const int at = there ? rank_of(S.c, c, n) : i;
        if (at >= k) continue;
        const float v = there ? value_of(c) : -INFINITY;
        const int col = there ? column_of(c) : -1;
        if (parts == 1) {
          a.top_ids[r * k + at] = o.bad ? -1 : col;
          if (a.top_logp) a.top_logp[r * k + at] = o.bad ? NAN : there ? o.logp(v) : -INFINITY;
        } else {
          out[4 + at] = v;
          out[4 + k + at] = __int_as_float(col);
        }
      }
    }
    __syncthreads();
  }
}

// Joins the parts of a row: one block per row, part p in lane p.  Of the parts' alternatives those stay that reach the k-th best of 64
// of them, the first few of every part.
constexpr size_t LLC_BYTES = (size_t)256 << 20;
constexpr int JOIN_NT = 256;
template <bool BF16>
__global__ __launch_bounds__(JOIN_NT) void token_logprobs_join_kernel(const TokenLogprobs a, int parts, const float *__restrict__ scratch) {
  constexpr int MOST = 64 * TOP_K_MAX;
  __shared__ alignas(16) Candidate list[MOST + RANK_STEP];
  __shared__ alignas(16) float set[64];
  __shared__ int n_cand;
  const int lane = threadIdx.x & 63, k = a.top_k;
  const size_t stride = part_floats(k);
  for (long long r = blockIdx.x; r < a.n; r += gridDim.x) {
    const int tok = a.logp ? a.token_ids[r] : -1;
    const bool given = tok >= 0 && tok < a.vocab;
    const float *in = scratch + (size_t)r * parts * stride;
    float4 t = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (lane < parts) t = *(const float4 *)(in + lane * stride);
    if (k && threadIdx.x < 64) {                 // lane p + parts * i: alternative i of part p
      const int p = lane % parts, i = lane / parts;
      set[lane] = i < min(k, 64 / parts) ? in[p * stride + 4 + i] : -INFINITY;
      if (lane == 0) n_cand = 0;
    }
    const float x_token = given ? ld_io<BF16>(a.logits, (size_t)r * a.ld + tok) : 0.f;
    State st;
    st.m = max_all(t.x);
    const float d = fmaxf(t.x - st.m, FAR), c = exp_of(d), s = t.y + t.z;
    const bool top = t.x == st.m;
    st.u = sum_all(c * (t.w + s * d));
    st.ones = sum_all(top ? t.y : 0.f);
    st.rest = sum_all(top ? t.z : c * s);
    const Row o = finish(st, a, (size_t)r, given, x_token, threadIdx.x == 0);
    __syncthreads();
    if (k) {
      const float tau = kth_of_64(set, k);
      for (int i0 = 0; i0 < parts * k; i0 += JOIN_NT) {
        const int i = i0 + (int)threadIdx.x, p = i / k;
        float v = -INFINITY;
        int col = -1;
        if (i < parts * k) {
          const float *y = in + p * stride + 4 + (i - p * k);
          v = y[0];
          col = __float_as_int(y[k]);
        }
        append(list, MOST, &n_cand, v >= tau, candidate(v, col));
      }
      __syncthreads();
      const int n = n_cand;
      for (int i = threadIdx.x; i < max(n, k); i += JOIN_NT) {
        const bool there = i < n;
        const Candidate x = there ? list[i] : 0;
        const int at = there ? rank_of(list, x, n) : i;
        if (at >= k) continue;
        a.top_ids[r * k + at] = there && !o.bad ? column_of(x) : -1;
        if (a.top_logp) a.top_logp[r * k + at] = o.bad ? NAN : there ? o.logp(value_of(x)) : -INFINITY;
      }
    }
    __syncthreads();
  }
}

template <typename V, bool STREAM>
__device__ __forceinline__ void put(char *out, size_t at, V v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, (V *)(out + at));
  else *(V *)(out + at) = v;
}
// A wave takes 64 x U 16-byte accesses of a row; HBM-bound, one read and one write a logit (16384 x 32000 fp32 to bf16: 522 us, 6.0 TB/s).
template <bool BF16, bool OUT_BF16, bool LEAD, bool STREAM>
__global__ __launch_bounds__(256) void token_logprobs_grad_kernel(const TokenLogprobsGrad a, int parts) {
  constexpr int N = Chunk<BF16>::N;
  const int lane = threadIdx.x & 63;
  for (long long w = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < (long long)a.n * parts; w += (long long)gridDim.x * 4) {
    const long long r = parts == 1 ? w : w / parts;
    const void *row = (const char *)a.logits + (size_t)r * a.ld * (BF16 ? 2 : 4);
    char *out = (char *)a.d_logits + (size_t)r * a.ld_d * (OUT_BF16 ? 2 : 4);
    const int c0 = (int)(w - r * parts) * 64 * U * N - (LEAD ? lead_of<OUT_BF16>(out) : 0);
    const int tok = a.d_logp ? a.token_ids[r] : -1;
    const float g = tok >= 0 && tok < a.vocab ? a.d_logp[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f;
    const float m = a.row_stats[2 * r], L = a.row_stats[2 * r + 1], H = a.d_entropy ? a.entropy[r] : 0.f;
    const bool zero = m == -INFINITY || (g == 0.f && h == 0.f);
    Chunk<BF16> x[U];
    if (!zero) {
#pragma unroll
      for (int i = 0; i < U; ++i) x[i].template load_edge<LEAD>(row, c0 + (i * 64 + lane) * N, a.vocab);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int col = c0 + (i * 64 + lane) * N;
      float o[N];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (zero) { o[j] = 0.f; continue; }
        const float lp = x[i].get(j) - m - L, p = exp_of(lp);
        o[j] = (col + j == tok ? g : 0.f) - g * p - h * p * (fmaxf(lp, FAR) + H);
      }
      if ((!LEAD || col >= 0) && col + N <= a.vocab) {
        if constexpr (OUT_BF16) {
          if constexpr (BF16) put<u32x4_a2, STREAM>(out, (size_t)col * 2, u32x4_a2{cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]), cvt_pk_bf16(o[4], o[5]), cvt_pk_bf16(o[6], o[7])});
          else put<u32x2_a2, STREAM>(out, (size_t)col * 2, u32x2_a2{cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3])});
        } else {
#pragma unroll
          for (int j = 0; j < N; j += 4) put<f32x4_a4, STREAM>(out, (size_t)(col + j) * 4, f32x4_a4{o[j], o[j + 1], o[j + 2], o[j + 3]});
        }
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if ((!LEAD || col + j >= 0) && col + j < a.vocab) st_io<OUT_BF16>(out, col + j, o[j]);
      }
    }
  }
}

// Places that a row can lie behind the beginning of a line; whether any row does.
constexpr int most_lead(bool bf16) { return LINE / (bf16 ? 2 : 4) - 1; }
bool off_lines(const void *rows, long long ld, bool bf16) { return ((uintptr_t)rows | (uintptr_t)(ld * (bf16 ? 2 : 4))) % LINE != 0; }

// Blocks (parts) of a row: of up to 256 rows, parts of eight turns (32768 fp32 columns).  us with 20 alternatives, fp32, one part / parts of eight turns / of four:
// one row of 128011 14.7 / 12.1 / 11.1, 64 16.4 / 16.2 / 16.7; but one of 65536 9.6 / 11.5 / 10.8 and 256 of 128011 29.2 / 34.4 / 34.4, where a single part runs in blocks
// of 512 threads.  A row of 32000 has eight turns and is not shared: two blocks a row would take 10.4 instead of 7.5 for one row, 13.7 instead of 9.2 for 128, 16.8 instead of 11.2
// for 256, as the join is a launch of its own.  Counted for fp32 whatever the type, so that the scratch does not depend on it.
int parts_of(int n, int vocab) {
  using T = Turn<false, 256>;
  const int turns = (vocab + most_lead(false) + T::COLS - 1) / T::COLS, least = (turns + T::MAX_TURNS - 1) / T::MAX_TURNS;
  return std::max(least, std::min({512 / n, turns / 8, 64}));
}

template <bool BF16, bool ENT, bool TOP, int NT>
auto rows_kernel(bool stream, bool lead) {
  if constexpr (NT == 256)
    if (lead && stream) return token_logprobs_kernel<BF16, ENT, TOP, NT, true, true>;
  if constexpr (NT == 256 && BF16)
    if (lead) return token_logprobs_kernel<BF16, ENT, TOP, NT, false, true>;
  if constexpr (NT == 512) return token_logprobs_kernel<BF16, ENT, TOP, NT, false, false>;      // (256 parts of 131072 columns at most: never past the cache)
  else return stream ? token_logprobs_kernel<BF16, ENT, TOP, NT, true, false> : token_logprobs_kernel<BF16, ENT, TOP, NT, false, false>;
}
template <bool BF16, int NT>
hipError_t launch_rows(const TokenLogprobs &a, int parts, float *scratch, hipStream_t st) {
  using T = Turn<BF16, NT>;
  // Logits that the last-level cache (256 MB) cannot hold are read past it: 16384 x 32000 fp32 354 -> 317 us, 2048 x 32000 49.0 -> 42.5; of
  // fewer the cache may hold what their producer left (512 x 32000, three inputs in turn that it holds: 13.5 -> 14.1).
  const bool stream = (size_t)a.n * a.vocab * (BF16 ? 2 : 4) > LLC_BYTES;
  // Where rows do not begin with a line, us without / with a lead: 2048 x 128011 fp32 170 / 156, 2048 x 50257 69 / 65, but 512 x 31999 12.6 / 12.8, 4096 x 31999
  // with 8 alternatives 92 / 98; bf16, every other row at an odd element, 2048 x 128011 119 / 96, 4096 x 31999 63 / 58, 1024 x 31999 17.1 / 16.3, 4096 x 15999 40.3 / 36.3, but
  // 512 x 31999 9.8 / 10.3, 1024 x 8191 7.4 / 11.0.
  const bool lead = NT == 256 && off_lines(a.logits, a.ld, BF16) && (BF16 ? a.vocab >= 12288 && (long long)a.n * a.vocab >= 30 << 20 : stream && a.vocab >= 49152);
  const int turns = (a.vocab + (lead ? most_lead(BF16) : 0) + T::COLS - 1) / T::COLS, part_turns = (turns + parts - 1) / parts;
  parts = (turns + part_turns - 1) / part_turns;
  const dim3 grid((unsigned)std::min<long long>((long long)a.n * parts, 1 << 22));
  // Without the entropy its sum is left out as well: 2048 x 128011 bf16 93 -> 87 us, one row of 32000 4.5 -> 4.1, 16384 x 32000 185 -> 166.
  auto *k = a.entropy ? (a.top_k ? rows_kernel<BF16, true, true, NT>(stream, lead) : rows_kernel<BF16, true, false, NT>(stream, lead))
                      : (a.top_k ? rows_kernel<BF16, false, true, NT>(stream, lead) : rows_kernel<BF16, false, false, NT>(stream, lead));
  hipLaunchKernelGGL(k, grid, dim3(NT), 0, st, a, parts, part_turns, scratch);
  if (parts > 1) hipLaunchKernelGGL(token_logprobs_join_kernel<BF16>, dim3((unsigned)std::min(a.n, 1 << 22)), dim3(JOIN_NT), 0, st, a, parts, (const float *)scratch);
  return hipGetLastError();
}
template <bool BF16>
hipError_t launch_rows(const TokenLogprobs &a, float *scratch, hipStream_t st) {
  const int parts = parts_of(a.n, a.vocab);
  // A wave per row for many short rows, and for rows so short that the quads of 256 threads hold fewer sets than there are alternatives.
  // us with 256 threads / one wave, without and with 20 alternatives: 2048 x 2048 fp32 7.0 / 5.9, 15.9 / 13.5; 8192 x 4000 26.4 / 26.8, 61.9 / 48.1;
  // 30000 x 7000 133 / 137, 250 / 236; but 512 x 2048 4.0 / 3.9, 7.6 / 10.6.  64 x 500 bf16 with 20 alternatives 35.7 / 11.0.
  const int few = 128 * Turn<BF16, 256>::N;      // 32 quads with a column
  const bool wave = parts == 1 && (a.vocab <= few || (a.n >= 2048 && a.vocab <= 8192));
  if (wave) return launch_rows<BF16, 64>(a, 1, scratch, st);
  // Blocks of 512 threads where a CU has no more than one and its turn is not much wider than the row.  us with 256 / 512 threads, 20 alternatives: one row of
  // 32000 fp32 9.2 / 8.0, 64 10.1 / 8.8, 256 12.1 / 11.6, 320 13.5 / 14.2; one of 8000 6.7 / 6.3, without alternatives 3.6 / 3.6, of 4000 3.2 / 3.5; one of 32000
  // bf16 9.6 / 8.3, 256 11.5 / 10.7, one of 8000 without alternatives 3.6 / 4.2.  1024 threads: 8.3 for one row of 32000, 12.6 for 256.
  const bool wide = (long long)a.n * parts <= 256 && 4ll * a.vocab > 3 * Turn<BF16, 512>::COLS;
  return wide ? launch_rows<BF16, 512>(a, parts, scratch, st) : launch_rows<BF16, 256>(a, parts, scratch, st);
}

template <bool BF16, bool OUT_BF16>
auto grad_kernel(bool lead, bool stream) {
  return lead ? (stream ? token_logprobs_grad_kernel<BF16, OUT_BF16, true, true> : token_logprobs_grad_kernel<BF16, OUT_BF16, true, false>)
              : (stream ? token_logprobs_grad_kernel<BF16, OUT_BF16, false, true> : token_logprobs_grad_kernel<BF16, OUT_BF16, false, false>);
}

}  // namespace

size_t token_logprobs_scratch_bytes(int n, int vocab, int top_k) {
  if (n <= 0) return 0;
  const int parts = parts_of(n, vocab);
  return parts == 1 ? 0 : (size_t)n * parts * part_floats(top_k) * sizeof(float);
}

hipError_t launch_token_logprobs(const TokenLogprobs &a, bool bf16, void *scratch, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  return bf16 ? launch_rows<true>(a, (float *)scratch, st) : launch_rows<false>(a, (float *)scratch, st);
}

hipError_t launch_token_logprobs_grad(const TokenLogprobsGrad &a, bool bf16, bool out_bf16, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  // Whole lines written where rows do not begin with one, us without / with a lead: 8192 x 31999 fp32 427 / 408, bf16 232 / 196, 2048 x 128011 bf16 204 / 184, 16000 x 8191
  // 111 / 101, but 30000 x 4097 99 / 110.
  const bool lead = a.vocab >= 8192 && off_lines(a.d_logits, a.ld_d, out_bf16);
  const int cols = 64 * U * (bf16 ? 8 : 4), parts = (a.vocab + (lead ? most_lead(out_bf16) : 0) + cols - 1) / cols;
  // Gradients that the last-level cache cannot hold are written past it: 16384 x 32000 fp32 to bf16 557 -> 540 us, bf16 to bf16 373 -> 363.
  const bool stream = (size_t)a.n * a.vocab * (out_bf16 ? 2 : 4) > LLC_BYTES;
  auto *k = bf16 ? (out_bf16 ? grad_kernel<true, true>(lead, stream) : grad_kernel<true, false>(lead, stream))
                 : (out_bf16 ? grad_kernel<false, true>(lead, stream) : grad_kernel<false, false>(lead, stream));
  hipLaunchKernelGGL(k, dim3((unsigned)std::min<long long>(((long long)a.n * parts + 3) / 4, 1 << 22)), dim3(256), 0, st, a, parts);
  return hipGetLastError();
}
