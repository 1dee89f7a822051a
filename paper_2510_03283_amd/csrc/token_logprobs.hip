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

constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.44269504088896340736f;
constexpr float FAR = -1e4f;            // differences of logits below this have e^x = 0; clamped, 0 times one is 0 and not NaN

// 16 bytes of a row: 4 fp32 or 8 bf16 values.  Rows start at any element (odd vocabularies, padded heads), and a 16-byte access needs
// no more than its elements' alignment: a wave's 1 KB then touches one cache line more.
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
template <bool BF16>
struct Chunk {
  static constexpr int N = BF16 ? 8 : 4;
  typedef typename std::conditional<BF16, u32x4_a2, u32x4_a4>::type raw_t;
  raw_t raw;
  __device__ __forceinline__ void load(const void *row, int col) { raw = *(const raw_t *)((const char *)row + (size_t)col * (BF16 ? 2 : 4)); }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (BF16) return __uint_as_float(i & 1 ? raw[i >> 1] & 0xffff0000u : raw[i >> 1] << 16);
    else return __uint_as_float(raw[i]);
  }
  // columns col .. col + N - 1, -inf from `end` on
  __device__ __forceinline__ void load_edge(const void *row, int col, int end) {
    if (col + N <= end) return load(row, col);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        const uint32_t lo = col + 2 * i < end ? ((const bf16_t *)row)[col + 2 * i] : 0xff80u, hi = col + 2 * i + 1 < end ? ((const bf16_t *)row)[col + 2 * i + 1] : 0xff80u;
        w[i] = lo | hi << 16;
      } else {
        w[i] = col + i < end ? ((const uint32_t *)row)[col + i] : 0xff800000u;
      }
    }
    raw = raw_t{w[0], w[1], w[2], w[3]};
  }
};

__device__ __forceinline__ float exp_of(float t) { return __builtin_amdgcn_exp2f(t * LOG2E); }
__device__ __forceinline__ bool better(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// What a set of columns contributes: ones + rest = sum e^(x - m), u = sum (x - m) e^(x - m).  `ones` counts columns that hold the
// maximum (at least one of each thread that met it; others are in rest), so that the logarithm of a sum just above 1 keeps its digits.
struct State {
  float m, ones, rest, u;
};
template <int NT>
__device__ __forceinline__ float3 block_sum3(float3 v, float (*red)[3]) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    v.x += __shfl_xor(v.x, o, 64);
    v.y += __shfl_xor(v.y, o, 64);
    v.z += __shfl_xor(v.z, o, 64);
  }
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) { red[w][0] = v.x; red[w][1] = v.y; red[w][2] = v.z; }
  __syncthreads();
  float3 t = make_float3(red[0][0], red[0][1], red[0][2]);
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) { t.x += red[i][0]; t.y += red[i][1]; t.z += red[i][2]; }
  return t;
}

struct Row {
  float m, L;          // statistics as they are reported
  bool empty, bad;
  __device__ __forceinline__ float logp(float x) const { return bad ? NAN : empty ? -INFINITY : x - m - L; }
};
__device__ __forceinline__ Row finish(const State &t, const TokenLogprobs &a, size_t r, float x_token, bool writes) {
  Row o;
  const float s = t.ones + t.rest;
  o.bad = s != s;
  o.empty = s == 0.f;
  o.m = o.bad ? NAN : o.empty ? -INFINITY : t.m;
  o.L = o.bad ? NAN : o.empty ? 0.f : log1pf((t.ones - 1.f) + t.rest);
  if (writes) {
    if (a.row_stats) {
      a.row_stats[2 * r] = o.m;
      a.row_stats[2 * r + 1] = o.L;
    }
    if (a.entropy) a.entropy[r] = o.empty ? 0.f : o.L - t.u / s;
    if (a.logp) {
      const int tok = a.token_ids[r];
      a.logp[r] = tok >= 0 && tok < a.vocab ? o.logp(x_token) : 0.f;
    }
  }
  return o;
}

constexpr int NT = 256, U = 4;                   // threads of a block; 16-byte accesses of a thread in a turn
constexpr int MAX_TURNS = 32;                    // turns of a part (LDS: 64 group maxima each)
constexpr int CAND = 1024;                       // candidates for the alternatives that LDS holds

// Columns [c0, c1) of a row.  A turn is NT * U consecutive 16-byte accesses; the four lanes of a quad hold U x 64 bytes of it, a
// group, whose maximum is kept: the alternatives are then found without a second pass over the row.
template <bool BF16>
struct Turn {
  static constexpr int N = Chunk<BF16>::N, COLS = NT * U * N, GROUPS = NT / 4, GROUP_COLS = 4 * U * N;
  static __device__ __forceinline__ int column(int turn, int u, int thread) { return turn * COLS + (u * NT + thread) * N; }
};

struct TopScratch {
  float group[MAX_TURNS * NT / 4];
  float quad[64];
  float v[CAND];
  int id[CAND];
  int list[MAX_TURNS * NT / 4];
  int n_list, n_cand, scan[4];
  float tau;
};

// Appends the columns of the listed groups whose value passes (strict ? > : >=) tau; a wave reads eight groups at a time.
template <bool BF16>
__device__ void collect(TopScratch &S, const void *row, int c0, int c1, float tau, bool strict) {
  using T = Turn<BF16>;
  constexpr int PER = T::GROUP_COLS / 64;        // values of a lane and group
  const int lane = threadIdx.x & 63, n = S.n_list;
  for (int i0 = (threadIdx.x >> 6) * 8; i0 < n; i0 += 32) {
    float x[8 * PER];
    int col[8 * PER];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int g = S.list[min(i0 + k, n - 1)];
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int at = lane + 64 * e, u = at / (4 * T::N), in = at % (4 * T::N);
        const int c = c0 + T::column(g / T::GROUPS, u, 4 * (g % T::GROUPS)) + in;
        col[k * PER + e] = i0 + k < n && c < c1 ? c : -1;
        x[k * PER + e] = ld_io<BF16>(row, min(c, c1 - 1));
      }
    }
#pragma unroll
    for (int k = 0; k < 8 * PER; ++k)
      if (col[k] >= 0 && (strict ? x[k] > tau : x[k] >= tau)) {
        const int at = atomicAdd(&S.n_cand, 1);
        if (at < CAND) { S.v[at] = x[k]; S.id[at] = col[k]; }
      }
  }
}

__device__ __forceinline__ void list_groups(TopScratch &S, int n_groups, float tau, bool strict) {
  for (int i = threadIdx.x; i < n_groups; i += NT)
    if (strict ? S.group[i] > tau : S.group[i] >= tau) S.list[atomicAdd(&S.n_list, 1)] = i;
}

__device__ __forceinline__ int rank_of(const TopScratch &S, int i, int n) {
  int r = 0;
  for (int j = 0; j < n; ++j) r += better(S.v[j], S.id[j], S.v[i], S.id[i]) ? 1 : 0;
  return r;
}

// The k best of columns [c0, c1): leaves at least min(k, allowed columns) of them, the best among them, in S.v / S.id and
// returns their number.  m: this thread's maximum, LOWEST if it met none.
//  - tau, the k-th largest of 64 maxima of disjoint sets (the quads' columns), has at least k columns at or above it, and no
//    more than about -64 log(1 - k / 64) where the values are spread by chance: 24 of them for k = 20, 44 for k = 32.
//  - groups whose maximum reaches tau are read again (k groups, 1 KB each, of a row of 125 or more).
//  - where more than CAND columns pass (many equal logits: a mask of the lowest value, or an ascending row), tau is raised to the
//    k-th largest of the CAND that were kept until the columns ABOVE it fit, and if those are fewer than k, columns equal to tau
//    fill up from the lowest on.
template <bool BF16>
__device__ int best_columns(TopScratch &S, const void *row, int c0, int c1, int turns, int k, float m) {
  using T = Turn<BF16>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_groups = turns * T::GROUPS;
  m = fmaxf(m, __shfl_xor(m, 1, 64));
  m = fmaxf(m, __shfl_xor(m, 2, 64));
  if ((lane & 3) == 0) S.quad[threadIdx.x >> 2] = m;
  if (threadIdx.x == 0) S.n_list = S.n_cand = 0;
  __syncthreads();
  if (wave == 0) {
    const float v = S.quad[lane];
    int r = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) r += better(S.quad[j], j, v, lane) ? 1 : 0;
    if (r == k - 1) S.tau = v;
  }
  __syncthreads();
  float tau = S.tau;
  list_groups(S, n_groups, tau, false);
  __syncthreads();
  collect<BF16>(S, row, c0, c1, tau, false);
  __syncthreads();
  int n = S.n_cand;
  if (n <= CAND) return n;
  for (bool first = true;; first = false) {
    if (!first) {                                // CAND columns above tau are here: their k-th best is above tau too
      for (int i = threadIdx.x; i < CAND; i += NT)
        if (rank_of(S, i, CAND) == k - 1) S.tau = S.v[i];
      __syncthreads();
      tau = S.tau;
    }
    __syncthreads();
    if (threadIdx.x == 0) S.n_list = S.n_cand = 0;
    __syncthreads();
    list_groups(S, n_groups, tau, true);
    __syncthreads();
    collect<BF16>(S, row, c0, c1, tau, true);
    __syncthreads();
    n = S.n_cand;
    if (n <= CAND) break;
  }
  for (int c = c0; c < c1 && n < k; c += NT) {
    const int col = c + threadIdx.x;
    const bool tie = col < c1 && ld_io<BF16>(row, col) == tau;
    const unsigned long long b = __ballot(tie);
    __syncthreads();
    if (lane == 0) S.scan[wave] = __popcll(b);
    __syncthreads();
    int at = n + __popcll(b & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) {
      if (w < wave) at += S.scan[w];
      n += S.scan[w];
    }
    if (tie && at < k) { S.v[at] = tau; S.id[at] = col; }
  }
  __syncthreads();
  return min(n, max(k, S.n_cand));
}

// Floats of the partial results of one part when a row is shared by several blocks: State, then the part's alternatives, best first.
__host__ __device__ __forceinline__ size_t part_floats(int k) { return (size_t)(4 + 2 * k + 3) & ~(size_t)3; }

// One block per row, or per part of a row where there are few rows.  One pass over the logits with the running maximum of every
// thread: 9.5 vector instructions a logit, of which the exponential takes 4 slots.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(NT) void token_logprobs_kernel(const TokenLogprobs a, int parts, int part_turns, float *__restrict__ scratch) {
  using T = Turn<BF16>;
  __shared__ float red[NT / 64][3];
  __shared__ float redm[NT / 64];
  __shared__ typename std::conditional<TOP, TopScratch, int>::type S;
  for (long long w = blockIdx.x; w < (long long)a.n * parts; w += gridDim.x) {
    const long long r = parts == 1 ? w : w / parts;
    const int part = (int)(w - r * parts);
    const void *row = (const char *)a.logits + (size_t)r * a.ld * (BF16 ? 2 : 4);
    const int c0 = part * part_turns * T::COLS, c1 = min((long long)a.vocab, (long long)c0 + part_turns * T::COLS);
    const int turns = (c1 - c0 + T::COLS - 1) / T::COLS;
    float x_token = 0.f;
    if (parts == 1 && a.logp && threadIdx.x == 0) {          // asked for ahead of the row
      const int tok = a.token_ids[r];
      if (tok >= 0 && tok < a.vocab) x_token = ld_io<BF16>(row, tok);
    }
    float m = LOWEST, s = 0.f, u = 0.f;
    for (int t = 0; t < turns; ++t) {
      Chunk<BF16> x[U];
      if (c0 + (t + 1) * T::COLS <= c1) {
#pragma unroll
        for (int i = 0; i < U; ++i) x[i].load(row, c0 + T::column(t, i, threadIdx.x));
      } else {
#pragma unroll
        for (int i = 0; i < U; ++i) x[i].load_edge(row, c0 + T::column(t, i, threadIdx.x), c1);
      }
      float g = LOWEST;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < T::N; ++j) g = fmaxf(g, x[i].get(j));
      const float mn = fmaxf(m, g), d = fmaxf(m - mn, FAR), c = exp_of(d);
      u = c * (u + s * d);
      s *= c;
      m = mn;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < T::N; ++j) {
          const float y = x[i].get(j) - m, e = exp_of(y);
          s += e;
          u += e * fmaxf(y, FAR);
        }
      if constexpr (TOP) {
        g = fmaxf(g, __shfl_xor(g, 1, 64));
        g = fmaxf(g, __shfl_xor(g, 2, 64));
        if ((threadIdx.x & 3) == 0) S.group[t * T::GROUPS + (threadIdx.x >> 2)] = g;
      }
    }
    State st;
    st.m = wave_max(m);
    if ((threadIdx.x & 63) == 0) redm[threadIdx.x >> 6] = st.m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) st.m = fmaxf(st.m, redm[i]);
    {
      const float d = fmaxf(m - st.m, FAR), c = exp_of(d);
      u = c * (u + s * d);
      s *= c;
      const bool one = m == st.m && s >= 1.f;
      const float3 t = block_sum3<NT>(make_float3(one ? 1.f : 0.f, one ? s - 1.f : s, u), red);
      st.ones = t.x; st.rest = t.y; st.u = t.z;
    }
    float *out = parts == 1 ? nullptr : scratch + (size_t)w * part_floats(a.top_k);
    Row o = {};
    if (parts == 1) o = finish(st, a, (size_t)r, x_token, threadIdx.x == 0);
    else if (threadIdx.x == 0) *(float4 *)out = make_float4(st.m, st.ones, st.rest, st.u);
    if constexpr (TOP) {
      const int k = a.top_k;
      const int n = best_columns<BF16>(S, row, c0, c1, turns, k, m);
      for (int i = threadIdx.x; i < n; i += NT) {
        const int at = rank_of(S, i, n);
        if (at >= k) continue;
        if (parts == 1) {
          a.top_ids[r * k + at] = o.bad ? -1 : S.id[i];
          if (a.top_logp) a.top_logp[r * k + at] = o.logp(S.v[i]);
        } else {
          out[4 + at] = S.v[i];
          out[4 + k + at] = __int_as_float(S.id[i]);
        }
      }
      for (int at = n + threadIdx.x; at < k; at += NT) {
        if (parts == 1) {
          a.top_ids[r * k + at] = -1;
          if (a.top_logp) a.top_logp[r * k + at] = o.bad ? NAN : -INFINITY;
        } else {
          out[4 + at] = -INFINITY;
          out[4 + k + at] = __int_as_float(-1);
        }
      }
    }
    __syncthreads();
  }
}

// Joins the parts of a row: one wave per row, part p in lane p.
template <bool BF16>
__global__ __launch_bounds__(64) void token_logprobs_join_kernel(const TokenLogprobs a, int parts, const float *__restrict__ scratch) {
  __shared__ float lv[64 * TOP_K_MAX];
  __shared__ int li[64 * TOP_K_MAX];
  const int lane = threadIdx.x, k = a.top_k;
  for (long long r = blockIdx.x; r < a.n; r += gridDim.x) {
    float x_token = 0.f;
    if (a.logp && lane == 0) {
      const int tok = a.token_ids[r];
      if (tok >= 0 && tok < a.vocab) x_token = ld_io<BF16>(a.logits, (size_t)r * a.ld + tok);
    }
    const float *in = scratch + (size_t)r * parts * part_floats(k);
    float4 t = make_float4(LOWEST, 0.f, 0.f, 0.f);
    if (lane < parts) t = *(const float4 *)(in + lane * part_floats(k));
    for (int i = lane; i < parts * k; i += 64) {
      const int p = i / k, at = i - p * k;
      lv[i] = in[p * part_floats(k) + 4 + at];
      li[i] = __float_as_int(in[p * part_floats(k) + 4 + k + at]);
    }
    State st;
    st.m = wave_max(t.x);
    const float d = fmaxf(t.x - st.m, FAR), c = exp_of(d), s = t.y + t.z;
    const bool top = t.x == st.m;
    st.u = wave_sum(c * (t.w + s * d));
    st.ones = wave_sum(top ? t.y : 0.f);
    st.rest = wave_sum(top ? t.z : c * s);
    const Row o = finish(st, a, (size_t)r, x_token, lane == 0);
    __syncthreads();
    int at = 0;
    for (int i = 0; i < k; ++i) {                // columns ascend with the part: on ties the lower lane
      float v = lane < parts && at < k ? lv[lane * k + at] : -INFINITY;
      const float best = wave_max(v);
      const unsigned long long who = __ballot(v == best && best > -INFINITY);
      const int winner = who ? __builtin_ctzll(who) : 0;
      if (lane == winner) {
        const bool none = !who;
        a.top_ids[r * k + i] = none || o.bad ? -1 : li[lane * k + at];
        if (a.top_logp) a.top_logp[r * k + i] = none && !o.bad ? -INFINITY : o.logp(v);
        if (!none) ++at;
      }
    }
    __syncthreads();
  }
}

// Blocks share the rows' columns, GRAD_U 16-byte accesses of a thread each; HBM-bound, one read and one write a logit.
constexpr int GRAD_U = 8;
template <bool BF16, bool OUT_BF16>
__global__ __launch_bounds__(NT) void token_logprobs_grad_kernel(const TokenLogprobsGrad a, int parts) {
  constexpr int N = Chunk<BF16>::N;
  for (long long w = blockIdx.x; w < (long long)a.n * parts; w += gridDim.x) {
    const long long r = parts == 1 ? w : w / parts;
    const int part = (int)(w - r * parts);
    const int tok = a.d_logp ? a.token_ids[r] : -1;
    const float g = tok >= 0 && tok < a.vocab ? a.d_logp[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f;
    const float m = a.row_stats[2 * r], L = a.row_stats[2 * r + 1], H = a.d_entropy ? a.entropy[r] : 0.f;
    const bool zero = m == -INFINITY || (g == 0.f && h == 0.f);
    const void *row = (const char *)a.logits + (size_t)r * a.ld * (BF16 ? 2 : 4);
    char *out = (char *)a.d_logits + (size_t)r * a.ld_d * (OUT_BF16 ? 2 : 4);
#pragma unroll
    for (int half = 0; half < GRAD_U / 4; ++half) {
      Chunk<BF16> x[4];
      const int base = (part * GRAD_U + half * 4) * NT * N;
      if (base >= a.vocab) break;
      if (!zero) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i].load_edge(row, base + (i * NT + (int)threadIdx.x) * N, a.vocab);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = base + (i * NT + (int)threadIdx.x) * N;
        float o[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          if (zero) { o[j] = 0.f; continue; }
          const float lp = x[i].get(j) - m - L, p = exp_of(lp);
          o[j] = (col + j == tok ? g : 0.f) - g * p - h * p * (fmaxf(lp, FAR) + H);
        }
        if (col + N <= a.vocab) {
          if constexpr (OUT_BF16) {
            if constexpr (BF16) *(u32x4_a2 *)(out + (size_t)col * 2) = u32x4_a2{cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]), cvt_pk_bf16(o[4], o[5]), cvt_pk_bf16(o[6], o[7])};
            else *(u32x2_a2 *)(out + (size_t)col * 2) = u32x2_a2{cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3])};
          } else {
#pragma unroll
            for (int j = 0; j < N; j += 4) *(f32x4_a4 *)(out + (size_t)(col + j) * 4) = f32x4_a4{o[j], o[j + 1], o[j + 2], o[j + 3]};
          }
        } else {
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (col + j < a.vocab) st_io<OUT_BF16>(out, col + j, o[j]);
        }
      }
    }
  }
}

// Parts of a row: one, unless there are too few rows to occupy the chip or a row is longer than the LDS has group maxima for.
// Counted for fp32 whatever the type, so that the scratch does not depend on it.
int parts_of(int n, int vocab) {
  const int turns = (vocab + Turn<false>::COLS - 1) / Turn<false>::COLS;
  int parts = (turns + MAX_TURNS - 1) / MAX_TURNS;
  if (n < 512) parts = std::max(parts, std::min({1024 / n, turns, 64}));
  return parts;
}

}  // namespace

size_t token_logprobs_scratch_bytes(int n, int vocab, int top_k) {
  if (n <= 0) return 0;
  const int parts = parts_of(n, vocab);
  return parts == 1 ? 0 : (size_t)n * parts * part_floats(top_k) * sizeof(float);
}

hipError_t launch_token_logprobs(const TokenLogprobs &a, bool bf16, void *scratch, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  int parts = parts_of(a.n, a.vocab);
  const int cols = bf16 ? Turn<true>::COLS : Turn<false>::COLS, turns = (a.vocab + cols - 1) / cols, part_turns = (turns + parts - 1) / parts;
  parts = (turns + part_turns - 1) / part_turns;
  const dim3 grid((unsigned)std::min<long long>((long long)a.n * parts, 1 << 22));
  auto *k = bf16 ? (a.top_k ? token_logprobs_kernel<true, true> : token_logprobs_kernel<true, false>)
                 : (a.top_k ? token_logprobs_kernel<false, true> : token_logprobs_kernel<false, false>);
  hipLaunchKernelGGL(k, grid, dim3(NT), 0, st, a, parts, part_turns, (float *)scratch);
  if (parts > 1) {
    const dim3 rows((unsigned)std::min(a.n, 1 << 22));
    if (bf16) hipLaunchKernelGGL(token_logprobs_join_kernel<true>, rows, dim3(64), 0, st, a, parts, (const float *)scratch);
    else hipLaunchKernelGGL(token_logprobs_join_kernel<false>, rows, dim3(64), 0, st, a, parts, (const float *)scratch);
  }
  return hipGetLastError();
}

hipError_t launch_token_logprobs_grad(const TokenLogprobsGrad &a, bool bf16, bool out_bf16, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  const int cols = GRAD_U * NT * (bf16 ? 8 : 4), parts = (a.vocab + cols - 1) / cols;
  auto *k = bf16 ? (out_bf16 ? token_logprobs_grad_kernel<true, true> : token_logprobs_grad_kernel<true, false>)
                 : (out_bf16 ? token_logprobs_grad_kernel<false, true> : token_logprobs_grad_kernel<false, false>);
  hipLaunchKernelGGL(k, dim3((unsigned)std::min<long long>((long long)a.n * parts, 1 << 22)), dim3(NT), 0, st, a, parts);
  return hipGetLastError();
}
