// Eviction: every (request, kv head) keeps the `budget` tokens of largest key - the first n_sink positions, then the newest n_recent, then by accumulated weight, the
// lower token on ties - and its new length is min(tokens, budget).  What stays behind the new length moves into the holes in front of it, the i-th into
// the i-th, so no token is read where another is written, and only what has to move does.
//
// A block of 1024 threads a (request, kv head) holds the keys in registers (ITEMS a thread, a wave's tokens side by side), finds the budget-th largest
// in three turns of 11, 11 and 10 bits with a histogram in LDS, and numbers holes and displaced tokens with ballots.  The moves follow in the same
// launch or, for long lists, in one of their own that the whole chip takes part in.
#include "kernels.h"

#include <algorithm>

namespace {

constexpr int THREADS = 1024, NWAVES = THREADS / 64, BINS = 2048;
constexpr int MAX_ITEMS = 32;                       // keys a thread holds; longer caches read them again

struct Where {
  const int32_t *table;
  int kvh;
};
__device__ __forceinline__ uint32_t token_of(const Kv4Cache &c, const Where &w, int t, bool &ok) {
  const int blk = w.table[t >> c.bshift];
  ok = blk >= 0 && (uint32_t)blk < c.num_blocks;
  return ok ? (((uint32_t)blk * c.Hkv + w.kvh) << c.bshift) + (t & ((1 << c.bshift) - 1)) : 0u;
}

// Larger is kept.  Weights (negative ones and NaN count as 0) below the newest, by position, below the first, by position.  A token in a block that
// does not exist is the first to go.
__device__ __forceinline__ uint32_t key_of(const Kv4Evict &a, const Where &w, int t, int newest) {
  bool ok;
  const uint32_t tok = token_of(a.c, w, t, ok);
  if (!ok) return 0u;
  const float x = a.c.weight[tok];
  const int pos = a.c.position[tok];
  const uint32_t p = (uint32_t)min(max(pos, 0), 0x3fffffff);
  if (pos < a.n_sink) return 0xffffffffu - p;
  if (pos >= newest) return 0x80000000u + p;
  return x > 0.f ? __float_as_uint(x) : 0u;
}

// Moves token `from` to token `to` with the lanes of LANES threads.
template <int HD, int LANES>
__device__ __forceinline__ void move_token(const Kv4Cache &c, uint32_t to, uint32_t from, int lane) {
  constexpr int W = HD / 32;                         // 16-byte pieces of K
  if (lane < W) ((uint4 *)c.k)[(size_t)to * W + lane] = ((const uint4 *)c.k)[(size_t)from * W + lane];
  else if (lane < 2 * W) ((uint4 *)c.v)[(size_t)to * W + lane - W] = ((const uint4 *)c.v)[(size_t)from * W + lane - W];
  static_assert(LANES >= 2 * W, "a lane a piece");
  if (lane == 0) c.weight[to] = c.weight[from];
  if (lane == 1) c.position[to] = c.position[from];
  if (lane == 2) {
    if constexpr (HD == 128) ((uint32_t *)c.k_scale)[to] = ((const uint32_t *)c.k_scale)[from];
    else ((uint16_t *)c.k_scale)[to] = ((const uint16_t *)c.k_scale)[from];
  }
  if (lane == 3) {
    if constexpr (HD == 128) ((uint32_t *)c.v_scale)[to] = ((const uint32_t *)c.v_scale)[from];
    else ((uint16_t *)c.v_scale)[to] = ((const uint16_t *)c.v_scale)[from];
  }
}

// lists: [n_req, Hkv, 2, most] token numbers: holes, displaced; counts [n_req, Hkv].
template <int HD, int ITEMS>
__global__ __launch_bounds__(THREADS) void kv4_evict_kernel(Kv4Evict a, int most, int32_t *__restrict__ lists, int32_t *__restrict__ counts, bool move) {
  __shared__ uint32_t hist[BINS];
  __shared__ int wsum[NWAVES][2];
  __shared__ uint32_t found[2];                      // digit, tokens above it
  const int kvh = blockIdx.x, req = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Where w = {a.tables + (size_t)req * a.max_blocks, kvh};
  const int room = (int)min((long long)a.max_blocks << a.c.bshift, (long long)INT32_MAX);
  const int len = min(min(max(a.lens[(size_t)req * a.len_heads + (a.len_heads > 1 ? kvh : 0)], 0), a.max_context), room);
  const int keep = min(len, max(a.budgets[(size_t)req * a.c.Hkv + kvh], 0));
  const int newest = a.n_recent > 0 ? max(a.seq_lens[req] - a.n_recent, 0) : INT32_MAX;
  const size_t id = (size_t)req * a.c.Hkv + kvh;
  int32_t *holes = lists + id * 2 * most, *moved = holes + most;
  __syncthreads();                                   // new_lens may be lens
  if (tid == 0) {
    a.new_lens[id] = keep;
    counts[id] = 0;
  }
  if (keep == len || keep == 0) return;

  constexpr bool HELD = ITEMS > 0;
  const int per = HELD ? ITEMS : (len + THREADS - 1) / THREADS, t0 = wave * 64 * per + lane;         // this thread's tokens: t0 + 64 n
  uint32_t key[HELD ? ITEMS : 1];
  if constexpr (HELD) {
#pragma unroll
    for (int n = 0; n < ITEMS; ++n) key[n] = t0 + 64 * n < len ? key_of(a, w, t0 + 64 * n, newest) : 0u;
  }
  auto each = [&](auto f) {
    if constexpr (HELD) {
#pragma unroll
      for (int n = 0; n < ITEMS; ++n) f(t0 + 64 * n, key[n]);
    } else {
      for (int n = 0; n < per; ++n) f(t0 + 64 * n, t0 + 64 * n < len ? key_of(a, w, t0 + 64 * n, newest) : 0u);
    }
  };

  // the keep-th largest key: digit by digit from the top
  uint32_t prefix = 0, left = keep;                  // of the keys that share the prefix the left-th largest is wanted
  int shift = 32;
#pragma unroll
  for (int turn = 0; turn < 3; ++turn) {
    const int bits = turn < 2 ? 11 : 10;
    shift -= bits;
    for (int b = tid; b < BINS; b += THREADS) hist[b] = 0;
    __syncthreads();
    each([&](int t, uint32_t k) {
      if (t < len && (turn == 0 || (k >> (shift + bits)) == prefix)) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    // sums from the top: each thread two bins, bin 2047 - 2 tid and the one below
    const int b0 = (1 << bits) - 1 - 2 * tid;
    const uint32_t h0 = b0 > 0 ? hist[b0] : 0, h1 = b0 > 0 ? hist[b0 - 1] : 0;
    uint32_t run = h0 + h1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = __shfl_up(run, o, 64);
      if (lane >= o) run += x;
    }
    if (lane == 63) wsum[wave][0] = (int)run;
    __syncthreads();
    uint32_t before = run - h0 - h1;
    for (int k = 0; k < wave; ++k) before += (uint32_t)wsum[k][0];
    if (before < left && left <= before + h0 + h1) {
      const bool second = left > before + h0;
      found[0] = (uint32_t)(b0 - second);
      found[1] = second ? before + h0 : before;
    }
    __syncthreads();
    prefix = (prefix << bits) | found[0];
    left -= found[1];
    __syncthreads();
  }
  // keys above `prefix` stay, and the `left` lowest tokens of those equal to it
  int ties = 0;
  each([&](int t, uint32_t k) { ties += __popcll(__ballot(t < len && k == prefix)); });
  if (lane == 0) wsum[wave][0] = ties;
  __syncthreads();
  int tie = 0;
  for (int k = 0; k < wave; ++k) tie += wsum[k][0];
  __syncthreads();
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  const int tie0 = tie;
  auto stays = [&](int t, uint32_t k) {
    const uint64_t eq = __ballot(t < len && k == prefix);
    const bool s = t < len && (k > prefix || (k == prefix && tie + __popcll(eq & below) < (int)left));
    tie += __popcll(eq);
    return s;
  };
  int nh = 0, nm = 0;
  each([&](int t, uint32_t k) {
    const bool s = stays(t, k);
    nh += __popcll(__ballot(!s && t < keep));
    nm += __popcll(__ballot(s && t >= keep));
  });
  if (lane == 0) { wsum[wave][0] = nh; wsum[wave][1] = nm; }
  __syncthreads();
  int ih = 0, im = 0, total = 0;
  for (int k = 0; k < NWAVES; ++k) {
    if (k < wave) { ih += wsum[k][0]; im += wsum[k][1]; }
    total += wsum[k][0];
  }
  tie = tie0;
  each([&](int t, uint32_t k) {
    const bool s = stays(t, k);
    const uint64_t h = __ballot(!s && t < keep), m = __ballot(s && t >= keep);
    if (!s && t < keep) holes[ih + __popcll(h & below)] = t;
    if (s && t >= keep) moved[im + __popcll(m & below)] = t;
    ih += __popcll(h);
    im += __popcll(m);
  });
  if (!move) {
    if (tid == 0) counts[id] = total;
    return;
  }
  __syncthreads();                                   // (a block's own global writes are seen by its threads behind a barrier)
  constexpr int LANES = HD == 128 ? 8 : 4;
  for (int n = tid / LANES; n < total; n += THREADS / LANES) {
    bool ok0, ok1;
    const uint32_t to = token_of(a.c, w, holes[n], ok0), from = token_of(a.c, w, moved[n], ok1);
    if (ok0 && ok1) move_token<HD, LANES>(a.c, to, from, tid % LANES);
  }
}

template <int HD>
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4Evict a, int most, const int32_t *__restrict__ lists, const int32_t *__restrict__ counts) {
  constexpr int LANES = HD == 128 ? 8 : 4;
  const size_t id = (size_t)blockIdx.z * a.c.Hkv + blockIdx.y;
  const int n = counts[id];
  const int32_t *holes = lists + id * 2 * most, *moved = holes + most;
  const Where w = {a.tables + (size_t)blockIdx.z * a.max_blocks, (int)blockIdx.y};
  for (int m = blockIdx.x * (256 / LANES) + threadIdx.x / LANES; m < n; m += gridDim.x * (256 / LANES)) {
    bool ok0, ok1;
    const uint32_t to = token_of(a.c, w, holes[m], ok0), from = token_of(a.c, w, moved[m], ok1);
    if (ok0 && ok1) move_token<HD, LANES>(a.c, to, from, threadIdx.x % LANES);
  }
}

constexpr int MOVE_INSIDE = 4096;                   // tokens up to which a block moves its own

int list_length(int max_context) { return max_context / 2 + 1; }

}  // namespace

// No more tokens can be displaced than there are holes in front of them: half of all.
size_t kv4_evict_scratch_bytes(int n_req, int max_context, int Hkv) {
  const size_t ids = (size_t)n_req * Hkv;
  return align_up(ids * sizeof(int32_t), 256) + ids * 2 * list_length(max_context) * sizeof(int32_t);
}

hipError_t launch_kv4_evict(const Kv4Evict &a, void *scratch, hipStream_t st) {
  if (a.n_req <= 0) return hipSuccess;
  int32_t *counts = (int32_t *)scratch, *lists = (int32_t *)((char *)scratch + align_up((size_t)a.n_req * a.c.Hkv * sizeof(int32_t), 256));
  const int most = list_length(a.max_context);
  const bool inside = a.max_context <= MOVE_INSIDE;
  auto select = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a.c.Hkv, a.n_req), dim3(THREADS), 0, st, a, most, lists, counts, inside); };
  const int items = cdiv(a.max_context, THREADS);
  if (a.c.hd == 128) items <= 2 ? select(kv4_evict_kernel<128, 2>) : items <= 8 ? select(kv4_evict_kernel<128, 8>) : items <= MAX_ITEMS ? select(kv4_evict_kernel<128, MAX_ITEMS>) : select(kv4_evict_kernel<128, 0>);
  else items <= 2 ? select(kv4_evict_kernel<64, 2>) : items <= 8 ? select(kv4_evict_kernel<64, 8>) : items <= MAX_ITEMS ? select(kv4_evict_kernel<64, MAX_ITEMS>) : select(kv4_evict_kernel<64, 0>);
  if (!inside) {
    auto move = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(std::max(1, std::min(cdiv(most, 256), cdiv(4096, a.n_req * a.c.Hkv))), a.c.Hkv, a.n_req), dim3(256), 0, st, a, most, lists, counts); };
    a.c.hd == 128 ? move(kv4_move_kernel<128>) : move(kv4_move_kernel<64>);
  }
  return hipGetLastError();
}
