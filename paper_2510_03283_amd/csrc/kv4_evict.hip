// Eviction: every (request, kv head) keeps the `budget` tokens of largest key - the first n_sink positions, then the newest n_recent, then by accumulated weight, the
// lower token on ties - and its new length is min(tokens, budget).  What stays behind the new length moves into the holes in front of it, the i-th into
// the i-th, so no token is read where another is written, and only what has to move does.
//
// A block of 1024 threads a (request, kv head) holds the keys in LDS (a wave's tokens side by side), finds the budget-th largest in three turns of 11, 11 and 10 bits with a
// histogram, and then every wave lists its holes and displaced tokens.  With few requests the instructions of these passes set the time (a block a CU, one head of
// 32768 tokens), so a pass does as little as it can: no token is compared with the length (key 0 is none), ties are counted only where some of them go, and the waves'
// lists stay apart: whoever moves finds the i-th hole by the waves' counts.  The moves follow in the same launch or, for long lists, in one of their own
// that the whole chip takes part in.  (8 requests x 8 heads of 20000 to 32768 tokens of 128, 12000 kept: 25 us and 47 of moves; the whole call 81, and 103 with the
// keys read again in every pass, as beyond MAX_HELD tokens.  32 x 8 heads of 1025 to 1088: 12.6 us, a chain of passes with a barrier each.)
#include "kernels.h"

#include <algorithm>

namespace {

constexpr int THREADS = 1024, NWAVES = THREADS / 64, BINS = 2048;
constexpr int BATCH = 4;                           // keys that a thread reads at once
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
constexpr int MAX_HELD = 32 * THREADS;              // keys that LDS has room for beside the histograms; longer caches read them again in every pass

struct Where {
  const int32_t *table;
  int kvh;
};
__device__ __forceinline__ uint32_t token_in(const Kv4Cache &c, const Where &w, int t, int blk, bool &ok) {
  ok = blk >= 0 && (uint32_t)blk < c.num_blocks;
  return ok ? (((uint32_t)blk * c.Hkv + w.kvh) << c.bshift) + (t & ((1 << c.bshift) - 1)) : 0u;
}
__device__ __forceinline__ uint32_t token_of(const Kv4Cache &c, const Where &w, int t, bool &ok) { return token_in(c, w, t, w.table[t >> c.bshift], ok); }

__device__ __forceinline__ int wave_total(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return __builtin_amdgcn_readfirstlane(v);
}

// Larger is kept.  Weights (negative ones and NaN count as 0) below the newest, by position, below the first, by position.  A token in a block that
// does not exist is the first to go.  0 is no token.  (Weights end at 0x7f800002, the newest at 0xbfffffff, and a sink in front of those is at least 0xc0000000.)
__device__ __forceinline__ uint32_t key_from(float weight, int pos, bool ok, int n_sink, int newest) {
  const uint32_t p = (uint32_t)min(max(pos, 0), 0x3fffffff);
  uint32_t key = (weight > 0.f ? __float_as_uint(weight) : 0u) + 2u;
  key = pos >= newest ? 0x80000000u + p : key;
  key = pos < n_sink ? 0xfffffffeu - p : key;
  return ok ? key : 1u;
}
// Keys of N tokens t, t + 64, ..: all their blocks are asked for first, then all their weights and positions (one after the other each would wait for two loads).
template <int N>
__device__ __forceinline__ void load_keys(const Kv4Evict &a, const Where &w, int t, int len, int newest, uint32_t *key) {
  int blk[N];
#pragma unroll
  for (int n = 0; n < N; ++n) blk[n] = w.table[min(t + 64 * n, len - 1) >> a.c.bshift];
  uint32_t tok[N];
  bool ok[N];
  float x[N];
  int pos[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    tok[n] = token_in(a.c, w, min(t + 64 * n, len - 1), blk[n], ok[n]);
    x[n] = a.c.weight[tok[n]];
    pos[n] = a.c.position[tok[n]];
  }
#pragma unroll
  for (int n = 0; n < N; ++n) key[n] = t + 64 * n < len ? key_from(x[n], pos[n], ok[n], a.n_sink, newest) : 0u;
}

// What the waves of a block have listed: wave w's holes and displaced tokens begin at w * stride of either list; before[w]: how many there are in the waves in front of it.
struct Lists {
  const int32_t *holes, *moved;
  int stride;
  const int (*before)[2];            // [NWAVES + 1], in LDS
};
__device__ __forceinline__ int entry_of(const Lists &l, int m, int which) {
  int w = 0;
#pragma unroll
  for (int k = 1; k < NWAVES; ++k) w += m >= l.before[k][which];
  return (which ? l.moved : l.holes)[w * l.stride + m - l.before[w][which]];
}
// Moves the m-th displaced token to the m-th hole (not where the hole lies in a block that does not exist) for m = first, first + step, .. below n, each by LANES lanes: a 16-byte piece of K or V a lane, and one of the small arrays in
// each of the first four.  AT_ONCE of them are under way, loads before stores (one after the other, with a branch for each array, the moves of 8 x 8 heads x 6300 tokens of 128
// took 60 us, now 47: 122 MB in pieces of 64 bytes).
template <int HD>
constexpr int LANES = HD / 16;
template <int HD, int AT_ONCE>
__device__ __forceinline__ void move_tokens(const Kv4Cache &c, const Where &w, const Lists &l, int n, int first, int step, int lane) {
  constexpr int PIECES = HD / 32;                    // of K, and of V
  // (pointers that a lane chooses are told to be global memory, or every access is checked for other address spaces)
  typedef __attribute__((address_space(1))) unsigned char *bytes;
  typedef __attribute__((address_space(1))) u32x4_t *quads;
  typedef __attribute__((address_space(1))) uint32_t *words;
  typedef __attribute__((address_space(1))) uint16_t *halves;
  const bytes rows = (bytes)(lane < PIECES ? c.k : c.v);
  const uint32_t piece = lane % PIECES;
  const bytes small = (bytes)(lane == 0 ? (unsigned char *)c.weight : lane == 1 ? (unsigned char *)c.position : lane == 2 ? c.k_scale : c.v_scale);
  for (int m = first; m < n; m += AT_ONCE * step) {
    uint32_t to[AT_ONCE], from[AT_ONCE];
    bool ok[AT_ONCE];
    int h[AT_ONCE], s[AT_ONCE], bh[AT_ONCE], bs[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int at = min(m + u * step, n - 1);
      h[u] = entry_of(l, at, 0);
      s[u] = entry_of(l, at, 1);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      bh[u] = w.table[h[u] >> c.bshift];
      bs[u] = w.table[s[u] >> c.bshift];
    }
    u32x4_t x[AT_ONCE];
    uint32_t y[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      bool there, here;
      to[u] = token_in(c, w, h[u], bh[u], there);
      from[u] = token_in(c, w, s[u], bs[u], here);
      ok[u] = there && here && m + u * step < n;
      x[u] = ((quads)rows)[(size_t)from[u] * PIECES + piece];
      if constexpr (HD == 128) y[u] = ((words)small)[from[u]];
      else y[u] = lane < 2 ? ((words)small)[from[u]] : ((halves)small)[from[u]];
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (!ok[u]) continue;
      ((quads)rows)[(size_t)to[u] * PIECES + piece] = x[u];
      if constexpr (HD == 128) {
        if (lane < 4) ((words)small)[to[u]] = y[u];
      } else {
        if (lane < 2) ((words)small)[to[u]] = y[u];
        else ((halves)small)[to[u]] = (uint16_t)y[u];
      }
    }
  }
}

// Bounds of a request's tokens up to which a block moves its own in any case, and moves up to which it does so in longer ones.  (64-wide heads, 8 of each request: 16 requests cut from 8192
// to 8000 tokens 33 us with a launch for the moves, 21 without, to 4000 41 and 44; 8 of 128-wide heads from 32768 to 32500 46 us with all moves in that launch, 42 with none left for it.)
constexpr int MOVE_INSIDE = 8192, MOVE_FEW = 512;
// lists: [n_req, Hkv, 2, most] token numbers: holes, displaced; counts [n_req, Hkv, NWAVES + 1]: of both lists of every wave (as many in all), and the lists' stride.
template <int HD, bool HELD>
__global__ __launch_bounds__(THREADS) void kv4_evict_kernel(Kv4Evict a, int most, int32_t *__restrict__ lists, int2 *__restrict__ counts, bool move) {
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t hist[3][BINS];
  __shared__ int wsum[NWAVES], before[NWAVES + 1][2];
  __shared__ uint32_t found[3];                      // digit, tokens above it, tokens that have it
  const int kvh = blockIdx.x, req = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Where w = {a.tables + (size_t)req * a.max_blocks, kvh};
  const int room = (int)min((long long)a.max_blocks << a.c.bshift, (long long)INT32_MAX);
  const int len = min(min(max(a.lens[(size_t)req * a.len_heads + (a.len_heads > 1 ? kvh : 0)], 0), a.max_context), room);
  const int keep = min(len, max(a.budgets[(size_t)req * a.c.Hkv + kvh], 0));
  const int newest = a.n_recent > 0 ? max(a.seq_lens[req] - a.n_recent, 0) : INT32_MAX;
  const size_t id = (size_t)req * a.c.Hkv + kvh;
  int32_t *holes = lists + id * 2 * most, *moved = holes + most;
  for (int b = tid; b < 3 * BINS; b += THREADS) (&hist[0][0])[b] = 0;
  __syncthreads();                                   // (and new_lens may be lens)
  if (tid == 0) a.new_lens[id] = keep;
  if (keep == len || keep == 0) {
    if (tid < NWAVES) counts[id * (NWAVES + 1) + tid] = make_int2(0, 0);
    return;
  }

  // per: tokens of a thread, in whole batches
  const int per = (len + THREADS * BATCH - 1) / (THREADS * BATCH) * BATCH, base = wave * 64 * per, t0 = base + lane;         // this thread's tokens: t0 + 64 n
  // f(first token of the wave's 64, this lane's key); a batch of keys is read before the first of them is used
  auto each = [&](auto f) {
    for (int n = 0; n < per && base + 64 * n < len; n += BATCH) {
      uint32_t k[BATCH];
      if constexpr (HELD) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) k[u] = keys[t0 + 64 * (n + u)];
      } else {
        load_keys<BATCH>(a, w, t0 + 64 * n, len, newest, k);
      }
#pragma unroll
      for (int u = 0; u < BATCH; ++u) f(base + 64 * (n + u), k[u]);
    }
  };

  // the keep-th largest key: digit by digit from the top
  uint32_t prefix = 0, left = keep;                  // of the keys that share the prefix the left-th largest is wanted
  int shift = 32;
#pragma unroll
  for (int turn = 0; turn < 3; ++turn) {
    const int bits = turn < 2 ? 11 : 10;
    shift -= bits;
    auto count = [&](uint32_t k) {
      if (turn == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&hist[turn][(k >> shift) & ((1u << bits) - 1)], 1u);
    };
    if (HELD && turn == 0) {
      for (int n = 0; n < per && base + 64 * n < len; n += 2 * BATCH) {
        uint32_t k[2 * BATCH];
        load_keys<2 * BATCH>(a, w, t0 + 64 * n, len, newest, k);
#pragma unroll
        for (int u = 0; u < 2 * BATCH; ++u)
          if (n + u < per) {
            keys[t0 + 64 * (n + u)] = k[u];
            count(k[u]);
          }
      }
    } else {
      each([&](int, uint32_t k) { count(k); });
    }
    __syncthreads();
    // sums from the top: each thread two bins, bin 2047 - 2 tid and the one below
    const int b0 = (1 << bits) - 1 - 2 * tid;
    const uint32_t h0 = b0 > 0 ? hist[turn][b0] : 0, h1 = b0 > 0 ? hist[turn][b0 - 1] : 0;
    uint32_t run = h0 + h1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = __shfl_up(run, o, 64);
      if (lane >= o) run += x;
    }
    if (lane == 63) wsum[wave] = (int)run;
    __syncthreads();
    uint32_t above = run - h0 - h1;
    for (int k = 0; k < wave; ++k) above += (uint32_t)wsum[k];
    if (above < left && left <= above + h0 + h1) {
      const bool second = left > above + h0;
      found[0] = (uint32_t)(b0 - second);
      found[1] = second ? above + h0 : above;
      found[2] = second ? h1 : h0;
    }
    __syncthreads();
    prefix = (prefix << bits) | found[0];
    left -= found[1];
  }
  // Keys above `prefix` stay, and the `left` lowest tokens of those equal to it: all of them in waves whose ties end below `left`, none in waves behind, and in one wave at most
  // the first ones, which it numbers.
  bool every = left == found[2], split = false;
  int tie = 0;
  if (!every) {
    int ties = 0;
    each([&](int, uint32_t k) { ties += k == prefix; });
    ties = wave_total(ties);
    if (lane == 0) before[wave][0] = ties;
    __syncthreads();
    for (int k = 0; k < wave; ++k) tie += before[k][0];
    tie = __builtin_amdgcn_readfirstlane(tie);
    __syncthreads();
    every = tie + ties <= (int)left;
    split = !every && tie < (int)left;
  }
  const uint32_t least = every ? prefix : prefix + 1;      // (keys are below 2^32 - 1)
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  int nh = 0, nm = 0;                                // of this wave
  each([&](int b0, uint32_t k) {
    uint64_t s = __ballot(k >= least);
    if (split) {
      const uint64_t eq = __ballot(k == prefix);
      s |= __ballot((eq >> lane & 1) && tie + __popcll(eq & below) < (int)left);
      tie += __popcll(eq);
    }
    if (b0 < keep) {                                 // some of these 64 can be holes
      const uint64_t h = b0 + 64 <= keep ? ~s : ~s & ((1ull << (keep - b0)) - 1);
      if (h >> lane & 1) holes[base + nh + __popcll(h & below)] = b0 + lane;
      nh += __popcll(h);
    }
    if (b0 + 64 > keep) {                            // some can be displaced
      const uint64_t m = b0 >= keep ? s : s & ~((1ull << (keep - b0)) - 1);
      if (m >> lane & 1) moved[base + nm + __popcll(m & below)] = b0 + lane;
      nm += __popcll(m);
    }
  });
  int2 *mine = counts + id * (NWAVES + 1);
  if (lane == 0) { before[wave + 1][0] = nh; before[wave + 1][1] = nm; }
  if (tid < 2) before[0][tid] = 0;
  __syncthreads();                                   // (a block's own global writes are seen by its threads behind a barrier)
  if (tid < 2)
    for (int k = 1; k <= NWAVES; ++k) before[k][tid] += before[k - 1][tid];
  __syncthreads();
  const bool mine_to_move = move || before[NWAVES][0] <= MOVE_FEW;
  if (!move) {                                       // what the next launch has to do
    if (lane == 0) mine[wave] = mine_to_move ? make_int2(0, 0) : make_int2(nh, nm);
    if (tid == 0) mine[NWAVES] = make_int2(64 * per, 0);
  }
  if (!mine_to_move) return;
  move_tokens<HD, 2>(a.c, w, Lists{holes, moved, 64 * per, before}, before[NWAVES][0], tid / LANES<HD>, THREADS / LANES<HD>, tid % LANES<HD>);
}

constexpr int MOVES_AT_ONCE = 4;
template <int HD>
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4Evict a, int most, const int32_t *__restrict__ lists, const int2 *__restrict__ counts) {
  __shared__ int before[NWAVES + 1][2];
  const size_t id = (size_t)blockIdx.z * a.c.Hkv + blockIdx.y;
  const int2 *mine = counts + id * (NWAVES + 1);
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {                            // sums in front of every wave
    int2 v = lane < NWAVES ? mine[lane] : make_int2(0, 0), sum = v;
#pragma unroll
    for (int o = 1; o <= NWAVES; o <<= 1) {
      const int x = __shfl_up(sum.x, o, 64), y = __shfl_up(sum.y, o, 64);
      if (lane >= o) { sum.x += x; sum.y += y; }
    }
    if (lane <= NWAVES) { before[lane][0] = sum.x - v.x; before[lane][1] = sum.y - v.y; }
  }
  __syncthreads();
  const int n = before[NWAVES][0];
  if (n == 0) return;                                // (the stride was not written either)
  const int32_t *holes = lists + id * 2 * most;
  const Where w = {a.tables + (size_t)blockIdx.z * a.max_blocks, (int)blockIdx.y};
  move_tokens<HD, MOVES_AT_ONCE>(a.c, w, Lists{holes, holes + most, mine[NWAVES].x, before}, n, blockIdx.x * (256 / LANES<HD>) + threadIdx.x / LANES<HD>, gridDim.x * (256 / LANES<HD>),
                                 threadIdx.x % LANES<HD>);
}

// Entries of a list: none lies behind the token that it names.
int list_length(int max_context) { return std::max(64, (max_context + 63) / 64 * 64); }
size_t counts_bytes(int n_req, int Hkv) { return align_up((size_t)n_req * Hkv * (NWAVES + 1) * sizeof(int2), 256); }

}  // namespace

size_t kv4_evict_scratch_bytes(int n_req, int max_context, int Hkv) {
  return counts_bytes(n_req, Hkv) + (size_t)n_req * Hkv * 2 * list_length(max_context) * sizeof(int32_t);
}

hipError_t launch_kv4_evict(const Kv4Evict &a, void *scratch, hipStream_t st) {
  if (a.n_req <= 0) return hipSuccess;
  int2 *counts = (int2 *)scratch;
  int32_t *lists = (int32_t *)((char *)scratch + counts_bytes(a.n_req, a.c.Hkv));
  const int most = list_length(a.max_context);
  const bool inside = a.max_context <= MOVE_INSIDE;
  const bool held = a.max_context <= MAX_HELD;
  const size_t lds = held ? (size_t)cdiv(a.max_context, THREADS * BATCH) * BATCH * THREADS * sizeof(uint32_t) : 0;
  hipError_t e = hipSuccess;
  auto select = [&](auto kernel, DeviceOnce &once) {
    if (held && !once.test()) {
      e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(MAX_HELD * sizeof(uint32_t)));
      if (e != hipSuccess) return;
      once.set();
    }
    hipLaunchKernelGGL(kernel, dim3(a.c.Hkv, a.n_req), dim3(THREADS), lds, st, a, most, lists, counts, inside);
  };
  static DeviceOnce once[4];
  if (a.c.hd == 128) held ? select(kv4_evict_kernel<128, true>, once[0]) : select(kv4_evict_kernel<128, false>, once[1]);
  else held ? select(kv4_evict_kernel<64, true>, once[2]) : select(kv4_evict_kernel<64, false>, once[3]);
  if (e != hipSuccess) return e;
  if (!inside) {
    auto move = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(std::max(1, std::min(cdiv(most, 256), cdiv(4096, a.n_req * a.c.Hkv))), a.c.Hkv, a.n_req), dim3(256), 0, st, a, most, lists, counts); };
    a.c.hd == 128 ? move(kv4_move_kernel<128>) : move(kv4_move_kernel<64>);
  }
  return hipGetLastError();
}
