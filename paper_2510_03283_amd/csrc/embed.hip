// Embedding rows of token ids, scaled, and the gradient of the table they come from.
//   forward   out[r, :] = io(scale * E[id_r, :])
//   backward  dE[v, :] (+)= scale * sum over the rows r with id_r = v, in order of r, of dx[r, :]
// A token id outside [0, vocab) is padding: its row of out is zero and its row of dx is not read.
#include "kernels.h"

#include <algorithm>

namespace {

constexpr size_t LLC_BYTES = (size_t)256 << 20;      // last-level cache

// ------------------------------------------------------------------ rows
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
// 2^lg threads per row, 16-byte accesses, four of them in flight a thread.  No branch around a load (a place behind the row reads its last one
// again, padding reads row 0): 66576 x 4096 bf16 151 -> 142 us, but with the rows written past the cache (as this many are) 126 -> 127 us,
// 5.2 TB/s of ids, distinct rows and output: HBM-bound.  Fewer blocks that go on to further rows were slower (2048: 155, past the cache 134).
template <bool BF16, bool STREAM>
__global__ __launch_bounds__(256) void embed_rows_kernel(const void *__restrict__ table, const int32_t *__restrict__ ids, int n, int vocab, int d,
                                                         float scale, void *__restrict__ out, int lg) {
  const int vecs = d / (BF16 ? 8 : 4), per = 1 << lg, lane = threadIdx.x & (per - 1), rows = 256 >> lg;
  for (size_t r = (size_t)blockIdx.x * rows + (threadIdx.x >> lg); r < (size_t)n; r += (size_t)gridDim.x * rows) {
    const int id = ids[r];
    const bool there = id >= 0 && id < vocab;
    const u32x4_t *src = (const u32x4_t *)table + (size_t)(there ? id : 0) * vecs;
    u32x4_t *dst = (u32x4_t *)out + r * vecs;
    for (int k0 = lane; k0 < vecs; k0 += 4 * per) {
      u32x4_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = src[min(k0 + i * per, vecs - 1)];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (k0 + i * per >= vecs) break;
        u32x4_t y = {0, 0, 0, 0};
        if (there) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (BF16) y[j] = cvt_pk_bf16(scale * __uint_as_float(x[i][j] << 16), scale * __uint_as_float(x[i][j] & 0xffff0000u));
            else y[j] = __float_as_uint(scale * __uint_as_float(x[i][j]));
          }
        }
        if constexpr (STREAM) __builtin_nontemporal_store(y, dst + k0 + i * per);
        else dst[k0 + i * per] = y;
      }
    }
  }
}

// ------------------------------------------------------------------ gradient of the table
// Three or four launches (one for few rows), no block of which waits for another, and no order of which depends on which block comes first.
//  bucket (many rows only) The ids are cut into chunks of 1024 rows; a block sorts its chunk by bucket, 2^lg adjacent tokens (stable: rows of a bucket
//         keep their order), and notes how many rows each bucket has in it.
//  place  A block per bucket collects the bucket's rows from all chunks in order and sorts them by token, again stably.  The rows of
//         lower buckets, counted over the chunks, say where the bucket begins.
//  sum    The sorted order is cut into windows of equal length, a wave per window and column strip, so that the work does not
//         depend on how often a token occurs.  A token whose rows all lie in the window is finished there; the sums of one that
//         began before the window or goes on behind it are set aside.  Further waves write the zeros of tokens that do not occur.
//  join   Per window: the token that goes on behind it, if it begins there, from the sums that were set aside, in window order.
// us of the launches, 65536 rows added to 32000 x 4096: bucket 4.9, place 11.6, sum 302 - 315 (1.57 GB behind the L2s, 5.0 - 5.2 TB/s of reads and
// writes mixed, what a large copy reaches: HBM-bound), join 14.7; 3347 rows added to 32000 x 2048: place 6.7, sum 10 - 13, join 4.2, each
// a chain of three or four dependent loads.
constexpr int WAVES = 16, CHUNK = 64 * WAVES, BUCKETS = 256, MAX_KEYS = 512;
struct Placed {
  int row, token;
};

// Lanes of this wave that hold the same key as this one (bits [0, bits) of it), of those that are `in`.
__device__ __forceinline__ unsigned long long lanes_like(int key, int bits, bool in) {
  unsigned long long same = __ballot(in);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long set = __ballot((key >> b) & 1);
    same &= (key >> b) & 1 ? set : ~set;
  }
  return same;
}
__device__ __forceinline__ int lower_lanes(unsigned long long m) { return __popcll(m & ((1ull << (threadIdx.x & 63)) - 1)); }
// Sum over the threads before this one (exclusive) of a block of 64 WAVES threads; red: WAVES ints that nothing else uses between two barriers.
__device__ __forceinline__ int sum_before(int x, int *red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(sum, o, 64);
    if (lane >= o) sum += y;
  }
  if (lane == 63) red[wave] = sum;
  __syncthreads();
  int at = sum - x;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) at += w < wave ? red[w] : 0;
  return at;
}

// begins[c][b]: rows of chunk c in buckets before b, b = 0 .. BUCKETS; the chunk's rows in order[CHUNK c ..].
__global__ __launch_bounds__(CHUNK) void embed_bucket_kernel(const int32_t *__restrict__ ids, int n, int vocab, int lg, int *__restrict__ begins,
                                                             Placed *__restrict__ order) {
  __shared__ int count[WAVES][BUCKETS];
  __shared__ int red[WAVES];
  const int wave = threadIdx.x >> 6;
  for (long long c = blockIdx.x; c * CHUNK < n; c += gridDim.x) {
    const long long i = c * CHUNK + threadIdx.x;
    const int id = i < n ? ids[i] : -1, bucket = id >> lg;
    for (int k = threadIdx.x; k < WAVES * BUCKETS; k += CHUNK) (&count[0][0])[k] = 0;
    __syncthreads();
    const bool in = id >= 0 && id < vocab;
    const unsigned long long same = lanes_like(bucket, 8, in);
    const int before = lower_lanes(same);
    if (in && before == 0) count[wave][bucket] = __popcll(same);
    __syncthreads();
    int mine = 0;
    if (threadIdx.x < BUCKETS)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) mine += count[w][threadIdx.x];
    int at = sum_before(mine, red);
    if (threadIdx.x < BUCKETS) {
      begins[c * (BUCKETS + 1) + threadIdx.x] = at;
      if (threadIdx.x == BUCKETS - 1) begins[c * (BUCKETS + 1) + BUCKETS] = at + mine;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const int x = count[w][threadIdx.x];
        count[w][threadIdx.x] = at;
        at += x;
      }
    }
    __syncthreads();
    if (in) order[c * CHUNK + count[wave][bucket] + before] = Placed{(int)i, id};
    __syncthreads();
  }
}

// The rows of a block's bucket in order, a contiguous share of them to every wave: f(row and token of this lane, whether it has one).
// From the chunks c0 .. c1 that the bucket kernel sorted.
template <typename F>
__device__ __forceinline__ void bucket_rows(const Placed *from, const int *begins, int bucket, int c0, int c1, F f) {
  const int lane = threadIdx.x & 63;
  for (int b0 = c0; b0 < c1; b0 += 64) {          // the extents of 64 chunks at a time, a lane each
    const int c = b0 + lane;
    const int s = c < c1 ? begins[(size_t)c * (BUCKETS + 1) + bucket] : 0, e = c < c1 ? begins[(size_t)c * (BUCKETS + 1) + bucket + 1] : 0;
    const int len = e - s;
    int sum = len;                               // inclusive
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(sum, o, 64);
      if (lane >= o) sum += y;
    }
    const int total = __shfl(sum, 63, 64);
    for (int k0 = 0; k0 < total; k0 += 64) {      // row k of these chunks: in the first chunk whose inclusive sum is above k
      const int k = k0 + lane;
      int lo = 0;
#pragma unroll
      for (int step = 32; step > 0; step >>= 1)
        if (__shfl(sum, lo + step - 1, 64) <= k) lo += step;
      lo = min(lo, 63);
      const int at = k - (__shfl(sum, lo, 64) - __shfl(len, lo, 64)) + __shfl(s, lo, 64);
      const bool in = k < total;
      Placed p = {0, 0};
      if (in) p = from[(size_t)(b0 + lo) * CHUNK + at];
      f(p, in);
    }
  }
}

// starts[v]: rows of tokens below v, v = 0 .. vocab; order: the rows by token.  From sorted chunks or, IDS > 0, from the n <= IDS * CHUNK ids
// themselves: every block looks through all of them, IDS a thread and read once, which saves the bucket kernel.
template <int IDS>
__global__ __launch_bounds__(64 * WAVES) void embed_place_kernel(const int32_t *__restrict__ ids, int n, const int *__restrict__ begins,
                                                                 const Placed *__restrict__ from, int chunks, int vocab, int lg, int *__restrict__ starts,
                                                                 Placed *__restrict__ order) {
  __shared__ int count[WAVES * MAX_KEYS];        // [wave][key]
  __shared__ int red[WAVES], lower[WAVES], after;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, keys = min(1 << lg, MAX_KEYS), bits = min(lg, 9), bucket = blockIdx.x;
  constexpr bool DIRECT = IDS > 0;
  const int per = DIRECT ? (n + CHUNK - 1) / CHUNK * 64 : (chunks + WAVES - 1) / WAVES;      // ids, chunks of a wave
  const int c0 = min(DIRECT ? n : chunks, per * wave), c1 = min(DIRECT ? n : chunks, c0 + per);
  int id[DIRECT ? IDS : 1];
  if constexpr (DIRECT)
#pragma unroll
    for (int k = 0; k < IDS; ++k) id[k] = c0 + 64 * k + lane < c1 ? ids[c0 + 64 * k + lane] : -1;
  const auto rows = [&](auto f) {
    if constexpr (DIRECT) {
#pragma unroll
      for (int k = 0; k < IDS; ++k) f(Placed{c0 + 64 * k + lane, id[k]}, true);
    } else {
      bucket_rows(from, begins, bucket, c0, c1, f);
    }
  };
  const long long begin = (long long)bucket << lg, end = min((long long)vocab, begin + (1ll << lg));
  int below = 0;                                 // rows of lower buckets
  if constexpr (!DIRECT)
    for (int c = threadIdx.x; c < chunks; c += 64 * WAVES) below += begins[(size_t)c * (BUCKETS + 1) + bucket];
  int here = 0;                                  // where this turn's tokens begin
  for (long long v0 = begin; v0 < end; v0 += MAX_KEYS) {       // (one turn for vocabularies of up to 131072)
    const int first = (int)v0, last = (int)min(end, v0 + keys);
    for (int k = threadIdx.x; k < WAVES * keys; k += 64 * WAVES) count[k] = 0;
    __syncthreads();
    rows([&](Placed p, bool in) {
      if (in && p.token >= first && p.token < last) atomicAdd(&count[wave * keys + p.token - first], 1);
      if (DIRECT && v0 == begin && p.token >= 0 && p.token < first) ++below;
    });
    if (v0 == begin) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, 64);
      if (lane == 0) lower[wave] = below;
    }
    __syncthreads();
    if (v0 == begin)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) here += lower[w];
    int mine = 0;
    if (threadIdx.x < keys)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) mine += count[w * keys + threadIdx.x];
    int at = sum_before(mine, red) + here;
    if (threadIdx.x < keys) {
      if (first + (int)threadIdx.x < last) starts[first + threadIdx.x] = at;
      if (first + (int)threadIdx.x == vocab - 1) starts[vocab] = at + mine;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const int x = count[w * keys + threadIdx.x];
        count[w * keys + threadIdx.x] = at;
        at += x;
      }
      if (threadIdx.x == keys - 1) after = at;
    }
    __syncthreads();
    here = after;
    rows([&](Placed p, bool has) {
      const bool in = has && p.token >= first && p.token < last;
      if (!__ballot(in)) return;
      const int key = p.token - first;
      const unsigned long long same = lanes_like(key, bits, in);
      const int leader = in ? __builtin_ctzll(same) : lane;
      int to = 0;
      if (in && lane == leader) to = atomicAdd(&count[wave * keys + key], __popcll(same));      // only this wave's lanes, one turn after the other
      to = __shfl(to, leader, 64) + lower_lanes(same);
      if (in) order[to] = p;
    });
    __syncthreads();
  }
}

constexpr int STRIP = 256, R = 8;     // columns of a wave, rows that it asks for together
constexpr int ZERO_ROWS = 8;          // rows of the table that a wave looks at for zeros
template <bool PAST>
__device__ __forceinline__ void put_zero(float *to) {
  const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
  if constexpr (PAST) __builtin_nontemporal_store(z, (f32x4_t *)to);
  else *(f32x4_t *)to = z;
}

// The whole gradient of at most FEW_ROWS rows in one launch instead of three (us, 32 rows of 4096 9.8 -> 3.5, 256 rows 11.7 -> 4.7; 256 rows of one
// token, the longest sum, 16.9 -> 29.7).  A unit is (row, strip of 256 columns): the first row of a token sums all of them, by looking
// through the ids; or (ZERO_ROWS tokens, strip) behind the rows' units.
constexpr int FEW_ROWS = 256;
template <bool ACC, bool PAST>
__global__ __launch_bounds__(256) void embed_few_kernel(const int32_t *__restrict__ ids, int n, const float *__restrict__ dx, int vocab, int d, float scale,
                                                        float *__restrict__ d_table, int strips) {
  constexpr int TURNS = FEW_ROWS / 64;
  const int lane = threadIdx.x & 63;
  const long long units = (n + (ACC ? 0 : ((long long)vocab + ZERO_ROWS - 1) / ZERO_ROWS)) * strips;
  int id[TURNS];
#pragma unroll
  for (int t = 0; t < TURNS; ++t) id[t] = 64 * t + lane < n ? ids[64 * t + lane] : -1;
  for (long long unit = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < units; unit += (long long)gridDim.x * 4) {
    const long long row = unit / strips;
    const int col = (int)(unit - row * strips) * STRIP + 4 * lane;
    const bool live = col < d;                   // other lanes of the last strip read its last column again and write nothing
    const int at_col = live ? col : d - 4;
    if (!ACC && row >= n) {
      const int v0 = (int)(row - n) * ZERO_ROWS;
      for (int i = 0; i < ZERO_ROWS && v0 + i < vocab; ++i) {
        bool has = false;
#pragma unroll
        for (int t = 0; t < TURNS; ++t) has = has || id[t] == v0 + i;
        if (!__ballot(has) && live) put_zero<PAST>(d_table + (size_t)(v0 + i) * d + col);
      }
      continue;
    }
    const int mine = (int)row, token = ids[mine];
    if (token < 0 || token >= vocab) continue;
    unsigned long long like[TURNS];
    bool first = true;
    int count = 0;
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      like[t] = __ballot(id[t] == token);
      const unsigned long long before = mine >= 64 * (t + 1) ? ~0ull : mine > 64 * t ? (1ull << (mine - 64 * t)) - 1 : 0ull;
      if (like[t] & before) first = false;
      count += __popcll(like[t]);
    }
    if (!first) continue;
    float *to = d_table + (size_t)token * d;
    f32x4_t old = {0.f, 0.f, 0.f, 0.f}, acc = {0.f, 0.f, 0.f, 0.f};
    if constexpr (ACC) old = *(const f32x4_t *)(to + at_col);
    int t = 0;                                   // rows left of turn t
    unsigned long long left = like[0];
    for (int i = 0; i < count; i += R) {
      f32x4_t x[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (i + k >= count) break;
#pragma unroll
        for (int q = 1; q < TURNS; ++q)
          if (!left && t < q) { t = q; left = like[q]; }
        const int r = 64 * t + __builtin_ctzll(left);
        left &= left - 1;
        x[k] = *(const f32x4_t *)(dx + (size_t)r * d + at_col);
      }
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (i + k < count) acc += x[k];
    }
    if (live) *(f32x4_t *)(to + col) = ACC ? old + scale * acc : scale * acc;
  }
}

// A unit is (window, strip of 256 columns), or (ZERO_ROWS tokens, strip) behind the windows' units.  Eight rows are asked for together, with
// the old values of the tokens that end among them: 8 to 16 KB of a wave in flight.
template <bool ACC, bool STREAM, bool PAST>
__global__ __launch_bounds__(256) void embed_sum_kernel(const int *__restrict__ starts, const Placed *__restrict__ order, const float *__restrict__ dx, int vocab,
                                                        int d, float scale, float *__restrict__ d_table, float *__restrict__ aside, int window,
                                                        long long windows, int strips) {
  const int lane = threadIdx.x & 63;
  const long long units = (windows + (ACC ? 0 : (vocab + ZERO_ROWS - 1) / ZERO_ROWS)) * strips;
  for (long long unit = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); unit < units; unit += (long long)gridDim.x * 4) {
    const long long win = unit / strips;
    const int col = (int)(unit - win * strips) * STRIP + 4 * lane;
    const bool live = col < d;                   // other lanes of the last strip read its last column again and write nothing
    const int at_col = live ? col : d - 4;
    if (!ACC && win >= windows) {
      const int v0 = (int)(win - windows) * ZERO_ROWS;
      const int s = starts[min(v0 + lane, vocab)], e = starts[min(v0 + lane + 1, vocab)];
      const unsigned long long none = __ballot(lane < ZERO_ROWS && v0 + lane < vocab && s == e);
      for (int i = 0; i < ZERO_ROWS; ++i)
        if (((none >> i) & 1) && live) put_zero<PAST>(d_table + (size_t)(v0 + i) * d + col);
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
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < cnt; i += R) {
      f32x4_t x[R], old[R];
      int token[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const int at = min(i + k, cnt - 1), row = __builtin_amdgcn_readlane(mine.row, at);
        token[k] = __builtin_amdgcn_readlane(mine.token, at);
        const f32x4_t *p = (const f32x4_t *)(dx + (size_t)row * d + at_col);
        if constexpr (STREAM) x[k] = __builtin_nontemporal_load(p);
        else x[k] = *p;
        if constexpr (ACC)
          if ((ends >> at) & 1) old[k] = *(const f32x4_t *)(d_table + (size_t)token[k] * d + at_col);
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (i + k >= cnt) break;
        acc += x[k];
        if (!((ends >> (i + k)) & 1)) continue;
        const bool before = from_before && token[k] == first, behind = goes_on && token[k] == last;
        if (live) {
          if (before || behind) *(f32x4_t *)(aside + (size_t)(2 * win + (before ? 0 : 1)) * d + col) = acc;
          else *(f32x4_t *)(d_table + (size_t)token[k] * d + col) = ACC ? old[k] + scale * acc : scale * acc;
        }
        acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
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
    f32x4_t acc = *(const f32x4_t *)(aside + (size_t)(2 * win + 1) * d + col), old = {0.f, 0.f, 0.f, 0.f};
    if constexpr (ACC) old = *(const f32x4_t *)(d_table + (size_t)token * d + col);
    for (long long w = win + 1; w <= last; w += 16) {
      f32x4_t x[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) x[k] = *(const f32x4_t *)(aside + (size_t)(2 * min(w + k, last)) * d + col);
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (w + k <= last) acc += x[k];
    }
    *(f32x4_t *)(d_table + (size_t)token * d + col) = ACC ? old + scale * acc : scale * acc;
  }
}

// Units wanted, four waves a CU: shorter windows put more sums aside.  us with 256 / 1024 / 4096: 1000 x 2048 17.8 / 14.3 / 14.2, 3347 x 2048 28.3 / 22.6 / 25.9,
// 8192 x 1024 31.2 / 27.6 / 30.4, 12288 x 4096 77.0 / 77.2 / 81.1, 65536 x 256 43.5 / 43.5 / 52.2.
constexpr int UNITS = 1024;
struct GradPlan {
  int strips, window, lg, chunks;
  long long windows;
  size_t begins_at, from_at, order_at, aside_at, bytes;
};
GradPlan plan_grad(int n, int vocab, int d) {
  GradPlan p;
  p.strips = (d + STRIP - 1) / STRIP;
  p.window = 64;
  while (p.window > 4 && ((long long)n + p.window - 1) / p.window * p.strips < UNITS) p.window >>= 1;
  p.windows = ((long long)n + p.window - 1) / p.window;
  p.lg = 0;
  while (((long long)vocab - 1) >> p.lg >= BUCKETS) ++p.lg;
  p.chunks = (int)(((long long)n + CHUNK - 1) / CHUNK);
  p.begins_at = align_up(((size_t)vocab + 1) * sizeof(int), 256);
  p.from_at = align_up(p.begins_at + (size_t)p.chunks * (BUCKETS + 1) * sizeof(int), 256);
  p.order_at = align_up(p.from_at + (size_t)p.chunks * CHUNK * sizeof(Placed), 256);
  p.aside_at = align_up(p.order_at + (size_t)n * sizeof(Placed), 256);
  // the windows of fewer rows may be shorter, and so more: never more than n / 4, nor, while they are shorter than 64, than 2 UNITS units
  const long long most = std::max<long long>(((long long)n + 63) / 64, std::min<long long>(((long long)n + 3) / 4, 2 * UNITS / p.strips + 1));
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
  // Rows that fill half the last-level cache or more are written past it, so that the table stays in it: 66576 x 4096 bf16 142 -> 127 us, 17000 x 4096 40.5 -> 35.0.
  const bool stream = (size_t)n * vecs * 16 >= LLC_BYTES / 2;
  auto *k = bf16 ? (stream ? embed_rows_kernel<true, true> : embed_rows_kernel<true, false>) : (stream ? embed_rows_kernel<false, true> : embed_rows_kernel<false, false>);
  hipLaunchKernelGGL(k, grid, dim3(256), 0, st, table, ids, n, vocab, d, scale, out, lg);
  return hipGetLastError();
}

size_t embed_grad_scratch_bytes(int n, int vocab, int d) { return plan_grad(n, vocab, d).bytes; }

hipError_t launch_embed_grad(const int32_t *ids, int n, int vocab, int d, const float *dx, float scale, float *d_table, bool accumulate, void *scratch,
                             hipStream_t st) {
  if (n <= 0 && accumulate) return hipSuccess;
  const GradPlan p = plan_grad(n, vocab, d);
  const long long zero_units = accumulate ? 0 : ((long long)vocab + ZERO_ROWS - 1) / ZERO_ROWS * p.strips;
  const auto blocks = [](long long units) { return dim3((unsigned)std::min<long long>((units + 3) / 4, 1 << 22)); };
  // The zeros of a table that the last-level cache cannot hold are written past it: 12288 rows into 32000 x 4096 155 -> 137 us.
  const bool past = (size_t)vocab * d * sizeof(float) > LLC_BYTES;
  if (n <= FEW_ROWS) {
    auto *few = accumulate ? embed_few_kernel<true, false> : past ? embed_few_kernel<false, true> : embed_few_kernel<false, false>;
    hipLaunchKernelGGL(few, blocks((long long)n * p.strips + zero_units), dim3(256), 0, st, ids, n, dx, vocab, d, scale, d_table, p.strips);
    return hipGetLastError();
  }
  int *starts = (int *)scratch;
  int *begins = (int *)((char *)scratch + p.begins_at);
  Placed *from = (Placed *)((char *)scratch + p.from_at), *order = (Placed *)((char *)scratch + p.order_at);
  float *aside = (float *)((char *)scratch + p.aside_at);
  const int buckets = ((vocab - 1) >> p.lg) + 1;
  // us in all with the bucket kernel / four / eight / sixteen ids a thread: 300 x 4096 18.1 / 13.5 / 14.1 / 15.2, 3347 x 2048 26.6 / 23.0 / 23.7 / 24.7,
  // 6000 x 1024 26.1 / - / 23.5 / 25.2, 8192 x 1024 27.6 / - / 26.7 / 27.9, 16384 x 1024 40.0 / - / - / 43.4.
  if (n <= 8 * CHUNK) {
    hipLaunchKernelGGL(n <= 4 * CHUNK ? embed_place_kernel<4> : embed_place_kernel<8>, dim3(buckets), dim3(64 * WAVES), 0, st, ids, n, (const int *)nullptr,
                       (const Placed *)nullptr, 0, vocab, p.lg, starts, order);
  } else {
    hipLaunchKernelGGL(embed_bucket_kernel, dim3(std::min(p.chunks, 1 << 20)), dim3(CHUNK), 0, st, ids, n, vocab, p.lg, begins, from);
    hipLaunchKernelGGL(embed_place_kernel<0>, dim3(buckets), dim3(64 * WAVES), 0, st, (const int32_t *)nullptr, 0, begins, from, p.chunks, vocab, p.lg, starts, order);
  }
  // Row gradients of half the last-level cache or more are read past it, so that the table stays: 12288 x 4096 99 -> 79 us, 65536 x 4096 358 -> 345;
  // 3347 x 2048, which fit, 23.4 -> 24.6.
  const bool stream = (size_t)n * d * sizeof(float) >= LLC_BYTES / 2;
  auto *sum = accumulate ? (stream ? embed_sum_kernel<true, true, false> : embed_sum_kernel<true, false, false>)
              : past     ? (stream ? embed_sum_kernel<false, true, true> : embed_sum_kernel<false, false, true>)
                         : (stream ? embed_sum_kernel<false, true, false> : embed_sum_kernel<false, false, false>);
  hipLaunchKernelGGL(sum, blocks(p.windows * p.strips + zero_units), dim3(256), 0, st, starts, order, dx, vocab, d, scale, d_table, aside, p.window, p.windows, p.strips);
  const int join_strips = (d + 1023) / 1024;
  const dim3 joins((unsigned)std::min<long long>(p.windows * join_strips, 1 << 22));       // (more than FEW_ROWS rows: always several windows)
  auto *join = accumulate ? embed_join_kernel<true> : embed_join_kernel<false>;
  hipLaunchKernelGGL(join, joins, dim3(256), 0, st, starts, order, vocab, d, scale, d_table, aside, p.window, p.windows, join_strips);
  return hipGetLastError();
}
