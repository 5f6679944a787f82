// Attention over the cache: what its two kernels share.  attend.cu has few query rows per sequence and key/value head (decoding), attend_rows.cu many (a prompt, or a
// whole batch behind a shared prefix).  Both walk a list of (sequence, key/value head, tile of query rows, chunk of tokens), cut into one share per CTA on the device.
#pragma once

#include <limits.h>

#include "kv_common.cuh"

namespace rosaq {

// Weights are exponentials of u - top (base 2), top a value kUp below the greatest u when it was last renewed: the greatest weight is 2^kUp then, and top is renewed when one would
// pass 2^kGrow, which fp16 still holds.  A long context has most of its weight in tokens far below the greatest, and fp16 is subnormal from 2^-14 on (against 64 bits, 131071 tokens
// at 4 bits: 3.5e-4 with a greatest weight of one).
constexpr float kNone = -1e30f;                     // top of a row that has seen nothing
constexpr float kLeastScale = 5.9604644775390625e-8f;   // of a value: what writing puts in the place of zero, which pages that were never written may hold
constexpr float kUp = 10.f, kGrow = 15.f;

struct AtParams {
  KvView kv;
  KvBatchView b;                                    // prefix launch: one sequence, all rows
  int last_row;                                     // index in b.row_start of the end of the rows of a prefix launch
  int prefix_tokens;                                // > 0: this launch attends to the prefix
  const __half *q;
  __half *out;
  long long ldq, ldo;
  int group;                                        // query heads of a key/value head
  float scale_log2;                                 // scale * log2(e)
  float *partials;                                  // [2 * CTA]: shared tiles
  int *arrived;                                     // [CTA], zero between launches
  float *prefix;                                    // [row][q head][head_dim + 4]: what the prefix launch found; or nullptr
  int *status;
  long long wait_limit;
};

struct Seq {
  int row, rows, len, chunks, tiles;                // chunks: at least one, so that every row is written
  long long cost;                                   // (head, tile, chunk) triples
};

template <int kRows, int kTokens>
__device__ __forceinline__ Seq load_seq(const AtParams &p, int i, bool report) {
  Seq s;
  const int first = p.b.row_start[i], end = p.b.row_start[p.prefix_tokens > 0 ? p.last_row : i + 1];
  const int cap = p.b.width * (kKvBlock << p.kv.page_shift);   // (checked on the host: at most 2^30)
  s.row = min(max(first, 0), p.b.n_rows);
  const int last = min(max(end, s.row), p.b.n_rows);
  s.rows = last - s.row;
  const int len = p.prefix_tokens > 0 ? p.prefix_tokens : p.b.kv_len[i];
  s.len = min(max(len, 0), cap);
  if (report && (first != s.row || end != last || len != s.len)) kv_report(p.status);
  s.chunks = max((s.len + kTokens - 1) / kTokens, 1);
  s.tiles = (int)(((long long)s.rows * p.group + kRows - 1) / kRows);
  s.cost = (long long)s.tiles * p.kv.n_heads * s.chunks;
  return s;
}

__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two weights: 2^x and 2^y rounded to 11 bits, which fp16 holds without rounding from 2^-14 on.  The sums of a row's weights take the same number, so that what all of them lose cancels, and what is
// left is as little as rounding leaves (with sums of unrounded weights 131000 tokens at 4 bits were 3.6e-4 off instead of 2.8e-4).  Below 2^-14 only the product loses more:
// weights of values next to nothing, whose scale is small, may vanish in fp16 and yet have most of the softmax.
__device__ __forceinline__ float2 weights(float x, float y) {
  // (Veltkamp's splitting: the upper 24 - 13 bits, to nearest; what is no number stays none)
  const float2 w = make_float2(ex2(x), ex2(y)), g = __fmul2_rn(w, make_float2(8193.f, 8193.f));
  return __fadd2_rn(g, __ffma2_rn(g, make_float2(-1.f, -1.f), w));
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_h2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}
// Two results: fp16, 65504 at most, as rosaq_kv_read has it.  (The greatest code of a head that reaches to the end of fp16 stands for up to 65566.)  A NaN stays one.
__device__ __forceinline__ uint32_t pack_out(float a, float b) {
  const __half2 h = __hmin2_nan(__floats2half2_rn(a, b), __half2half2(__ushort_as_half(0x7bff)));
  return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ uint32_t h2_fma(uint32_t v, uint32_t mul, uint32_t add) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&mul), *reinterpret_cast<const __half2 *>(&add));
  return *reinterpret_cast<const uint32_t *>(&r);
}

// The next chunk of a walk over the list: sequence, (head, tile) in it, chunk of that.
struct Cursor {
  int seq, unit, chunk;
  Seq s;
};
// brings `chunk`, which may have run past the tile's last one, back into its range; there has to be such a chunk in the list
template <int kRows, int kTokens>
__device__ __forceinline__ void settle(const AtParams &p, Cursor &c) {
  while (c.chunk >= c.s.chunks) {
    const int skip = c.chunk / c.s.chunks, left = c.s.tiles * p.kv.n_heads - c.unit;
    if (skip < left) {
      c.unit += skip, c.chunk -= skip * c.s.chunks;
    } else {
      c.chunk -= left * c.s.chunks, c.unit = 0;
      do c.s = load_seq<kRows, kTokens>(p, ++c.seq, false);
      while (c.s.cost == 0);
    }
  }
}

// Divisions are 32-bit ones wherever the numbers are small: a 64-bit one takes a lone warp 0.2 us.
__device__ __forceinline__ long long divide(long long a, int b) { return a >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); }

// How the list is cut.  Even shares, except that
//   - tiles of few chunks are not cut where there is no need: joining the parts of several CTAs takes about 5 us, a chunk of a warp 1.0 (one sequence of 333 tokens, 32
//     heads: 13.9 us in 50 shares of seven chunks, 9.9 in 32 shares of a tile), and
//   - where all tiles are short, a cut moves to the nearer end of the tile it falls into: then there is nothing to join (64 x 200 tokens, 32 heads: 29.9 and 21.0 us).
struct Shares {
  long long total, part;                            // part = total / ctas, and what is left
  int ctas, left, near;
  __device__ __forceinline__ long long even(int c) const { return part * c + (uint32_t)(left * c) / (uint32_t)ctas; }
  // the last CTA whose even share begins at or before `at`
  __device__ __forceinline__ int owner(long long at) const {
    int c = min(max((int)((float)at * (float)ctas / (float)total), 0), ctas - 1);   // within one of it
    while (even(c) > at) --c;
    while (c + 1 < ctas && even(c + 1) <= at) ++c;
    return c;
  }
  __device__ __forceinline__ int snap(int chunk, int chunks) const { return chunk <= near ? -chunk : chunks - chunk <= near ? chunks - chunk : 0; }
  // the CTAs that hold chunks of the tile [at, at + chunks)
  __device__ __forceinline__ int first(long long at, int chunks) const { return owner(at + min(near, chunks - 1)); }
  __device__ __forceinline__ int last(long long at, int chunks) const { return max(first(at, chunks), owner(at + max(chunks - 1 - near, 0))); }
};

// What CTA `cta` of at most `most` does: chunks [begin, end) of the list (none if they are equal), `cur` at the first one.  A whole warp, `out` in shared memory.  A CTA takes at
// least `least` chunks, and tiles of fewer than `few` on average are not cut.
struct Share {
  Shares all;
  long long begin, end;
  Cursor cur;
};
template <int kRows, int kTokens>
__device__ __forceinline__ void find_share(const AtParams &p, int cta, int most, int few, int least, bool report, Share &out) {
  if ((threadIdx.x & 31) == 0) out.begin = out.end = 0;
  const int lane = threadIdx.x & 31;
  long long total = 0;
  int units = 0, longest = 0;
#pragma unroll 4
  for (int i = lane; i < p.b.n_seqs; i += 32) {
    const Seq s = load_seq<kRows, kTokens>(p, i, report);
    total += s.cost, units += s.tiles;
    if (s.cost) longest = max(longest, s.chunks);
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) {
    total += __shfl_xor_sync(0xffffffffu, total, d), units += __shfl_xor_sync(0xffffffffu, units, d);
    longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, d));
  }
  units *= p.kv.n_heads;
  if (total == 0) return;
  Shares sh;
  sh.total = total;
  sh.ctas = (int)min((long long)most, total < (long long)few * units ? (long long)units : max(divide(total, least), 1ll));
  if (cta >= sh.ctas) return;
  sh.part = divide(total, sh.ctas), sh.left = (int)(total - sh.part * sh.ctas);
  sh.near = (longest + 1) / 2;
  if (sh.near > min(8ll, sh.part / 8)) sh.near = 0;
  // the sequence that holds the first chunk of an even share
  const long long even = sh.even(cta);
  long long base = 0;
  Cursor cur;
  cur.seq = 0;
  for (int i = 0; i < p.b.n_seqs; i += 32) {
    const long long c = i + lane < p.b.n_seqs ? load_seq<kRows, kTokens>(p, i + lane, false).cost : 0;
    long long sum = c;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const long long o = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += o;
    }
    const unsigned past = __ballot_sync(0xffffffffu, base + sum > even);
    if (past) {
      const int k = __ffs(past) - 1;
      cur.seq = i + k;
      base += __shfl_sync(0xffffffffu, sum - c, k);
      break;
    }
    base += __shfl_sync(0xffffffffu, sum, 31);
  }
  cur.s = load_seq<kRows, kTokens>(p, cur.seq, false);
  cur.unit = (int)divide(even - base, cur.s.chunks), cur.chunk = (int)((even - base) - (long long)cur.unit * cur.s.chunks);
  const int moved = sh.snap(cur.chunk, cur.s.chunks);
  const long long begin = even + moved;
  cur.chunk += moved;
  // and where the next CTA's begins, by the same rule
  long long end = total;
  if (cta + 1 < sh.ctas) {
    const long long next = sh.even(cta + 1);
    Cursor c = cur;
    c.chunk += (int)(next - begin);
    settle<kRows, kTokens>(p, c);
    end = next + sh.snap(c.chunk, c.s.chunks);
  }
  settle<kRows, kTokens>(p, cur);
  if (lane == 0) out.all = sh, out.begin = begin, out.end = end, out.cur = cur;
}

// A finished row: its place in out and in what the prefix launch found.
struct RowAt {
  __half *out;
  float *prefix;        // [kHd], {maximum, sum}
};
template <int kHd>
__device__ __forceinline__ RowAt row_at(const AtParams &p, int first_row, int head, int flat) {
  const int tok = flat / p.group, qh = head * p.group + flat - tok * p.group;
  const long long row = first_row + tok;
  return RowAt{p.out + row * p.ldo + (long long)qh * kHd, p.prefix ? p.prefix + (row * p.kv.n_heads * p.group + qh) * (kHd + 4) : nullptr};
}
// Four channels of it: out, or, in a prefix launch, the sums of the prefix.
template <int kHd>
__device__ __forceinline__ void store_row4(const AtParams &p, const RowAt &at, int ch, float4 a, float m, float l) {
  if (p.prefix_tokens > 0) {
    *reinterpret_cast<float4 *>(at.prefix + ch) = a;
    if (ch == 0) *reinterpret_cast<float2 *>(at.prefix + kHd) = make_float2(m, l);
    return;
  }
  if (at.prefix) {
    const float4 x = *reinterpret_cast<const float4 *>(at.prefix + ch);
    const float2 ml = *reinterpret_cast<const float2 *>(at.prefix + kHd);
    const float mm = fmaxf(m, ml.x), f = ex2(m - mm), g = ex2(ml.x - mm);
    a = make_float4(a.x * f + x.x * g, a.y * f + x.y * g, a.z * f + x.z * g, a.w * f + x.w * g);
    l = l * f + ml.y * g;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;        // no token: zeros
  uint2 h;
  h.x = pack_out(a.x * inv, a.y * inv), h.y = pack_out(a.z * inv, a.w * inv);
  *reinterpret_cast<uint2 *>(at.out + ch) = h;
}

// (maximum, sum, channels) of two parts of a row's tokens
__device__ __forceinline__ void join(float4 &a, float &m, float &l, float4 x, float mx, float lx) {
  const float mm = fmaxf(m, mx), f = ex2(m - mm), g = ex2(mx - mm);
  a = make_float4(a.x * f + x.x * g, a.y * f + x.y * g, a.z * f + x.z * g, a.w * f + x.w * g);
  l = l * f + lx * g, m = mm;
}

// A tile of which this CTA holds a part only.
struct OpenTile {
  int from;             // its first chunk, counted from the CTA's first; kNoTile: there is none
  int seq, unit, chunks;
};
constexpr int kNoTile = INT_MIN;
__host__ __device__ constexpr int at_partial(int hd, int rows) { return rows * (hd + 4); }   // floats of a partial tile: [row][hd], then [row]{maximum, sum}, padded
__device__ __forceinline__ float *my_partial(const AtParams &p, int from, int floats) {
  return p.partials + (2ll * blockIdx.x + (from < 0 ? 0 : 1)) * floats;
}

// Adds the parts of CTAs first, first + step, ... c1 of a row's channels ch ... ch + 3; the tile begins in CTA c0's share.
template <int kHd, int kRows>
__device__ __forceinline__ void gather(const AtParams &p, int row, int ch, int c0, int c1, int first, int step, float4 &a, float &m, float &l) {
  constexpr int kAhead = 8;                      // loads in flight
  for (int k = first; k <= c1; k += kAhead * step) {
    float4 x[kAhead];
    float2 ml[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int kk = k + u * step;
      const float *const from = p.partials + (2ll * kk + (kk == c0)) * at_partial(kHd, kRows);
      ml[u] = make_float2(kNone, 0.f), x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (kk <= c1) {
        x[u] = __ldcg(reinterpret_cast<const float4 *>(from + row * kHd + ch));
        ml[u] = __ldcg(reinterpret_cast<const float2 *>(from + kRows * kHd + 2 * row));
      }
    }
    float mm = m;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) mm = fmaxf(mm, ml[u].x);
    float f = ex2(m - mm);
    a = make_float4(a.x * f, a.y * f, a.z * f, a.w * f), l *= f, m = mm;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      f = ex2(ml[u].x - m);
      a.x = __fmaf_rn(x[u].x, f, a.x), a.y = __fmaf_rn(x[u].y, f, a.y), a.z = __fmaf_rn(x[u].z, f, a.z), a.w = __fmaf_rn(x[u].w, f, a.w);
      l = __fmaf_rn(ml[u].y, f, l);
    }
  }
}

// Tiles that other CTAs hold parts of too: one that began before this share, one that is left to the next ones (`tiles`, shared memory).  The CTA has stored its partial tiles; the
// CTA that arrives last joins all of them, in the order of the shares: no CTA waits for another, and the bits are the same every time.  Threads 0 ... kThreads - 1, named barrier 1;
// `span`: four ints, `scratch`: 32 bytes per thread of shared memory.
template <int kHd, int kRows, int kTokens, int kThreads>
__device__ __forceinline__ void join_shares(const AtParams &p, const Shares &shares, long long begin, const OpenTile *tiles, int *span, float4 *scratch) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  if (tiles[0].from == kNoTile && tiles[1].from == kNoTile) return;
  const bool mine = warp < 2 && lane == 0 && tiles[warp].from != kNoTile;
  if (mine) {
    span[2 * warp] = shares.first(begin + tiles[warp].from, tiles[warp].chunks);
    span[2 * warp + 1] = shares.last(begin + tiles[warp].from, tiles[warp].chunks);
  }
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
  if (mine) {
    // (cumulative: what the barrier has made this thread see is visible to whoever sees the count, and the other way round)
    fence_gpu();
    const bool all = atomicAdd(p.arrived + span[2 * warp], 1) == span[2 * warp + 1] - span[2 * warp];
    fence_gpu();
    if (all) p.arrived[span[2 * warp]] = 0;
    else span[2 * warp] = -1;
  }
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
#pragma unroll 1
  for (int o = 0; o < 2; ++o) {
    const OpenTile f = tiles[o];
    const int c0 = span[2 * o], c1 = span[2 * o + 1];
    if (f.from == kNoTile || c0 < 0) continue;
    const Seq s = load_seq<kRows, kTokens>(p, f.seq, false);
    const int head = f.unit / s.tiles, first_row = (f.unit - head * s.tiles) * kRows, rows = min(kRows, s.rows * p.group - first_row);
    // an item is four channels of a row; where there are fewer than threads, several threads take every `split`-th partial tile each
    const int items = rows * (kHd / 4), split = max(1, kThreads / items);
#pragma unroll 1
    for (int i = threadIdx.x; i < items * split; i += kThreads) {
      const int item = i % items, row = item / (kHd / 4), ch = 4 * (item % (kHd / 4));
      float m = kNone, l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      gather<kHd, kRows>(p, row, ch, c0, c1, c0 + i / items, split, a, m, l);
      if (split == 1) store_row4<kHd>(p, row_at<kHd>(p, s.row, head, first_row + row), ch, a, m, l);
      else scratch[2 * i] = a, scratch[2 * i + 1] = make_float4(m, l, 0.f, 0.f);
    }
    if (split == 1) continue;
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
    for (int i = threadIdx.x; i < items; i += kThreads) {
      float m = kNone, l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int u = 0; u < split; ++u) join(a, m, l, scratch[2 * (u * items + i)], scratch[2 * (u * items + i) + 1].x, scratch[2 * (u * items + i) + 1].y);
      store_row4<kHd>(p, row_at<kHd>(p, s.row, head, first_row + i / (kHd / 4)), 4 * (i % (kHd / 4)), a, m, l);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");   // the scratch is free again
  }
}

int launch_attend_rows(rosaq_ctx *ctx, AtParams p, int hd, int bits, cudaStream_t s);   // attend_rows.cu

}  // namespace rosaq
