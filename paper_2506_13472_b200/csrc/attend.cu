// rosaq_attend: softmax(scale q k^T) v of new rows over the quantized paged cache, with an optional prefix shared by all sequences.
//
// With k = lo_k + s_k c and v = lo_v + s_v d (codes c, d; one pair (s, lo) per token) the sums split into products of codes and sums over tokens:
//   q . k = s_k (q . c) + lo_k sum(q),      sum_t p_t v_t = sum_t (p_t s_t) d_t + sum_t p_t lo_t.
// So no key is dequantised: nibbles and bytes, masked out of their words, ARE fp16 numbers (subnormal: code * 2^-24), exact operands of the
// tensor core.  Value codes are taken about the middle of their range, d_t - 2^(bits - 1), which costs an addition per pair and keeps the sums as small as
// the result: of positive codes the roundings of the weights and of the accumulators would all point one way (against 64 bits, 26000 tokens
// at 8 bits: 1.2e-3 that way).  The weights of the second product are kept near one whatever the size of the values: with 2^e the power of two in s_t,
// u_t = score_t log2(e) + e is what the running maximum M is taken of, and p_t s_t = 2^(u_t - M) (s_t 2^-e) has its greatest value in [1, 2)
// before the rounding to fp16 (2^-11 relative, 2^-25 of the greatest weight absolute), while sum(p_t) and sum(p_t lo_t) stay in fp32.
//
// Tokens are the rows of the first MMA (m16n8k16: 16 tokens x 8 query rows) and the k of the second one (16 channels x 8 query rows), so a group of
// up to eight query heads costs no more than one, and a lane's words of a block (kv_common.cuh) are its A fragments in both.
//
// Bound: memory for one row per sequence.  What moves is the cache, once; a block of 16 tokens and one key/value head (2176 bytes at 4 bits, head of
// 128) takes a warp about 190 instructions, half of what an SM issues in the time in which its share of the HBM bandwidth delivers the block.
// The list of (sequence, head, tile of query rows, block) is cut into equal shares, one per CTA, whatever the lengths: CTAs read lengths on the
// device, so a captured launch follows them.  Every warp streams a run
// of its own through slots of its own and refills them itself.
// A tile whose blocks several CTAs share is finished by the CTA that arrives last, in the order of the shares: no CTA waits for another, and the
// bits are the same every time.
#include <limits.h>

#include <algorithm>

#include "kv_common.cuh"

#ifndef W1
#define W1 7
#endif
#ifndef W8
#define W8 5
#endif
#ifndef AT4
#define AT4 16
#endif
#ifndef AT8
#define AT8 12
#endif
#ifndef ILP1
#define ILP1 2
#endif
#ifndef QS1
#define QS1 0
#endif
namespace rosaq {
namespace {

constexpr float kNone = -1e30f;                     // running maximum of a row that has seen nothing
constexpr float kGrow = 8.f;                        // a maximum is renewed when it is exceeded by this factor of two
constexpr int kChunk = 2;                           // blocks that a warp takes at a time

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

template <int kRows>
__device__ __forceinline__ Seq load_seq(const AtParams &p, int i, bool report) {
  Seq s;
  const int first = p.b.row_start[i], end = p.b.row_start[p.prefix_tokens > 0 ? p.last_row : i + 1];
  const int cap = p.b.ld_table * (kKvBlock << p.kv.page_shift);   // (checked on the host: below 2^31)
  s.row = min(max(first, 0), p.b.n_rows);
  const int last = min(max(end, s.row), p.b.n_rows);
  s.rows = last - s.row;
  const int len = p.prefix_tokens > 0 ? p.prefix_tokens : p.b.kv_len[i];
  s.len = min(max(len, 0), cap);
  if (report && (first != s.row || end != last || len != s.len)) kv_report(p.status);
  s.chunks = max((s.len + kChunk * kKvBlock - 1) / (kChunk * kKvBlock), 1);
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
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_h2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t v, uint32_t mul, uint32_t add) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&mul), *reinterpret_cast<const __half2 *>(&add));
  return *reinterpret_cast<const uint32_t *>(&r);
}
// A fragment of step j of a block in units of 2^-24.  Four bits, keys (token, channel): the codes, of channels 8-15 sixteen times the codes.  Four bits, values (channel,
// token): the whole bytes, i.e. code + 16 * (code of the channel eight further on), in the rows of channels 0-7, sixteen times the code in those of channels 8-15; what
// is too much in the first is taken off the sums (one operation less per word).
template <int kBits, bool kValue>
__device__ __forceinline__ void code_fragment(const uint32_t *w, int j, uint32_t *a) {
  if (kBits == 4 && kValue) {
    a[0] = w[j] & 0x00ff00ffu, a[1] = w[j] & 0x00f000f0u, a[2] = __byte_perm(w[j], 0, 0x4341), a[3] = a[2] & 0x00f000f0u;
  } else if (kBits == 4) {
    const uint32_t u = w[j], v = u >> 8;
    a[0] = u & 0x000f000fu, a[2] = u & 0x00f000f0u, a[1] = v & 0x000f000fu, a[3] = v & 0x00f000f0u;
  } else {
    const uint32_t u = w[2 * j], v = w[2 * j + 1];
    a[0] = __byte_perm(u, 0, 0x4140), a[1] = __byte_perm(v, 0, 0x4140), a[2] = __byte_perm(u, 0, 0x4342), a[3] = __byte_perm(v, 0, 0x4342);
  }
}
// of values as code - 2^(bits - 1), by way of 1024 + code (upper nibbles: 1024 + 16 code)
template <int kBits>
__device__ __forceinline__ void value_fragment(const uint32_t *w, int j, uint32_t *a) {
  constexpr uint32_t kOne = 0x3c003c00u, kSixteenth = 0x2c002c00u;
  if (kBits == 4) {
    constexpr uint32_t kLow = 0xe408e408u, kHigh = 0xd480d480u;   // -1032, -72
    const uint32_t u = w[j], v = u >> 8;
    a[0] = h2_fma(lop_and_or(u, 0x000f000fu, 0x64006400u), kOne, kLow), a[1] = h2_fma(lop_and_or(u, 0x00f000f0u, 0x64006400u), kSixteenth, kHigh);
    a[2] = h2_fma(lop_and_or(v, 0x000f000fu, 0x64006400u), kOne, kLow), a[3] = h2_fma(lop_and_or(v, 0x00f000f0u, 0x64006400u), kSixteenth, kHigh);
  } else {
    constexpr uint32_t kMid = 0xe480e480u;                        // -1152
    const uint32_t u = w[2 * j], v = w[2 * j + 1];
    a[0] = h2_fma(__byte_perm(u, 0x64646464u, 0x4140), kOne, kMid), a[1] = h2_fma(__byte_perm(v, 0x64646464u, 0x4140), kOne, kMid);
    a[2] = h2_fma(__byte_perm(u, 0x64646464u, 0x4342), kOne, kMid), a[3] = h2_fma(__byte_perm(v, 0x64646464u, 0x4342), kOne, kMid);
  }
}

template <int kHd, int kBits, int kTiles, int kWarps>
struct Cfg {
  static constexpr int kRows = 8 * kTiles;
  static constexpr int kStageBytes = kChunk * kv_block_bytes(kHd, kBits);
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kPerSm = kTiles == 1 ? (kBits == 4 ? AT4 : AT8) / (kWarps + 1) : kTiles == 2 ? 12 / (kWarps + 1) : 1;   // CTAs that the registers are to leave room for
  static constexpr int kIlp = kTiles == 1 ? ILP1 : 1;   // blocks computed at a time
  static constexpr int kAccLd = kHd + 4;            // floats: two rows of a pair on different banks
  static constexpr int kFragBytes = kRows * (4 * kAccLd + 16);   // a part of a tile: [row][kAccLd], then [row]{maximum, sum, sum of least values, -}
  static constexpr bool kQShared = kTiles > 2 || (kTiles == 1 && QS1);      // B fragments of the queries in shared memory rather than in registers, each warp its own
  static constexpr int kQBytes = kQShared ? kWarps * kTiles * kHd / 16 * 256 : 0;
  static constexpr int kPairBytes = kChunk * kKvBlock * 20;   // of a warp: what its tokens' pairs become
  static constexpr int kRoom = 222 * 1024 / kPerSm - kQBytes - 1024 - (kPairBytes + 64 + 64) * kWarps;
  static constexpr int kDepth = kRoom / kStageBytes / kWarps < 32 / kWarps ? kRoom / kStageBytes / kWarps : 32 / kWarps;   // slots of a warp, next to each other
  static constexpr int kStages = kWarps * kDepth;
  static constexpr int kSmem = kStages * kStageBytes + kQBytes + kPairBytes * kWarps + 16 * kStages + 64 * kWarps + 64;
  static constexpr bool kSlotsHold = kDepth * kStageBytes >= kFragBytes;   // a part of a tile
  static constexpr int kPartial = kRows * (kHd + 4);   // floats of a partial tile: [row][kHd], then [row]{maximum, sum}, padded
  static constexpr long long kWorkBytes = 2 * 4 * kPartial + 2 * kWarps * kFragBytes;   // of a CTA: partial tiles, parts that the slots do not hold
  static_assert(kChunk == 2 && kDepth >= 1 && kStages <= 32, "slots");
};

// The next chunk of a walk over the list: sequence, (head, tile) in it, chunk of that.
struct Cursor {
  int seq, unit, chunk;
  Seq s;
};
// brings `chunk`, which may have run past the tile's last one, back into its range; there has to be such a chunk in the list
template <int kRows>
__device__ __forceinline__ bool settle(const AtParams &p, Cursor &c) {
  if (c.chunk < c.s.chunks) return false;
  do {
    const int skip = c.chunk / c.s.chunks, left = c.s.tiles * p.kv.n_heads - c.unit;
    if (skip < left) {
      c.unit += skip, c.chunk -= skip * c.s.chunks;
    } else {
      c.chunk -= left * c.s.chunks, c.unit = 0;
      do c.s = load_seq<kRows>(p, ++c.seq, false);
      while (c.s.cost == 0);
    }
  } while (c.chunk >= c.s.chunks);
  return true;
}

// How the list is cut.  Even shares, except that
//   - tiles of few chunks are not cut where there is no need: joining the parts of several CTAs takes about 5 us, a warp's chunk 0.8 (one sequence of 333 tokens,
//     32 heads: 13.8 us in 50 shares of seven chunks, .. in 32 shares of a tile), and
//   - a cut that would fall within `near` chunks of the end of a tile moves there.
// Divisions are 32-bit ones wherever the numbers are small: a 64-bit one takes a lone warp 0.2 us.
__device__ __forceinline__ long long divide(long long a, int b) { return a >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b); }
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
__device__ __forceinline__ Shares make_shares(long long total, int units, int warps, int tiles, int most) {
  Shares s;
  s.total = total;
  s.ctas = (int)min((long long)most, total < 8ll * warps * units ? (long long)units : divide(total, warps));
  s.part = divide(total, s.ctas), s.left = (int)(total - s.part * s.ctas);
  s.near = (int)min(8ll / tiles, s.part / 8);
  return s;
}

// A part of a tile, as its warp leaves it.
struct Frag {
  int from;             // first chunk of the tile, counted from the CTA's first; kNoFrag: none
  int seq, unit, chunks;
  const float *data;
};
constexpr int kNoFrag = INT_MIN;

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
  h.x = pack_h2(a.x * inv, a.y * inv), h.y = pack_h2(a.z * inv, a.w * inv);
  *reinterpret_cast<uint2 *>(at.out + ch) = h;
}

// (maximum, sum, channels) of two parts of a row's tokens
__device__ __forceinline__ void join(float4 &a, float &m, float &l, float4 x, float mx, float lx) {
  const float mm = fmaxf(m, mx), f = ex2(m - mm), g = ex2(mx - mm);
  a = make_float4(a.x * f + x.x * g, a.y * f + x.y * g, a.z * f + x.z * g, a.w * f + x.w * g);
  l = l * f + lx * g, m = mm;
}

template <int kHd, int kBits, int kTiles, int kWarps>
__global__ void __launch_bounds__(32 * (kWarps + 1), Cfg<kHd, kBits, kTiles, kWarps>::kPerSm)
attend_kernel(const __grid_constant__ AtParams p) {
  using C = Cfg<kHd, kBits, kTiles, kWarps>;
  constexpr int kSteps = kHd / 16, kWords = kSteps * (kBits / 4), kRows = C::kRows, kConsumers = 32 * kWarps;
  constexpr int kBlockBytes = kv_block_bytes(kHd, kBits);
  // Value codes about the middle of their range: by an addition per pair, or, while there is one tile of rows, by a second MMA that takes the middle off
  // again (eight of them in the place of 32 additions).
  constexpr bool kTakeOff = kTiles == 1;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t *const ring = smem;                                                             // [warp][kDepth] slots
  uint2 *const q_frags = reinterpret_cast<uint2 *>(smem + C::kStages * C::kStageBytes);   // [warp][step][tile][lane]
  float4 *const pair_terms = reinterpret_cast<float4 *>(q_frags + C::kQBytes / 8);        // [warp][token]{s_k', lo_k, log2 s_v, 1 / s_v}, [token] lo_v / s_v + middle
  uint64_t *const bars = reinterpret_cast<uint64_t *>(pair_terms + C::kPairBytes / 16 * kWarps);
  Frag *const frags = reinterpret_cast<Frag *>(bars + 2 * C::kStages);                    // [warp]{first part of a tile that began before, last one}
  int *const flag = reinterpret_cast<int *>(frags + 2 * kWarps);                          // [2]{first, last CTA} of tiles that other CTAs hold parts of
  // Parts of tiles: a warp's last one lies in its slots, where they are large enough, an earlier one behind the partial tiles of all CTAs.
  uint8_t *const parts = reinterpret_cast<uint8_t *>(p.partials + 2ll * gridDim.x * C::kPartial) + (long long)blockIdx.x * 2 * kWarps * C::kFragBytes;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;

  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * C::kStages;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(full0 + 8 * i, 1), mbar_init(empty0 + 8 * i, 1);
    mbar_init_fence();
  }
  if (threadIdx.x < 2 * kWarps) frags[threadIdx.x].from = kNoFrag;
  grid_dep_launch_dependents();
  __syncthreads();
  grid_dep_wait();                                  // q, the batch, the pages, the partial tiles: all may be the previous kernel's

  // ---- the share of this CTA; every warp works it out
  long long total = 0;
  int units = 0;
#pragma unroll 4
  for (int i = lane; i < p.b.n_seqs; i += 32) {
    const Seq s = load_seq<kRows>(p, i, blockIdx.x == 0 && warp == 0);
    total += s.cost, units += s.tiles;
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) total += __shfl_xor_sync(0xffffffffu, total, d), units += __shfl_xor_sync(0xffffffffu, units, d);
  units *= p.kv.n_heads;
  if (total == 0) return;
  const Shares shares = make_shares(total, units, kWarps, kTiles, gridDim.x);
  const int ctas = shares.ctas, cta = blockIdx.x;
  if (cta >= ctas) return;
  long long begin, end;
  Cursor cur;
  {
    // the sequence that holds the first chunk of an even share
    const long long even = shares.even(cta);
    long long base = 0;
    cur.seq = 0;
    for (int i = 0; i < p.b.n_seqs; i += 32) {
      const long long c = i + lane < p.b.n_seqs ? load_seq<kRows>(p, i + lane, false).cost : 0;
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
    cur.s = load_seq<kRows>(p, cur.seq, false);
    cur.unit = (int)divide(even - base, cur.s.chunks), cur.chunk = (int)((even - base) - (long long)cur.unit * cur.s.chunks);
    const int moved = shares.snap(cur.chunk, cur.s.chunks);
    begin = even + moved, cur.chunk += moved;        // (perhaps behind the tile's last chunk: settled below)
    // and where the next CTA's begins, by the same rule
    end = total;
    if (cta + 1 < ctas) {
      const long long next = shares.even(cta + 1);
      Cursor c = cur;
      c.chunk += (int)(next - begin);
      settle<kRows>(p, c);
      end = next + shares.snap(c.chunk, c.s.chunks);
    }
  }
  const int n = (int)(end - begin);                 // chunks of this CTA (a share of 2^31 would be 4 TB of cache)
  // warp w takes chunks [n w / kWarps, n (w + 1) / kWarps), rounded up (warp 0 always has one), of the CTA's: long runs, so that a warp seldom changes its tile and never waits for another
  auto bound = [&](int w) { return (int)(((long long)n * w + kWarps - 1) / kWarps); };

  if (warp == kWarps) {
    // ---- producer: lane i fills slot i, with chunks i % kDepth, i % kDepth + kDepth, ... of warp i / kDepth.  The lanes go round together and none waits for
    // another's slot; the page of a chunk is looked up a fill ahead.
    const int owner = min(lane / C::kDepth, kWarps - 1);
    const int last = lane < C::kStages ? bound(owner + 1) : 0;
    int j = bound(owner) + lane % C::kDepth;
    uint32_t parity = 1;                             // of the phase that frees the slot; the other one's end brings its chunk
    bool copied = false;
    long long tries = 0;
    const uint64_t keep = policy_evict_first();
    cur.chunk += j;
    const uint8_t *first = nullptr, *second = nullptr;   // the next chunk: a run of blocks, and the second block when it lies elsewhere
    int run = 0, rest = 0;                           // their bytes
    auto look_up = [&]() {
      run = rest = 0;
      if (j >= last) return;
      settle<kRows>(p, cur);
      const int head = cur.unit / cur.s.tiles, block = kChunk * cur.chunk;
      const int blocks = min(kChunk, (cur.s.len + kKvBlock - 1) / kKvBlock - block);   // (0: a sequence of no tokens)
      if (blocks <= 0) return;
      const uint8_t *const heads = p.kv.pages + ((long long)head << p.kv.page_shift) * kBlockBytes;
      const int page = kv_page(p.kv, p.b, cur.seq, block), near = min(blocks, 1 << p.kv.page_shift);
      if (page < 0) kv_report(p.status);             // (the first page of the cache in its place)
      first = heads + kv_offset(p.kv, max(page, 0), block, kBlockBytes), run = near * kBlockBytes;
      if (near < blocks) {
        const int other = kv_page(p.kv, p.b, cur.seq, block + 1);
        if (other < 0) kv_report(p.status);
        second = heads + kv_offset(p.kv, max(other, 0), block + 1, kBlockBytes), rest = kBlockBytes;
      }
    };
    look_up();
    while (__any_sync(0xffffffffu, j < last)) {
      const bool ready = j < last && mbar_test_wait(empty0 + 8 * lane, parity);
      if (ready) {
        const uint32_t bar = full0 + 8 * lane, dst = smem_u32(ring + lane * C::kStageBytes);
        if (run == 0) {
          mbar_arrive(bar);
        } else {
          mbar_arrive_expect_tx(bar, run + rest);
          bulk_copy_g2s_hint(dst, first, run, bar, keep);
          if (rest) bulk_copy_g2s_hint(dst + kBlockBytes, second, rest, bar, keep);
        }
        copied = true, parity ^= 1, tries = 0;
        j += C::kDepth, cur.chunk += C::kDepth;
        look_up();
      } else if (j < last && ++tries > p.wait_limit) {   // the consumers give up too, one wait each
        atomicExch(p.status, (int)ROSAQ_ERR_TIMEOUT);
        j = last;
      }
      if (!__any_sync(0xffffffffu, ready)) __nanosleep(40);
    }
    // the CTA outlasts its copies, also when the consumers have given up on them
    if (copied)
      for (int i = 0; i < 1 << 20 && !mbar_test_wait(full0 + 8 * lane, parity); ++i) __nanosleep(100);
    return;
  }

  // ---- consumers
  const int r = lane >> 2, c = lane & 3;
  uint2 *const q_frag = q_frags + warp * (C::kQBytes / 8 / kWarps);
  float4 *const terms = pair_terms + warp * (C::kPairBytes / 16);
  float *const term_vl = reinterpret_cast<float *>(terms + kChunk * kKvBlock);
  bool lost = false;
  int j = bound(warp);                               // this warp's next chunk
  const int last = bound(warp + 1);
  int slot = warp * C::kDepth;
  uint32_t parity = 0;
  cur.chunk += j;
  while (j < last) {
    settle<kRows>(p, cur);
    const Seq &s = cur.s;
    const int head = cur.unit / s.tiles, tile = cur.unit - head * s.tiles, chunk0 = cur.chunk, j0 = j;
    const int j1 = min(last, j0 + s.chunks - chunk0);   // the chunks [j0, j1) are this tile's
    const int first_row = tile * kRows, n_flat = s.rows * p.group;

    // ---- query rows of the tile: B fragments, scaled by a power of two so that the greatest value of all rows lies in [2^12, 2^13); of the channels whose
    // nibbles read sixteen times too large a sixteenth.  Rows that are not finite do not count for it.
    uint32_t qf[kTiles][kSteps][2];
    float row_b[2 * kTiles];                         // scale log2(e) sum(q) of this lane's columns 2 c, 2 c + 1 of each tile of eight rows
    int lim[2 * kTiles];                             // tokens that the row sees
    const int seen0 = s.len - s.rows + 1;            // by the first row of the sequence
    float most_q = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int flat = first_row + 8 * t + r;
      const bool valid = flat < n_flat;
      const int tok = valid ? flat / p.group : 0, qh = head * p.group + (valid ? flat - tok * p.group : 0);
      const __half *const src = p.q + (long long)(s.row + tok) * p.ldq + (long long)qh * kHd + 2 * c;
      float most = 0.f, sum = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) qf[t][k][h] = valid ? *reinterpret_cast<const uint32_t *>(src + 16 * k + 8 * h) : 0u;
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&qf[t][k][h]));
          most = fmaxf(most, fmaxf(fabsf(x.x), fabsf(x.y)));
          sum += x.x + x.y;
        }
      most_q = fmaxf(most_q, most <= 65504.f ? most : 0.f);
      sum += __shfl_xor_sync(0xffffffffu, sum, 1), sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const float b = p.scale_log2 * sum;
      const int seen = p.prefix_tokens > 0 ? s.len : valid ? min(max(seen0 + tok, 0), s.len) : s.len;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        row_b[2 * t + e] = __shfl_sync(0xffffffffu, b, 4 * (2 * c + e));
        lim[2 * t + e] = __shfl_sync(0xffffffffu, seen, 4 * (2 * c + e));
      }
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) most_q = fmaxf(most_q, __shfl_xor_sync(0xffffffffu, most_q, d));
    const int up = most_q > 0.f ? 12 - ((int)(__float_as_uint(most_q) >> 23) - 127) : 0;   // (fp16 values: never an fp32 subnormal)
    const float key_scale = p.scale_log2 * __uint_as_float((uint32_t)(127 + 24 - up) << 23);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float f = __uint_as_float((uint32_t)(127 + up - (kBits == 4 && h ? 4 : 0)) << 23);
          const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&qf[t][k][h]));
          qf[t][k][h] = pack_h2(x.x * f, x.y * f);
        }
        if (C::kQShared) q_frag[(k * kTiles + t) * 32 + lane] = make_uint2(qf[t][k][0], qf[t][k][1]);
      }
    if (C::kQShared) __syncwarp();
    int least = s.len, most_seen = s.len;            // tokens that every row, that any row of the tile sees
    if (p.prefix_tokens == 0) {
      const int t0 = first_row / p.group, t1 = (min(first_row + kRows, n_flat) - 1) / p.group;
      least = min(max(seen0 + t0, 0), s.len), most_seen = min(max(seen0 + t1, 0), s.len);
    }

    float acc[kSteps][kTiles][4], top[2 * kTiles], den[2 * kTiles], off[2 * kTiles];
#pragma unroll
    for (int i = 0; i < 2 * kTiles; ++i) top[i] = kNone, den[i] = off[i] = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][t][e] = 0.f;

    // Value codes about the middle of their range (kTakeOff): the sums of the weights, as the tensor core has them, gather in `low`, and every
    // kFlush chunks the middle times them is taken off.
    float low[4] = {0.f, 0.f, 0.f, 0.f};
    auto take_off = [&]() {
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][0][e] += low[e];
#pragma unroll
      for (int e = 0; e < 4; ++e) low[e] = 0.f;
    };

    // ---- this warp's chunks of the tile
#pragma unroll 1
    for (; j < j1; ++j) {
      const uint32_t base = smem_u32(ring + slot * C::kStageBytes);
      if (!lost) {
        bool here = mbar_try_wait(full0 + 8 * slot, parity);
        if (!__all_sync(0xffffffffu, here)) {
          for (long long i = 0; !here && i < p.wait_limit; ++i) here = mbar_try_wait(full0 + 8 * slot, parity);
          lost = !__all_sync(0xffffffffu, here);
          if (lost && lane == 0) atomicExch(p.status, (int)ROSAQ_ERR_TIMEOUT);
        }
      }
      if (lost) continue;                            // (waits once; the barriers and counters below are still served)
      const int tok0 = (chunk0 + j - j0) * (kChunk * kKvBlock);
      {
        // what a token's pairs come to, one token per lane
        constexpr int kPairs = 2 * kv_code_bytes(kHd, kBits);
        const uint32_t at = base + (lane >> 4) * kBlockBytes + kPairs + 4 * (lane & 15);
        uint32_t kp = lds32(at), vp = lds32(at + 64);
        if (tok0 + lane >= most_seen) kp = vp = 0x00000001u;   // whatever lies behind the last token
        const float2 kf = __half22float2(*reinterpret_cast<__half2 *>(&kp)), vf = __half22float2(*reinterpret_cast<__half2 *>(&vp));
        const float lv = lg2(vf.x), vi = ex2(-lv);   // log2(s) and 1 / s as that has it
        terms[lane] = make_float4(kf.x * key_scale, kf.y, lv, vi);
        term_vl[lane] = __fmaf_rn(vf.y, vi, kBits == 4 ? 8.f : 128.f);   // (lo + s 2^(bits - 1)) / s
        __syncwarp();
      }
      constexpr int kN = C::kIlp;
#pragma unroll 1
      for (int b0 = 0; b0 < kChunk; b0 += kN) {
        const int tok_b = tok0 + b0 * kKvBlock;
        if (tok_b >= most_seen) break;
        const uint32_t at = base + b0 * kBlockBytes + 16 * lane;
        // ---- scores.  A second block that is not there (or holds nothing that is seen) is computed from what lies in the slot and masked.
        float sc[kN][kTiles][4];
#pragma unroll
        for (int b = 0; b < kN; ++b)
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[b][t][e] = 0.f;
        constexpr int kPer = kBits == 4 ? 4 : 2;     // steps of a 16-byte chunk
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
          uint32_t w[kN][4];
#pragma unroll
          for (int b = 0; b < kN; ++b) {
            const uint4 v = lds128(at + b * kBlockBytes + 512 * i);
            w[b][0] = v.x, w[b][1] = v.y, w[b][2] = v.z, w[b][3] = v.w;
          }
#pragma unroll
          for (int e = 0; e < kPer; ++e) {
            const int k = kPer * i + e;
            uint2 qs[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) qs[t] = C::kQShared ? q_frag[(k * kTiles + t) * 32 + lane] : make_uint2(qf[t][k][0], qf[t][k][1]);
#pragma unroll
            for (int b = 0; b < kN; ++b) {
              uint32_t a[4];
              code_fragment<kBits, false>(w[b], e, a);
#pragma unroll
              for (int t = 0; t < kTiles; ++t) mma16816(sc[b][t], a, qs[t].x, qs[t].y);
            }
          }
        }
        // ---- u = score log2(e) + log2(s_v)
        float vi[kN][2], vl[kN][2];
#pragma unroll
        for (int b = 0; b < kN; ++b)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int tk = kKvBlock * (b0 + b) + 8 * h + r;
            const float4 x = terms[tk];
            vi[b][h] = x.w, vl[b][h] = term_vl[tk];
#pragma unroll
            for (int i = 0; i < 2 * kTiles; ++i) {
              float &y = sc[b][i >> 1][2 * h + (i & 1)];
              y = __fmaf_rn(y, x.x, __fmaf_rn(row_b[i], x.y, x.z));
            }
          }
        if (tok_b + kN * kKvBlock > least) {
          // the border: tokens that a row does not see
#pragma unroll
          for (int b = 0; b < kN; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int i = 0; i < 2 * kTiles; ++i)
                if (tok_b + kKvBlock * b + 8 * h + r >= min(lim[i], most_seen)) sc[b][i >> 1][2 * h + (i & 1)] = -INFINITY;
        }
        float most[2 * kTiles];
        bool grow = false;
#pragma unroll
        for (int i = 0; i < 2 * kTiles; ++i) {
          most[i] = fmaxf(sc[0][i >> 1][i & 1], sc[0][i >> 1][(i & 1) + 2]);
#pragma unroll
          for (int b = 1; b < kN; ++b) most[i] = fmaxf(most[i], fmaxf(sc[b][i >> 1][i & 1], sc[b][i >> 1][(i & 1) + 2]));
          grow |= most[i] > top[i] + kGrow;
        }
        if (__any_sync(0xffffffffu, grow)) {
          if (kTakeOff) take_off();
#pragma unroll
          for (int i = 0; i < 2 * kTiles; ++i) {
            const int t = i >> 1, e = i & 1;
            float m = most[i];
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4)), m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)), top[i]);
            const float f = ex2(top[i] - m);
            top[i] = m, den[i] *= f, off[i] *= f;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) acc[k][t][e] *= f, acc[k][t][e + 2] *= f;
          }
        }
        // ---- weights p s_v, their sums, and the product with the value codes
        uint32_t pf[kN][kTiles][2];
#pragma unroll
        for (int b = 0; b < kN; ++b)
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = 2 * t + (e & 1), h = e >> 1;
              const float x = ex2(sc[b][t][e] - top[i]);
              den[i] = __fmaf_rn(x, vi[b][h], den[i]);
              off[i] = __fmaf_rn(x, vl[b][h], off[i]);
              sc[b][t][e] = x;
            }
            pf[b][t][0] = transpose8(pack_h2(sc[b][t][0], sc[b][t][1])), pf[b][t][1] = transpose8(pack_h2(sc[b][t][2], sc[b][t][3]));
          }
        if (kTakeOff) {
          // minus the middle of what the fragments hold: 8 + 16 * 8 and 16 * 8, or 128
          const uint32_t mid[4] = {kBits == 4 ? 0x80888088u : 0x80808080u, 0x80808080u, kBits == 4 ? 0x80888088u : 0x80808080u, 0x80808080u};
#pragma unroll
          for (int b = 0; b < kN; ++b) mma16816(low, mid, pf[b][0][0], pf[b][0][1]);
        }
#pragma unroll
        for (int b = 0; b < kN; ++b)
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint4 v = lds128(at + b * kBlockBytes + kv_code_bytes(kHd, kBits) + 512 * i);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
              uint32_t a[4];
              if (kTakeOff) code_fragment<kBits, true>(w, e, a);
              else value_fragment<kBits>(w, e, a);
#pragma unroll
              for (int t = 0; t < kTiles; ++t) mma16816(acc[kPer * i + e][t], a, pf[b][t][0], pf[b][t][1]);
            }
          }
      }
      constexpr int kFlush = 4;
      if (kTakeOff && (j & (kFlush - 1)) == 0) take_off();
      __syncwarp();
      if (lane == 0) mbar_arrive(empty0 + 8 * slot);   // (every lane's loads from the slot have been used by now)
      if (++slot == (warp + 1) * C::kDepth) slot = warp * C::kDepth, parity ^= 1;
    }
    if (kTakeOff) take_off();
    cur.chunk = chunk0 + j1 - j0;

    // ---- the tile's rows, or this warp's part of them
    const bool whole = chunk0 == 0 && j1 - j0 == s.chunks;
    const int which = chunk0 != 0 ? 0 : 1;
    // (no chunk left: the slots are free)
    float *const part = reinterpret_cast<float *>(C::kSlotsHold && j == last ? ring + warp * C::kDepth * C::kStageBytes : parts + (2 * warp + which) * C::kFragBytes);
#pragma unroll
    for (int i = 0; i < 2 * kTiles; ++i) {
      const int t = i >> 1, e = i & 1, row = 8 * t + 2 * c + e;
#pragma unroll
      for (int d = 4; d < 32; d *= 2) den[i] += __shfl_xor_sync(0xffffffffu, den[i], d), off[i] += __shfl_xor_sync(0xffffffffu, off[i], d);
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        if (kTakeOff && kBits == 4) acc[k][t][e] -= acc[k][t][e + 2];
        acc[k][t][e] *= kTakeOff ? 16777216.f : 1.f;
        acc[k][t][e + 2] *= !kTakeOff ? 1.f : kBits == 4 ? 1048576.f : 16777216.f;
      }
      if (!whole) {
        if (r == 0) reinterpret_cast<float4 *>(part + kRows * C::kAccLd)[row] = make_float4(top[i], den[i], off[i], 0.f);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) part[row * C::kAccLd + 16 * k + r] = acc[k][t][e], part[row * C::kAccLd + 16 * k + 8 + r] = acc[k][t][e + 2];
      } else if (first_row + row < n_flat) {
        const RowAt to = row_at<kHd>(p, s.row, head, first_row + row);
        float l = den[i];
        if (p.prefix_tokens > 0) {
#pragma unroll
          for (int k = 0; k < kSteps; ++k) to.prefix[16 * k + r] = acc[k][t][e] + off[i], to.prefix[16 * k + 8 + r] = acc[k][t][e + 2] + off[i];
          if (r == 0) *reinterpret_cast<float2 *>(to.prefix + kHd) = make_float2(top[i], l);
        } else {
          float f = 1.f, g = 0.f;
          if (to.prefix) {
            const float2 ml = *reinterpret_cast<const float2 *>(to.prefix + kHd);
            const float mm = fmaxf(top[i], ml.x);
            f = ex2(top[i] - mm), g = ex2(ml.x - mm);
            l = l * f + ml.y * g;
          }
          const float inv = l == 0.f ? 0.f : 1.f / l;
          f *= inv, g *= inv;
#pragma unroll
          for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float x = (acc[k][t][e + 2 * h] + off[i]) * f;
              if (to.prefix) x = __fmaf_rn(to.prefix[16 * k + 8 * h + r], g, x);
              to.out[16 * k + 8 * h + r] = __float2half_rn(x);
            }
        }
      }
    }
    if (!whole && lane == 0) frags[2 * warp + which] = Frag{j0 - chunk0, cur.seq, cur.unit, s.chunks, part};
  }

  // ---- tiles that several warps hold parts of: chains of the last part of one warp (or the first one of warp 0, when the CTA's share begins inside a tile) and the first
  // parts of those behind it
  asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
  // One warp per chain, or all on the only one and on those of large tiles.
  int chains = 0;
#pragma unroll 1
  for (int lead = -1; lead < kWarps; ++lead) chains += frags[lead < 0 ? 0 : 2 * lead + 1].from != kNoFrag;
  const bool alone = kTiles == 1 && chains > 1;
  int open = -1;                                     // the chain that is left to other CTAs, if it begins here
#pragma unroll 1
  for (int lead = -1, k = 0; lead < kWarps; ++lead) {
    const Frag f = frags[lead < 0 ? 0 : 2 * lead + 1];
    if (f.from == kNoFrag) continue;
    const bool whole = f.from >= 0 && f.from + f.chunks <= n;
    if (!whole && lead >= 0) open = lead;
    if (alone && k++ % kWarps != warp) continue;
    const Seq s = load_seq<kRows>(p, f.seq, false);
    const int head = f.unit / s.tiles, first_row = (f.unit - head * s.tiles) * kRows, rows = min(kRows, s.rows * p.group - first_row);
    const float *member[kWarps];                     // the parts that belong to it
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const Frag &g = frags[2 * w + (w == lead)];
      member[w] = w >= lead && g.from == f.from ? g.data : nullptr;
    }
    float *const to = p.partials + (long long)(2 * cta + (f.from < 0 ? 0 : 1)) * C::kPartial;
#pragma unroll 1
    for (int i = alone ? lane : threadIdx.x; i < rows * (kHd / 4); i += alone ? 32 : kConsumers) {
      const int row = i / (kHd / 4), ch = 4 * (i % (kHd / 4));
      float m = kNone, l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), u[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        u[w] = member[w] ? reinterpret_cast<const float4 *>(member[w] + kRows * C::kAccLd)[row] : make_float4(kNone, 0.f, 0.f, 0.f);
        m = fmaxf(m, u[w].x);
      }
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (!member[w]) continue;
        const float4 v = *reinterpret_cast<const float4 *>(member[w] + row * C::kAccLd + ch);
        const float g = ex2(u[w].x - m);
        a.x = __fmaf_rn(g, v.x + u[w].z, a.x), a.y = __fmaf_rn(g, v.y + u[w].z, a.y), a.z = __fmaf_rn(g, v.z + u[w].z, a.z), a.w = __fmaf_rn(g, v.w + u[w].z, a.w);
        l = __fmaf_rn(g, u[w].y, l);
      }
      if (whole) {
        store_row4<kHd>(p, row_at<kHd>(p, s.row, head, first_row + row), ch, a, m, l);
      } else {
        *reinterpret_cast<float4 *>(to + row * kHd + ch) = a;
        if (ch == 0) *reinterpret_cast<float2 *>(to + kRows * kHd + 2 * row) = make_float2(m, l);
      }
    }
  }
  // ---- tiles that other CTAs hold parts of too: one that began before this share, one that is left to the next ones
  const bool enters = frags[0].from != kNoFrag;
  if (!enters && open < 0) return;
  const int mine = warp == 0 && enters ? 0 : warp == 1 && open >= 0 ? 2 * open + 1 : -1;   // warp 0 sees to the one, warp 1 to the other
  int *const span = flag + 2 * warp;                 // [2][first, last]
  if (mine >= 0 && lane == 0) span[0] = shares.first(begin + frags[mine].from, frags[mine].chunks), span[1] = shares.last(begin + frags[mine].from, frags[mine].chunks);
  asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
  if (mine >= 0 && lane == 0) {
    // (cumulative: what the barrier has made this thread see is visible to whoever sees the count, and the other way round)
    fence_gpu();
    const bool all = atomicAdd(p.arrived + span[0], 1) == span[1] - span[0];
    fence_gpu();
    if (all) p.arrived[span[0]] = 0;
    else span[0] = -1;
  }
  asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
  float4 *const scratch = reinterpret_cast<float4 *>(ring);   // (nothing in the slots is needed any more)
#pragma unroll 1
  for (int o = 0; o < 2; ++o) {
    const int c0 = flag[2 * o], c1 = flag[2 * o + 1];
    if ((o == 0 ? !enters : open < 0) || c0 < 0) continue;
    // ---- this CTA is the last one: the partial tiles of all, in the order of the list
    const Frag f = frags[o == 0 ? 0 : 2 * open + 1];
    const Seq s = load_seq<kRows>(p, f.seq, false);
    const int head = f.unit / s.tiles, first_row = (f.unit - head * s.tiles) * kRows, rows = min(kRows, s.rows * p.group - first_row);
    // an item is four channels of a row; where there are fewer than threads, several threads take every `split`-th partial tile each
    const int items = rows * (kHd / 4), split = max(1, kConsumers / items);
#pragma unroll 1
    for (int i = threadIdx.x; i < items * split; i += kConsumers) {
      const int item = i % items, row = item / (kHd / 4), ch = 4 * (item % (kHd / 4));
      float m = kNone, l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      constexpr int kAhead = 8;                      // loads in flight
      for (int k = c0 + i / items; k <= c1; k += kAhead * split) {
        float4 x[kAhead];
        float2 ml[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int kk = k + u * split;
          const float *const from = p.partials + (long long)(2 * kk + (kk == c0)) * C::kPartial;
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
      if (split == 1) store_row4<kHd>(p, row_at<kHd>(p, s.row, head, first_row + row), ch, a, m, l);
      else scratch[2 * i] = a, scratch[2 * i + 1] = make_float4(m, l, 0.f, 0.f);
    }
    if (split == 1) continue;
    asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
    for (int i = threadIdx.x; i < items; i += kConsumers) {
      float m = kNone, l = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int u = 0; u < split; ++u) join(a, m, l, scratch[2 * (u * items + i)], scratch[2 * (u * items + i) + 1].x, scratch[2 * (u * items + i) + 1].y);
      store_row4<kHd>(p, row_at<kHd>(p, s.row, head, first_row + i / (kHd / 4)), 4 * (i % (kHd / 4)), a, m, l);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");   // the scratch is free again
  }
}

template <int kHd, int kBits, int kTiles, int kWarps>
int launch_pass(rosaq_ctx *ctx, AtParams p, cudaStream_t s) {
  using C = Cfg<kHd, kBits, kTiles, kWarps>;
  static_assert(C::kSmem <= 227 * 1024, "shared memory of an SM");
  static_assert(2 * 16 * 32 <= C::kDepth * C::kStageBytes, "scratch of a merged tile");
  auto *const kern = attend_kernel<kHd, kBits, kTiles, kWarps>;
  int &per_sm = ctx->at_per_sm[(kHd == 64) + 2 * (kBits == 8) + 4 * (kTiles / 2)];
  if (per_sm == 0) {
    int n = 0;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, C::kThreads, C::kSmem) != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      return ROSAQ_ERR_CUDA;
    }
    per_sm = n;
  }
  const int ctas = std::min(per_sm * ctx->sm_count, kAtMaxCtas);
  const int st = grow_workspace(ctx, reinterpret_cast<void **>(&ctx->at_partials), &ctx->at_partial_bytes, (size_t)(ctas * C::kWorkBytes));
  if (st != ROSAQ_OK) return st;
  p.partials = ctx->at_partials;
  return kv_launch(kern, dim3(ctas), C::kThreads, C::kSmem, s, p);
}

#ifndef W1
#define W1 8
#endif
#ifndef W2
#define W2 5
#endif
#ifndef W4
#define W4 6
#endif
template <int kHd, int kBits>
int launch_rows_pass(rosaq_ctx *ctx, const AtParams &p, long long rows_of_seq, cudaStream_t s) {
  if (rows_of_seq <= 8) return launch_pass<kHd, kBits, 1, kBits == 4 ? W1 : W8>(ctx, p, s);
  if (rows_of_seq <= 16) return launch_pass<kHd, kBits, 2, W2>(ctx, p, s);
  return launch_pass<kHd, kBits, 4, W4>(ctx, p, s);
}

int launch_any(rosaq_ctx *ctx, int hd, int bits, const AtParams &p, long long rows_of_seq, cudaStream_t s) {
  if (hd == 128) return bits == 4 ? launch_rows_pass<128, 4>(ctx, p, rows_of_seq, s) : launch_rows_pass<128, 8>(ctx, p, rows_of_seq, s);
  return bits == 4 ? launch_rows_pass<64, 4>(ctx, p, rows_of_seq, s) : launch_rows_pass<64, 8>(ctx, p, rows_of_seq, s);
}

}  // namespace

int launch_attend(rosaq_ctx *ctx, const KvView &kv, int hd, int bits, const KvBatchView &b, const int32_t *prefix_table, int prefix_tokens,
                  const __half *q, long long ldq, int n_q_heads, float scale, __half *out, long long ldo, cudaStream_t s) {
  AtParams p{};
  p.kv = kv, p.b = b, p.q = q, p.out = out, p.ldq = ldq, p.ldo = ldo, p.group = n_q_heads / kv.n_heads;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = ctx->d_status, p.wait_limit = ctx->wait_limit;
  const size_t prefix_bytes = prefix_tokens > 0 ? (size_t)b.n_rows * n_q_heads * (hd + 4) * sizeof(float) : 0;
  int st = ROSAQ_OK;
  if (prefix_bytes) st = grow_workspace(ctx, reinterpret_cast<void **>(&ctx->at_prefix), &ctx->at_prefix_bytes, prefix_bytes);
  if (st != ROSAQ_OK) return st;
  p.arrived = ctx->at_arrived;
  const long long rows_of_seq = ((long long)b.n_rows + b.n_seqs - 1) / b.n_seqs * p.group;
  if (prefix_tokens > 0) {
    p.prefix = ctx->at_prefix;
    AtParams f = p;
    f.prefix_tokens = prefix_tokens, f.last_row = b.n_seqs;
    f.b.n_seqs = 1, f.b.table = prefix_table;
    f.b.ld_table = (int)(((long long)prefix_tokens + (kKvBlock << kv.page_shift) - 1) / (kKvBlock << kv.page_shift));
    st = launch_any(ctx, hd, bits, f, (long long)b.n_rows * p.group, s);
    if (st != ROSAQ_OK) return st;
  }
  return launch_any(ctx, hd, bits, p, rows_of_seq, s);
}

}  // namespace rosaq
