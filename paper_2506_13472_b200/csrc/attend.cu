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
// device, so a captured launch follows them.  A producer warp copies blocks into a ring (one lane per slot), the other warps take them in turn.
// A tile whose blocks several CTAs share is finished by the CTA that arrives last, in the order of the shares: no CTA waits for another, and the
// bits are the same every time.
#include <algorithm>

#include "kv_common.cuh"

namespace rosaq {
namespace {

constexpr float kNone = -1e30f;                     // running maximum of a row that has seen nothing
constexpr float kGrow = 8.f;                        // a maximum is renewed when it is exceeded by this factor of two

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
  float *prefix;                                    // [row][q head][head_dim + 2]: what the prefix launch found; or nullptr
  int *status;
  long long wait_limit;
};

struct Seq {
  int row, rows, len, blocks, tiles;
  long long cost;                                   // (head, tile, block) triples; one per tile at least, so that every row is written
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
  s.blocks = (s.len + kKvBlock - 1) / kKvBlock;
  s.tiles = (int)(((long long)s.rows * p.group + kRows - 1) / kRows);
  s.cost = (long long)s.tiles * p.kv.n_heads * max(s.blocks, 1);
  return s;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
// A fragment of step j of a block of keys (token, channel): code * 2^-24, of the upper nibbles (channels 8-15) code * 2^-20
template <int kBits>
__device__ __forceinline__ void key_fragment(const uint32_t *w, int j, uint32_t *a) {
  if (kBits == 4) {
    const uint32_t u = w[j], v = u >> 8;
    a[0] = u & 0x000f000fu, a[2] = u & 0x00f000f0u, a[1] = v & 0x000f000fu, a[3] = v & 0x00f000f0u;
  } else {
    const uint32_t u = w[2 * j], v = w[2 * j + 1];
    a[0] = __byte_perm(u, 0, 0x4140), a[1] = __byte_perm(v, 0, 0x4140), a[2] = __byte_perm(u, 0, 0x4342), a[3] = __byte_perm(v, 0, 0x4342);
  }
}
// of values (channel, token): code - 2^(bits - 1), by way of 1024 + code (upper nibbles: 1024 + 16 code)
__device__ __forceinline__ uint32_t h2_fma(uint32_t v, uint32_t mul, uint32_t add) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&mul), *reinterpret_cast<const __half2 *>(&add));
  return *reinterpret_cast<const uint32_t *>(&r);
}
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
  static constexpr int kStages = kBits == 4 ? (kTiles == 1 && kWarps <= 4 ? 16 : 32) : (kWarps <= 4 ? 8 : 16);
  static constexpr int kBlockBytes = kv_block_bytes(kHd, kBits);
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kAccLd = kHd + 4;            // floats: rows of the accumulators of a warp, two rows of a pair on different banks
  static constexpr int kSumBytes = kWarps * kRows * 4 * 4;
  static constexpr int kBarBytes = 2 * kStages * 8;
  static constexpr int kSmem = kStages * kBlockBytes + kWarps * kRows * kAccLd * 4 + kSumBytes + kBarBytes + 64;
  static constexpr int kPartial = kRows * (kHd + 2);   // floats of a partial tile
  static constexpr int kLeast = 2 * kWarps;         // blocks that make a CTA of its own worth while
};

// Adds the partial tiles of a tile of query rows and writes the rows (or, in a prefix launch, the sums of the prefix).
// acc(i, row, channel) / sum(i, row): i-th partial; n of them.
template <int kHd>
__device__ __forceinline__ void store_row4(const AtParams &p, int row, int qhead, int n_q_heads, int ch, float4 a, float m, float l) {
  if (p.prefix_tokens > 0) {
    float *const to = p.prefix + ((long long)row * n_q_heads + qhead) * (kHd + 2);
    *reinterpret_cast<float2 *>(to + ch) = make_float2(a.x, a.y);
    *reinterpret_cast<float2 *>(to + ch + 2) = make_float2(a.z, a.w);
    if (ch == 0) *reinterpret_cast<float2 *>(to + kHd) = make_float2(m, l);
    return;
  }
  if (p.prefix) {
    const float *const from = p.prefix + ((long long)row * n_q_heads + qhead) * (kHd + 2);
    const float2 x = *reinterpret_cast<const float2 *>(from + ch), y = *reinterpret_cast<const float2 *>(from + ch + 2);
    const float2 ml = *reinterpret_cast<const float2 *>(from + kHd);
    const float mm = fmaxf(m, ml.x), f = ex2(m - mm), g = ex2(ml.x - mm);
    a = make_float4(a.x * f + x.x * g, a.y * f + x.y * g, a.z * f + y.x * g, a.w * f + y.y * g);
    l = l * f + ml.y * g;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;        // no token: zeros
  uint2 h;
  h.x = pack_h2(a.x * inv, a.y * inv), h.y = pack_h2(a.z * inv, a.w * inv);
  *reinterpret_cast<uint2 *>(p.out + (long long)row * p.ldo + (long long)qhead * kHd + ch) = h;
}

template <int kHd, int kBits, int kTiles, int kWarps>
__global__ void __launch_bounds__(32 * (kWarps + 1)) attend_kernel(const __grid_constant__ AtParams p) {
  using C = Cfg<kHd, kBits, kTiles, kWarps>;
  constexpr int kSteps = kHd / 16, kWords = kSteps * (kBits / 4), kRows = C::kRows, kConsumers = 32 * kWarps;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t *const ring = smem;
  float *const accs = reinterpret_cast<float *>(smem + C::kStages * C::kBlockBytes);      // [warp][row][kAccLd]
  float4 *const sums = reinterpret_cast<float4 *>(accs + kWarps * kRows * C::kAccLd);     // [warp][row]: maximum, sum, sum of least values
  uint64_t *const bars = reinterpret_cast<uint64_t *>(sums + kWarps * kRows);
  long long *const scan = reinterpret_cast<long long *>(bars + 2 * C::kStages);           // total cost; then flags
  int *const flag = reinterpret_cast<int *>(scan + 1);
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * C::kStages;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(full0 + 8 * i, 1), mbar_init(empty0 + 8 * i, 1);
    mbar_init_fence();
    scan[0] = 0;
    flag[1] = 0;
  }
  grid_dep_launch_dependents();
  __syncthreads();
  grid_dep_wait();                                  // q, the batch, the pages, the partial tiles: all may be the previous kernel's

  // ---- the share of this CTA
  long long mine = 0;
  for (int i = threadIdx.x; i < p.b.n_seqs; i += C::kThreads) mine += load_seq<kRows>(p, i, blockIdx.x == 0).cost;
  if (mine) atomicAdd(reinterpret_cast<unsigned long long *>(scan), (unsigned long long)mine);
  __syncthreads();
  const long long total = scan[0];
  const int ctas = (int)max(1ll, min((long long)gridDim.x, total / C::kLeast)), cta = blockIdx.x;
  if (cta >= ctas || total == 0) return;
  const long long begin = total * cta / ctas, end = total * (cta + 1) / ctas;
  // the sequence that holds `begin`
  int seq0 = 0;
  long long seq0_at = 0;
  {
    long long base = 0;
    for (int i = 0; i < p.b.n_seqs; i += 32) {
      long long c = i + lane < p.b.n_seqs ? load_seq<kRows>(p, i + lane, false).cost : 0, sum = c;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const long long o = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += o;
      }
      const unsigned past = __ballot_sync(0xffffffffu, base + sum > begin);
      if (past) {
        const int k = __ffs(past) - 1;
        seq0 = i + k;
        seq0_at = base + __shfl_sync(0xffffffffu, sum - c, k);
        break;
      }
      base += __shfl_sync(0xffffffffu, sum, 31);
    }
  }
  const int n = (int)(end - begin);                 // blocks of this CTA (a share of 2^31 would be 4 TB of cache)

  if (warp == kWarps) {
    // ---- producer: lane i owns slot i and brings blocks i, i + kStages, ...
    if (lane < C::kStages) {
      int seq = seq0;
      long long at = seq0_at;
      Seq s = load_seq<kRows>(p, seq, false);
      uint32_t parity = 1;                           // of the phase that frees the slot; the other one's end brings its block
      uint32_t filled = 0;                           // parity of the last fill
      bool copied = false;
      const uint64_t keep = policy_evict_first();
      for (int j = lane; j < n; j += C::kStages, parity ^= 1) {
        while (begin + j >= at + s.cost) at += s.cost, s = load_seq<kRows>(p, ++seq, false);
        const int per = max(s.blocks, 1);
        const long long in = begin + j - at;
        const int unit = (int)(in / per), block = (int)(in - (long long)unit * per), head = unit / s.tiles;
        const uint8_t *src = nullptr;
        if (s.blocks > 0) {
          int page = kv_page(p.kv, p.b, seq, block);
          if (page < 0) kv_report(p.status), page = 0;   // (a page of the cache all the same)
          src = p.kv.pages + kv_offset(p.kv, page, block, C::kBlockBytes) + ((long long)head << p.kv.page_shift) * C::kBlockBytes;
        }
        bool free = mbar_test_wait(empty0 + 8 * lane, parity);
        for (long long i = 0; !free && i < p.wait_limit; ++i) {
          __nanosleep(100);
          free = mbar_test_wait(empty0 + 8 * lane, parity);
        }
        if (!free) {                                 // the consumers give up too, one wait each
          atomicExch(p.status, (int)ROSAQ_ERR_TIMEOUT);
          break;
        }
        copied = true, filled = parity ^ 1;
        if (src) {
          mbar_arrive_expect_tx(full0 + 8 * lane, C::kBlockBytes);
          bulk_copy_g2s_hint(smem_u32(ring + lane * C::kBlockBytes), src, C::kBlockBytes, full0 + 8 * lane, keep);
        } else {
          mbar_arrive(full0 + 8 * lane);
        }
      }
      // the CTA outlasts its copies, also when the consumers have given up on them
      if (copied)
        for (int i = 0; i < 1 << 20 && !mbar_test_wait(full0 + 8 * lane, filled); ++i) __nanosleep(100);
    }
    return;
  }

  // ---- consumers: warp w takes blocks w, w + kWarps, ... of the CTA's share, whichever tile they belong to
  const int r = lane >> 2, c = lane & 3;
  const int n_q_heads = p.kv.n_heads * p.group;
  int seq = seq0;
  long long at = seq0_at;
  Seq s = load_seq<kRows>(p, seq, false);
  bool lost = false;
  for (int j0 = 0; j0 < n;) {
    while (begin + j0 >= at + s.cost) at += s.cost, s = load_seq<kRows>(p, ++seq, false);
    const int per = max(s.blocks, 1);
    const long long in = begin + j0 - at;
    const int unit = (int)(in / per), block0 = (int)(in - (long long)unit * per);
    const int head = unit / s.tiles, tile = unit - head * s.tiles;
    const int j1 = (int)min((long long)n, (long long)j0 + per - block0);   // the blocks [j0, j1) are this tile's
    const long long first_row = (long long)tile * kRows, n_flat = (long long)s.rows * p.group;

    // ---- query rows of the tile: B fragments, scaled by a power of two per row so that the greatest value lies in [2^12, 2^13); of
    // the channels whose nibbles read sixteen times too large a sixteenth.  A row that is not finite is left as it is.
    uint32_t qf[kTiles][kSteps][2];
    float row_a[2 * kTiles], row_b[2 * kTiles];      // of this lane's columns 2 c, 2 c + 1 of each tile of eight rows
    int lim[2 * kTiles];                             // tokens that the row sees
    const int seen0 = s.len - s.rows + 1;            // by the first row of the sequence
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const long long flat = first_row + 8 * t + r;
      const bool valid = flat < n_flat;
      const int tok = valid ? (int)(flat / p.group) : 0, qh = head * p.group + (valid ? (int)(flat - (long long)tok * p.group) : 0);
      const __half *const src = p.q + (long long)(s.row + tok) * p.ldq + (long long)qh * kHd + 2 * c;
      float most = 0.f, sum = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          qf[t][k][h] = valid ? *reinterpret_cast<const uint32_t *>(src + 16 * k + 8 * h) : 0u;
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&qf[t][k][h]));
          most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
          sum += f.x + f.y;
        }
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1)), most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      sum += __shfl_xor_sync(0xffffffffu, sum, 1), sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      int up = 12 - ((int)(__float_as_uint(most) >> 23) - 127);          // (fp16 values: never an fp32 subnormal)
      if (!(most > 0.f) || most > 65504.f) up = 0;
      const float f0 = __uint_as_float((uint32_t)(127 + up) << 23), f1 = kBits == 4 ? f0 * 0.0625f : f0;
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&qf[t][k][h]));
          qf[t][k][h] = pack_h2(f.x * (h ? f1 : f0), f.y * (h ? f1 : f0));
        }
      const float a = p.scale_log2 * __uint_as_float((uint32_t)(127 + 24 - up) << 23), b = p.scale_log2 * sum;
      const int seen = p.prefix_tokens > 0 ? s.len : valid ? min(max(seen0 + tok, 0), s.len) : s.len;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        row_a[2 * t + e] = __shfl_sync(0xffffffffu, a, 4 * (2 * c + e));
        row_b[2 * t + e] = __shfl_sync(0xffffffffu, b, 4 * (2 * c + e));
        lim[2 * t + e] = __shfl_sync(0xffffffffu, seen, 4 * (2 * c + e));
      }
    }
    int least = s.len, most_seen = s.len;            // tokens that every row, that any row of the tile sees
    if (p.prefix_tokens == 0) {
      const int t0 = (int)(first_row / p.group), t1 = (int)((min(first_row + kRows, n_flat) - 1) / p.group);
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

    // ---- this warp's blocks
    int j = j0 + ((warp - j0) % kWarps + kWarps) % kWarps;
    for (; j < j1; j += kWarps) {
      const int slot = j % C::kStages;
      const uint32_t parity = (j / C::kStages) & 1, base = smem_u32(ring + slot * C::kBlockBytes);
      if (!lost) {
        bool here = mbar_try_wait(full0 + 8 * slot, parity);
        for (long long i = 0; !here && i < p.wait_limit; ++i) here = mbar_try_wait(full0 + 8 * slot, parity);
        lost = !__all_sync(0xffffffffu, here);
        if (lost && lane == 0) atomicExch(p.status, (int)ROSAQ_ERR_TIMEOUT);
      }
      if (lost) continue;                            // (waits once; the barriers and counters below are still served)
      const int tok0 = (block0 + j - j0) * kKvBlock;
      if (tok0 < most_seen) {
        // scores
        float sc[kTiles][4];
        {
          uint32_t w[kWords];
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint4 v = lds128(base + 512 * i + 16 * lane);
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
          }
          float alt[kTiles][4];
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][e] = alt[t][e] = 0.f;
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            uint32_t a[4];
            key_fragment<kBits>(w, k, a);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) mma16816(k & 1 ? alt[t] : sc[t], a[0], a[1], a[2], a[3], qf[t][k][0], qf[t][k][1]);
          }
#pragma unroll
          for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][e] += alt[t][e];
        }
        // pairs (scale, least value) of tokens r and r + 8
        constexpr int kPairs = 2 * kv_code_bytes(kHd, kBits);
        float ks[2], kl[2], vm[2], vi[2], vl[2], ve[2];
        const bool border = tok0 + kKvBlock > least;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t kp = lds32(base + kPairs + 4 * r + 32 * h), vp = lds32(base + kPairs + 64 + 4 * r + 32 * h);
          if (border && tok0 + r + 8 * h >= most_seen) kp = vp = 0x00000001u;   // whatever lies behind the last token
          const float2 kf = __half22float2(*reinterpret_cast<__half2 *>(&kp)), vf = __half22float2(*reinterpret_cast<__half2 *>(&vp));
          const uint32_t bits = __float_as_uint(vf.x), expo = bits >> 23;
          ks[h] = kf.x, kl[h] = kf.y;
          vm[h] = __uint_as_float((bits & 0x007fffffu) | 0x3f800000u);   // s 2^-e
          vi[h] = __uint_as_float((254u - expo) << 23);                  // 2^-e
          vl[h] = __fmaf_rn(vf.y, vi[h], vm[h] * (kBits == 4 ? 8.f : 128.f));   // (lo + s 2^(bits - 1)) 2^-e
          ve[h] = (float)((int)expo - 127);
        }
        float most = 0.f;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 2 * t + (e & 1), h = e >> 1;
            sc[t][e] = __fmaf_rn(sc[t][e], row_a[i] * ks[h], __fmaf_rn(row_b[i], kl[h], ve[h]));
            if (border && tok0 + r + 8 * h >= lim[i]) sc[t][e] = -INFINITY;
            most = fmaxf(most, sc[t][e] - top[i]);
          }
        if (__any_sync(0xffffffffu, most > kGrow)) {
#pragma unroll
          for (int i = 0; i < 2 * kTiles; ++i) {
            float m = fmaxf(sc[i >> 1][i & 1], sc[i >> 1][(i & 1) + 2]);
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4)), m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)), top[i]);
            const float f = ex2(top[i] - m);
            top[i] = m, den[i] *= f, off[i] *= f;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) acc[k][i >> 1][i & 1] *= f, acc[k][i >> 1][(i & 1) + 2] *= f;
          }
        }
        uint32_t pf[kTiles][2];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 2 * t + (e & 1), h = e >> 1;
            const float x = ex2(sc[t][e] - top[i]);
            den[i] = __fmaf_rn(x, vi[h], den[i]);
            off[i] = __fmaf_rn(x, vl[h], off[i]);
            sc[t][e] = x * vm[h];
          }
          pf[t][0] = transpose8(pack_h2(sc[t][0], sc[t][1])), pf[t][1] = transpose8(pack_h2(sc[t][2], sc[t][3]));
        }
        {
          uint32_t w[kWords];
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint4 v = lds128(base + kv_code_bytes(kHd, kBits) + 512 * i + 16 * lane);
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
          }
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            uint32_t a[4];
            value_fragment<kBits>(w, k, a);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) mma16816(acc[k][t], a[0], a[1], a[2], a[3], pf[t][0], pf[t][1]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty0 + 8 * slot);
    }

    // ---- the warps' sums together
#pragma unroll
    for (int i = 0; i < 2 * kTiles; ++i) {
#pragma unroll
      for (int d = 4; d < 32; d *= 2) den[i] += __shfl_xor_sync(0xffffffffu, den[i], d), off[i] += __shfl_xor_sync(0xffffffffu, off[i], d);
      const int row = 8 * (i >> 1) + 2 * c + (i & 1);
      if (r == 0) sums[warp * kRows + row] = make_float4(top[i], den[i], off[i], 0.f);
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        float *const to = accs + (warp * kRows + row) * C::kAccLd + 16 * k + r;
        to[0] = acc[k][i >> 1][i & 1];
        to[8] = acc[k][i >> 1][(i & 1) + 2];
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
    const int rows = (int)min((long long)kRows, n_flat - first_row);
    const bool whole = block0 == 0 && j1 - j0 == per;
    float *const slot = p.partials + (long long)(2 * cta + (block0 == 0 ? 1 : 0)) * C::kPartial;
    for (int i = threadIdx.x; i < rows * (kHd / 4); i += kConsumers) {
      const int row = i / (kHd / 4), ch = 4 * (i % (kHd / 4));
      float m = kNone;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) m = fmaxf(m, sums[w * kRows + row].x);
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f, o = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 u = sums[w * kRows + row];
        const float f = ex2(u.x - m);
        const float4 v = *reinterpret_cast<const float4 *>(accs + (w * kRows + row) * C::kAccLd + ch);
        a.x += f * v.x, a.y += f * v.y, a.z += f * v.z, a.w += f * v.w;
        l += f * u.y, o += f * u.z;
      }
      a.x += o, a.y += o, a.z += o, a.w += o;
      if (whole) {
        const long long flat = first_row + row;
        const int tok = (int)(flat / p.group), qh = head * p.group + (int)(flat - (long long)tok * p.group);
        store_row4<kHd>(p, s.row + tok, qh, n_q_heads, ch, a, m, l);
      } else {
        float *const to = slot + row * (kHd + 2);
        *reinterpret_cast<float2 *>(to + ch) = make_float2(a.x, a.y);
        *reinterpret_cast<float2 *>(to + ch + 2) = make_float2(a.z, a.w);
        if (ch == 0) *reinterpret_cast<float2 *>(to + kHd) = make_float2(m, l);
      }
    }
    if (!whole) {
      // the CTAs that hold blocks [unit0, unit0 + per) of the list
      const long long unit0 = at + (long long)unit * per;
      const int c0 = (int)(((unit0 + 1) * ctas + total - 1) / total) - 1, c1 = (int)(((unit0 + per) * ctas + total - 1) / total) - 1;
      __threadfence();
      asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
      if (threadIdx.x == 0) {
        const bool last = atomicAdd(p.arrived + c0, 1) == c1 - c0;
        if (last) p.arrived[c0] = 0;
        flag[1] = last;
      }
      asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
      if (flag[1]) {
        __threadfence();
        for (int i = threadIdx.x; i < rows * (kHd / 4); i += kConsumers) {
          const int row = i / (kHd / 4), ch = 4 * (i % (kHd / 4));
          const float *const from = p.partials + (long long)row * (kHd + 2);
          float m = kNone, l = 0.f;
          float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int k = c0; k <= c1; ++k) m = fmaxf(m, __ldcg(from + (long long)(2 * k + (k == c0)) * C::kPartial + kHd));
#pragma unroll 4
          for (int k = c0; k <= c1; ++k) {
            const float *const x = from + (long long)(2 * k + (k == c0)) * C::kPartial;
            const float2 u = __ldcg(reinterpret_cast<const float2 *>(x + ch)), v = __ldcg(reinterpret_cast<const float2 *>(x + ch + 2));
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(x + kHd));
            const float f = ex2(ml.x - m);
            a.x += f * u.x, a.y += f * u.y, a.z += f * v.x, a.w += f * v.y, l += f * ml.y;
          }
          const long long flat = first_row + row;
          const int tok = (int)(flat / p.group), qh = head * p.group + (int)(flat - (long long)tok * p.group);
          store_row4<kHd>(p, s.row + tok, qh, n_q_heads, ch, a, m, l);
        }
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");   // the sums are free again
    j0 = j1;
  }
}

template <int kHd, int kBits, int kTiles, int kWarps>
int launch_pass(rosaq_ctx *ctx, AtParams p, cudaStream_t s) {
  using C = Cfg<kHd, kBits, kTiles, kWarps>;
  static_assert(C::kSmem <= 227 * 1024, "shared memory of an SM");
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
  const int st = grow_workspace(ctx, reinterpret_cast<void **>(&ctx->at_partials), &ctx->at_partial_bytes, (size_t)2 * ctas * C::kPartial * sizeof(float));
  if (st != ROSAQ_OK) return st;
  p.partials = ctx->at_partials;
  return kv_launch(kern, dim3(ctas), C::kThreads, C::kSmem, s, p);
}

template <int kHd, int kBits>
int launch_rows_pass(rosaq_ctx *ctx, const AtParams &p, long long rows_of_seq, cudaStream_t s) {
  if (rows_of_seq <= 8) return launch_pass<kHd, kBits, 1, 4>(ctx, p, s);
  if (rows_of_seq <= 16) return launch_pass<kHd, kBits, 2, 4>(ctx, p, s);
  return launch_pass<kHd, kBits, 4, 4>(ctx, p, s);
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
  const size_t prefix_bytes = prefix_tokens > 0 ? (size_t)b.n_rows * n_q_heads * (hd + 2) * sizeof(float) : 0;
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
