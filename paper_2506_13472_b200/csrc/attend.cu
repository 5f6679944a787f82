// rosaq_attend: softmax(scale q k^T) v of new rows over the quantized paged cache, with an optional prefix shared by all sequences.
//
// With k = lo_k + s_k c and v = lo_v + s_v d (codes c, d; one pair (s, lo) per token) the sums split into products of codes and sums over tokens:
//   q . k = s_k (q . c) + lo_k sum(q),      sum_t p_t v_t = sum_t (p_t s_t) d_t + sum_t p_t lo_t.
// So no key is dequantised: nibbles and bytes, masked out of their words, ARE fp16 numbers (subnormal: code * 2^-24), exact operands of the
// tensor core.  Value codes are taken about the middle of their range, d_t - 10 or d_t - 128, which costs an addition per pair and keeps the sums as small as
// the result: of positive codes the roundings of the weights and of the accumulators would all point one way (against 64 bits, 26000 tokens
// at 8 bits: 1.2e-3 that way).  The weights of the second product keep their size whatever that of the values: u_t = score_t log2(e) + log2(s_t) is what the
// running maximum is taken of, so that p_t s_t has its greatest value between 2^10 and 2^15 and is cut to 11 bits, an fp16 number (2^-35 of
// the greatest weight absolute), while sum(p_t) and sum(p_t lo_t) are in fp32, of the same weights.
//
// Tokens are the rows of the first MMA (m16n8k16: 16 tokens x 8 query rows) and the k of the second one (16 channels x 8 query rows), so a group of
// up to eight query heads costs no more than one, and a lane's words of a block (kv_common.cuh) are its A fragments in both.
//
// Bound: memory for one row per sequence and long contexts at 8 bits (16 sequences of 20000 to 32767 tokens, 8 heads of 128: 0.93 of the copy bandwidth); at 4 bits the instructions, about 484 per pair
// of blocks of 16 tokens and one key/value head (4352 bytes, head of 128), of which a scheduler issues one in two cycles: 64 x 2250 tokens, 32 heads, take 133 us, 119 without the
// arithmetic, 95 at the copy bandwidth.  With one query head per key/value head seven of an MMA's eight columns are empty, and half of the softmax's instructions work on a column that always is.
// Short calls are bound by latency: 5.7 us for one chunk, 1.0 to 1.3 us per further chunk of a warp, 5 us to join CTAs.
// The list of (sequence, head, tile of query rows, chunk) is cut into equal shares, one per CTA, whatever the lengths: CTAs read lengths on the device, so a captured launch
// follows them.  A CTA's share is cut into one run per warp, each with slots of its own, all filled by one more warp, a lane per slot (warps that fill their own: 153 to 168 us
// instead of 152).  A tile whose chunks several CTAs share is finished by the CTA that arrives last, in the order of the shares: no CTA waits for another, and the bits are the
// same every time.
#include <algorithm>

#include "attend_common.cuh"

namespace rosaq {
namespace {

constexpr int kChunk = 2, kTokens = kChunk * kKvBlock;   // blocks that a warp takes at a time
constexpr int kRows = 8;                            // query rows of a tile
// From kManyRows query rows per sequence and key/value head on, and from kManyWork of (row, key/value head, token that the table has room for) in all: attend_rows.cu, which takes 10 us
// more for any call and a third to a half of the time per row and token.  (us here and there, 32 query and 8 key/value heads of 128 at 4 bits: 32 rows of each of 16 sequences of 1000
// tokens 34 and 36, 64 rows 47 and 38; of one sequence of 500 tokens 64 rows 12 and 24; of 4000 tokens 64 rows 26 and 25, 128 rows 33 and 26; of 30000 tokens 64 rows 67 and 52;
// 128 rows behind a prefix of 500 tokens 20 and 32, of 4000 40 and 35, of 16000 77 and 47.)
constexpr long long kManyRows = 64, kManyWork = 1ll << 22;
// Greatest wait limit.  A warp that gives up leaves others to give up by themselves, so every wait has to end in a time that somebody can wait for; and some poll 32 times as often.
constexpr long long kMostPolls = 1ll << 24;

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
// A fragment of step j of a block, keys (token, channel) or values (channel, token), in units of 2^-24: the codes; at four bits sixteen times the codes of the second nibbles, which
// are channels 8-15.  (Values: whole bytes in the rows of channels 0-7, what is too much taken off at the end, are an operation less per word; but what the accumulators cut off
// is relative to the sixteenfold sum then: 131071 tokens 3.5e-4 off, 3.2e-4 so.)
template <int kBits, bool kValue>
__device__ __forceinline__ void code_fragment(const uint32_t *w, int j, uint32_t *a) {
  if (kBits == 4) {
    const uint32_t u = w[j], v = u >> 8;
    const uint32_t a1 = u & 0x00f000f0u, a2 = v & 0x000f000fu;
    a[0] = u & 0x000f000fu, a[1] = kValue ? a1 : a2, a[2] = kValue ? a2 : a1, a[3] = v & 0x00f000f0u;
  } else {
    const uint32_t u = w[2 * j], v = w[2 * j + 1];
    a[0] = __byte_perm(u, 0, 0x4140), a[1] = __byte_perm(v, 0, 0x4140), a[2] = __byte_perm(u, 0, 0x4342), a[3] = __byte_perm(v, 0, 0x4342);
  }
}

template <int kHd, int kBits, int kWarps>
struct Cfg {
  static constexpr int kStageBytes = kChunk * kv_block_bytes(kHd, kBits);
  static constexpr int kThreads = 32 * (kWarps + 1);
  // Two CTAs on an SM: at 4 bits 14 warps with 128 registers, at 8 bits ten with two slots each.  More warps with fewer registers that compute one block at a time are slower:
  // 64 x 2250 tokens 141 us when this was measured, 20 warps with 96 registers 157, 24 with 80 183 to 197.  (The instance of heads of 128 at 4 bits needs a little more than 128: by
  // -Xptxas -v it spills 8 bytes and loads 20.)
  static constexpr int kPerSm = 2;
  static constexpr int kAccLd = kHd + 4;            // floats: two rows of a pair on different banks
  static constexpr int kPartBytes = kRows * (4 * kAccLd + 16);   // a part of a tile: [row][kAccLd], then [row]{maximum, sum, sum of least values, -}
  static constexpr int kPairBytes = kTokens * 20 + kRows * 4;   // of a warp: what its tokens' pairs become, and what brings the scores of rows back that were scaled by themselves
  static constexpr int kFixed = kPairBytes + 2 * (int)sizeof(OpenTile) + 16;   // of a warp, besides its slots
  static constexpr int kRoom = 222 * 1024 / kPerSm - 1024 - 128 - (kFixed + 64) * kWarps;
  static constexpr int kDepth = kRoom / kStageBytes / kWarps < 32 / kWarps ? kRoom / kStageBytes / kWarps : 32 / kWarps;   // slots of a warp, next to each other
  static constexpr int kStages = kWarps * kDepth;
  static constexpr int kSmem = kStages * (kStageBytes + 16) + kFixed * kWarps + 128;
  static constexpr long long kWorkBytes = 2 * 4 * at_partial(kHd, kRows) + 2 * kWarps * kPartBytes;   // of a CTA: partial tiles, parts that the slots do not hold
  static_assert(kDepth >= 1 && kStages <= 32 && kStageBytes >= kPartBytes && kStageBytes >= 32 * 32, "slots");
};

template <int kHd, int kBits, int kWarps>
__global__ void __launch_bounds__(32 * (kWarps + 1), Cfg<kHd, kBits, kWarps>::kPerSm) attend_kernel(const __grid_constant__ AtParams p) {
  using C = Cfg<kHd, kBits, kWarps>;
  constexpr int kSteps = kHd / 16, kWords = kSteps * (kBits / 4), kConsumers = 32 * kWarps;
  constexpr int kBlockBytes = kv_block_bytes(kHd, kBits);
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t *const ring = smem;                                                             // [warp][kDepth] slots
  float4 *const pair_terms = reinterpret_cast<float4 *>(smem + C::kStages * C::kStageBytes);   // [warp][token]{s_k', lo_k, log2 s_v, 1 / s_v}, [token] lo_v / s_v + middle, [row]
  uint64_t *const bars = reinterpret_cast<uint64_t *>(pair_terms + C::kPairBytes / 16 * kWarps);
  const float **const data = reinterpret_cast<const float **>(bars + 2 * C::kStages);     // [warp][2]: where the parts below lie
  OpenTile *const parts = reinterpret_cast<OpenTile *>(data + 2 * kWarps);                // [warp]{first part of a tile that began before, last one}
  OpenTile *const open = parts + 2 * kWarps;                                              // [2] tiles that other CTAs hold parts of too
  int *const span = reinterpret_cast<int *>(open + 2);
  // A warp's last part lies in its slots, which are free by then, an earlier one behind the partial tiles of all CTAs.
  uint8_t *const earlier = reinterpret_cast<uint8_t *>(p.partials + 2ll * gridDim.x * at_partial(kHd, kRows)) + (long long)blockIdx.x * 2 * kWarps * C::kPartBytes;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * C::kStages;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) mbar_init(full0 + 8 * i, 1), mbar_init(empty0 + 8 * i, 1);
    mbar_init_fence();
  }
  if (threadIdx.x < 2 * kWarps + 2) parts[threadIdx.x].from = kNoTile;
  grid_dep_launch_dependents();
  grid_dep_wait();                                  // q, the batch, the pages, the partial tiles: all may be the previous kernel's

  __shared__ Share share;                           // (by one warp: eight that compute the same take turns)
  if (warp == 0) find_share<kRows, kTokens>(p, blockIdx.x, gridDim.x, 8 * kWarps, kWarps, blockIdx.x == 0, share);
  __syncthreads();
  if (share.begin == share.end) return;
  Cursor cur = share.cur;
  const int n = (int)(share.end - share.begin);     // chunks of this CTA (a share of 2^31 would be 4 TB of cache)
  // warp w takes chunks [n w / kWarps, n (w + 1) / kWarps) of them, rounded up (warp 0 always has one): long runs, so that a warp seldom changes its tile and never waits for another
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
      settle<kRows, kTokens>(p, cur);
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
  float4 *const terms = pair_terms + warp * (C::kPairBytes / 16);
  float *const term_vl = reinterpret_cast<float *>(terms + kTokens), *const back = term_vl + kTokens;
  bool lost = false;
  int j = bound(warp);                               // this warp's next chunk
  const int last = bound(warp + 1);
  int slot = warp * C::kDepth;
  uint32_t parity = 0;
  cur.chunk += j;
  while (j < last) {
    settle<kRows, kTokens>(p, cur);
    const Seq &s = cur.s;
    const int head = cur.unit / s.tiles, tile = cur.unit - head * s.tiles, chunk0 = cur.chunk, j0 = j;
    const int j1 = min(last, j0 + s.chunks - chunk0);   // the chunks [j0, j1) are this tile's
    const int first_row = tile * kRows, n_flat = s.rows * p.group;

    // ---- query rows of the tile: B fragments, scaled by a power of two so that the greatest value of all rows lies in [2^12, 2^13); of the channels whose
    // nibbles read sixteen times too large a sixteenth.  Rows that are not finite do not count for it.  fp16 holds what is left of a row exactly down to 2^-16 of its greatest value, and
    // what lies below to 2^-27 of it, as long as that is no more than 2^kQuiet below the tile's; where one is, every row is scaled by itself, and its scores are brought back by a product.
    uint32_t qf[kSteps][2];
    float row_b[2];                                  // scale log2(e) sum(q) of this lane's columns 2 c, 2 c + 1
    int lim[2];                                      // tokens that the row sees
    const int seen0 = s.len - s.rows + 1;            // by the first row of the sequence
    const int flat = first_row + r;
    const bool valid = flat < n_flat;
    const int tok = valid ? flat / p.group : 0, qh = head * p.group + (valid ? flat - tok * p.group : 0);
    const __half *const src = p.q + (long long)(s.row + tok) * p.ldq + (long long)qh * kHd + 2 * c;
    float most_q = 0.f, sum = 0.f;
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) qf[k][h] = valid ? *reinterpret_cast<const uint32_t *>(src + 16 * k + 8 * h) : 0u;
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&qf[k][h]));
        most_q = fmaxf(most_q, fmaxf(fabsf(x.x), fabsf(x.y)));
        sum += x.x + x.y;
      }
    if (!(most_q <= 65504.f)) most_q = 0.f;
    most_q = fmaxf(most_q, __shfl_xor_sync(0xffffffffu, most_q, 1)), most_q = fmaxf(most_q, __shfl_xor_sync(0xffffffffu, most_q, 2));
    const float own_q = most_q;                      // of this lane's row
#pragma unroll
    for (int d = 16; d > 2; d /= 2) most_q = fmaxf(most_q, __shfl_xor_sync(0xffffffffu, most_q, d));
    sum += __shfl_xor_sync(0xffffffffu, sum, 1), sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    // (Infinities among the queries make all scores NaN: over keys of one sign they would all be minus infinity, and the row like one that sees nothing.)
    const float row_sum = isfinite(sum) ? p.scale_log2 * sum : NAN;
    const int seen = p.prefix_tokens > 0 || !valid ? s.len : min(max(seen0 + tok, 0), s.len);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      row_b[e] = __shfl_sync(0xffffffffu, row_sum, 4 * (2 * c + e));
      lim[e] = __shfl_sync(0xffffffffu, seen, 4 * (2 * c + e));
    }
    const int up = most_q > 0.f ? 12 - ((int)(__float_as_uint(most_q) >> 23) - 127) : 0;   // (fp16 values: never an fp32 subnormal)
    const float key_scale = p.scale_log2 * __uint_as_float((uint32_t)(127 + 24 - up) << 23);
    constexpr int kQuiet = 6;
    const int own_up = own_q > 0.f ? 12 - ((int)(__float_as_uint(own_q) >> 23) - 127) : up;
    const bool apart = __any_sync(0xffffffffu, own_up > up + kQuiet);
    const int row_up = apart ? own_up : up;
    if (apart && c == 0) back[r] = __uint_as_float((uint32_t)(127 + up - own_up) << 23);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float f = __uint_as_float((uint32_t)(127 + row_up - (kBits == 4 && h ? 4 : 0)) << 23);
        const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&qf[k][h]));
        qf[k][h] = pack_h2(x.x * f, x.y * f);
      }
    int least = s.len, most_seen = s.len;            // tokens that every row, that any row of the tile sees
    if (p.prefix_tokens == 0) {
      const int t0 = first_row / p.group, t1 = (min(first_row + kRows, n_flat) - 1) / p.group;
      least = min(max(seen0 + t0, 0), s.len), most_seen = min(max(seen0 + t1, 0), s.len);
    }

    float acc[kSteps][4], top[2], den[2], off[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) top[e] = kNone, den[e] = off[e] = 0.f;
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[k][e] = 0.f;
    // Value codes about the middle of their range: the sums of the weights, as the tensor core has them, times minus the middle gather in `low` (one MMA per block), and every
    // kFlush chunks they are added to the accumulators.
    constexpr int kFlush = 4;
    // (The tensor core cuts off the sums' last bits.  What it cuts off the codes' sums and off the middle's goes the other way, and cancels when the middle has about as many zeros at
    // its end as codes have: else all parts of a long context are off to one side.  131000 tokens at 4 bits: signed error -1.7e-4 with 8, +9e-5 with 7, below 3e-5 with 6 and 10.)
    constexpr float kMiddle = kBits == 4 ? 10.f : 128.f;
    constexpr uint32_t kLow = kBits == 4 ? 0x800a800au : 0x80808080u, kHigh = kBits == 4 ? 0x80a080a0u : 0x80808080u;   // minus that times 2^-24, and times 2^-20
    float low[4] = {0.f, 0.f, 0.f, 0.f};
    auto take_off = [&]() {
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] += low[e];
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
      const int tok0 = (chunk0 + j - j0) * kTokens;
      if (tok0 < most_seen) {
        {
          // what a token's pairs come to, one token per lane
          constexpr int kPairs = 2 * kv_code_bytes(kHd, kBits);
          const uint32_t at = base + (lane >> 4) * kBlockBytes + kPairs + 4 * (lane & 15);
          uint32_t kp = lds32(at), vp = lds32(at + 64);
          if (tok0 + lane >= most_seen) kp = vp = 0x00000001u;   // whatever lies behind the last token
          const float2 kf = __half22float2(*reinterpret_cast<__half2 *>(&kp)), vf = __half22float2(*reinterpret_cast<__half2 *>(&vp));
          const float lv = lg2(fmaxf(vf.x, kLeastScale)), vi = ex2(-lv);   // log2(s) and 1 / s as that has it
          terms[lane] = make_float4(kf.x * key_scale, kf.y, lv, vi);
          term_vl[lane] = __fmaf_rn(vf.y, vi, kMiddle);   // (lo + s middle) / s
          __syncwarp();
        }
        const uint32_t at = base + 16 * lane;
        // ---- scores.  A second block that is not there (or holds nothing that is seen) is computed from what lies in the slot and masked.
        float sc[kChunk][4];
#pragma unroll
        for (int b = 0; b < kChunk; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[b][e] = 0.f;
        constexpr int kPer = kBits == 4 ? 4 : 2;     // steps of a 16-byte chunk
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
          uint32_t w[kChunk][4];
#pragma unroll
          for (int b = 0; b < kChunk; ++b) {
            const uint4 v = lds128(at + b * kBlockBytes + 512 * i);
            w[b][0] = v.x, w[b][1] = v.y, w[b][2] = v.z, w[b][3] = v.w;
          }
#pragma unroll
          for (int e = 0; e < kPer; ++e)
#pragma unroll
            for (int b = 0; b < kChunk; ++b) {
              uint32_t a[4];
              code_fragment<kBits, false>(w[b], e, a);
              mma16816(sc[b], a, qf[kPer * i + e][0], qf[kPer * i + e][1]);
            }
        }
        if (apart) {
          const float2 f = *reinterpret_cast<const float2 *>(back + 2 * c);
#pragma unroll
          for (int b = 0; b < kChunk; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) sc[b][2 * h] *= f.x, sc[b][2 * h + 1] *= f.y;
        }
        // ---- u = score log2(e) + log2(s_v)
        float vi[kChunk][2], vl[kChunk][2];
#pragma unroll
        for (int b = 0; b < kChunk; ++b)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int tk = kKvBlock * b + 8 * h + r;
            const float4 x = terms[tk];
            vi[b][h] = x.w, vl[b][h] = term_vl[tk];
#pragma unroll
            for (int e = 0; e < 2; ++e) sc[b][2 * h + e] = __fmaf_rn(sc[b][2 * h + e], x.x, __fmaf_rn(row_b[e], x.y, x.z));
          }
        if (tok0 + kTokens > least) {
          // the border: tokens that a row does not see
#pragma unroll
          for (int b = 0; b < kChunk; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (tok0 + kKvBlock * b + 8 * (e >> 1) + r >= min(lim[e & 1], most_seen)) sc[b][e] = -INFINITY;
        }
        float most[2];
        bool grow = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          most[e] = fmaxf(fmaxf(sc[0][e], sc[0][e + 2]), fmaxf(sc[1][e], sc[1][e + 2]));
          grow |= most[e] > top[e] + kGrow;
        }
        if (__any_sync(0xffffffffu, grow)) {
          take_off();
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float m = most[e];
            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4)), m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
            m = fmaxf(fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16)) - kUp, top[e]);
            const float f = ex2(top[e] - m);
            top[e] = m, den[e] *= f, off[e] *= f;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) acc[k][e] *= f, acc[k][e + 2] *= f;
          }
        }
        // ---- weights p s_v, their sums, and the product with the value codes
        uint32_t pf[kChunk][2];
#pragma unroll
        for (int b = 0; b < kChunk; ++b) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 x = weights(sc[b][2 * h] - top[0], sc[b][2 * h + 1] - top[1]);
            den[0] = __fmaf_rn(x.x, vi[b][h], den[0]), den[1] = __fmaf_rn(x.y, vi[b][h], den[1]);
            off[0] = __fmaf_rn(x.x, vl[b][h], off[0]), off[1] = __fmaf_rn(x.y, vl[b][h], off[1]);
            pf[b][h] = transpose8(pack_h2(x.x, x.y));
          }
        }
        // minus the middle of the codes, as the fragments have them
        const uint32_t mid[4] = {kLow, kHigh, kLow, kHigh};
#pragma unroll
        for (int b = 0; b < kChunk; ++b) mma16816(low, mid, pf[b][0], pf[b][1]);
#pragma unroll
        for (int b = 0; b < kChunk; ++b)
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint4 v = lds128(at + b * kBlockBytes + kv_code_bytes(kHd, kBits) + 512 * i);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
              uint32_t a[4];
              code_fragment<kBits, true>(w, e, a);
              mma16816(acc[kPer * i + e], a, pf[b][0], pf[b][1]);
            }
          }
        if (j % kFlush == 0) take_off();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty0 + 8 * slot);   // (every lane's loads from the slot have been used by now)
      if (++slot == (warp + 1) * C::kDepth) slot = warp * C::kDepth, parity ^= 1;
    }
    take_off();
    cur.chunk = chunk0 + j1 - j0;

    // ---- the tile's rows, or this warp's part of them
    const bool whole = chunk0 == 0 && j1 - j0 == s.chunks;
    const int which = chunk0 != 0 ? 0 : 1;
    // (no chunk left: the slots are free)
    float *const part = reinterpret_cast<float *>(j == last ? ring + warp * C::kDepth * C::kStageBytes : earlier + (2 * warp + which) * C::kPartBytes);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 2 * c + e;
#pragma unroll
      for (int d = 4; d < 32; d *= 2) den[e] += __shfl_xor_sync(0xffffffffu, den[e], d), off[e] += __shfl_xor_sync(0xffffffffu, off[e], d);
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        acc[k][e] *= 16777216.f, acc[k][e + 2] *= kBits == 4 ? 1048576.f : 16777216.f;
      }
      if (!whole) {
        if (r == 0) reinterpret_cast<float4 *>(part + kRows * C::kAccLd)[row] = make_float4(top[e], den[e], off[e], 0.f);
#pragma unroll
        for (int k = 0; k < kSteps; ++k) part[row * C::kAccLd + 16 * k + r] = acc[k][e], part[row * C::kAccLd + 16 * k + 8 + r] = acc[k][e + 2];
      } else if (first_row + row < n_flat) {
        const RowAt to = row_at<kHd>(p, s.row, head, first_row + row);
        float l = den[e];
        if (p.prefix_tokens > 0) {
#pragma unroll
          for (int k = 0; k < kSteps; ++k) to.prefix[16 * k + r] = acc[k][e] + off[e], to.prefix[16 * k + 8 + r] = acc[k][e + 2] + off[e];
          if (r == 0) *reinterpret_cast<float2 *>(to.prefix + kHd) = make_float2(top[e], l);
        } else {
          // (the prefix's sums before the first store, which might be to the same memory for all the compiler knows: one trip, not 32)
          float f = 1.f, g = 0.f, pre[kSteps][2];
          if (to.prefix) {
            const float2 ml = *reinterpret_cast<const float2 *>(to.prefix + kHd);
#pragma unroll
            for (int k = 0; k < kSteps; ++k) pre[k][0] = to.prefix[16 * k + r], pre[k][1] = to.prefix[16 * k + 8 + r];
            const float mm = fmaxf(top[e], ml.x);
            f = ex2(top[e] - mm), g = ex2(ml.x - mm);
            l = l * f + ml.y * g;
          }
          const float inv = l == 0.f ? 0.f : 1.f / l;   // no token: zeros
          f *= inv, g *= inv;
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            float x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              x[h] = (acc[k][e + 2 * h] + off[e]) * f;
              if (to.prefix) x[h] = __fmaf_rn(pre[k][h], g, x[h]);
            }
            const uint32_t both = pack_out(x[0], x[1]);
            to.out[16 * k + r] = __ushort_as_half((unsigned short)both), to.out[16 * k + 8 + r] = __ushort_as_half((unsigned short)(both >> 16));
          }
        }
      }
    }
    if (!whole && lane == 0) parts[2 * warp + which] = OpenTile{j0 - chunk0, cur.seq, cur.unit, s.chunks}, data[2 * warp + which] = part;
  }

  // ---- tiles that several warps hold parts of: chains of the last part of one warp (or the first one of warp 0, when the CTA's share begins inside a tile) and the first
  // parts of those behind it.  One warp per chain, or all on the only one.
  asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
  int chains = 0;
#pragma unroll 1
  for (int lead = -1; lead < kWarps; ++lead) chains += parts[lead < 0 ? 0 : 2 * lead + 1].from != kNoTile;
  const bool alone = chains > 1;
#pragma unroll 1
  for (int lead = -1, k = 0; lead < kWarps; ++lead) {
    const OpenTile f = parts[lead < 0 ? 0 : 2 * lead + 1];
    if (f.from == kNoTile) continue;
    const bool whole = f.from >= 0 && f.from + f.chunks <= n;
    if (!whole && threadIdx.x == 0) open[f.from < 0 ? 0 : 1] = f;
    if (alone && k++ % kWarps != warp) continue;
    const Seq s = load_seq<kRows, kTokens>(p, f.seq, false);
    const int head = f.unit / s.tiles, first_row = (f.unit - head * s.tiles) * kRows, rows = min(kRows, s.rows * p.group - first_row);
    const float *member[kWarps];                     // the parts that belong to it
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const int g = 2 * w + (w == lead);
      member[w] = w >= lead && parts[g].from == f.from ? data[g] : nullptr;
    }
    float *const to = my_partial(p, f.from, at_partial(kHd, kRows));
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
  asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory");
  join_shares<kHd, kRows, kTokens, kConsumers>(p, share.all, share.begin, open, span, reinterpret_cast<float4 *>(ring));   // (nothing in the slots is needed any more)
}

template <int kHd, int kBits>
int launch_few(rosaq_ctx *ctx, AtParams p, cudaStream_t s) {
  constexpr int kWarps = kBits == 4 ? 7 : 5;
  using C = Cfg<kHd, kBits, kWarps>;
  static_assert(C::kSmem <= 113 * 1024, "two CTAs on an SM");
  auto *const kern = attend_kernel<kHd, kBits, kWarps>;
  int &per_sm = ctx->at_per_sm[(kHd == 64) + 2 * (kBits == 8)];
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

int launch_any(rosaq_ctx *ctx, int hd, int bits, const AtParams &p, bool many, cudaStream_t s) {
  if (many) return launch_attend_rows(ctx, p, hd, bits, s);
  if (hd == 128) return bits == 4 ? launch_few<128, 4>(ctx, p, s) : launch_few<128, 8>(ctx, p, s);
  return bits == 4 ? launch_few<64, 4>(ctx, p, s) : launch_few<64, 8>(ctx, p, s);
}

}  // namespace

int attend_forms(const KvView &kv, const KvBatchView &b, int prefix_tokens, int n_q_heads) {
  const long long group = n_q_heads / kv.n_heads;
  auto many = [&](long long rows_of_seq, int n_seqs, long long room) {
    return rows_of_seq >= kManyRows && (double)rows_of_seq * n_seqs * kv.n_heads * (double)room >= (double)kManyWork;
  };
  const bool own = many(((long long)b.n_rows + b.n_seqs - 1) / b.n_seqs * group, b.n_seqs, (long long)b.width * (kKvBlock << kv.page_shift));
  return (own ? 1 : 0) + (prefix_tokens > 0 && many(b.n_rows * group, 1, prefix_tokens) ? 2 : 0);
}

int launch_attend(rosaq_ctx *ctx, const KvView &kv, int hd, int bits, const KvBatchView &b, const int32_t *prefix_table, int prefix_tokens,
                  const __half *q, long long ldq, int n_q_heads, float scale, __half *out, long long ldo, cudaStream_t s) {
  AtParams p{};
  p.kv = kv, p.b = b, p.q = q, p.out = out, p.ldq = ldq, p.ldo = ldo, p.group = n_q_heads / kv.n_heads;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = ctx->d_status, p.wait_limit = std::min<long long>(ctx->wait_limit, kMostPolls);
  const size_t prefix_bytes = prefix_tokens > 0 ? (size_t)b.n_rows * n_q_heads * (hd + 4) * sizeof(float) : 0;
  int st = ROSAQ_OK;
  if (prefix_bytes) st = grow_workspace(ctx, reinterpret_cast<void **>(&ctx->at_prefix), &ctx->at_prefix_bytes, prefix_bytes);
  if (st != ROSAQ_OK) return st;
  p.arrived = ctx->at_arrived;
  const int forms = attend_forms(kv, b, prefix_tokens, n_q_heads);
  if (prefix_tokens > 0) {
    p.prefix = ctx->at_prefix;
    AtParams f = p;
    f.prefix_tokens = prefix_tokens, f.last_row = b.n_seqs;
    f.b.n_seqs = 1, f.b.table = prefix_table;
    f.b.ld_table = f.b.width = (int)(((long long)prefix_tokens + (kKvBlock << kv.page_shift) - 1) / (kKvBlock << kv.page_shift));
    st = launch_any(ctx, hd, bits, f, forms & 2, s);
    if (st != ROSAQ_OK) return st;
  }
  return launch_any(ctx, hd, bits, p, forms & 1, s);
}

}  // namespace rosaq
