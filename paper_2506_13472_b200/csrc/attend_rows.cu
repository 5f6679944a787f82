// rosaq_attend for many query rows per sequence and key/value head: a prompt, or a batch behind a shared prefix.
//
// tcgen05: per chunk of 64 tokens S = Q C^T (128 rows x 64 tokens, both operands in shared memory) and O += P D (P in tensor memory over its scores, D in shared memory), fp32
// accumulators in tensor memory.  C and D are the codes less the middle of their range (8 or 128), exact in fp16, so nothing but the softmax weights loses bits, as in
// attend.cu; with A = scale s_k, B = scale (lo_k + middle s_k), L = log2 s_v, M = lo_v / s_v + middle of a token (scale: with log2 e)
//   u = A S + (B sum(q) + L),   p s_v = 2^(u - top),   out = (sum (p s_v) D + sum (p s_v) M) / sum (p s_v) / s_v.
// (Keys and values rounded to fp16 instead need none of the terms: 1.25 us per chunk of 256 rows, and an error of 6.5e-4 where this has 2.7e-4 and the rounding of the result alone
// 2.1e-4: some channels of keys are several times larger than others, and their roundings move the scores.)
// A CTA has up to two tiles of 128 rows, which share the operands that four warps make of the codes, in the fragment order of the cache's words: one stmatrix stores four 8 x 8
// pieces, rows of keys (channels contiguous) and rows of channels of values (tokens contiguous), both K-major with the 128-byte swizzle.  Softmax: a row per thread, four warps per
// tile; the scores of the next chunk go to a second buffer.  What the weights of a row are relative to is seldom renewed: then its accumulators are rescaled in tensor memory.
//
// Measured: 1.75 us per chunk and pair of tiles (head of 128), 3300 cycles: the tensor core takes 1280 of them (an MMA of 64 tokens 48 for its operands from shared memory, of 128
// channels 64), the exponentials 1024, the terms 2560 of the shared memory's bandwidth (20 bytes per row and token: a broadcast costs as much as any load).  Softmax warps have 176
// registers, so that terms are loaded while scores are on their way (all warps with 128: 2 % slower).  Before the first chunk
// and behind the last one about 8 us: the share, the queries and the first codes 4, the rows 4 (135 KB of partial sums per CTA).
#include <algorithm>
#include <type_traits>

#include "attend_common.cuh"

namespace rosaq {
namespace {

constexpr int kTile = 128, kRows = 2 * kTile;       // query rows of an MMA, of a CTA's tile
constexpr int kTokens = 64, kBlocks = kTokens / kKvBlock;
constexpr int kWorkers = 8;                         // softmax warps
constexpr int kMakers = 4;                          // a block of sixteen tokens each
constexpr int kIssuers = kWorkers + kMakers;        // first of the two warps that issue MMAs, one per tile
constexpr int kThreads = 32 * (kIssuers + 4);        // (whole groups of four warps, which registers are shared out to; the last one waits at the end)
constexpr int kRegsSoftmax = 176, kRegsMaker = 80, kRegsRest = 80;   // 512 in all
static_assert(2 * kRegsSoftmax + kRegsMaker + kRegsRest <= 512, "registers");
constexpr int kFew = 16, kLeast = 4;                // chunks: of tiles that are not cut, of a CTA
constexpr int kJoinRows = 16, kJoinThreads = 256;

// What the pairs of a chunk's tokens come to, two tokens (t, t + 1) at a time: {A_t, A_t+1, B_t, B_t+1}, {1 / s_v twice, M twice}, and behind both L of all
constexpr int kTermBytes = kTokens * 20;

// A tile that begins in a CTA's share and does not end there, for the launch that joins the parts: behind the partial tiles of all CTAs, one per CTA.
struct OpenRows {
  int rows;             // 0: there is none
  int head, first_row, seq_row, last_cta, pad[3];
};

template <int kHd, int kBits>
struct RCfg {
  static constexpr int kHalves = kHd / 64;          // 64 channels: a row of 128 bytes
  static constexpr int kQBytes = kTile * 2 * kHd, kKBytes = kTokens * 2 * kHd, kVBytes = kKBytes;
  static constexpr int kRawBytes = kBlocks * kv_block_bytes(kHd, kBits);
  static constexpr int kRaw = kBits == 4 ? 6 : kHd == 64 ? 4 : 3;   // chunks of codes under way: three of 8.7 KB do not cover the latency of the memory
  static constexpr int kKv = 3;                     // chunks of keys and values: with two, the makers wait for the tensor core and it for them
  static constexpr int kOffK = 2 * kQBytes, kOffV = kOffK + kKv * kKBytes, kOffRaw = kOffV + kKv * kVBytes, kOffTerms = kOffRaw + kRaw * kRawBytes,
                       kOffBars = kOffTerms + kKv * kTermBytes;
  static constexpr int kSmem = kOffBars + 512 + 1024;   // (the swizzled operands start at a multiple of 1024)
  static constexpr long long kWorkBytes = 2 * 4 * at_partial(kHd, kRows) + (int)sizeof(OpenRows);   // of a CTA
};
// barriers
constexpr int kRawFull = 0, kRawEmpty = 6, kKFull = 12, kVFull = 15, kKFree = 18, kVFree = 21, kSFull = 24 /* [tile][buffer] */, kPFull = 28, kODone = 32 /* [tile][buffer] */, kQFull = 36,
              kDone = 38, kBars = 40;
// tensor memory
__device__ __forceinline__ uint32_t s_col(int tile, int buf) { return 128 * tile + 64 * buf; }
__device__ __forceinline__ uint32_t o_col(int tile) { return 256 + 128 * tile; }

__device__ __forceinline__ void stmatrix4(uint32_t addr, const uint32_t *a) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3])
               : "memory");
}
// D (+)= A B over 64 of k: four MMAs, both operands K-major in shared memory (A: 128 rows; rows of 128 bytes, swizzled)
__device__ __forceinline__ void mma4_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q, e;\n\t.reg .b64 ta, tb;\n\t"
      "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "add.u64 ta, %1, 2;\n\tadd.u64 tb, %2, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], ta, tb, %3, q;\n\t"
      "add.u64 ta, %1, 4;\n\tadd.u64 tb, %2, 4;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], ta, tb, %3, q;\n\t"
      "add.u64 ta, %1, 6;\n\tadd.u64 tb, %2, 6;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], ta, tb, %3, q;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// the same with A in tensor memory: 16 of k are eight columns
__device__ __forceinline__ void mma4_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q, e;\n\t.reg .b64 tb;\n\t.reg .b32 ta;\n\t"
      "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "add.u32 ta, %1, 8;\n\tadd.u64 tb, %2, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], tb, %3, q;\n\t"
      "add.u32 ta, %1, 16;\n\tadd.u64 tb, %2, 4;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], tb, %3, q;\n\t"
      "add.u32 ta, %1, 24;\n\tadd.u64 tb, %2, 6;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [ta], tb, %3, q;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// the chunks of a tile that a CTA goes through, and what it may skip: everything behind the last token that a row sees
struct Segment {
  int head, tile, chunk0, count, rows;              // count: chunks that are worked on (none: nothing is seen)
  bool whole;
};
__device__ __forceinline__ Segment segment(const AtParams &p, const Cursor &c, int left) {
  Segment g;
  const Seq &s = c.s;
  g.head = c.unit / s.tiles, g.tile = c.unit - g.head * s.tiles, g.chunk0 = c.chunk;
  const int first_row = g.tile * kRows, n_flat = s.rows * p.group;
  g.rows = min(kRows, n_flat - first_row);
  const int take = min(left, s.chunks - c.chunk);
  g.whole = c.chunk == 0 && take == s.chunks;
  int seen = s.len;
  if (p.prefix_tokens == 0) seen = min(max(s.len - s.rows + 1 + (first_row + g.rows - 1) / p.group, 0), s.len);
  g.count = min(take, max((seen + kTokens - 1) / kTokens - c.chunk, 0));
  return g;
}

template <int kHd, int kBits>
__global__ void __launch_bounds__(kThreads, 1) attend_rows_kernel(const __grid_constant__ AtParams p) {
  using C = RCfg<kHd, kBits>;
  constexpr int kWords = kHd / 16 * (kBits / 4), kBlockBytes = kv_block_bytes(kHd, kBits);
  extern __shared__ uint8_t dyn[];
  uint8_t *const smem = dyn + ((1024 - (smem_u32(dyn) & 1023)) & 1023);
  const uint32_t base = smem_u32(smem), bars = base + C::kOffBars;
  uint32_t *const tmem_at = reinterpret_cast<uint32_t *>(smem + C::kOffBars + 8 * kBars);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31;
  auto bar = [&](int i) { return bars + 8 * i; };

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kRaw; ++i) mbar_init(bar(kRawFull + i), 1), mbar_init(bar(kRawEmpty + i), kMakers);
    for (int i = 0; i < C::kKv; ++i) mbar_init(bar(kKFull + i), 4), mbar_init(bar(kVFull + i), 4), mbar_init(bar(kKFree + i), 2), mbar_init(bar(kVFree + i), 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(kQFull + i), 4);
      for (int b = 0; b < 2; ++b) mbar_init(bar(kSFull + 2 * i + b), 1), mbar_init(bar(kPFull + 2 * i + b), 4), mbar_init(bar(kODone + 2 * i + b), 1);
    }
    mbar_init(bar(kDone), 1), mbar_init(bar(kDone + 1), 1);
    mbar_init_fence();
  }
  // The launch before this one is over before the tensor memory is asked for, and those behind begin when this CTA has it: a CTA takes all that an SM has, and neither side may
  // hold what the other one waits for.
  grid_dep_wait();
  __shared__ Share share;
  OpenRows *const open = reinterpret_cast<OpenRows *>(p.partials + 2ll * gridDim.x * at_partial(kHd, kRows)) + blockIdx.x;
  if (warp == kIssuers) tmem_alloc<512>(smem_u32(tmem_at));
  if (warp == 0) {
    if (lane == 0) open->rows = 0;
    find_share<kRows, kTokens>(p, blockIdx.x, gridDim.x, kFew, kLeast, blockIdx.x == 0, share);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_at, 0);
  grid_dep_launch_dependents();
  if (share.begin == share.end) {
    if (warp == kIssuers) tmem_dealloc<512>(tmem);
    return;
  }
  Cursor cur = share.cur;
  const int n = (int)(share.end - share.begin);

  // A wait that expires is reported, and the warp waits no more: it goes on through what the others rely on.
  bool lost = false;
  auto wait = [&](int b, uint32_t parity) {
    if (lost) return;
    bool here = mbar_try_wait(bar(b), parity);
    if (!__all_sync(0xffffffffu, here)) {
      for (long long i = 0; !here && i < p.wait_limit; ++i) here = mbar_try_wait(bar(b), parity);
      lost = !__all_sync(0xffffffffu, here);
      if (lost && lane == 0) atomicExch(p.status, (int)ROSAQ_ERR_TIMEOUT);
    }
  };

  // The same without the suspension of mbarrier.try_wait, which takes its time to end: for the one warp that everybody waits for.
  auto spin = [&](int b, uint32_t parity) {
    if (lost) return;
    bool here = mbar_test_wait(bar(b), parity);
    if (__all_sync(0xffffffffu, here)) return;
    for (long long i = 0; !here && i < 32 * p.wait_limit; ++i) here = mbar_test_wait(bar(b), parity);
    lost = !__all_sync(0xffffffffu, here);
    if (lost && lane == 0) atomicExch(p.status, (int)ROSAQ_ERR_TIMEOUT);
  };

  if (warp < kWorkers) {
    reg_inc<kRegsSoftmax>();
    // ================================================================ softmax: warps 0-3 the first tile, 4-7 the second; a row per thread
    const int x = warp >> 2, row = 32 * (warp & 3) + lane;
    const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    uint32_t g = 0, all = 0;                         // chunks of this tile so far, of both
    // Products of chunk k end phase k / 2 of one of two barriers.  A phase is waited for only when the one before it on its barrier is known to have ended: chunk g waits for those
    // of chunk g - 2, and those of chunk g - 1 only when it rescales.
    for (int left = n; left > 0;) {
      settle<kRows, kTokens>(p, cur);
      const Segment sg = segment(p, cur, left);
      const Seq &s = cur.s;
      const int take = min(left, s.chunks - cur.chunk), flat = sg.tile * kRows + kTile * x + row;
      const bool active = sg.rows > kTile * x, valid = kTile * x + row < sg.rows;
      const int tok = valid ? flat / p.group : 0;
      float top = kNone, den = 0.f, off = 0.f;
      if (active && sg.count > 0) {
        // ---- the queries
        const __half *const src = p.q + (long long)(s.row + tok) * p.ldq + (long long)(sg.head * p.group + (valid ? flat - tok * p.group : 0)) * kHd;
        // (kLanes lanes per row, so that a row's bytes are read together; a loop of few instructions, which are fetched for the first time here)
        constexpr int kLanes = kHd / 8, kPer = 32 / kLanes;
        const int piece = lane % kLanes;
        uint8_t *const rows = smem + x * C::kQBytes + (piece / 8) * (128 * kTile);
#pragma unroll 1
        for (int i = 0; i < 32; i += kPer) {
          const int of = i + lane / kLanes, to = 32 * (warp & 3) + of;
          const __half *const from = reinterpret_cast<const __half *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(src), of));
          const int bytes = __shfl_sync(0xffffffffu, valid, of) ? 16 : 0;   // (the others are zeros)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(rows + 128 * to + (((piece & 7) ^ (to & 7)) << 4))), "l"(from + 8 * piece), "r"(bytes)
                       : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kQFull + x));
        float sum_q = 0.f;
#pragma unroll 1
        for (int i = 0; i < kLanes; ++i) {
          const uint4 v = *reinterpret_cast<const uint4 *>(smem + x * C::kQBytes + (i / 8) * (128 * kTile) + 128 * row + (((i & 7) ^ (row & 7)) << 4));
          const __half2 *const h = reinterpret_cast<const __half2 *>(&v);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum_q += __low2float(h[k]) + __high2float(h[k]);
        }
        if (!isfinite(sum_q)) sum_q = NAN;           // all scores are NaN then: over keys of one sign they could all be minus infinity, and the row like one that sees nothing
        const int lim = p.prefix_tokens > 0 ? s.len : valid ? min(max(s.len - s.rows + 1 + tok, 0), s.len) : s.len;
        const int least = __reduce_min_sync(0xffffffffu, lim);
        for (int j = 0; j < sg.count; ++j, ++g) {
          const int buf = g & 1, tok0 = (sg.chunk0 + j) * kTokens;
          // Scores of this chunk, terms of its tokens, and products of the last but one before it (which are older): asked for at once, as an answer takes more than 100 cycles.
          const uint32_t slot = (all + j) % C::kKv, turn = (all + j) / C::kKv;
          {
            // (the scores first: once they are there, the terms three chunks back are, and the parity is that of this chunk)
            const bool here = lost || mbar_try_wait(bar(kSFull + 2 * x + buf), (g >> 1) & 1), made = lost || mbar_try_wait(bar(kVFull + slot), turn & 1),
                       old = lost || g < 2 || mbar_try_wait(bar(kODone + 2 * x + buf), ((g >> 1) - 1) & 1);
            if (!__all_sync(0xffffffffu, here && made && old)) {
              wait(kSFull + 2 * x + buf, (g >> 1) & 1);
              wait(kVFull + slot, turn & 1);
              if (g >= 2) wait(kODone + 2 * x + buf, ((g >> 1) - 1) & 1);
            }
          }
          tc_fence_after();
          const float4 *const t_ab = reinterpret_cast<const float4 *>(smem + C::kOffTerms + slot * kTermBytes), *const t_vm = t_ab + kTokens / 2, *const t_l = t_vm + kTokens / 2;
          // u, two tokens at a time; those of the second half go back to tensor memory until the first half's exponentials are done
          const bool border = tok0 + kTokens > least;
          const float2 q2 = make_float2(sum_q, sum_q);
          float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          float sc[32];
          auto load = [&](int half) {
            tmem_ld16(lanes + s_col(x, buf) + 32 * half, reinterpret_cast<uint32_t *>(sc));
            tmem_ld16(lanes + s_col(x, buf) + 32 * half + 16, reinterpret_cast<uint32_t *>(sc + 16));
          };
          float2 aa[16], cc[16];                     // of the scores that are on their way
          auto terms = [&](int half) {
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const float4 l = t_l[8 * half + i / 2], x0 = t_ab[16 * half + i], x1 = t_ab[16 * half + i + 1];
              aa[i] = make_float2(x0.x, x0.y), aa[i + 1] = make_float2(x1.x, x1.y);
              cc[i] = __ffma2_rn(make_float2(x0.z, x0.w), q2, make_float2(l.x, l.y)), cc[i + 1] = __ffma2_rn(make_float2(x1.z, x1.w), q2, make_float2(l.z, l.w));
            }
          };
          auto scale = [&](int half) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 u = __ffma2_rn(make_float2(sc[2 * i], sc[2 * i + 1]), aa[i], cc[i]);
              sc[2 * i] = u.x, sc[2 * i + 1] = u.y;
            }
            if (border) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (tok0 + 32 * half + i >= lim) sc[i] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < 32; i += 2) m[(i >> 1) & 3] = fmaxf(m[(i >> 1) & 3], fmaxf(sc[i], sc[i + 1]));
          };
          load(1);
          terms(1);
          tc_wait_ld();
          scale(1);
          tmem_st16(lanes + s_col(x, buf) + 32, reinterpret_cast<const uint32_t *>(sc));
          tmem_st16(lanes + s_col(x, buf) + 48, reinterpret_cast<const uint32_t *>(sc + 16));
          load(0);
          terms(0);
          tc_wait_ld();
          scale(0);
          const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
          if (__any_sync(0xffffffffu, most > top + kGrow)) {
            const float now = fmaxf(most - kUp, top), f = ex2(top - now);
            top = now, den *= f, off *= f;
            if (j > 0) {
              wait(kODone + 2 * x + (buf ^ 1), ((g - 1) >> 1) & 1);
              tc_fence_after();
#pragma unroll 1
              for (int i = 0; i < kHd; i += 16) {
                float o[16];
                tmem_ld16(lanes + o_col(x) + i, reinterpret_cast<uint32_t *>(o));
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] *= f;
                tmem_st16(lanes + o_col(x) + i, reinterpret_cast<const uint32_t *>(o));
              }
            }
          }
          float2 d2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)}, o2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 minus = make_float2(-top, -top);
          float4 vms[16];
          auto ahead = [&](int half) {
#pragma unroll
            for (int i = 0; i < 16; ++i) vms[i] = t_vm[16 * half + i];
          };
          auto weigh = [&](int half) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float4 vm = vms[i];
              const float2 e = __fadd2_rn(make_float2(sc[2 * i], sc[2 * i + 1]), minus), x2 = weights(e.x, e.y);
              w[i] = pack_h2(x2.x, x2.y);
              d2[i & 1] = __ffma2_rn(x2, make_float2(vm.x, vm.y), d2[i & 1]);
              o2[i & 1] = __ffma2_rn(x2, make_float2(vm.z, vm.w), o2[i & 1]);
            }
            // the weights over scores that have been read: sixteen columns hold 32 of them
            tmem_st16(lanes + s_col(x, buf) + 16 * half, w);
          };
          ahead(0);
          weigh(0);
          tc_wait_st();                              // (the second half's u)
          load(1);
          ahead(1);
          tc_wait_ld();
          weigh(1);
          den += (d2[0].x + d2[0].y) + (d2[1].x + d2[1].y), off += (o2[0].x + o2[0].y) + (o2[1].x + o2[1].y);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kPFull + 2 * x + buf));
        }
        wait(kODone + 2 * x + ((g - 1) & 1), ((g - 1) >> 1) & 1);
        tc_fence_after();
      }
      all += max(sg.count, 0);
      // ---- the rows, or this CTA's part of them
      const int from = n - left - sg.chunk0;
      if (active) {
        // By way of shared memory (the place of this warp's queries), 32 channels at a time, so that eight lanes write to a row: a row per lane takes 32 sectors per
        // instruction (a tile of one chunk 20.2 us that way).
        const int r = kTile * x + row;
        const RowAt to = row_at<kHd>(p, s.row, sg.head, valid ? flat : 0);
        float *const sums = !sg.whole ? my_partial(p, from, at_partial(kHd, kRows)) + r * kHd : to.prefix;   // where a part, or a prefix launch's result, goes
        const bool finish = sg.whole && p.prefix_tokens == 0;
        float f = 1.f, g = 0.f;
        if (finish) {
          float l = den;
          if (to.prefix && valid) {
            const float2 ml = *reinterpret_cast<const float2 *>(to.prefix + kHd);
            const float mm = fmaxf(top, ml.x);
            f = ex2(top - mm), g = ex2(ml.x - mm), l = l * f + ml.y * g;
          }
          const float inv = l == 0.f ? 0.f : 1.f / l;   // no token: zeros
          f *= inv, g *= inv;
        } else if (valid) {
          float *const at = sg.whole ? to.prefix + kHd : sums - r * kHd + kRows * kHd + 2 * r;
          *reinterpret_cast<float2 *>(at) = make_float2(top, den);
        }
        uint8_t *const stage = smem + x * C::kQBytes + 4096 * (warp & 3);
#pragma unroll 1
        for (int ch = 0; ch < kHd; ch += 32) {
          float o[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
          if (sg.count > 0) {
            tmem_ld16(lanes + o_col(x) + ch, reinterpret_cast<uint32_t *>(o));
            tmem_ld16(lanes + o_col(x) + ch + 16, reinterpret_cast<uint32_t *>(o + 16));
            tc_wait_ld();
          }
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4 *>(stage + 128 * lane + (((e / 4) ^ (lane & 7)) << 4)) = make_float4((o[e] + off) * f, (o[e + 1] + off) * f, (o[e + 2] + off) * f, (o[e + 3] + off) * f);
          __syncwarp();
          if (!sg.whole) {
            float *const part = sums + (lane / 8 - lane) * kHd + ch + 4 * (lane & 7);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int of = 4 * i + lane / 8;
              if (r - lane + of < sg.rows) *reinterpret_cast<float4 *>(part + 4 * i * kHd) = *reinterpret_cast<const float4 *>(stage + 128 * of + (((lane & 7) ^ (of & 7)) << 4));
            }
            continue;
          }
#pragma unroll 2
          for (int i = 0; i < 8; ++i) {
            const int of = 4 * i + lane / 8, at = ch + 4 * (lane & 7);
            float4 v = *reinterpret_cast<const float4 *>(stage + 128 * of + (((lane & 7) ^ (of & 7)) << 4));
            const bool there = __shfl_sync(0xffffffffu, valid, of);
            float *const to_sums = reinterpret_cast<float *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(sums), of));
            __half *const to_out = reinterpret_cast<__half *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to.out), of));
            const float gg = __shfl_sync(0xffffffffu, g, of);
            if (!there) continue;
            if (finish) {
              if (p.prefix) {
                const float4 w = *reinterpret_cast<const float4 *>(to_sums + at);
                v = make_float4(__fmaf_rn(w.x, gg, v.x), __fmaf_rn(w.y, gg, v.y), __fmaf_rn(w.z, gg, v.z), __fmaf_rn(w.w, gg, v.w));
              }
              uint2 h;
              h.x = pack_out(v.x, v.y), h.y = pack_out(v.z, v.w);
              *reinterpret_cast<uint2 *>(to_out + at) = h;
            } else {
              *reinterpret_cast<float4 *>(to_sums + at) = v;
            }
          }
        }
      }
      if (threadIdx.x == 0 && from >= 0 && from + s.chunks > n) {
        open->head = sg.head, open->first_row = sg.tile * kRows, open->seq_row = s.row, open->rows = sg.rows;
        open->last_cta = share.all.last(share.begin + from, s.chunks);
      }
      tc_fence_before();
      left -= take, cur.chunk += take;
    }
  } else if (warp < kWorkers + kMakers) {
    reg_dec<kRegsMaker>();
    // ================================================================ keys, then values from codes: a block of sixteen tokens per warp
    const int blk = warp - kWorkers;
    // where stmatrix puts the four pieces of a step: this lane names row lane & 7 of piece lane >> 3
    const int h1 = (lane >> 3) & 1, h2 = lane >> 4;
    uint32_t g = 0;
    for (int left = n; left > 0;) {
      settle<kRows, kTokens>(p, cur);
      const Segment sg = segment(p, cur, left);
      const int take = min(left, cur.s.chunks - cur.chunk);
      for (int j = 0; j < sg.count; ++j, ++g) {
        const int st = g % C::kKv, raw = g % C::kRaw;
        const uint32_t from = base + C::kOffRaw + raw * C::kRawBytes + blk * kBlockBytes;
        const int tok0 = (sg.chunk0 + j) * kTokens + blk * kKvBlock;
        wait(kRawFull + raw, (g / C::kRaw) & 1);
        constexpr int kPairs = 2 * kv_code_bytes(kHd, kBits);
        constexpr float kMid = kBits == 4 ? 8.f : 128.f;
        auto make = [&](auto kind) {
          constexpr bool value = decltype(kind)::value;
          if (g >= (uint32_t)C::kKv) wait((value ? kVFree : kKFree) + st, (g / C::kKv - 1) & 1);
          if (value && lane < kKvBlock) {
            // what the pairs of this token come to; whatever lies behind the last one is finite
            const int t = kKvBlock * blk + lane;
            uint32_t kp = lds32(from + kPairs + 4 * lane), vp = lds32(from + kPairs + 64 + 4 * lane);
            if (tok0 + lane >= cur.s.len) kp = vp = 1u;
            const float2 kf = __half22float2(*reinterpret_cast<__half2 *>(&kp)), vf = __half22float2(*reinterpret_cast<__half2 *>(&vp));
            const float l = lg2(fmaxf(vf.x, kLeastScale)), vi = ex2(-l);   // log2(s) and 1 / s as that has it
            float *const terms = reinterpret_cast<float *>(smem + C::kOffTerms + st * kTermBytes);
            float *const ab = terms + 4 * (t / 2) + (t & 1), *const vm = ab + 2 * kTokens;
            ab[0] = kf.x * p.scale_log2, ab[2] = __fmaf_rn(kf.x, kMid, kf.y) * p.scale_log2;
            vm[0] = vi, vm[2] = __fmaf_rn(vf.y, vi, kMid);
            terms[4 * kTokens + t] = l;
          }
          uint32_t to;                               // of step 0; keys advance by two 16-byte pieces of a row, values by sixteen rows
          if (value) to = base + C::kOffV + st * C::kVBytes + 128 * (8 * h1 + (lane & 7)) + (((2 * blk + h2) ^ (lane & 7)) << 4);
          else to = base + C::kOffK + st * C::kKBytes + 128 * (kKvBlock * blk + 8 * h1 + (lane & 7));
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint4 v4 = lds128(from + value * kv_code_bytes(kHd, kBits) + 512 * i + 16 * lane);
            const uint32_t w[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
            for (int e = 0; e < (kBits == 4 ? 4 : 2); ++e) {
              const int k = (kBits == 4 ? 4 : 2) * i + e;
              uint32_t f[4];                         // codes less the middle; pieces in the order (row half, k half) = (0, 0), (1, 0), (0, 1), (1, 1)
              if (kBits == 4) {
                constexpr uint32_t kOne = 0x3c003c00u, kSixteenth = 0x2c002c00u, kLow = 0xe408e408u, kHigh = 0xd480d480u;   // -1032, -72
                const uint32_t u = w[e], v = u >> 8;
                const uint32_t n0 = h2_fma(lop_and_or(u, 0x000f000fu, 0x64006400u), kOne, kLow), n1 = h2_fma(lop_and_or(u, 0x00f000f0u, 0x64006400u), kSixteenth, kHigh);
                const uint32_t n2 = h2_fma(lop_and_or(v, 0x000f000fu, 0x64006400u), kOne, kLow), n3 = h2_fma(lop_and_or(v, 0x00f000f0u, 0x64006400u), kSixteenth, kHigh);
                f[0] = n0, f[1] = value ? n1 : n2, f[2] = value ? n2 : n1, f[3] = n3;
              } else {
                constexpr uint32_t kOne = 0x3c003c00u, kMiddle = 0xe480e480u;   // -1152
                const uint32_t u = w[2 * e], v = w[2 * e + 1];
                f[0] = h2_fma(__byte_perm(u, 0x64646464u, 0x4140), kOne, kMiddle), f[1] = h2_fma(__byte_perm(v, 0x64646464u, 0x4140), kOne, kMiddle);
                f[2] = h2_fma(__byte_perm(u, 0x64646464u, 0x4342), kOne, kMiddle), f[3] = h2_fma(__byte_perm(v, 0x64646464u, 0x4342), kOne, kMiddle);
              }
              if (value) stmatrix4(to + 2048 * k, f);
              else stmatrix4(to + (k / 4) * (128 * kTokens) + ((((2 * k + h2) & 7) ^ (lane & 7)) << 4), f);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(bar((value ? kVFull : kKFull) + st));
        };
        make(std::false_type{});
        make(std::true_type{});
        if (lane == 0 && !lost) mbar_arrive(bar(kRawEmpty + raw));   // (a slot whose copy was given up on is not filled again)
      }
      left -= take, cur.chunk += take;
    }
  } else {
    reg_dec<kRegsRest>();                            // (one instruction for the whole warpgroup)
    if (warp < kIssuers + 2) {
      // ================================================================ MMAs.  Everything that addresses them is the same in all lanes, and the compiler can see it (what came
      // from memory by way of a shuffle): it then lies in uniform registers.  A warp per tile: one warp for both leaves the tensor core idle in each of its waits, which take 100 to 200
      // cycles also when there is nothing to wait for (1.41 us per chunk of two tiles).
      constexpr uint32_t idesc_s = (1u << 4) | ((uint32_t)(kTokens >> 3) << 17) | (8u << 24), idesc_o = (1u << 4) | ((uint32_t)(kHd >> 3) << 17) | (8u << 24);
      const uint32_t ubase = __shfl_sync(0xffffffffu, base, 0), ubars = ubase + C::kOffBars;
      const uint64_t q_desc = make_b_desc(ubase + (warp - kIssuers) * C::kQBytes), k_desc = make_b_desc(ubase + C::kOffK), v_desc = make_b_desc(ubase + C::kOffV);
      constexpr uint32_t kQHalf16 = 8 * kTile, kK16 = C::kKBytes / 16, kKHalf16 = 8 * kTokens, kV16 = C::kVBytes / 16;
      auto ubar = [&](int i) { return ubars + 8 * i; };
      const int x = warp - kIssuers;
      int k_at = 0, v_at = 0;                          // slots of the next keys and values ...
      uint32_t k_turn = 0, v_turn = 0;                 // ... and the parity of their barriers
      uint32_t scored = 0, weighed = 0, tiles = 0;     // chunks whose scores, whose products have been issued; tiles of queries
      // scores of the next chunk.  (A second tile without rows lets go of the keys and values all the same, when they are there: their barriers count two arrivals.)
      auto scores = [&](bool active) {
        spin(kKFull + k_at, k_turn);
        if (active) {
          tc_fence_after();
          if (!lost) {
#pragma unroll
            for (int h = 0; h < C::kHalves; ++h)
              mma4_ss(tmem + s_col(x, scored & 1), q_desc + h * kQHalf16, k_desc + (uint64_t)(k_at * kK16 + h * kKHalf16), idesc_s, h);
          }
          tc_commit(ubar(kSFull + 2 * x + (scored & 1)));
          ++scored;
        }
        tc_commit(ubar(kKFree + k_at));
        if (++k_at == C::kKv) k_at = 0, k_turn ^= 1;
      };
      for (int left = __shfl_sync(0xffffffffu, n, 0); left > 0;) {
        settle<kRows, kTokens>(p, cur);
        const Segment sg = segment(p, cur, left);
        const int take = __shfl_sync(0xffffffffu, min(left, cur.s.chunks - cur.chunk), 0);
        const int count = __shfl_sync(0xffffffffu, sg.count, 0);
        const bool active = __shfl_sync(0xffffffffu, sg.rows > kTile * x, 0);
        if (count > 0) {
          if (active) spin(kQFull + x, tiles++ & 1);
          scores(active);
          for (int j = 0; j < count; ++j) {
            if (j + 1 < count) scores(active);
            spin(kVFull + v_at, v_turn);
            if (active) {
              spin(kPFull + 2 * x + (weighed & 1), (weighed >> 1) & 1);
              tc_fence_after();
              if (!lost) mma4_ts(tmem + o_col(x), tmem + s_col(x, weighed & 1), v_desc + (uint64_t)(v_at * kV16), idesc_o, j > 0);
              tc_commit(ubar(kODone + 2 * x + (weighed & 1)));
              ++weighed;
            }
            tc_commit(ubar(kVFree + v_at));
            if (++v_at == C::kKv) v_at = 0, v_turn ^= 1;
          }
        }
        left -= take, cur.chunk += take;
      }
      // everything issued is over before the tensor memory is given back, whatever was waited for
      tc_commit(bar(kDone + x));
      for (int i = 0; i < 1 << 20 && !mbar_test_wait(bar(kDone + x), 0); ++i) __nanosleep(100);
    } else if (warp == kIssuers + 2) {
      // ================================================================ copies: lane i brings block i of the chunk; its page is looked up a chunk ahead
      uint32_t g = 0;
      const uint64_t keep = policy_evict_first();
      const int run = min(1 << p.kv.page_shift, kBlocks);   // blocks next to each other: one copy, by the lane of the first one
      int block = 0, blocks = 0, page = 0;
      const uint8_t *heads = nullptr;
      auto look_up = [&](const Segment &sg, int j) {
        block = (sg.chunk0 + j) * kBlocks, blocks = min(kBlocks, (cur.s.len + kKvBlock - 1) / kKvBlock - block);
        heads = p.kv.pages + ((long long)sg.head << p.kv.page_shift) * kBlockBytes;
        page = lane < blocks && lane % run == 0 ? kv_page(p.kv, p.b, cur.seq, block + lane) : 0;
      };
      for (int left = n; left > 0;) {
        settle<kRows, kTokens>(p, cur);
        const Segment sg = segment(p, cur, left);
        const int take = min(left, cur.s.chunks - cur.chunk);
        if (sg.count > 0) look_up(sg, 0);
        for (int j = 0; j < sg.count && !lost; ++j, ++g) {
          const int raw = g % C::kRaw;
          if (g >= (uint32_t)C::kRaw) wait(kRawEmpty + raw, (g / C::kRaw - 1) & 1);
          if (lost) break;
          if (lane == 0) mbar_arrive_expect_tx(bar(kRawFull + raw), blocks * kBlockBytes);
          __syncwarp();
          if (page < 0) kv_report(p.status), page = 0;         // (the first page of the cache in its place)
          if (lane < blocks && lane % run == 0)
            bulk_copy_g2s_hint(base + C::kOffRaw + raw * C::kRawBytes + lane * kBlockBytes, heads + kv_offset(p.kv, page, block + lane, kBlockBytes),
                               min(run, blocks - lane) * kBlockBytes, bar(kRawFull + raw), keep);
          if (j + 1 < sg.count) look_up(sg, j + 1);
        }
        left -= take, cur.chunk += take;
      }
      // the CTA outlasts its copies, also when nobody waits for them any more
      for (uint32_t k = g < (uint32_t)C::kRaw ? 0 : g - C::kRaw; k < g; ++k)
        for (int i = 0; i < 1 << 20 && !mbar_test_wait(bar(kRawFull + k % C::kRaw), (k / C::kRaw) & 1); ++i) __nanosleep(100);
    }
  }
  __syncthreads();
  if (warp == kIssuers) tmem_dealloc<512>(tmem);
}

// The parts of tiles that several CTAs hold, in the order of the list: kJoinRows rows of the tile that begins in share blockIdx.x and does not end there.  (One CTA that arrives last
// would have 135 KB per part to read: behind a prefix of 16001 tokens, 18 parts of 256 rows, 220 us in all.)
template <int kHd>
__global__ void __launch_bounds__(kJoinThreads) attend_rows_join_kernel(const __grid_constant__ AtParams p, int ctas) {
  grid_dep_launch_dependents();
  grid_dep_wait();
  const OpenRows open = reinterpret_cast<const OpenRows *>(p.partials + 2ll * ctas * at_partial(kHd, kRows))[blockIdx.x];
  const int c0 = blockIdx.x;
  for (int i = threadIdx.x; i < kJoinRows * (kHd / 4); i += kJoinThreads) {
    const int row = blockIdx.y * kJoinRows + i / (kHd / 4), ch = 4 * (i % (kHd / 4));
    if (row >= open.rows) break;
    float m = kNone, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    gather<kHd, kRows>(p, row, ch, c0, open.last_cta, c0, 1, a, m, l);
    store_row4<kHd>(p, row_at<kHd>(p, open.seq_row, open.head, open.first_row + row), ch, a, m, l);
  }
}

template <int kHd, int kBits>
int launch(rosaq_ctx *ctx, AtParams p, cudaStream_t s) {
  using C = RCfg<kHd, kBits>;
  static_assert(C::kSmem + (int)sizeof(Share) <= 227 * 1024 && 8 * kBars + 16 <= 512, "shared memory");
  auto *const kern = attend_rows_kernel<kHd, kBits>;
  int &ready = ctx->at_per_sm[4 + (kHd == 64) + 2 * (kBits == 8)];
  if (ready == 0 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess) {
    (void)cudaGetLastError();
    return ROSAQ_ERR_CUDA;
  }
  cudaFuncAttributes attr{};
  if (ready == 0 && (cudaFuncGetAttributes(&attr, kern) != cudaSuccess || attr.numRegs * 4 < 2 * kRegsSoftmax + kRegsMaker + kRegsRest)) {
    (void)cudaGetLastError();
    return ROSAQ_ERR_CUDA;                           // (the warpgroups would wait for registers that the block does not have)
  }
  ready = 1;
  const int ctas = std::min(ctx->sm_count, kAtMaxCtas);
  const int st = grow_workspace(ctx, reinterpret_cast<void **>(&ctx->at_partials), &ctx->at_partial_bytes, (size_t)(ctas * C::kWorkBytes));
  if (st != ROSAQ_OK) return st;
  p.partials = ctx->at_partials;
  const int launched = kv_launch(kern, dim3(ctas), kThreads, C::kSmem, s, p);
  if (launched != ROSAQ_OK) return launched;
  return kv_launch(attend_rows_join_kernel<kHd>, dim3(ctas, kRows / kJoinRows), kJoinThreads, 0, s, p, ctas);
}

}  // namespace

int launch_attend_rows(rosaq_ctx *ctx, AtParams p, int hd, int bits, cudaStream_t s) {
  if (hd == 128) return bits == 4 ? launch<128, 4>(ctx, p, s) : launch<128, 8>(ctx, p, s);
  return bits == 4 ? launch<64, 4>(ctx, p, s) : launch<64, 8>(ctx, p, s);
}

}  // namespace rosaq
