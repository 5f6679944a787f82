// rosaq_kv_write and rosaq_kv_read: fp16 rows into the quantized paged cache and back.
//
// A head of a token (64 or 128 channels) is one group: lo = its least value, scale = fp16((hi - lo) / (2^bits - 1)),
// code = rint((x - lo) / scale), value = lo + scale * code.  lo is an input value, so it is held without rounding, and a group that
// lies on one side of zero loses no range (the weights' integer zero-point would).
//
// Bound: memory (rows in, 0.27 or 0.52 of their bytes out).  One warp takes one block of 16 tokens of one head, keys or values: rows
// arrive as 16 bytes per lane (a row is contiguous over 16 or 8 lanes), codes go through 4 KB of shared memory as 16-bit numbers, and
// ldmatrix hands every lane the pairs whose nibbles or bytes make up its words: plain for keys, transposed for values.  Whole
// blocks leave as 16-byte stores; the bytes of a block that begins or ends inside it are stored one by one.
#include "kv_common.cuh"

namespace rosaq {
namespace {

constexpr int kWarps = 8;                           // four heads, keys and values
constexpr int kHeadsPerCta = kWarps / 2;

__device__ __forceinline__ uint32_t h2_bits(__half2 v) { return *reinterpret_cast<uint32_t *>(&v); }
__device__ __forceinline__ __half2 bits_h2(uint32_t v) { return *reinterpret_cast<__half2 *>(&v); }

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t *a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t *a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void stmatrix4(uint32_t addr, const uint32_t *a) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3])
               : "memory");
}
__device__ __forceinline__ void stmatrix4_trans(uint32_t addr, const uint32_t *a) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3])
               : "memory");
}

// Shared address of the row that this lane names to ldmatrix / stmatrix for channels [16 j, 16 j + 16) of 16 tokens.  The four 8 x 8
// matrices are the A fragment's: keys (tokens 0-7, channels 0-7), (8-15, 0-7), (0-7, 8-15), (8-15, 8-15); values, whose rows are
// channels, the same with the parts of tokens and channels exchanged.
template <bool kValue>
__device__ __forceinline__ uint32_t frag_addr(uint32_t tile, int row_bytes, int lane, int j) {
  const int a = (lane >> 3) & 1, b = lane >> 4;
  const int tok = (lane & 7) + 8 * (kValue ? b : a), ch = 16 * j + 8 * (kValue ? a : b);
  return tile + tok * row_bytes + 2 * ch;
}

template <int kHd, int kBits, bool kValue>
__device__ __forceinline__ void write_block(const KvPiece &p, const __half *x, long long ldx, uint8_t *block, uint32_t tile) {
  constexpr int kLanes = kHd / 8, kPer = 32 / kLanes, kSteps = kKvBlock / kPer;   // lanes of a token, tokens and loads of a step
  constexpr int kRowBytes = 2 * kHd + 16;                                         // 16 more: rows on different banks
  constexpr int kWords = kHd / 16 * (kBits / 4);
  constexpr float kMax = kBits == 4 ? 15.f : 255.f;
  const int lane = threadIdx.x & 31, part = lane % kLanes, mine = lane / kLanes;
  uint4 in[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int t = i * kPer + mine - p.slot;
    in[i] = make_uint4(0, 0, 0, 0);
    if (t >= 0 && t < p.n) in[i] = __ldg(reinterpret_cast<const uint4 *>(x + (p.row + t) * ldx + 8 * part));
  }
  uint8_t *const params = block + 2 * kv_code_bytes(kHd, kBits) + (kValue ? 4 * kKvBlock : 0);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int t = i * kPer + mine;
    const bool valid = t >= p.slot && t < p.slot + p.n;
    if (!__any_sync(0xffffffffu, valid)) continue;
    const uint32_t w[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
    // (least, minus the greatest); a NaN is in neither
    __half2 lo2 = __hmin2(__hmin2(bits_h2(w[0]), bits_h2(w[1])), __hmin2(bits_h2(w[2]), bits_h2(w[3])));
    __half2 hi2 = __hmax2(__hmax2(bits_h2(w[0]), bits_h2(w[1])), __hmax2(bits_h2(w[2]), bits_h2(w[3])));
    __half2 m = __halves2half2(__hmin(__low2half(lo2), __high2half(lo2)), __hneg(__hmax(__low2half(hi2), __high2half(hi2))));
#pragma unroll
    for (int d = kLanes / 2; d > 0; d /= 2) m = __hmin2(m, bits_h2(__shfl_xor_sync(0xffffffffu, h2_bits(m), d)));
    float lo = __low2float(m), hi = -__high2float(m);
    if (isnan(lo)) lo = hi = 0.f;
    lo = fminf(fmaxf(lo, -65504.f), 65504.f) + 0.f, hi = fminf(fmaxf(hi, -65504.f), 65504.f);
    __half sh = __float2half_rn(__fdiv_rn(hi - lo, kMax));
    if (__half_as_ushort(sh) == 0) sh = __ushort_as_half(1);
    const float s = __half2float(sh), inv = __frcp_rn(s);
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // infinities end up at the ends of the range, a NaN at its least value
      const __half2 c = __hmin2(__hmax2(bits_h2(w[e]), bits_h2(0xfbfffbffu)), bits_h2(0x7bff7bffu));
      const float xs[2] = {__low2float(c), __high2float(c)};
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        // (x - lo) / s rounded correctly from the rounded reciprocal: one residual and one correction (Markstein, "Computation of
        // elementary functions on the IBM RISC System/6000 processor", 1990).  A product with the reciprocal alone would move the
        // ties, which fp16 data meets once in some thousand values, to either side.
        const float d = xs[f] - lo, q = d * inv;
        const float t1 = fminf(fmaxf(__fmaf_rn(__fmaf_rn(-q, s, d), inv, q), 0.f), kMax);
        code[2 * e + f] = __float_as_uint(t1 + 12582912.f);   // 1.5 * 2^23: rounds to nearest, ties to even, into the low bits
      }
    }
    uint32_t out[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = __byte_perm(code[2 * e], code[2 * e + 1], 0x5410);
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(tile + t * kRowBytes + 16 * part), "r"(out[0]), "r"(out[1]), "r"(out[2]),
                 "r"(out[3])
                 : "memory");
    if (valid && part == 0)
      *reinterpret_cast<uint32_t *>(params + 4 * t) = (uint32_t)__half_as_ushort(sh) | ((uint32_t)__half_as_ushort(__float2half_rn(lo)) << 16);
  }
  __syncwarp();
  uint8_t *const codes = block + (kValue ? kv_code_bytes(kHd, kBits) : 0);
#pragma unroll
  for (int q = 0; q < kWords / 4; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < (kBits == 4 ? 4 : 2); ++e) {
      uint32_t a[4];
      const uint32_t at = frag_addr<kValue>(tile, kRowBytes, lane, (kBits == 4 ? 4 : 2) * q + e);
      if (kValue) ldmatrix4_trans(at, a);
      else ldmatrix4(at, a);
      if (kBits == 4) {
        if (p.n != kKvBlock) {                       // rows of other tokens hold whatever was there
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] &= 0x000f000fu;
        }
        w[e] = kValue ? (a[0] | a[1] << 4 | a[2] << 8 | a[3] << 12) : (a[0] | a[2] << 4 | a[1] << 8 | a[3] << 12);
      } else {
        w[2 * e] = __byte_perm(a[0], a[2], 0x6420), w[2 * e + 1] = __byte_perm(a[1], a[3], 0x6420);
      }
    }
    uint8_t *const to = codes + 512 * q + 16 * lane;
    if (p.n == kKvBlock) {
      *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = kv_byte_token<kBits, kValue>(lane, e, j) - p.slot;   // (4 q is even: w's parity is e's)
          if (t >= 0 && t < p.n) to[4 * e + j] = (uint8_t)(w[e] >> (8 * j));
        }
    }
  }
  __syncwarp();
}

template <int kHd, int kBits, bool kValue>
__device__ __forceinline__ void read_block(const KvPiece &p, __half *x, long long ldx, const uint8_t *block, uint32_t tile) {
  constexpr int kLanes = kHd / 8, kPer = 32 / kLanes, kSteps = kKvBlock / kPer;
  constexpr int kRowBytes = 2 * kHd + 16;
  constexpr int kWords = kHd / 16 * (kBits / 4);
  const int lane = threadIdx.x & 31, part = lane % kLanes, mine = lane / kLanes;
  const uint8_t *const params = block + 2 * kv_code_bytes(kHd, kBits) + (kValue ? 4 * kKvBlock : 0);
  const uint8_t *const codes = block + (kValue ? kv_code_bytes(kHd, kBits) : 0) + 16 * lane;
  uint4 in[kWords / 4];
#pragma unroll
  for (int q = 0; q < kWords / 4; ++q) in[q] = __ldg(reinterpret_cast<const uint4 *>(codes + 512 * q));
  // scale and least value of the four (two: keys) tokens whose codes this lane holds
  uint32_t prm[4];
  if (kValue) {
    const uint2 u = __ldg(reinterpret_cast<const uint2 *>(params + 8 * (lane & 3))), v = __ldg(reinterpret_cast<const uint2 *>(params + 32 + 8 * (lane & 3)));
    prm[0] = u.x, prm[1] = u.y, prm[2] = v.x, prm[3] = v.y;
  } else {
    prm[0] = prm[1] = __ldg(reinterpret_cast<const uint32_t *>(params + 4 * (lane >> 2)));
    prm[2] = prm[3] = __ldg(reinterpret_cast<const uint32_t *>(params + 32 + 4 * (lane >> 2)));
  }
  float s[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = __low2float(bits_h2(prm[i])), lo[i] = __high2float(bits_h2(prm[i]));
#pragma unroll
  for (int j = 0; j < kHd / 16; ++j) {
    const uint32_t *const w = reinterpret_cast<const uint32_t *>(in);
    uint32_t a[4];                                   // A fragment order: keys (h, p) = a[h + 2 p], values (h, p) = a[p + 2 h]
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        uint32_t pair;
        if (kBits == 4) pair = (w[j] >> (8 * h + 4 * q)) & 0x000f000fu;
        else pair = kValue ? __byte_perm(w[2 * j + q], 0, h ? 0x4342 : 0x4140) : __byte_perm(w[2 * j + h], 0, q ? 0x4342 : 0x4140);
        const __half2 c = __hsub2(bits_h2(pair | 0x64006400u), bits_h2(0x64006400u));   // 1024 + code, less 1024
        // (the greatest code of a group that reaches to the end of fp16 may stand for a little more)
        const float x0 = fminf(__fmaf_rn(__low2float(c), s[2 * h], lo[2 * h]), 65504.f);
        const float x1 = fminf(__fmaf_rn(__high2float(c), s[2 * h + 1], lo[2 * h + 1]), 65504.f);
        a[kValue ? q + 2 * h : h + 2 * q] = h2_bits(__floats2half2_rn(x0, x1));
      }
    const uint32_t at = frag_addr<kValue>(tile, kRowBytes, lane, j);
    if (kValue) stmatrix4_trans(at, a);
    else stmatrix4(at, a);
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int t = i * kPer + mine;
    if (t >= p.slot && t < p.slot + p.n)
      *reinterpret_cast<uint4 *>(x + (p.row + t - p.slot) * ldx + 8 * part) = lds128(tile + t * kRowBytes + 16 * part);
  }
  __syncwarp();
}

struct KvParams {
  KvView kv;
  KvBatchView b;
  __half *k, *v;
  long long ldk, ldv;
  int rows_per_cta;
  int *status;
};

template <int kHd, int kBits, bool kWrite>
__global__ void __launch_bounds__(32 * kWarps) kv_rows_kernel(KvParams p) {
  __shared__ __align__(16) uint8_t tiles[kWarps][kKvBlock * (2 * kHd + 16)];
  grid_dep_launch_dependents();
  grid_dep_wait();                                   // the rows, the batch and the pages may be the previous kernel's output
  constexpr int kBlockBytes = kv_block_bytes(kHd, kBits);
  const int warp = threadIdx.x / 32, head = blockIdx.y * kHeadsPerCta + warp / 2;
  if (head >= p.kv.n_heads) return;
  const uint32_t tile = smem_u32(tiles[warp]);
  const long long head_at = (long long)head * (kBlockBytes << p.kv.page_shift);
  const int first = blockIdx.x * p.rows_per_cta;
  kv_pieces(p.kv, p.b, kBlockBytes, first, first + p.rows_per_cta, p.status, [&](const KvPiece &piece) {
    uint8_t *const block = p.kv.pages + piece.offset + head_at;
    if (warp & 1) {
      if (kWrite) write_block<kHd, kBits, true>(piece, p.v + head * kHd, p.ldv, block, tile);
      else read_block<kHd, kBits, true>(piece, p.v + head * kHd, p.ldv, block, tile);
    } else {
      if (kWrite) write_block<kHd, kBits, false>(piece, p.k + head * kHd, p.ldk, block, tile);
      else read_block<kHd, kBits, false>(piece, p.k + head * kHd, p.ldk, block, tile);
    }
  });
}

template <bool kWrite>
int launch_rows(const KvView &kv, int hd, int bits, const KvBatchView &b, __half *k, long long ldk, __half *v, long long ldv, int *status,
                cudaStream_t s) {
  // A piece belongs to the CTA in whose rows it begins.  Sixteen rows per CTA give a long run of rows one piece each; where
  // sequences bring a few rows each, every row is likely to be a piece of its own and gets a CTA.
  KvParams p{kv, b, k, v, ldk, ldv, b.n_rows >= 8 * b.n_seqs ? kKvBlock : 1, status};
  const dim3 grid((b.n_rows + p.rows_per_cta - 1) / p.rows_per_cta, (kv.n_heads + kHeadsPerCta - 1) / kHeadsPerCta);
  if (grid.y > 65535) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  if (hd == 128) return bits == 4 ? kv_launch(kv_rows_kernel<128, 4, kWrite>, grid, 32 * kWarps, 0, s, p) : kv_launch(kv_rows_kernel<128, 8, kWrite>, grid, 32 * kWarps, 0, s, p);
  return bits == 4 ? kv_launch(kv_rows_kernel<64, 4, kWrite>, grid, 32 * kWarps, 0, s, p) : kv_launch(kv_rows_kernel<64, 8, kWrite>, grid, 32 * kWarps, 0, s, p);
}

}  // namespace

int launch_kv_write(const KvView &kv, int hd, int bits, const KvBatchView &b, const __half *k, long long ldk, const __half *v, long long ldv,
                    int *status, cudaStream_t s) {
  return launch_rows<true>(kv, hd, bits, b, const_cast<__half *>(k), ldk, const_cast<__half *>(v), ldv, status, s);
}
int launch_kv_read(const KvView &kv, int hd, int bits, const KvBatchView &b, __half *k, long long ldk, __half *v, long long ldv, int *status,
                   cudaStream_t s) {
  return launch_rows<false>(kv, hd, bits, b, k, ldk, v, ldv, status, s);
}

}  // namespace rosaq
