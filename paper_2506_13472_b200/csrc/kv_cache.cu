// rosaq_kv_write and rosaq_kv_read: fp16 rows into the quantized paged cache and back.
//
// A head of a token (64 or 128 channels) is one group: lo = its least value, scale = fp16((hi - lo) / (2^bits - 1)),
// code = rint((x - lo) / scale), value = lo + scale * code.  lo is an input value, so it is held without rounding, and a group that
// lies on one side of zero loses no range (the weights' integer zero-point would).
//
// Bound: memory (rows in, 0.27 or 0.52 of their bytes out).  One warp takes one block of 16 tokens of one head, keys or values: rows
// arrive as 16 bytes per lane in 4 KB of shared memory (a row is contiguous over 16 or 8 lanes), codes take their place as 16-bit numbers, and
// ldmatrix hands every lane the pairs whose nibbles or bytes make up its words: plain for keys, transposed for values.  Whole
// blocks leave as 16-byte stores; into those that begin or end inside a block the bytes of the other tokens are read first (bytes stored one by one would be 190 partial
// sectors per token and head, 64 x 32 of them 6.9 us).  One warp of a call writes to a block, so nothing comes between.
//
// Measured (heads of 128): 2048 rows of 32 heads at 4 bits written in 12.6 us, read in 8.5 (floor 6.5 each way); 13200 rows of 40 heads read in 63 to 73 (343 MB, floor 55: four fifths are
// writes, of which a fill kernel does 3.9 TB/s, 69 us for this much); 64 single rows of 32 heads written in 5.5, latency of lengths, table, rows and quantizer in turn.
#include "kv_common.cuh"

namespace rosaq {
namespace {

constexpr int kWarps = 4;                           // two heads, keys and values
constexpr int kHeadsPerCta = kWarps / 2;

__device__ __forceinline__ uint32_t h2_bits(__half2 v) { return *reinterpret_cast<uint32_t *>(&v); }
__device__ __forceinline__ __half2 bits_h2(uint32_t v) { return *reinterpret_cast<__half2 *>(&v); }

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
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
__device__ __forceinline__ uint32_t frag_addr(uint32_t tile, int row_bytes, int lane, int j, bool value) {
  const int a = (lane >> 3) & 1, b = lane >> 4;
  const int tok = (lane & 7) + 8 * (value ? b : a), ch = 16 * j + 8 * (value ? a : b);
  return tile + tok * row_bytes + 2 * ch;
}

// (least, minus the greatest) of 8 n values; kSkip: of those that are numbers, else a NaN where one is
template <int n, bool kSkip>
__device__ __forceinline__ __half2 range(const uint32_t (*w)[4]) {
  __half2 lo = bits_h2(w[0][0]), hi = lo;
#pragma unroll
  for (int i = 1; i < 4 * n; ++i) {
    const __half2 x = bits_h2(w[i / 4][i % 4]);
    lo = kSkip ? __hmin2(lo, x) : __hmin2_nan(lo, x), hi = kSkip ? __hmax2(hi, x) : __hmax2_nan(hi, x);
  }
  const __half l = kSkip ? __hmin(__low2half(lo), __high2half(lo)) : __hmin_nan(__low2half(lo), __high2half(lo));
  const __half h = kSkip ? __hmax(__low2half(hi), __high2half(hi)) : __hmax_nan(__low2half(hi), __high2half(hi));
  return __halves2half2(l, __hneg(h));
}

// Keys and values take the same code (which of them is uniform in a warp) and its loops are rolled: small calls spend more time on fetching instructions than on anything else.
template <int kHd, int kBits>
__device__ __forceinline__ void write_block(bool value, const KvPiece &p, const __half *x, long long ldx, uint8_t *block, uint32_t tile) {
  constexpr int kLanes = kHd / 8, kPer = 32 / kLanes, kSteps = kKvBlock / kPer;   // lanes of a token, tokens and loads of a step
  constexpr int kRowBytes = 2 * kHd + 16;                                         // 16 more: rows on different banks
  constexpr int kWords = kHd / 16 * (kBits / 4);
  constexpr float kMax = kBits == 4 ? 15.f : 255.f;
  const int lane = threadIdx.x & 31, part = lane % kLanes, mine = lane / kLanes;
  // ---- the rows, as far as shared memory
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int t = i * kPer + mine - p.slot;
    if (t >= 0 && t < p.n) copy16(tile + (i * kPer + mine) * kRowBytes + 16 * part, x + (p.row + t) * ldx + 8 * part);
  }
  uint8_t *const codes = block + (value ? kv_code_bytes(kHd, kBits) : 0) + 16 * lane;
  // which bytes of this lane's words (even and odd ones) are this piece's, and what is there now
  uint32_t ours[2] = {0xffffffffu, 0xffffffffu};
  uint4 old[kWords / 4];
  if (p.n != kKvBlock) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      ours[e] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = (value ? kv_byte_token<kBits, true>(lane, e, j) : kv_byte_token<kBits, false>(lane, e, j)) - p.slot;
        if (t >= 0 && t < p.n) ours[e] |= 0xffu << (8 * j);
      }
    }
#pragma unroll
    for (int q = 0; q < kWords / 4; ++q)
      if (ours[0] | ours[1]) old[q] = *reinterpret_cast<const uint4 *>(codes + 512 * q);
  }
  copy_wait_all();
  __syncwarp();
  uint8_t *const params = block + 2 * kv_code_bytes(kHd, kBits) + (value ? 4 * kKvBlock : 0);
  // ---- codes in the values' place.  Four lanes per token, each every fourth 16 bytes: what a token costs besides its values (two divisions, the exchange) is shared by 32
  // of them (2048 rows x 32 heads: 12.6 us, with sixteen lanes per token 15.9)
  const int quad = lane & 3;
#pragma unroll 1
  for (int t0 = p.slot & ~7; t0 < p.slot + p.n; t0 += 8) {
    const int t = t0 + (lane >> 2);
    const bool valid = t >= p.slot && t < p.slot + p.n;
    const uint32_t cell = tile + t * kRowBytes + 16 * quad;
    uint32_t w[kHd / 32][4];
#pragma unroll
    for (int k = 0; k < kHd / 32; ++k) {
      const uint4 v = lds128(cell + 64 * k);         // (of tokens that are not this piece's: whatever was there)
      w[k][0] = v.x, w[k][1] = v.y, w[k][2] = v.z, w[k][3] = v.w;
    }
    // (least, minus the greatest).  Almost always all are numbers: NaNs come through this way, and what is not finite is seen to apart.
    __half2 m = range<kHd / 32, false>(w);
    m = __hmin2_nan(m, bits_h2(__shfl_xor_sync(0xffffffffu, h2_bits(m), 1))), m = __hmin2_nan(m, bits_h2(__shfl_xor_sync(0xffffffffu, h2_bits(m), 2)));
    float lo = __low2float(m), hi = -__high2float(m);
    if (__any_sync(0xffffffffu, valid && !(lo >= -65504.f && hi <= 65504.f))) {
      m = range<kHd / 32, true>(w);                  // a NaN is in neither
      m = __hmin2(m, bits_h2(__shfl_xor_sync(0xffffffffu, h2_bits(m), 1))), m = __hmin2(m, bits_h2(__shfl_xor_sync(0xffffffffu, h2_bits(m), 2)));
      lo = __low2float(m), hi = -__high2float(m);
      if (isnan(lo)) lo = hi = 0.f;
      lo = fminf(fmaxf(lo, -65504.f), 65504.f), hi = fminf(fmaxf(hi, -65504.f), 65504.f);
      // infinities end up at the ends of the range, a NaN at its least value
      const __half2 least = __float2half2_rn(lo);
#pragma unroll
      for (int k = 0; k < kHd / 32; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __half2 c = __hmin2(__hmax2(bits_h2(w[k][e]), bits_h2(0xfbfffbffu)), bits_h2(0x7bff7bffu));
          w[k][e] = h2_bits(__hmax2(c, least));      // (a NaN came out of the two before as -65504)
        }
    }
    lo += 0.f;                                       // (no negative zero)
    __half sh = __float2half_rn(__fdiv_rn(hi - lo, kMax));
    if (__half_as_ushort(sh) == 0) sh = __ushort_as_half(1);
    const float s = __half2float(sh), inv = __frcp_rn(s);
#pragma unroll
    for (int k = 0; k < kHd / 32; ++k) {
      uint32_t out[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 v = __half22float2(bits_h2(w[k][e]));
        // (x - lo) / s rounded correctly from the rounded reciprocal: one residual and one correction (Markstein, "Computation of
        // elementary functions on the IBM RISC System/6000 processor", 1990).  A product with the reciprocal alone would move the
        // ties, which fp16 data meets once in some thousand values, to either side.
        const float d0 = v.x - lo, d1 = v.y - lo, q0 = d0 * inv, q1 = d1 * inv;
        const float u0 = __fmaf_rn(__fmaf_rn(-q0, s, d0), inv, q0), u1 = __fmaf_rn(__fmaf_rn(-q1, s, d1), inv, q1);
        // 1.5 * 2^23 rounds to nearest, ties to even, into the low bits; the greatest code is the limit (s may have been rounded down)
        out[e] = __vminu2(__byte_perm(__float_as_uint(u0 + 12582912.f), __float_as_uint(u1 + 12582912.f), 0x5410), kBits == 4 ? 0x000f000fu : 0x00ff00ffu);
      }
      asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(cell + 64 * k), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]) : "memory");
    }
    if (valid && quad == 0)
      *reinterpret_cast<uint32_t *>(params + 4 * t) = (uint32_t)__half_as_ushort(sh) | ((uint32_t)__half_as_ushort(__float2half_rn(lo)) << 16);
  }
  __syncwarp();
#pragma unroll
  for (int q = 0; q < kWords / 4; ++q) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < (kBits == 4 ? 4 : 2); ++e) {
      uint32_t a[4];                                 // keys: (token half, channel half) at 1 and 2; values: (channel half, token half)
      const uint32_t at = frag_addr(tile, kRowBytes, lane, (kBits == 4 ? 4 : 2) * q + e, value);
      if (value) ldmatrix4_trans(at, a);
      else ldmatrix4(at, a);
      if (kBits == 4) {
        // (the rows of other tokens hold whatever was there)
        const uint32_t mask = 0x000f000fu, nibble = value ? a[1] : a[2], byte = value ? a[2] : a[1];
        w[e] = (a[0] & mask) | (nibble & mask) << 4 | (byte & mask) << 8 | (a[3] & mask) << 12;
      } else {
        w[2 * e] = __byte_perm(a[0], a[2], 0x6420), w[2 * e + 1] = __byte_perm(a[1], a[3], 0x6420);
      }
    }
    if (p.n != kKvBlock) {
      w[0] = (w[0] & ours[0]) | (old[q].x & ~ours[0]), w[1] = (w[1] & ours[1]) | (old[q].y & ~ours[1]);
      w[2] = (w[2] & ours[0]) | (old[q].z & ~ours[0]), w[3] = (w[3] & ours[1]) | (old[q].w & ~ours[1]);
    }
    if (ours[0] | ours[1]) *reinterpret_cast<uint4 *>(codes + 512 * q) = make_uint4(w[0], w[1], w[2], w[3]);
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
  // (plain loads: the launch before may have been writing these bytes after this one had begun, which loads by way of the read-only path do not allow)
  uint4 in[kWords / 4];
#pragma unroll
  for (int q = 0; q < kWords / 4; ++q) in[q] = *reinterpret_cast<const uint4 *>(codes + 512 * q);
  // scale and least value of the four (two: keys) tokens whose codes this lane holds
  uint32_t prm[4];
  if (kValue) {
    const uint2 u = *reinterpret_cast<const uint2 *>(params + 8 * (lane & 3)), v = *reinterpret_cast<const uint2 *>(params + 32 + 8 * (lane & 3));
    prm[0] = u.x, prm[1] = u.y, prm[2] = v.x, prm[3] = v.y;
  } else {
    prm[0] = prm[1] = *reinterpret_cast<const uint32_t *>(params + 4 * (lane >> 2));
    prm[2] = prm[3] = *reinterpret_cast<const uint32_t *>(params + 32 + 4 * (lane >> 2));
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
    const uint32_t at = frag_addr(tile, kRowBytes, lane, j, kValue);
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
    const bool value = warp & 1;
    __half *const x = (value ? p.v : p.k) + head * kHd;
    const long long ldx = value ? p.ldv : p.ldk;
    if (kWrite) write_block<kHd, kBits>(value, piece, x, ldx, block, tile);
    else if (value) read_block<kHd, kBits, true>(piece, x, ldx, block, tile);
    else read_block<kHd, kBits, false>(piece, x, ldx, block, tile);
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
