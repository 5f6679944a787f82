// The paged cache of quantized keys and values: layout, the batch that a call describes, and the walk over its new rows.
#pragma once

#include "ptx.cuh"
#include "rosaq_internal.cuh"

namespace rosaq {

// ------------------------------------------------------------------------------------
// A page holds page_tokens tokens of one sequence for every key/value head: [head][page_tokens / 16] blocks of 16 tokens,
//
//   key codes | value codes | 16 x {fp16 scale, fp16 least value} of the keys | the same of the values
//
// 2176 bytes for a head of 128 at four bits, so that one bulk copy brings a block into shared memory.  Codes lie as the A operand
// of m16n8k16 MMAs: lane 4 r + c (r < 8, c < 4) owns head_dim / 16 * (bits / 4) words of 32 bits, word w in the 16-byte
// chunk w / 4 at 512 (w / 4) + 16 lane, so a warp reads 512 contiguous bytes per load and needs no exchange.  With
// i = 16 (multiples of the words) and halves h, p, b in {0, 1}:
//
//   keys (row = token, k = channel)      token 8 h + r,        channel i + 8 p + 2 c + b
//   values (row = channel, k = token)    token 8 h + 2 c + b,  channel i + 8 p + r
//
//   4 bits: byte 2 b + h, nibble p: (word & 0x000f000f) is the pair b = 0, 1 in two fp16 mantissas, i.e. subnormal numbers
//           code * 2^-24 that the tensor core multiplies as they are; (word & 0x00f000f0) the same times 16
//   8 bits: keys byte 2 p + b of the word of h, values byte 2 h + b of the word of p
//
// No byte is shared by two tokens: what lies around a token is kept by whole bytes.
// ------------------------------------------------------------------------------------
constexpr int kKvBlock = 16;                        // tokens of a block

__host__ __device__ constexpr int kv_code_bytes(int hd, int bits) { return kKvBlock * hd * bits / 8; }
__host__ __device__ constexpr int kv_block_bytes(int hd, int bits) { return 2 * kv_code_bytes(hd, bits) + 2 * 4 * kKvBlock; }

struct KvView {
  uint8_t *pages;
  long long page_bytes;
  int n_pages;
  int page_shift;       // log2 of the blocks of a page
  int n_heads;
};

struct KvBatchView {
  const int32_t *row_start, *kv_len, *table;
  int n_seqs, ld_table;
  int width;            // entries of a row of the table that belong to it
  int n_rows;           // rows of the caller's buffers
};

// Status words are only ever set: the first launch that finds something wrong is reported.
__device__ __forceinline__ void kv_report(int *status) { atomicExch(status, (int)ROSAQ_ERR_INVALID_ARG); }

// Page of a block of a sequence, or -1: every access to the pages goes through this or a block that kv_place found.
__host__ __device__ inline int kv_page(const KvView &kv, const KvBatchView &b, int seq, int block) {
  const int page = b.table[(long long)seq * b.ld_table + (block >> kv.page_shift)];
  return page >= 0 && page < kv.n_pages ? page : -1;
}
__host__ __device__ inline long long kv_offset(const KvView &kv, int page, int block, int block_bytes) {
  return page * kv.page_bytes + (long long)(block & ((1 << kv.page_shift) - 1)) * block_bytes;
}

// One run of new rows inside one block of one sequence.
struct KvPiece {
  int row, n;           // first row, rows (1 ... 16)
  int slot;             // its position in the block
  long long offset;     // in the pages, of the block of head 0
};

// The run that begins at `row` of sequence `seq` (the last one with row_start[seq] <= row), cut to rows below `total`.
enum KvPlace { kPlaced, kBadPage, kBadSequence, kBadRows };   // nothing else of the block / of the sequence / of the batch is usable
__host__ __device__ inline KvPlace kv_place(const KvView &kv, const KvBatchView &b, int block_bytes, int seq, int row, int total, KvPiece *p) {
  const int begin = b.row_start[seq], stop = b.row_start[seq + 1], end = stop < total ? stop : total;
  const long long len = b.kv_len[seq];
  p->row = row, p->n = end - row, p->slot = 0, p->offset = -1;
  if (end <= row) return kBadRows;                    // (not ascending)
  if (begin < 0 || begin > row || len < (long long)stop - begin || len > ((long long)b.width << kv.page_shift) * kKvBlock) return kBadSequence;
  const long long pos = len - (stop - row);
  p->slot = (int)(pos % kKvBlock);
  if (p->n > kKvBlock - p->slot) p->n = kKvBlock - p->slot;
  const int block = (int)(pos / kKvBlock), page = kv_page(kv, b, seq, block);
  if (page < 0) return kBadPage;
  p->offset = kv_offset(kv, page, block, block_bytes);
  return kPlaced;
}

// The sequence that `row` belongs to: the last i with row_start[i] <= row.  A whole warp; 32 probes per step.
__device__ __forceinline__ int kv_find_seq(const int32_t *row_start, int n_seqs, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n_seqs;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const unsigned below = __ballot_sync(0xffffffffu, at < hi && row_start[at] <= row);
    const int k = below ? 31 - __clz(below) : 0;
    lo += k * step;
    hi = min(lo + step, hi);
  }
  return lo;
}

// Calls f(piece) for every piece that begins in rows [first, last).  Uniform in a warp.  Nothing the batch says makes an access out of
// bounds: rows are cut to n_rows, positions to the page list, pages to the cache, and what had to be cut is reported.
template <typename F>
__device__ __forceinline__ void kv_pieces(const KvView &kv, const KvBatchView &b, int block_bytes, int first, int last, int *status, F f) {
  const int all = b.row_start[b.n_seqs], total = min(all, b.n_rows);
  if (all > b.n_rows && first == 0) kv_report(status);
  first = max(first, b.row_start[0]);
  last = min(last, total);
  if (first >= last) return;
  // decoding, a row per sequence: row r is sequence r's, which takes one round of loads to see
  const int guess = min(first, b.n_seqs - 1);
  int seq = b.row_start[guess] <= first && first < b.row_start[guess + 1] ? guess : kv_find_seq(b.row_start, b.n_seqs, first);
  for (int row = first; row < last;) {
    while (seq + 1 < b.n_seqs && b.row_start[seq + 1] <= row) ++seq;
    KvPiece p;
    const KvPlace place = kv_place(kv, b, block_bytes, seq, row, total, &p);
    if (place != kPlaced) kv_report(status);
    if (place == kBadRows) return;
    if (place == kPlaced && (row == b.row_start[seq] || p.slot == 0)) f(p);
    row += p.n;
  }
}

// The token whose code byte `byte` of word w of a lane is (4 r + c = lane).
template <int kBits, bool kValue>
__device__ __forceinline__ int kv_byte_token(int lane, int w, int byte) {
  const int r = lane >> 2, c = lane & 3;
  if (kBits == 4) return kValue ? 8 * (byte & 1) + 2 * c + (byte >> 1) : 8 * (byte & 1) + r;
  return kValue ? 8 * (byte >> 1) + 2 * c + (byte & 1) : 8 * (w & 1) + r;
}

// launchers; all return a rosaq_status
struct RopeTable {
  uint64_t turn[128];   // per pair: the part of a turn that one position adds, in 2^-64 turns
};
int launch_rope(int sm_count, const RopeTable &t, int head_dim, int rot_dim, int interleaved, float magnitude, const __half *x, int n_rows, long long ldx,
                int n_heads, const int32_t *positions, __half *y, long long ldy, cudaStream_t s);
int launch_kv_write(const KvView &kv, int hd, int bits, const KvBatchView &b, const __half *k, long long ldk, const __half *v, long long ldv,
                    int *status, cudaStream_t s);
int launch_kv_read(const KvView &kv, int hd, int bits, const KvBatchView &b, __half *k, long long ldk, __half *v, long long ldv, int *status,
                   cudaStream_t s);
int attend_forms(const KvView &kv, const KvBatchView &b, int prefix_tokens, int n_q_heads);   // which passes run on attend_rows.cu: the sequences' own (1), the prefix (2)
int launch_attend(rosaq_ctx *ctx, const KvView &kv, int hd, int bits, const KvBatchView &b, const int32_t *prefix_table, int prefix_tokens,
                  const __half *q, long long ldq, int n_q_heads, float scale, __half *out, long long ldo, cudaStream_t s);

// A launch that may start while the one before it drains; the kernel waits (griddepcontrol) before it touches anything.
template <typename K, typename... A>
inline int kv_launch(K kern, dim3 grid, int threads, int smem, cudaStream_t s, const A &...args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kern, args...) != cudaSuccess) {
    (void)cudaGetLastError();
    return ROSAQ_ERR_CUDA;
  }
  return ROSAQ_OK;
}

}  // namespace rosaq
