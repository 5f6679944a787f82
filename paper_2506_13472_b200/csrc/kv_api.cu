// extern "C" entry points of the operators between the q/k/v linears and the o_proj rotation: rotary positions, the paged cache of
// quantized keys and values, and the attention that reads it.  Argument checks and dispatch.
#include <algorithm>
#include <cmath>
#include <new>

#include "kv_common.cuh"

using namespace rosaq;

struct rosaq_rope {
  RopeTable table;
  int head_dim, rot_dim, interleaved;
  float magnitude;
};

namespace {

int check_rows(const void *p, int n_rows, int64_t ld, int64_t d) {
  if (n_rows < 0 || (!p && n_rows > 0) || ld < d) return ROSAQ_ERR_INVALID_ARG;
  if (!aligned16(p) || (ld % 8) != 0) return ROSAQ_ERR_ALIGNMENT;
  return ROSAQ_OK;
}

int check_kv(const rosaq_kv *kv, KvView *out) {
  if (!kv || !kv->pages || kv->n_pages < 1) return ROSAQ_ERR_INVALID_ARG;
  const int64_t bytes = rosaq_kv_page_bytes(kv->n_kv_heads, kv->head_dim, kv->bits, kv->page_tokens);
  if (bytes < 0) return (int)bytes;
  if (!aligned16(kv->pages)) return ROSAQ_ERR_ALIGNMENT;
  int shift = 0;
  while ((kKvBlock << shift) < kv->page_tokens) ++shift;
  *out = KvView{static_cast<uint8_t *>(kv->pages), bytes, kv->n_pages, shift, kv->n_kv_heads};
  return ROSAQ_OK;
}

int check_batch(const rosaq_kv_batch *b, const rosaq_kv *kv, int n_rows, KvBatchView *out) {
  if (b && b->n_seqs == 0 && n_rows == 0) {         // nothing of it is looked at
    *out = KvBatchView{};
    return ROSAQ_OK;
  }
  if (!b || b->n_seqs < 1 || b->ld_table < 1 || !b->row_start || !b->kv_len || !b->table) return ROSAQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(b->row_start) | reinterpret_cast<uintptr_t>(b->kv_len) | reinterpret_cast<uintptr_t>(b->table)) & 3)
    return ROSAQ_ERR_ALIGNMENT;
  if (b->table_pages < 0 || b->table_pages > b->ld_table) return ROSAQ_ERR_INVALID_ARG;
  const int width = b->table_pages > 0 ? b->table_pages : b->ld_table;
  if ((int64_t)width * kv->page_tokens > (int64_t)1 << 30) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  *out = KvBatchView{b->row_start, b->kv_len, b->table, b->n_seqs, b->ld_table, width, n_rows};
  return ROSAQ_OK;
}

// rows of fp16 against the pages of a cache
bool in_pages(const KvView &kv, const void *p, int n_rows, int64_t ld, int64_t d) {
  const char *const lo = static_cast<const char *>(p), *const hi = lo + sizeof(__half) * ((size_t)(n_rows - 1) * (size_t)ld + (size_t)d);
  const char *const a = reinterpret_cast<const char *>(kv.pages), *const b = a + kv.page_bytes * kv.n_pages;
  return lo < b && a < hi;
}

}  // namespace

extern "C" {

int rosaq_rope_create(rosaq_ctx *ctx, const rosaq_rope_desc *d, rosaq_rope **out) {
  if (!out) return ROSAQ_ERR_INVALID_ARG;
  *out = nullptr;
  if (!ctx || !d || d->head_dim < 2 || d->rot_dim < 2 || d->rot_dim > d->head_dim || d->rot_dim % 2 != 0) return ROSAQ_ERR_INVALID_ARG;
  if (d->interleaved != 0 && d->interleaved != 1) return ROSAQ_ERR_INVALID_ARG;
  if (!(d->base > 0) || !std::isfinite(d->base) || !std::isfinite(d->magnitude)) return ROSAQ_ERR_INVALID_ARG;
  if (d->scaling < ROSAQ_ROPE_PLAIN || d->scaling > ROSAQ_ROPE_BY_PARTS) return ROSAQ_ERR_INVALID_ARG;
  if (d->scaling != ROSAQ_ROPE_PLAIN && (!(d->factor > 0) || !std::isfinite(d->factor))) return ROSAQ_ERR_INVALID_ARG;
  if (d->scaling == ROSAQ_ROPE_NTK && d->rot_dim < 4) return ROSAQ_ERR_INVALID_ARG;
  if (d->scaling == ROSAQ_ROPE_BY_PARTS &&
      (!(d->low >= 0) || !(d->high > d->low) || !std::isfinite(d->high) || !(d->context > 0) || !std::isfinite(d->context)))
    return ROSAQ_ERR_INVALID_ARG;
  if (d->rot_dim > 256 || d->head_dim > 65536) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  rosaq_rope *r = new (std::nothrow) rosaq_rope();
  if (!r) return ROSAQ_ERR_ALLOC;
  r->head_dim = d->head_dim, r->rot_dim = d->rot_dim, r->interleaved = d->interleaved, r->magnitude = d->magnitude;
  const long double two_pi = 6.283185307179586476925286766559L;
  const double base = d->scaling == ROSAQ_ROPE_NTK ? d->base * std::pow(d->factor, (double)d->rot_dim / (d->rot_dim - 2)) : d->base;
  for (int i = 0; i < d->rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / d->rot_dim);
    if (d->scaling == ROSAQ_ROPE_LINEAR) f /= d->factor;
    if (d->scaling == ROSAQ_ROPE_BY_PARTS) {
      const double turns = d->context * f / (double)two_pi, keep = std::fmin(std::fmax((turns - d->low) / (d->high - d->low), 0.0), 1.0);
      f *= keep + (1.0 - keep) / d->factor;
    }
    if (!std::isfinite(f)) {
      delete r;
      return ROSAQ_ERR_INVALID_ARG;
    }
    const long double turn = (long double)f / two_pi, part = turn - std::floor(turn);   // positions are whole numbers: whole turns drop out
    const long double scaled = std::floor(part * 18446744073709551616.0L + 0.5L);
    r->table.turn[i] = scaled >= 18446744073709551616.0L ? 0 : (uint64_t)scaled;
  }
  *out = r;
  return ROSAQ_OK;
}

int rosaq_rope_free(rosaq_rope *r) {
  if (!r) return ROSAQ_ERR_INVALID_ARG;
  delete r;
  return ROSAQ_OK;
}

int rosaq_rope_apply(rosaq_ctx *ctx, const rosaq_rope *r, const void *x, int n_rows, int64_t ldx, int n_heads, const int32_t *positions,
                     void *y, int64_t ldy, void *stream) {
  if (!ctx || !r || n_heads < 1) return ROSAQ_ERR_INVALID_ARG;
  const int64_t d = (int64_t)n_heads * r->head_dim;
  int st = check_rows(x, n_rows, ldx, d);
  if (st == ROSAQ_OK) st = check_rows(y, n_rows, ldy, d);
  if (st == ROSAQ_OK && !positions && n_rows > 0) st = ROSAQ_ERR_INVALID_ARG;
  if (st == ROSAQ_OK && (reinterpret_cast<uintptr_t>(positions) & 3)) st = ROSAQ_ERR_ALIGNMENT;
  if (st != ROSAQ_OK || n_rows == 0) return st;
  if (!(x == y && ldx == ldy) && views_overlap(n_rows, x, ldx, d, y, ldy, d)) return ROSAQ_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return ROSAQ_ERR_CUDA;
  return launch_rope(ctx->sm_count, r->table, r->head_dim, r->rot_dim, r->interleaved, r->magnitude, static_cast<const __half *>(x), n_rows,
                     ldx, n_heads, positions, static_cast<__half *>(y), ldy, static_cast<cudaStream_t>(stream));
}

int64_t rosaq_kv_page_bytes(int n_kv_heads, int head_dim, int bits, int page_tokens) {
  if (n_kv_heads < 1 || page_tokens < 1 || (bits != 4 && bits != 8)) return ROSAQ_ERR_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || n_kv_heads > 65536) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  if (page_tokens < kKvBlock || page_tokens > 1024 || (page_tokens & (page_tokens - 1)) != 0) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  return (int64_t)n_kv_heads * (page_tokens / kKvBlock) * kv_block_bytes(head_dim, bits);
}

int rosaq_kv_locate(const rosaq_kv *kv, const rosaq_kv_batch *batch, int n_rows, int64_t *offset, int32_t *slot) {
  KvView view;
  KvBatchView b;
  int st = check_kv(kv, &view);
  if (st == ROSAQ_OK) st = check_batch(batch, kv, n_rows, &b);
  if (st == ROSAQ_OK && (n_rows < 0 || !offset || !slot)) st = ROSAQ_ERR_INVALID_ARG;
  if (st != ROSAQ_OK || b.n_seqs == 0) return st;
  for (int i = 0; i < n_rows; ++i) offset[i] = slot[i] = -1;
  const int all = b.row_start[b.n_seqs], total = std::min(all, n_rows), bytes = kv_block_bytes(kv->head_dim, kv->bits);
  if (all > n_rows) st = ROSAQ_ERR_INVALID_ARG;
  int seq = 0;
  for (int row = std::max(b.row_start[0], 0); row < total;) {
    while (seq + 1 < b.n_seqs && b.row_start[seq + 1] <= row) ++seq;
    KvPiece p;
    const KvPlace place = kv_place(view, b, bytes, seq, row, total, &p);
    if (place != kPlaced) st = ROSAQ_ERR_INVALID_ARG;
    if (place == kBadRows) break;
    for (int i = 0; place == kPlaced && i < p.n; ++i) offset[row + i] = p.offset, slot[row + i] = p.slot + i;
    row += p.n;
  }
  return st;
}

int rosaq_kv_write(rosaq_ctx *ctx, const rosaq_kv *kv, const rosaq_kv_batch *batch, const void *k, int64_t ldk, const void *v, int64_t ldv,
                   int n_rows, void *stream) {
  if (!ctx) return ROSAQ_ERR_INVALID_ARG;
  KvView view;
  KvBatchView b;
  int st = check_kv(kv, &view);
  if (st == ROSAQ_OK) st = check_batch(batch, kv, n_rows, &b);
  const int64_t d = st == ROSAQ_OK ? (int64_t)kv->n_kv_heads * kv->head_dim : 0;
  if (st == ROSAQ_OK) st = check_rows(k, n_rows, ldk, d);
  if (st == ROSAQ_OK) st = check_rows(v, n_rows, ldv, d);
  if (st != ROSAQ_OK || n_rows == 0) return st;
  if (in_pages(view, k, n_rows, ldk, d) || in_pages(view, v, n_rows, ldv, d)) return ROSAQ_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return ROSAQ_ERR_CUDA;
  return launch_kv_write(view, kv->head_dim, kv->bits, b, static_cast<const __half *>(k), ldk, static_cast<const __half *>(v), ldv,
                         ctx->d_status, static_cast<cudaStream_t>(stream));
}

int rosaq_kv_read(rosaq_ctx *ctx, const rosaq_kv *kv, const rosaq_kv_batch *batch, void *k, int64_t ldk, void *v, int64_t ldv, int n_rows,
                  void *stream) {
  if (!ctx) return ROSAQ_ERR_INVALID_ARG;
  KvView view;
  KvBatchView b;
  int st = check_kv(kv, &view);
  if (st == ROSAQ_OK) st = check_batch(batch, kv, n_rows, &b);
  const int64_t d = st == ROSAQ_OK ? (int64_t)kv->n_kv_heads * kv->head_dim : 0;
  if (st == ROSAQ_OK) st = check_rows(k, n_rows, ldk, d);
  if (st == ROSAQ_OK) st = check_rows(v, n_rows, ldv, d);
  if (st != ROSAQ_OK || n_rows == 0) return st;
  if (in_pages(view, k, n_rows, ldk, d) || in_pages(view, v, n_rows, ldv, d) || views_overlap(n_rows, k, ldk, d, v, ldv, d))
    return ROSAQ_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return ROSAQ_ERR_CUDA;
  return launch_kv_read(view, kv->head_dim, kv->bits, b, static_cast<__half *>(k), ldk, static_cast<__half *>(v), ldv, ctx->d_status,
                        static_cast<cudaStream_t>(stream));
}

int rosaq_attend_forms(const rosaq_kv *kv, const rosaq_kv_batch *batch, int n_rows, int n_q_heads) {
  KvView view;
  KvBatchView b;
  int st = check_kv(kv, &view);
  if (st == ROSAQ_OK) st = check_batch(batch, kv, n_rows, &b);
  if (st != ROSAQ_OK) return st;
  if (n_rows < 0 || n_q_heads < 1 || batch->prefix_tokens < 0) return ROSAQ_ERR_INVALID_ARG;
  if (n_q_heads % kv->n_kv_heads != 0) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  return n_rows == 0 ? 0 : attend_forms(view, b, batch->prefix_tokens, n_q_heads);
}

int rosaq_attend(rosaq_ctx *ctx, const rosaq_kv *kv, const rosaq_kv_batch *batch, const void *q, int64_t ldq, int n_q_heads, float scale,
                 void *out, int64_t ldo, int n_rows, void *stream) {
  if (!ctx || n_q_heads < 1) return ROSAQ_ERR_INVALID_ARG;
  // scores of fp16 numbers stay below 2^99.2 then, above what the kernels take for a row that has seen nothing (-10^30)
  if (!(std::fabs(scale) <= 288230376151711744.f)) return ROSAQ_ERR_INVALID_ARG;
  KvView view;
  KvBatchView b;
  int st = check_kv(kv, &view);
  if (st == ROSAQ_OK) st = check_batch(batch, kv, n_rows, &b);
  if (st != ROSAQ_OK) return st;
  if (n_q_heads % kv->n_kv_heads != 0) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  const int64_t d = (int64_t)n_q_heads * kv->head_dim;
  if (batch->prefix_tokens < 0 || (batch->prefix_tokens > 0 && !batch->prefix_table)) return ROSAQ_ERR_INVALID_ARG;
  if (batch->prefix_tokens > 1 << 30) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  if (batch->prefix_tokens > 0 && (reinterpret_cast<uintptr_t>(batch->prefix_table) & 3)) return ROSAQ_ERR_ALIGNMENT;
  if ((int64_t)n_rows * n_q_heads > (int64_t)1 << 30) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  st = check_rows(q, n_rows, ldq, d);
  if (st == ROSAQ_OK) st = check_rows(out, n_rows, ldo, d);
  if (st != ROSAQ_OK || n_rows == 0) return st;
  if (in_pages(view, out, n_rows, ldo, d)) return ROSAQ_ERR_INVALID_ARG;
  // q may be overwritten by its own result: a row's head is written when every CTA that reads it has
  if (!(q == out && ldq == ldo) && views_overlap(n_rows, q, ldq, d, out, ldo, d)) return ROSAQ_ERR_INVALID_ARG;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return ROSAQ_ERR_CUDA;
  return launch_attend(ctx, view, kv->head_dim, kv->bits, b, batch->prefix_table, batch->prefix_tokens, static_cast<const __half *>(q), ldq,
                       n_q_heads, scale, static_cast<__half *>(out), ldo, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
