// rosaq_rope: rotary positions.  The pair (a, b) of channels i of a head turns by t = position * f_i:
//   a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t)
// in the interleaved layout (2 i, 2 i + 1), in the half layout (i, i + rot_dim / 2).
//
// Angles: position * f_i in fp32 would be off by 0.06 radians at a million positions, so the host gives f_i as a 64-bit fraction of a turn;
// the integer product with the position is the angle modulo one turn, off by 2^-33 turns at most, and its upper 32 bits, as a signed number,
// go to sincosf with no range left to reduce (as an fp32 number of radians: up to half a turn, off by less than 2^-23 turns).  A negative position turns back.
//
// Bound: memory, and waves of CTAs that do not fill it.  A thread holds 16 channels of a head, works out their angles once and walks over the heads of its row.  Measured: 8191 rows of
// 40 heads of 128 in 35.4 us (168 MB, 4.7 TB/s; an elementwise kernel takes 28.7 over as much, the floor at the copy bandwidth is 25.6): the grid is made for eight CTAs per SM, registers
// admit four, so that these 1024 CTAs are 1.7 waves, and a thread's first loads wait for eight sines and cosines.  64 rows of 64 heads: 2.9 us.
#include <algorithm>

#include "kv_common.cuh"

namespace rosaq {
namespace {

constexpr int kThreads = 256;

struct RopeParams {
  RopeTable table;
  const __half *x;
  __half *y;
  const int32_t *positions;
  long long ldx, ldy;
  int n_rows, n_heads, heads_per_cta, head_dim, rot_dim, turns, copies;   // items of a head that turn, that are only copied
  float magnitude;
};

// kPairs: pairs of an item, eight (two accesses of 16 bytes) where rows allow them, else one
// kCopies: some items only copy (else the loads and stores need no conditions)
template <bool kInterleaved, int kPairs, bool kCopies>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ RopeParams p) {
  __shared__ uint64_t turn[128];
  for (int i = threadIdx.x; i < p.rot_dim / 2; i += kThreads) turn[i] = p.table.turn[i];
  grid_dep_launch_dependents();
  grid_dep_wait();                                   // x and the positions may be the previous kernel's output
  __syncthreads();
  const int items = p.turns + p.copies;
  const long long id = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long row = id / items;
  const int item = (int)(id - row * items);
  if (row >= p.n_rows) return;
  const int h0 = blockIdx.y * p.heads_per_cta, h1 = min(h0 + p.heads_per_cta, p.n_heads);
  const __half *x = p.x + row * p.ldx + (long long)h0 * p.head_dim;
  __half *y = p.y + row * p.ldy + (long long)h0 * p.head_dim;
  // An item is kPairs pairs that turn, or as many channels behind them that are only copied: the same loads and stores, so that the lanes of a warp stay together.
  const bool turns = !kCopies || item < p.turns;
  const int half = p.rot_dim / 2, pair = turns ? item * kPairs : 0;
  // where its channels are: 2 kPairs next to each other (interleaved), or two lots of kPairs
  const int at0 = turns ? (kInterleaved ? 2 : 1) * kPairs * item : p.rot_dim + 2 * kPairs * (item - p.turns);
  const int at1 = turns && !kInterleaved ? at0 + half : at0 + kPairs;
  const bool second = turns || at1 < p.head_dim;     // (the last copied item may have one lot only)
  float c[kPairs], s[kPairs];
  const long long pos = p.positions[row];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const int32_t t = (int32_t)(((uint64_t)pos * turn[pair + i] + 0x80000000ull) >> 32);
    sincosf((float)t * 1.4629180792671596e-9f, &s[i], &c[i]);   // 2 pi / 2^32
    s[i] *= p.magnitude, c[i] *= p.magnitude;
  }
#pragma unroll 4
  for (int h = h0; h < h1; ++h, x += p.head_dim, y += p.head_dim) {
    if (kPairs == 1) {
      const int i1 = kInterleaved ? at0 + 1 : at1;
      const __half a = x[at0], b = second ? x[i1] : a;
      const float fa = __half2float(a), fb = __half2float(b);
      y[at0] = turns ? __float2half_rn(fa * c[0] - fb * s[0]) : a;
      if (second) y[i1] = turns ? __float2half_rn(fb * c[0] + fa * s[0]) : b;
    } else if (kInterleaved) {
      uint4 va = *reinterpret_cast<const uint4 *>(x + at0), vb = second ? *reinterpret_cast<const uint4 *>(x + at1) : va;
      __half2 *const ea = reinterpret_cast<__half2 *>(&va), *const eb = reinterpret_cast<__half2 *>(&vb);
#pragma unroll
      for (int i = 0; i < kPairs / 2; ++i) {
        const int k = i + kPairs / 2;
        const float2 a = __half22float2(ea[i]), b = __half22float2(eb[i]);
        const __half2 u = __floats2half2_rn(a.x * c[i] - a.y * s[i], a.y * c[i] + a.x * s[i]);
        const __half2 w = __floats2half2_rn(b.x * c[k] - b.y * s[k], b.y * c[k] + b.x * s[k]);
        if (turns) ea[i] = u, eb[i] = w;
      }
      *reinterpret_cast<uint4 *>(y + at0) = va;
      if (second) *reinterpret_cast<uint4 *>(y + at1) = vb;
    } else {
      uint4 va = *reinterpret_cast<const uint4 *>(x + at0), vb = second ? *reinterpret_cast<const uint4 *>(x + at1) : va;
      __half2 *const ea = reinterpret_cast<__half2 *>(&va), *const eb = reinterpret_cast<__half2 *>(&vb);
#pragma unroll
      for (int i = 0; i < kPairs / 2; ++i) {
        const float2 a = __half22float2(ea[i]), b = __half22float2(eb[i]);
        const __half2 u = __floats2half2_rn(a.x * c[2 * i] - b.x * s[2 * i], a.y * c[2 * i + 1] - b.y * s[2 * i + 1]);
        const __half2 w = __floats2half2_rn(b.x * c[2 * i] + a.x * s[2 * i], b.y * c[2 * i + 1] + a.y * s[2 * i + 1]);
        if (turns) ea[i] = u, eb[i] = w;
      }
      *reinterpret_cast<uint4 *>(y + at0) = va;
      if (second) *reinterpret_cast<uint4 *>(y + at1) = vb;
    }
  }
}

}  // namespace

int launch_rope(int sm_count, const RopeTable &t, int head_dim, int rot_dim, int interleaved, float magnitude, const __half *x, int n_rows, long long ldx,
                int n_heads, const int32_t *positions, __half *y, long long ldy, cudaStream_t s) {
  RopeParams p{t, x, y, positions, ldx, ldy, n_rows, n_heads, 0, head_dim, rot_dim, 0, 0, magnitude};
  const bool wide = head_dim % 8 == 0 && rot_dim % 16 == 0;
  p.turns = wide ? rot_dim / 16 : rot_dim / 2;
  const int rest = x == y ? 0 : head_dim - rot_dim, each = wide ? 16 : 2;
  p.copies = (rest + each - 1) / each;
  const long long ctas = ((long long)n_rows * (p.turns + p.copies) + kThreads - 1) / kThreads;
  if (ctas > 0x7fffffffll) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  // Heads are shared out as long as the device is not full: the angles of a row are worked out once per share.
  const int shares = (int)std::min<long long>(std::min(n_heads, 65535), std::max<long long>(1, 8 * sm_count / ctas));
  p.heads_per_cta = (n_heads + shares - 1) / shares;
  const dim3 grid((unsigned)ctas, (n_heads + p.heads_per_cta - 1) / p.heads_per_cta);
  auto go = [&](auto with, auto without) { return p.copies ? kv_launch(with, grid, kThreads, 0, s, p) : kv_launch(without, grid, kThreads, 0, s, p); };
  if (interleaved) return wide ? go(rope_kernel<true, 8, true>, rope_kernel<true, 8, false>) : go(rope_kernel<true, 1, true>, rope_kernel<true, 1, false>);
  return wide ? go(rope_kernel<false, 8, true>, rope_kernel<false, 8, false>) : go(rope_kernel<false, 1, true>, rope_kernel<false, 1, false>);
}

}  // namespace rosaq
