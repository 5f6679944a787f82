// rosaq_rope: rotary positions.  The pair (a, b) of channels i of a head turns by t = position * f_i:
//   a' = m (a cos t - b sin t),  b' = m (b cos t + a sin t)
// in the interleaved layout (2 i, 2 i + 1), in the half layout (i, i + rot_dim / 2).
//
// Angles: position * f_i in fp32 would be off by 0.06 radians at a million positions, so the host gives f_i as a 64-bit fraction of a turn;
// the integer product with the position is the angle modulo one turn, off by 2^-33 turns at most, and its upper 32 bits, as a signed number,
// go to sincosf with no range left to reduce.  A negative position turns back.
//
// Bound: memory.  A thread holds 16 (interleaved: 8) channels of a head, works out their angles once and walks over the heads of its row.
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
  int n_rows, n_heads, heads_per_cta, head_dim, rot_dim, turns, copies;   // work items of a head that turn, and that are only copied
  float magnitude;
};

// kPairs: pairs of a work item, 8 in the half layout and 4 in the interleaved one, where rows allow 16-byte accesses, else 1
template <bool kInterleaved, int kPairs>
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
  if (item >= p.turns) {                             // behind the part that turns
    constexpr int kCopy = kPairs > 1 ? 8 : 1;
    const int at = p.rot_dim + (item - p.turns) * kCopy;
    for (int h = h0; h < h1; ++h, x += p.head_dim, y += p.head_dim) {
      if (kCopy == 8) *reinterpret_cast<uint4 *>(y + at) = *reinterpret_cast<const uint4 *>(x + at);
      else y[at] = x[at];
    }
    return;
  }
  const int first = item * kPairs, half = p.rot_dim / 2;
  float c[kPairs], s[kPairs];
  const long long pos = p.positions[row];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const int32_t t = (int32_t)(((uint64_t)pos * turn[first + i] + 0x80000000ull) >> 32);
    sincosf((float)t * 1.4629180792671596e-9f, &s[i], &c[i]);   // 2 pi / 2^32
    s[i] *= p.magnitude, c[i] *= p.magnitude;
  }
#pragma unroll 2
  for (int h = h0; h < h1; ++h, x += p.head_dim, y += p.head_dim) {
    if (kPairs == 1) {
      const int ia = kInterleaved ? 2 * first : first, ib = kInterleaved ? ia + 1 : first + half;
      const float a = __half2float(x[ia]), b = __half2float(x[ib]);
      y[ia] = __float2half_rn(a * c[0] - b * s[0]);
      y[ib] = __float2half_rn(b * c[0] + a * s[0]);
    } else if (kInterleaved) {
      uint4 v = *reinterpret_cast<const uint4 *>(x + 2 * first);
      __half2 *const e = reinterpret_cast<__half2 *>(&v);
#pragma unroll
      for (int i = 0; i < (kInterleaved ? kPairs : 0); ++i) {
        const float2 u = __half22float2(e[i]);
        e[i] = __floats2half2_rn(u.x * c[i] - u.y * s[i], u.y * c[i] + u.x * s[i]);
      }
      *reinterpret_cast<uint4 *>(y + 2 * first) = v;
    } else {
      uint4 va = *reinterpret_cast<const uint4 *>(x + first), vb = *reinterpret_cast<const uint4 *>(x + first + half);
      __half2 *const ea = reinterpret_cast<__half2 *>(&va), *const eb = reinterpret_cast<__half2 *>(&vb);
#pragma unroll
      for (int i = 0; i < kPairs / 2; ++i) {
        const float2 a = __half22float2(ea[i]), b = __half22float2(eb[i]);
        ea[i] = __floats2half2_rn(a.x * c[2 * i] - b.x * s[2 * i], a.y * c[2 * i + 1] - b.y * s[2 * i + 1]);
        eb[i] = __floats2half2_rn(b.x * c[2 * i] + a.x * s[2 * i], b.y * c[2 * i + 1] + a.y * s[2 * i + 1]);
      }
      *reinterpret_cast<uint4 *>(y + first) = va;
      *reinterpret_cast<uint4 *>(y + first + half) = vb;
    }
  }
}

}  // namespace

int launch_rope(int sm_count, const RopeTable &t, int head_dim, int rot_dim, int interleaved, float magnitude, const __half *x, int n_rows, long long ldx,
                int n_heads, const int32_t *positions, __half *y, long long ldy, cudaStream_t s) {
  RopeParams p{t, x, y, positions, ldx, ldy, n_rows, n_heads, 0, head_dim, rot_dim, 0, 0, magnitude};
  const bool wide = head_dim % 8 == 0 && rot_dim % (interleaved ? 8 : 16) == 0;
  p.turns = wide ? rot_dim / (interleaved ? 8 : 16) : rot_dim / 2;
  p.copies = x == y ? 0 : (head_dim - rot_dim) / (wide ? 8 : 1);
  const long long ctas = ((long long)n_rows * (p.turns + p.copies) + kThreads - 1) / kThreads;
  if (ctas > 0x7fffffffll) return ROSAQ_ERR_UNSUPPORTED_SHAPE;
  // Heads are shared out as long as the device is not full: the angles of a row are worked out once per share.
  const int shares = (int)std::min<long long>(std::min(n_heads, 65535), std::max<long long>(1, 8 * sm_count / ctas));
  p.heads_per_cta = (n_heads + shares - 1) / shares;
  const dim3 grid((unsigned)ctas, (n_heads + p.heads_per_cta - 1) / p.heads_per_cta);
  if (interleaved) return wide ? kv_launch(rope_kernel<true, 4>, grid, kThreads, 0, s, p) : kv_launch(rope_kernel<true, 1>, grid, kThreads, 0, s, p);
  return wide ? kv_launch(rope_kernel<false, 8>, grid, kThreads, 0, s, p) : kv_launch(rope_kernel<false, 1>, grid, kThreads, 0, s, p);
}

}  // namespace rosaq
