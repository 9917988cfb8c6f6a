// The parts of a query row joined: the largest M, the parts' o weighted by 2^(M_i - M) and divided by their weighted l.
// A row has 32 threads of four channels each; the few (M, l) of its parts are read by all of them.
#include "attend_internal.h"

namespace rkv {

namespace {

// PER_TOKEN: blocks over all (token, head) rows; otherwise over the rows of the few-rows kernel alone.
template <bool PER_TOKEN>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, int blocks_per) {
  const int Hq = a.H * a.G;
  const int outer = blockIdx.x / blocks_per, inner = (blockIdx.x - outer * blocks_per) * 8 + (threadIdx.x >> 5);
  const int piece = threadIdx.x & 31;
  int p, token, hq, count, first;
  if constexpr (PER_TOKEN) {
    token = outer; hq = inner;
    p = count_not_above(a.starts, a.P + 1, token) - 1;
    if (p < 0 || p >= a.P) return;
    const Tokens tk = tokens_between(a, p, p + 1);
    count = tk.count; first = tk.first;
    if (hq >= Hq) return;
  } else {
    p = outer / a.H;
    const Tokens tk = tokens_between(a, p, p + 1);
    count = tk.count; first = tk.first;
    if (count > kSmallRows || inner >= count * a.G) return;
    token = first + inner / a.G;
    hq = (outer - p * a.H) * a.G + inner % a.G;
  }
  const int h = hq / a.G;
  const int64_t row = (int64_t)token * Hq + hq, slots = (int64_t)a.T * Hq;
  const bool small = a.small_splits > 0 && count <= kSmallRows && count * a.G <= a.small_rows;
  const int prefixes = group_of(a, p) >= 0 ? a.prefix_splits : 0;
  const int own = small ? a.small_splits : a.tile_splits;
  if (own == 0 || (own == 1 && a.prefix_splits == 0)) return;     // written whole, or by nobody
  // the parts behind the prefix's lie `own_step` apart
  const int64_t own_at = small ? ((int64_t)p * a.small_splits * a.H + h) * a.small_rows + (token - first) * a.G + (hq - h * a.G) : row;
  const int64_t own_step = small ? (int64_t)a.H * a.small_rows : slots;
  const float* own_o = small ? a.small_o : a.tile_o;
  const float2* own_ml = small ? a.small_ml : a.tile_ml;

  float top = -INFINITY, l = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  auto take = [&](const float2* mls, const float* os, int64_t at, int64_t step, int n) {
    for (int i = 0; i < n; ++i, at += step) {
      const float2 part = mls[at];
      if (part.x == -INFINITY && part.y == 0.f) continue;        // nothing visible there (its o is not written)
      const float next = fmaxf(top, part.x);
      const float fade = exp2_raw(top - safe_max(next)), weight = exp2_raw(part.x - safe_max(next));
      x = x * fade + *reinterpret_cast<const f32x4*>(os + at * kHeadDim + piece * 4) * weight;
      l = l * fade + part.y * weight;
      top = next;
    }
  };
  take(a.prefix_ml, a.prefix_o, row, slots, prefixes);
  take(own_ml, own_o, own_at, own_step, own);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(a.out + token * a.ost + hq * a.osh + piece * 4) = pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if (a.lse != nullptr && piece == 0) a.lse[row] = lse_of(top, l);
}

}  // namespace

hipError_t launch_attend_join(const AttendArgs& a, bool per_token, hipStream_t stream) {
  if (per_token) {
    const int per = (a.H * a.G + 7) / 8;
    hipLaunchKernelGGL(attend_join_kernel<true>, dim3((unsigned)((int64_t)a.T * per)), dim3(256), 0, stream, a, per);
  } else {
    const int per = a.small_rows / 8;
    hipLaunchKernelGGL(attend_join_kernel<false>, dim3((unsigned)((int64_t)a.P * a.H * per)), dim3(256), 0, stream, a, per);
  }
  return hipGetLastError();
}

}  // namespace rkv
