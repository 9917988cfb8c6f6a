// The parts of a query row joined: the largest M, the parts' o weighted by 2^(M_i - M) and divided by their weighted l.
// Half a wave has four channels a lane; its lanes first read one part's (M, l) each, all at once, and then all of its lanes read the
// parts' o one after the other without waiting in between.  From eight parts on a row has a whole workgroup, an eighth of the parts each half
// wave, else eight rows share it: bound by latency, not by bytes (one row's parts 3 us behind the kernel that wrote them, most of it the
// launch: with its reads beside each other it is no faster; 14 000 rows in four parts 7 us).
#include "attend_internal.h"

namespace rkv {

namespace {

// How the rows are gone through.  All parts [split][t][hq], own ones of one kind (kTokens: nothing but the row's own parts is read before
// them); of both kinds, or by unit, with others beside them (kMixed) or alone (kUnits: over the few-rows kernel's units).
enum JoinMode { kTokens, kMixed, kUnits };

template <JoinMode MODE, int SHARE>                    // SHARE: half waves per row, 1 or 8
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, int rows_per) {
  __shared__ float4 shared_o[SHARE > 1 ? 8 : 1][32];
  __shared__ float2 shared_ml[8];
  const int Hq = a.H * a.G;
  const int sub = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = (rows_per + 8 / SHARE - 1) / (8 / SHARE);
  const int outer = blockIdx.x / per, inner = (blockIdx.x - outer * per) * (8 / SHARE) + (SHARE > 1 ? 0 : sub);
  bool here = inner < rows_per, small = false;
  int token = outer, hq = inner, prefixes = a.prefix_splits;
  const int64_t slots = (int64_t)a.T * Hq;
  int64_t row, own_at, own_step = slots;
  if constexpr (MODE == kTokens) {
    here = here && token >= a.starts[0] && token < a.starts[a.P];
    small = a.small_splits > 0;
    own_at = row = (int64_t)token * Hq + hq;
  } else {
    int p;
    if constexpr (MODE == kMixed) {
      p = count_not_above(a.starts, a.P + 1, token) - 1;
      if (p < 0 || p >= a.P) return;                   // (the whole workgroup)
    } else {
      p = outer / a.H;
    }
    const Tokens tk = tokens_between(a, p, p + 1);
    small = a.small_splits > 0 && tk.count <= kSmallRows && tk.count * a.G <= a.small_rows;
    if constexpr (MODE == kUnits) {
      here = here && small && inner < tk.count * a.G;
      token = tk.first + inner / a.G;
      hq = (outer - p * a.H) * a.G + inner % a.G;
    }
    if (prefixes > 0 && group_of(a, p) < 0) prefixes = 0;
    own_at = row = (int64_t)token * Hq + hq;
    if (small) {
      const int h = hq / a.G;
      own_at = ((int64_t)p * a.small_splits * a.H + h) * a.small_rows + (token - tk.first) * a.G + (hq - h * a.G);
      own_step = (int64_t)a.H * a.small_rows;
    }
  }
  const int own = small ? a.small_splits : a.tile_splits;
  here = here && (own > 1 || a.prefix_splits > 0);     // else written whole
  if (SHARE > 1 && !here) return;
  const float* own_o = small ? a.small_o : a.tile_o;
  const float2* own_ml = small ? a.small_ml : a.tile_ml;

  // this half wave's parts: sub, sub + SHARE, ... (at most 32 of them), the prefix's first
  const int part = SHARE > 1 ? lane * SHARE + sub : lane;
  const int parts = here ? prefixes + own : 0;
  float2 ml = make_float2(-INFINITY, 0.f);
  const float* at = nullptr;
  if (part < parts) {
    const bool pre = part < prefixes;
    const int64_t slot = pre ? row + part * slots : own_at + (part - prefixes) * own_step;
    ml = (pre ? a.prefix_ml : own_ml)[slot];
    at = (pre ? a.prefix_o : own_o) + slot * kHeadDim;
  }
  float top = half_wave_max(ml.x);
  const bool some = ml.x != -INFINITY || ml.y != 0.f;              // (a part that saw nothing has written no o)
  const float weight = some ? exp2_raw(ml.x - safe_max(top)) : 0.f;
  float l = half_wave_sum(some ? ml.y * weight : 0.f);
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  const int base_lane = threadIdx.x & 32;
  const uint32_t mask = (uint32_t)(__ballot(some) >> base_lane);
  const int mine = 32 - __clz(mask);
  for (int i0 = 0; i0 < mine; i0 += 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = min(i0 + u, 31);
      const float w = __shfl(weight, base_lane + i);
      const uint64_t from = (uint64_t)__shfl((unsigned long long)(uintptr_t)at, base_lane + i);
      if ((mask >> i) & 1u && i == i0 + u) x += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(from) + lane * 4) * w;
    }
  }
  if constexpr (SHARE > 1) {
    shared_o[sub][lane] = make_float4(x[0], x[1], x[2], x[3]);
    if (lane == 0) shared_ml[sub] = make_float2(top, l);
    __syncthreads();
    if (sub != 0) return;
    float all = -INFINITY;
#pragma unroll
    for (int i = 0; i < SHARE; ++i) all = fmaxf(all, shared_ml[i].x);
    l = 0.f;
    x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < SHARE; ++i) {
      const float w = exp2_raw(shared_ml[i].x - safe_max(all));
      const float4 o = shared_o[i][lane];
      l += shared_ml[i].y * w;
      x += f32x4{o.x, o.y, o.z, o.w} * w;
    }
    top = all;
  }
  if (!here) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(a.out + token * a.ost + hq * a.osh + lane * 4) = pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if (a.lse != nullptr && lane == 0) a.lse[row] = lse_of(top, l);
}

}  // namespace

hipError_t launch_attend_join(const AttendArgs& a, hipStream_t stream) {
  // (by token alone only where every row that it reads has been written: the few-rows kernel says so of prefixes that a problem does not have)
  const JoinMode mode = a.small_by_token || (a.small_splits == 0 && a.prefix_splits == 0) ? kTokens :
                        (a.prefix_splits > 0 || a.tile_splits > 1 ? kMixed : kUnits);
  const int parts = a.prefix_splits + (a.small_splits > a.tile_splits || mode == kUnits ? a.small_splits : a.tile_splits);
  const int rows = mode == kUnits ? a.small_rows : a.H * a.G;
  const int64_t outer = mode == kUnits ? (int64_t)a.P * a.H : a.T;
  // (a workgroup per row where its parts are many and rows few, or where half a wave cannot hold them)
  const bool share = parts > 32 || (parts >= 8 && outer * rows <= 8192);
  const dim3 grid((unsigned)(outer * (share ? rows : (rows + 7) / 8)));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a, rows); };
  if (mode == kTokens) share ? go(attend_join_kernel<kTokens, 8>) : go(attend_join_kernel<kTokens, 1>);
  else if (mode == kMixed) share ? go(attend_join_kernel<kMixed, 8>) : go(attend_join_kernel<kMixed, 1>);
  else share ? go(attend_join_kernel<kUnits, 8>) : go(attend_join_kernel<kUnits, 1>);
  return hipGetLastError();
}

}  // namespace rkv
