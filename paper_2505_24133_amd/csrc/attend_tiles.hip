// Attention of many rows of queries per KV head (prompts, chunks of prompts, the queries of a group over its shared prefix): bound by
// the matrix pipe and by the exponentials.
//
// A workgroup has a tile of 128 query rows (new token, head of the group) of one KV head, 32 a wave, and walks over the cache rows that one
// of them sees, 64 at a time: copied to LDS by DMA one tile ahead, one barrier a tile.  S^T = K Q^T by MFMA 32x32x16: a lane has one
// query and half of the tile's rows, so that maxima and sums are register arithmetic and one exchange between the halves of the
// wave, and the weights are, without any movement, the second operand of O^T += V^T P^T.  V^T comes out of LDS by the transposing read.
// Two workgroups share a compute unit, so that one's products run beside the other's exponentials.
#include "attend_internal.h"

namespace rkv {

namespace {

constexpr int kKeys = 64;                            // cache rows of a step
constexpr int kKeyBytes = kKeys * kRowBytes;
constexpr int kThreads = 256;
constexpr float kSlack = 8.f;        // a maximum that grows by less than 2^8 leaves the weights' reference where it is (they stay below 2^8)

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) x = min(x, __shfl_xor(x, m));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) x = max(x, __shfl_xor(x, m));
  return __builtin_amdgcn_readfirstlane(x);
}

// PREFIX: the query rows are those of a group's problems, the cache rows the group's shared ones.
template <bool PAGED, bool PREFIX>
__global__ __launch_bounds__(kThreads, 2) void attend_tiles_kernel(AttendArgs a, int splits) {
  __shared__ __attribute__((aligned(256))) unsigned char lds[2 * 2 * kKeyBytes];
  __shared__ int bounds[4][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int h = blockIdx.x % a.H;
  const int rest = blockIdx.x / a.H;
  const int split = rest % splits;

  // the problem (or group) that this tile belongs to, and which of its tiles it is: the tiles of all problems are counted through
  int tile = rest / splits, owner = -1;
  Tokens tk{0, 0};
  const int owners = PREFIX ? a.groups : a.P;
  for (int at = 0; at < owners; at += 64) {
    const int o = at + lane;
    Tokens mine{0, 0};
    if (o < owners) mine = PREFIX ? tokens_between(a, clampi(a.group_starts[o], 0, a.P), clampi(a.group_starts[o + 1], 0, a.P)) : tokens_between(a, o, o + 1);
    const bool small = !PREFIX && a.small_splits > 0 && (int64_t)mine.count * a.G <= a.small_rows;
    const int tiles = small ? 0 : (int)(((int64_t)mine.count * a.G + kTileRows - 1) / kTileRows);
    const int upto = (int)wave_inclusive_scan((uint32_t)tiles);
    const uint64_t past = __ballot(upto > tile);
    if (past != 0) {
      const int l = __ffsll((unsigned long long)past) - 1;
      owner = at + l;
      tk.first = __shfl(mine.first, l);
      tk.count = __shfl(mine.count, l);
      tile = __shfl(upto, l) - 1 - tile;               // the last tile, which sees the most rows, first
      break;
    }
    tile -= __shfl(upto, 63);
  }
  if (owner < 0) return;
  owner = __builtin_amdgcn_readfirstlane(owner);
  tk.first = __builtin_amdgcn_readfirstlane(tk.first);
  tk.count = __builtin_amdgcn_readfirstlane(tk.count);
  tile = __builtin_amdgcn_readfirstlane(tile);

  // this lane's query: element j of step s is channel 16 s + 8 (lane >> 5) + j
  const int rows = tk.count * a.G;
  const int col = lane & 31, half = lane >> 5;
  const int row = tile * kTileRows + wave * 32 + col;
  const int j = min(row, rows - 1) / a.G;
  const int g = min(row, rows - 1) - j * a.G;
  const int token = tk.first + j, hq = h * a.G + g;
  bf16x8 qf[8];
  const uint16_t* qr = a.q + (int64_t)token * a.qst + (int64_t)hq * a.qsh + half * 8;
#pragma unroll
  for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qr + s * 16);

  int p0 = owner, base = 0, lim = a.N;
  Sight see;
  if constexpr (PREFIX) {
    p0 = clampi(a.group_starts[owner], 0, a.P - 1);
    lim = prefix_of(a, owner);
    // the problem of the lane's token: the last one of the group that starts at or before it
    int lo = p0, hi = clampi(a.group_starts[owner + 1], p0 + 1, a.P);
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.starts[mid] <= token) lo = mid; else hi = mid;
    }
    const int end = clampi(a.starts[lo + 1], 0, a.T);
    see = sight(a, clampi(a.kv_len[lo], 0, a.N) - (end - token));
  } else {
    base = prefix_of(a, group_of(a, owner));
    see = sight(a, clampi(a.kv_len[owner], 0, a.N) - (tk.count - j));
  }
  const int sinks = a.window > 0 ? a.sinks : 0;
  const int hi_min = wave_min(see.hi), hi_max = wave_max(see.hi), lo_min = wave_min(see.lo), lo_max = wave_max(see.lo);
  if (lane == 0) {
    bounds[wave][0] = hi_max;
    bounds[wave][1] = lo_min;
  }
  __syncthreads();
  const int all_hi = max(max(bounds[0][0], bounds[1][0]), max(bounds[2][0], bounds[3][0]));
  const int all_lo = min(min(bounds[0][1], bounds[1][1]), min(bounds[2][1], bounds[3][1]));
  const Span<kKeys> span(base, lim, __builtin_amdgcn_readfirstlane(all_lo), __builtin_amdgcn_readfirstlane(all_hi), sinks);
  const int used = clampi(span.tiles, 1, splits);
  const int t_lo = split < used ? (int)((int64_t)span.tiles * split / used) : 0;
  const int t_hi = split < used ? (int)((int64_t)span.tiles * (split + 1) / used) : 0;

  f32x16 o[4];
  float mx = -INFINITY, sum = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  Rows<PAGED> rs(a, p0, h);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
  auto copy = [&](int t, int buf) {
    const int start = span.start(t), end = span.end(t);
    rs.reload(start, min(start + kKeys, end) - 1);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + buf * 2 * kKeyBytes + wave * 16 * kRowBytes);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int r = wave * 16 + c * 4 + (lane >> 4);
      const uint16_t *kp, *vp;
      rs.find(min(start + r, end - 1), key_chunk(r, lane & 15), value_chunk(r, lane & 15), &kp, &vp);
      dma16_from(kp, to + c * 1024);
      dma16_from(vp, to + kKeyBytes + c * 1024);
    }
  };

  if (t_lo < t_hi) copy(t_lo, 0);
  for (int t = t_lo; t < t_hi; ++t) {
    const int buf = (t - t_lo) & 1;
    // this wave's copies have arrived and its reads of the other buffer are done; behind the barrier that holds for all
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 1 < t_hi) copy(t + 1, buf ^ 1);
    const int start = span.start(t), stop = min(span.end(t), start + kKeys);
    if (start >= hi_max || (stop <= lo_min && start >= sinks)) continue;      // none of this wave's queries sees any of it
    const uint32_t kt = lds0 + buf * 2 * kKeyBytes, vt = kt + kKeyBytes;
    f32x16 s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int st = 0; st < 8; ++st)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int r = b * 32 + col;
        const bf16x8 kf = *(__attribute__((address_space(3))) const bf16x8*)(uintptr_t)(kt + r * kRowBytes + (key_chunk(r, 2 * st + half) << 4));
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], s[b], 0, 0, 0);
      }
    // element i of block b is row 32 b + 8 (i >> 2) + 4 half + (i & 3)
    const bool edge = !(start + kKeys <= min(hi_min, span.end(t)) && (start >= lo_max || start + kKeys <= sinks));
    if (edge) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int c = start + b * 32 + 8 * (i >> 2) + 4 * half + (i & 3);
          const bool seen = c < min(see.hi, stop) && (c >= see.lo || c < sinks);
          s[b][i] = seen ? s[b][i] : -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[1][i]);
    top = fmaxf(top, __shfl_xor(top, 32)) * a.scale2;
    // the reference moves only where some query's maximum has outgrown it
    if (__any(top > mx + kSlack || mx == -INFINITY)) {
      const float next = fmaxf(mx, top);
      const float fade = exp2_raw(mx - safe_max(next));
      mx = next;
      sum *= fade;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= fade;
    }
    const float ref = safe_max(mx);
    Frag pf[4];
    float add = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = exp2_raw(__fmaf_rn(s[b][i], a.scale2, -ref));
        add += w;
        pf[2 * b + (i >> 3)].b[i & 7] = (__bf16)w;
      }
    sum += add;                                          // of this lane's rows; the two halves are added up at the end
    // values: block d has channels 16 d .. 16 d + 15 and 64 + 16 d ..; element j of step st is row 16 st + 8 (j >> 2) + 4 half + (j & 3)
    const int vrow = 4 * half + ((lane & 15) >> 2);
    const int vchunk = 8 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      Frag vf[4];
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int jh = 0; jh < 2; ++jh) {
          const int r = 16 * st + 8 * jh + vrow;
          vf[st].s[jh] = read_transposed(vt + r * kRowBytes + (value_chunk(r, 2 * d + vchunk) << 4) + ((lane & 1) << 3));
        }
      if (edge && __any(not_finite(vf[0]) | not_finite(vf[1]) | not_finite(vf[2]) | not_finite(vf[3]))) {
        f32x16 ups, downs;
#pragma unroll
        for (int i = 0; i < 16; ++i) ups[i] = downs[i] = 0.f;
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          Frag up, down;
          split_not_finite(vf[st], up, down);
          const Frag w = given_weight(pf[st]);
          ups = __builtin_amdgcn_mfma_f32_32x32x16_bf16(up.b, w.b, ups, 0, 0, 0);
          downs = __builtin_amdgcn_mfma_f32_32x32x16_bf16(down.b, w.b, downs, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (ups[i] > 0.f) o[d][i] += INFINITY;
          if (downs[i] > 0.f) o[d][i] -= INFINITY;
        }
      }
#pragma unroll
      for (int st = 0; st < 4; ++st) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[st].b, pf[st].b, o[d], 0, 0, 0);
    }
  }

  sum += __shfl_xor(sum, 32);
  if (row >= rows) return;
  const int64_t at = (int64_t)token * (a.H * a.G) + hq;
  if (!PREFIX && splits == 1 && a.prefix_splits == 0) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* to = a.out + (int64_t)token * a.ost + (int64_t)hq * a.osh + 4 * half;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<uint2*>(to + 64 * (i >> 3) + 16 * d + 8 * ((i >> 2) & 1)) = pack4(o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv);
    if (a.lse != nullptr && half == 0) a.lse[at] = lse_of(mx, sum);
  } else {
    const int64_t slot = (int64_t)split * a.T * (a.H * a.G) + at;
    float* to = (PREFIX ? a.prefix_o : a.tile_o) + slot * kHeadDim + 4 * half;
    if (t_lo < t_hi)
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(to + 64 * (i >> 3) + 16 * d + 8 * ((i >> 2) & 1)) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
    if (half == 0) (PREFIX ? a.prefix_ml : a.tile_ml)[slot] = make_float2(mx, sum);
  }
}

}  // namespace

// The most tiles that T tokens of `owners` problems or groups can make.
int64_t attend_tile_bound(int64_t T, int G, int64_t owners) { return T * G / kTileRows + (owners < T ? owners : T); }

hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool prefix, hipStream_t stream) {
  const int splits = prefix ? a.prefix_splits : a.tile_splits;
  const dim3 grid((unsigned)(attend_tile_bound(a.T, a.G, prefix ? a.groups : a.P) * a.H * splits));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a, splits); };
  if (prefix) paged ? go(attend_tiles_kernel<true, true>) : go(attend_tiles_kernel<false, true>);
  else paged ? go(attend_tiles_kernel<true, false>) : go(attend_tiles_kernel<false, false>);
  return hipGetLastError();
}

}  // namespace rkv
