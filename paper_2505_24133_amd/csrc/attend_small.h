// Attention of few rows of queries per KV head (single tokens, some tokens of a draft): bound by reading the cache.
//
// A workgroup has one (problem, KV head) and a share of its rows; its two waves take parts of that share, each by itself: rows are copied to
// LDS by DMA in tiles of 32, two tiles in the wave's own buffers, so that no wave waits for another and a compute unit, which holds two
// workgroups, has up to 128 KB of copies under way.  All G query heads of all new tokens (rows) use what is read: MT tiles of 16 query rows.
// S^T = K Q^T by MFMA 16x16x32 puts a query in a lane and rows in its registers, so that the softmax is register arithmetic and two lane
// exchanges, and its result is, without any movement, the second operand of O^T += V^T P^T; V^T comes out of LDS by the transposing
// read.  The waves are joined through LDS, workgroups of a unit by attend_join.hip.
// 64 sequences of 1152 rows, 8 KV heads (303 MB): 48 to 51 us, 6.0 to 6.3 TB/s, 57 (5.3) with caches that were not used before, where nothing
// but reads of 8 GiB reach 6.0 TB/s; one sequence of 32768 rows 24 us (5.6 TB/s) and the join; of 1152 rows 5 us, most of it the reads that
// follow each other (starts, then the length, the page, the rows).
#pragma once

#include "attend_internal.h"

namespace rkv {

namespace small {

constexpr int kTile = 32;                            // rows of a tile
constexpr int kTileBytes = kTile * kRowBytes;        // of keys, and of values
constexpr int kWaveBytes = 4 * kTileBytes;           // two buffers of both
constexpr int kWaves = 2;
constexpr int kThreads = kWaves * 64;

template <int MT>
struct Lds {
  unsigned char buffers[kWaves * kWaveBytes];
  float2 ml[kWaves][MT * 16];
};

template <int MT, bool PAGED>
__device__ __forceinline__ void attend(const AttendArgs& a, int block, Lds<MT>& shared) {
  unsigned char* lds = shared.buffers;
  float2(*ml)[MT * 16] = shared.ml;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int units = a.P * a.H;
  const int split = block / units, unit = block - split * units;
  const int p = unit / a.H, h = unit - p * a.H;
  const Tokens tk = tokens_between(a, p, p + 1);
  const int rows = min(tk.count, kSmallRows) * a.G;              // (a count past it is not this kernel's, and no product overflows)
  if (rows == 0 || tk.count > kSmallRows || rows > a.small_rows) return;
  const int len = clampi(a.kv_len[p], 0, a.N);
  const int group = group_of(a, p), base = prefix_of(a, group);
  const int r0 = len - tk.count;                                 // row of the first new token
  const Sight first = sight(a, r0), last = sight(a, len - 1);
  const int sinks = a.window > 0 ? a.sinks : 0;
  const Span<kTile> span(base, a.N, first.lo, last.hi, sinks);

  // this wave's tiles: a unit's tiles are dealt to as many workgroups as are worth it
  const int used = clampi((span.tiles * kTile + a.small_share - 1) / a.small_share, 1, a.small_splits);
  const int64_t part = split * kWaves + wave, parts = (int64_t)used * kWaves;
  const int t_lo = split < used ? (int)(span.tiles * part / parts) : 0;
  const int t_hi = split < used ? (int)(span.tiles * (part + 1) / parts) : 0;

  // 16 query rows a tile: lane & 15; channel 32 s + 8 (lane >> 4) + j of element j
  const int col = lane & 15, g4 = lane >> 4;
  bf16x8 qf[MT][4];
  Sight see[MT];
  int hi_min = 0x7fffffff, lo_max = 0;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = min(m * 16 + col, rows - 1);
    const int j = row / a.G, g = row - j * a.G;
    see[m] = sight(a, r0 + j);
    const uint16_t* qr = a.q + (int64_t)(tk.first + j) * a.qst + (int64_t)(h * a.G + g) * a.qsh + g4 * 8;
#pragma unroll
    for (int s = 0; s < 4; ++s) qf[m][s] = *reinterpret_cast<const bf16x8*>(qr + s * 32);
  }
  hi_min = first.hi;
  lo_max = last.lo;

  f32x4 o[MT][8];
  float mx[MT], sum[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    mx[m] = -INFINITY; sum[m] = 0.f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[m][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  Rows<PAGED, 4> rs(a, p, h, 0);
  const uint32_t mine = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + wave * kWaveBytes;
  auto copy = [&](int tile, int buf) {
    const int start = span.start(tile);
    rs.reload(start, start + kTile - 1);
    const uint32_t to = __builtin_amdgcn_readfirstlane(mine + buf * 2 * kTileBytes);
#pragma unroll
    for (int c = 0; c < kTile; c += 16) rs.copy(rs.place(start + c), to + c * kRowBytes, to + kTileBytes + c * kRowBytes);   // eight copies
  };

  if (t_lo < t_hi) copy(t_lo, 0);
  for (int t = t_lo; t < t_hi; ++t) {
    const int buf = (t - t_lo) & 1;
    if (t + 1 < t_hi) {
      copy(t + 1, buf ^ 1);
      asm volatile("s_waitcnt vmcnt(16)" ::: "memory");          // all but the copies just issued
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    const uint32_t kt = mine + buf * 2 * kTileBytes, vt = kt + kTileBytes;
    const int start = span.start(t);
    // keys of 16 rows at 4 steps of 32 channels; element i of a tile of S^T is row 4 g4 + i
    f32x4 s[MT][2];
#pragma unroll
    for (int m = 0; m < MT; ++m) s[m][0] = s[m][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int row = b * 16 + col;
        const bf16x8 kf = read16(kt + row * kRowBytes + (key_chunk(row, 4 * st + g4) << 4));
#pragma unroll
        for (int m = 0; m < MT; ++m) s[m][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[m][st], s[m][b], 0, 0, 0);
      }
    const bool edge = !(start + kTile <= min(hi_min, span.end(t)) && (start >= lo_max || start + kTile <= sinks) && start >= base);
    Frag pf[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[m][i >> 2][i & 3] * a.scale2;
      if (edge) {                                                // bit 16 (i >> 2) + (i & 3) from row start + 4 g4 on
        const int from = start + 4 * g4;
        const uint32_t seen = (bits_from(max(see[m].lo, base) - from) | (bits_from(base - from) & ~bits_from(sinks - from))) &
                              ~bits_from(min(see[m].hi, span.end(t)) - from);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = seen_or(x[i], seen, 16 * (i >> 2) + (i & 3));
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      top = fmaxf(top, mx[m]);
      const float ref = safe_max(top);
      const float fade = exp2_raw(mx[m] - ref);
      mx[m] = top;
      float add = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = exp2_raw(x[i] - ref);
        add += x[i];
      }
      sum[m] = sum[m] * fade + add;                              // of this lane's rows; lanes are added up at the end
      // the weights as bf16, which the matrix pipe takes: o moves by at most 2^-8 sum w |v| (0.0020 relative to 64 bits where 32-bit weights
      // have 0.0017, most of either o's own rounding); the sum is that of the weights before, for lse has 32 bits
#pragma unroll
      for (int i = 0; i < 8; ++i) pf[m].b[i] = (__bf16)x[i];
#pragma unroll
      for (int d = 0; d < 8; ++d) o[m][d] *= fade;
    }
    // values: 16 channels a block; element j of a lane is row 16 (j >> 2) + 4 g4 + (j & 3), as in pf
    const int vrow = 4 * g4 + (col >> 2);
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      Frag vf;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int row = vrow + half * 16, chunk = 2 * d + ((col & 3) >> 1);
        vf.s[half] = read_transposed(vt + row * kRowBytes + (value_chunk(row, chunk) << 4) + ((col & 1) << 3));
      }
      if (edge && __any(not_finite(largest_magnitudes(0, vf)))) {
        const Frag bad = take_not_finite(vf);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
          const f32x4 met = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad.b, given_weight(pf[m]).b, zero, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[m][d][i] += met_value(met[i]);
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) o[m][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.b, pf[m].b, o[m][d], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // read before this buffer is copied over
  }

  // join the waves: (M, l) of each, then the sum of their o; the buffers are free now (16 floats of padding spread the rows over the banks)
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float l = sum[m];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g4 == 0) ml[wave][m * 16 + col] = make_float2(mx[m], l);
  }
  float* mine_o = reinterpret_cast<float*>(lds + wave * kWaveBytes);   // [MT * 16][128], rows' 16-byte pieces xor-ed by the row
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int row = m * 16 + col, piece = (4 * d + g4) ^ (row & 7);
      *reinterpret_cast<f32x4*>(mine_o + row * kHeadDim + piece * 4) = o[m][d];
    }
  __syncthreads();
  const bool whole = a.small_splits == 1 && a.prefix_splits == 0;
  for (int i = threadIdx.x; i < rows * 32; i += kThreads) {
    const int row = i >> 5, piece = i & 31;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][row].x);
    float l = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float weight = exp2_raw(ml[w][row].x - safe_max(top));
      // (a wave without a visible row has o = 0 and weight 0)
      l += ml[w][row].y * weight;
      x += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds + w * kWaveBytes) + row * kHeadDim + (piece ^ (row & 7)) * 4) * weight;
    }
    if (whole) {
      const int j = row / a.G, hq = h * a.G + row - j * a.G;
      const int64_t token = tk.first + j;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      *reinterpret_cast<uint2*>(a.out + token * a.ost + hq * a.osh + piece * 4) = pack4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
      if (a.lse != nullptr && piece == 0) a.lse[token * (a.H * a.G) + hq] = lse_of(top, l);
    } else {
      const int j = row / a.G;
      const int64_t place = (int64_t)(tk.first + j) * (a.H * a.G) + h * a.G + row - j * a.G, places = (int64_t)a.T * (a.H * a.G);
      const int64_t at = a.small_by_token ? split * places + place : (((int64_t)p * a.small_splits + split) * a.H + h) * a.small_rows + row;
      if (split < used) *reinterpret_cast<f32x4*>(a.small_o + at * kHeadDim + piece * 4) = x;
      if (piece == 0) {
        a.small_ml[at] = make_float2(top, l);                    // of a workgroup without rows: -inf, 0
        if (split == 0 && group < 0)                             // no prefix: nothing for the join to find
          for (int i = 0; i < a.prefix_splits; ++i) a.prefix_ml[i * places + place] = make_float2(-INFINITY, 0.f);
      }
    }
  }
}

}  // namespace small
}  // namespace rkv
