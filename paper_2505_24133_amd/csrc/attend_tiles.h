// Attention of many rows of queries per KV head (prompts, chunks of prompts, the queries of a group over its shared prefix): bound by
// the matrix pipe and by the exponentials.
//
// A workgroup has a tile of 128 query rows (new token, head of the group) of one KV head, 32 a wave, and walks over the cache rows that one
// of them sees in steps of 32: copied to LDS by DMA three steps ahead, into rings of four, one barrier a step.  S^T = K Q^T by MFMA
// 32x32x16: a lane has one query and half of the step's rows, so that maxima and sums are register arithmetic and one exchange
// between the halves of the wave, and the weights are, without any movement, the second operand of O^T += V^T P^T.  V^T comes out of
// LDS by the transposing read.  The next step's scores are formed beside this step's exponentials, and two workgroups share a compute unit, so
// that one's products run beside the other's maxima.  Two workgroups leave a lane 256 registers, and the loop stays in them: one that is
// spilled is read back behind a wait for all copies under way (12 % of a long prompt).  Beside few-rows units (attend_beside.hip) 15 to 31
// scalar registers spill to vector registers, and for shared prefixes in contiguous caches four vector registers to memory, where values that
// are not finite are taken out.
//
// The weights are the second product's operand, and the matrix pipe takes 16 bits at this rate: they are rounded to bf16, which moves o by
// at most 2^-8 sum w |v| (measured against 64 bits: 0.0021 to 0.0023 relative where a plain form with 32-bit weights has 0.0017, most of
// either o's own rounding).  The sum l adds them before the rounding, for lse has 32 bits; and as the reference may lag behind the maximum by
// 2^8, the largest weight is rounded as well.  M, l and o are held in 32 bits.
//
// The largest prompts run at 0.97 to 1.05 PFLOP/s (three of up to 15000 tokens, 32 heads on 8: 590 to 640 us by the card), where a library
// product of 8192^3 reaches 1.22 to 1.30 and the loop's matrix and vector instructions by themselves, in registers, 1.56: the matrix pipe is
// busy in 55 % of the cycles.  At its full rate 32 query rows a wave would read 120 of the 128 bytes a cycle that LDS delivers, and the
// clock falls with the power that the products draw.  48 query rows a wave (16x16x32) win 3 % there and lose 7 to 18 where there are
// edges or few tiles; 64, one wave a SIMD, take 1.5 times as long.
#pragma once

#include <type_traits>

#include "attend_internal.h"

namespace rkv {

namespace tiles {

constexpr int kKeys = 32;                            // cache rows of a step
constexpr int kKeyBytes = kKeys * kRowBytes;
constexpr int kThreads = 256;
constexpr float kSlack = 8.f;        // a maximum that grows by less than 2^8 leaves the weights' reference where it is (they stay below 2^8)

// Over the 32 queries of a wave (in both of its halves); rows are below 2^24, which a float holds.
__device__ __forceinline__ int wave_max(int x) { return __builtin_amdgcn_readfirstlane((int)half_wave_max((float)x)); }
__device__ __forceinline__ int wave_min(int x) { return -wave_max(-x); }

struct Lds {
  unsigned char rings[2 * 4 * kKeyBytes];                // of keys, then of values
  int bounds[4][2];
  int2 places[kTileRows];                                // token and head of every query, and what it may see: for the edges and the end,
  Sight sights[kTileRows];                               // registers are short
};

// PREFIX: the query rows are those of a group's problems, the cache rows the group's shared ones.
template <bool PAGED, bool PREFIX>
__device__ __forceinline__ void attend(const AttendArgs& a, int splits, int block, Lds& shared) {
  unsigned char* lds = shared.rings;
  int(*bounds)[2] = shared.bounds;
  int2* places = shared.places;
  Sight* sights = shared.sights;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = block % a.H;
  const int rest = block / a.H;
  const int split = rest % splits;

  // The problem (or group) that this tile belongs to, and which of its tiles it is: the tiles of all problems are counted through, 64
  // at a time.  What else is needed of a problem is read with its tokens: reads that follow each other are what a short call waits for.
  int tile = rest / splits, owner = -1;
  Tokens tk{0, 0};
  int p0 = 0, p1 = 0, length = 0;                        // the owner's problems (PREFIX), and its rows: of the cache, or of the shared prefix
  const int owners = PREFIX ? a.groups : a.P;
  for (int at = 0; at < owners; at += 64) {
    const int o = min(at + lane, owners - 1);
    int q0 = o, q1 = o + 1;
    if constexpr (PREFIX) {
      q0 = clampi(a.group_starts[o], 0, a.P);
      q1 = clampi(a.group_starts[o + 1], 0, a.P);
    }
    const int rows_of = clampi(PREFIX ? a.prefix_len[o] : a.kv_len[o], 0, a.N);
    Tokens mine = tokens_between(a, q0, q1);
    if (at + lane >= owners) mine.count = 0;
    const bool small = !PREFIX && a.small_splits > 0 && (int64_t)mine.count * a.G <= a.small_rows;
    const int tiles = small ? 0 : (int)(((int64_t)mine.count * a.G + kTileRows - 1) / kTileRows);
    const int upto = (int)wave_inclusive_scan((uint32_t)tiles);
    const uint64_t past = __ballot(upto > tile);
    if (past != 0) {
      const int l = __ffsll((unsigned long long)past) - 1;
      owner = at + l;
      tk.first = __builtin_amdgcn_readlane(mine.first, l);
      tk.count = __builtin_amdgcn_readlane(mine.count, l);
      p0 = __builtin_amdgcn_readlane(q0, l);
      p1 = __builtin_amdgcn_readlane(q1, l);
      length = __builtin_amdgcn_readlane(rows_of, l);
      tile = __builtin_amdgcn_readlane(upto, l) - 1 - tile;         // the last tile, which sees the most rows, first
      break;
    }
    tile -= __builtin_amdgcn_readlane(upto, 63);
  }
  if (owner < 0) return;

  // this lane's query: element j of step s is channel 16 s + 8 (lane >> 5) + j
  const int rows = tk.count * a.G;
  const int col = lane & 31, half = lane >> 5;
  bf16x8 qf[8];
  int hi_min, hi_max, lo_min, lo_max, all_hi, all_lo, base = 0, lim = a.N;
  const int sinks = a.window > 0 ? a.sinks : 0;
  {
    const int row = min(tile * kTileRows + wave * 32 + col, rows - 1);
    const int j = row / a.G;
    const int token = tk.first + j, hq = h * a.G + row - j * a.G;
    const uint16_t* qr = a.q + (int64_t)token * a.qst + (int64_t)hq * a.qsh + half * 8;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qr + s * 16);

    Sight see;
    if constexpr (PREFIX) {
      lim = length;
      // the problem of the lane's token is the last one of the group that starts at or before it: the problems' starts and lengths
      // are read 64 at a time, and every lane bisects the lanes that hold them
      int end = 0, rows_of = 0;
      for (int at = p0; at < p1; at += 64) {
        const int p = min(at + lane, a.P - 1), n = min(64, p1 - at);
        const int begins = a.starts[p], ends = clampi(a.starts[p + 1], 0, a.T), held = clampi(a.kv_len[p], 0, a.N);
        int upto = 0;                                    // of these problems
        for (int step = 32; step > 0; step >>= 1) {
          const int begin = __shfl(begins, upto + step - 1);
          if (upto + step <= n && begin <= token) upto += step;
        }
        const int begin_63 = __builtin_amdgcn_readlane(begins, 63);
        if (upto == 63 && n == 64 && begin_63 <= token) upto = 64;
        const int l = max(upto - 1, 0), end_l = __shfl(ends, l), held_l = __shfl(held, l);
        if (upto > 0 || at == p0) { end = end_l; rows_of = held_l; }
      }
      see = sight(a, rows_of - (end - token));
      hi_min = wave_min(see.hi); hi_max = wave_max(see.hi); lo_min = wave_min(see.lo); lo_max = wave_max(see.lo);
      if (lane == 0) {
        bounds[wave][0] = hi_max;
        bounds[wave][1] = lo_min;
      }
    } else {
      base = prefix_of(a, group_of(a, owner));
      const int r0 = length - tk.count;                  // a later token sees no less, and nothing earlier
      see = sight(a, r0 + j);
      hi_min = __builtin_amdgcn_readlane(see.hi, 0); hi_max = __builtin_amdgcn_readlane(see.hi, 31);
      lo_min = __builtin_amdgcn_readlane(see.lo, 0); lo_max = __builtin_amdgcn_readlane(see.lo, 31);
      all_lo = sight(a, r0 + (int)((uint32_t)(tile * kTileRows) / (uint32_t)a.G)).lo;
      all_hi = sight(a, r0 + (int)((uint32_t)min(tile * kTileRows + kTileRows - 1, rows - 1) / (uint32_t)a.G)).hi;
    }
    if (half == 0) {
      places[wave * 32 + col] = make_int2(token, hq);
      sights[wave * 32 + col] = see;
    }
  }
  if constexpr (PREFIX) {
    __syncthreads();
    all_hi = max(max(bounds[0][0], bounds[1][0]), max(bounds[2][0], bounds[3][0]));
    all_lo = min(min(bounds[0][1], bounds[1][1]), min(bounds[2][1], bounds[3][1]));
  }
  const Span<kKeys> span(base, lim, __builtin_amdgcn_readfirstlane(all_lo), __builtin_amdgcn_readfirstlane(all_hi), sinks);
  const int used = clampi(span.tiles, 1, splits);
  const int t_lo = split < used ? (int)((int64_t)span.tiles * split / used) : 0;
  const int t_hi = split < used ? (int)((int64_t)span.tiles * (split + 1) / used) : 0;

  f32x16 o[4];
  float mx = -INFINITY, sum = 0.f;                       // of this lane's rows; the two halves of the wave are added up at the end
  float minus_ref = 0.f;                                 // what the exponents are taken from: mx, or 0 as long as nothing was visible
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;

  if (t_lo < t_hi) {
    Rows<PAGED, 2> rs(a, p0, h, 2 * (wave & 1));
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    // Batch i: the keys and the values of step i, eight rows a wave, to the rings' places i & 3 (past the last step that one again, for a
    // constant number of copies).
    int batch_start = span.start(t_lo);
    auto batch = [&](int i, int ring) {
      if (i < t_hi && i != t_lo) batch_start = i == span.tiles_a ? span.start_b : batch_start + kKeys;
      rs.reload(batch_start, batch_start + kKeys - 1);
      const auto at = rs.place(batch_start + 16 * (wave >> 1));
      const uint32_t to = lds0 + wave * 8 * kRowBytes + ring * kKeyBytes;
      rs.copy(at, to, to + 4 * kKeyBytes);
    };
    // Steps [plain_lo, plain_hi) are seen whole by all of the wave's queries.
    const int plain_lo = span.tiles_a + max(0, (max(base, lo_max) - span.start_b + kKeys - 1) / kKeys);
    const int plain_hi = span.tiles_a + max(0, min(hi_min, span.end_b) - span.start_b) / kKeys;
    // places of the fragments in a ring: keys by step of 16 channels, values by block of channels
    const uint32_t k_at = lds0 + col * kRowBytes + (key_chunk(col, half) << 4);
    const int vrow = 4 * half + ((lane & 15) >> 2);
    const uint32_t v_at = lds0 + 4 * kKeyBytes + vrow * kRowBytes + (value_chunk(vrow, 8 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) + ((lane & 1) << 3);
    auto keys = [&](int st, int ring) { return read16((k_at ^ (st << 5)) + ring * kKeyBytes); };
    // block d has channels 16 d .. 16 d + 15 and 64 + 16 d ..; element j of st is row 16 st + 8 (j >> 2) + 4 half + (j & 3)
    auto values = [&](int d, int st, int ring) {
      Frag f;
#pragma unroll
      for (int jh = 0; jh < 2; ++jh) f.s[jh] = read_transposed((v_at ^ (d << 5)) + ring * kKeyBytes + (16 * st + 8 * jh) * kRowBytes);
      return f;
    };

    f32x16 s;                                            // element i is row 8 (i >> 2) + 4 half + (i & 3)
    // One step: its scores s are there; behind them come the next step's scores, beside the weights, and the values' product.
    auto step = [&](int t, auto ring_of_t) {
      constexpr int RING = decltype(ring_of_t)::value, NEXT = (RING + 1) & 3;
      // this wave's copies of step t's values and the next one's keys have arrived (behind them: two copies of values and the batch after)
      // and its reads of step t - 1 are done; behind the barrier that holds for all
      asm volatile("s_waitcnt vmcnt(6) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      batch(t + 3, (RING + 3) & 3);
      bf16x8 kf[8];
#pragma unroll
      for (int st = 0; st < 4; ++st) kf[st] = keys(st, NEXT);
      const bool edge = t < plain_lo || t >= plain_hi;
      if (__builtin_expect(edge, 0)) {
        asm volatile("" ::: "memory");                   // (a branch, not a selection made for every step)
        // the rows that this lane's query sees, a bit each from row start + 4 half on; element i has bit 8 (i >> 2) + (i & 3)
        const int from = span.start(t) + 4 * half, stop = min(span.end(t), span.start(t) + kKeys);
        const Sight see = sights[wave * 32 + col];
        const uint32_t seen = (bits_from(max(see.lo, base) - from) | (bits_from(base - from) & ~bits_from(sinks - from))) & ~bits_from(min(see.hi, stop) - from);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = seen_or(s[i], seen, 8 * (i >> 2) + (i & 3));
      }
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      top = pair_max32(top) * a.scale2;
      // the reference moves only where some query's maximum has outgrown it
      if (__builtin_expect(__any(top > mx + kSlack), 0)) {
        const float next = fmaxf(mx, top);
        const float fade = exp2_raw(mx - safe_max(next));
        mx = next;
        minus_ref = -safe_max(next);
        sum *= fade;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= fade;
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);                     // a wave that has its products goes before the one that looks for its maxima: 3 to 9 %
#pragma unroll
      for (int st = 4; st < 8; ++st) kf[st] = keys(st, NEXT);
      f32x16 next;
#pragma unroll
      for (int i = 0; i < 16; ++i) next[i] = 0.f;
#pragma unroll
      for (int st = 0; st < 8; ++st) next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[st], qf[st], next, 0, 0, 0);
      Frag w[2], vf[8];
      float add = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = exp2_raw(__fmaf_rn(s[i], a.scale2, minus_ref));
        add += x;
        w[i >> 3].b[i & 7] = (__bf16)x;
      }
      sum += add;
#pragma unroll
      for (int i = 0; i < 8; ++i) vf[i] = values(i & 3, i >> 2, RING);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(w[i].u[0]), "+v"(w[i].u[1]), "+v"(w[i].u[2]), "+v"(w[i].u[3]));
      asm volatile("" : "+v"(sum));
      __builtin_amdgcn_sched_barrier(0);
      if (__builtin_expect(edge, 0)) {
        // what is not finite is taken out of the values, and added where a weight meets it
        bool some = false;
        {
          uint32_t largest = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) largest = largest_magnitudes(largest, vf[i]);
          some = __any(not_finite(largest));
        }
        if (__builtin_expect(some, 0)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            __builtin_amdgcn_sched_barrier(0);           // (one fragment at a time: there are no registers for more)
            f32x16 met;
#pragma unroll
            for (int e = 0; e < 16; ++e) met[e] = 0.f;
            const Frag bad = take_not_finite(vf[i]);
            met = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bad.b, given_weight(w[i >> 2]).b, met, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i & 3][e] += met_value(met[e]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i].b, w[i >> 2].b, o[i & 3], 0, 0, 0);
      __builtin_amdgcn_s_setprio(0);
      s = next;
    };

    batch(t_lo, 0);
    batch(t_lo + 1, 1);
    batch(t_lo + 2, 2);
    asm volatile("s_waitcnt vmcnt(10)\n\ts_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int st = 0; st < 8; ++st) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys(st, 0), qf[st], s, 0, 0, 0);
    for (int t = t_lo;;) {
      step(t, std::integral_constant<int, 0>());
      if (++t == t_hi) break;
      step(t, std::integral_constant<int, 1>());
      if (++t == t_hi) break;
      step(t, std::integral_constant<int, 2>());
      if (++t == t_hi) break;
      step(t, std::integral_constant<int, 3>());
      if (++t == t_hi) break;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no copy outlives the workgroup
  }

  // The wave's rows go out through LDS (its 16 KB of the rings, behind a barrier), so that whole rows are written: row col's 16-byte
  // pieces lie xor-ed by the row.
  sum += __shfl_xor(sum, 32);
  const bool whole = !PREFIX && splits == 1 && a.prefix_splits == 0;
  const int64_t slots = (int64_t)split * a.T * (a.H * a.G);
  const int left = rows - tile * kTileRows - wave * 32;  // of this wave's 32 rows there are so many
  if (col < left && half == 0) {
    const int2 place = places[wave * 32 + col];
    const int64_t at = (int64_t)place.x * (a.H * a.G) + place.y;
    if (!whole) (PREFIX ? a.prefix_ml : a.tile_ml)[slots + at] = make_float2(mx, sum);
    else if (a.lse != nullptr) a.lse[at] = lse_of(mx, sum);
  }
  if (!whole && t_lo == t_hi) return;                    // (of a part without rows -inf, 0 is all that is read)
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  float* mine = reinterpret_cast<float*>(lds) + wave * 32 * kHeadDim;
  const float inv = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int piece = 16 * (i >> 3) + 4 * d + 2 * ((i >> 2) & 1) + half;
      *reinterpret_cast<f32x4*>(mine + col * kHeadDim + ((piece ^ col) & 31) * 4) = f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]} * inv;
    }
  if (whole) {
    for (int r = lane >> 4; r < min(left, 32); r += 4) {
      const int2 place = places[wave * 32 + r];
      const int piece = 2 * (lane & 15);
      const f32x4 x = *reinterpret_cast<const f32x4*>(mine + r * kHeadDim + (piece ^ r) * 4), y = *reinterpret_cast<const f32x4*>(mine + r * kHeadDim + ((piece + 1) ^ r) * 4);
      const uint2 lo = pack4(x[0], x[1], x[2], x[3]), hi = pack4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<uint4*>(a.out + (int64_t)place.x * a.ost + (int64_t)place.y * a.osh + piece * 4) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  } else {
    for (int r = lane >> 5; r < min(left, 32); r += 2) {
      const int2 place = places[wave * 32 + r];
      const int64_t slot = slots + (int64_t)place.x * (a.H * a.G) + place.y;
      *reinterpret_cast<f32x4*>((PREFIX ? a.prefix_o : a.tile_o) + slot * kHeadDim + (lane & 31) * 4) = *reinterpret_cast<const f32x4*>(mine + r * kHeadDim + ((lane & 31) ^ r) * 4);
    }
  }
}

}  // namespace tiles
}  // namespace rkv
