// Shared parts of the attention kernels over the cache (gfx950): which rows a block of queries reads, how rows are found and
// copied to LDS, and the one-pass softmax.
//
// For a query q with visible rows c:  s_c = scale log2(e) q . k_c,  M = max s_c,  l = sum 2^(s_c - M),  o = sum 2^(s_c - M) v_c / l.
// M, l and the unnormalised o are carried over the rows; a part of the rows is described by its (M, l, o), and parts are joined by
// M = max M_i, weights 2^(M_i - M).  A part without a visible row has M = -inf, l = 0.
#pragma once

#include <math.h>

#include "rkv_attend.h"
#include "rkv_internal.h"

namespace rkv {

typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

constexpr int kSmallRows = 32;       // query rows per KV head (new tokens * G) that the kernel for few rows takes at most
constexpr int kTileRows = 128;       // query rows of a tile of the kernel for many

struct AttendArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* out;
  float* lse;                  // or nullptr
  const int32_t* starts;
  const int32_t* kv_len;
  const int32_t* group_starts; // groups > 0: problems that share their first rows
  const int32_t* prefix_len;
  int P, H, G, N, T, groups, window, sinks, num_pages;
  KvLayout kl, vl;
  int64_t qst, qsh, ost, osh;
  float scale2;                // scale * log2(e)
  // Parts of the rows, unnormalised, [split][t][hq]; those of the few-rows kernel without small_by_token [p][split][h][small_rows]
  int small_splits, tile_splits, prefix_splits;   // 0: the kernel does not run
  int small_rows;              // most query rows of a unit of the few-rows kernel: 16 or 32
  bool small_by_token;
  int small_share;             // rows of the cache that are worth a workgroup of it
  float* small_o;
  float2* small_ml;
  float* tile_o;
  float2* tile_ml;
  float* prefix_o;
  float2* prefix_ml;
};

// ------------------------------------------------------------------------------------------------ which rows
__device__ __forceinline__ int clampi(int x, int lo, int hi) { return min(max(x, lo), hi); }

// Number of entries of the ascending array a[0 .. n) that are <= t; t is the same in all lanes.  64 of them are compared at a time.
__device__ __forceinline__ int count_not_above(const int32_t* a, int n, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;
  while (len > 0) {
    const int step = (len + 63) >> 6;
    const int at = (lane + 1) * step - 1;
    const bool le = at < len && a[lo + min(at, len - 1)] <= t;
    const int c = __popcll(__ballot(le));
    lo += c * step;
    if (step == 1) break;
    len = min(step, len - c * step);
  }
  return lo;
}

struct Tokens { int first, count; };       // of a problem, or of a group
__device__ __forceinline__ Tokens tokens_between(const AttendArgs& a, int p0, int p1) {
  const int lo = clampi(a.starts[p0], 0, a.T), hi = clampi(a.starts[p1], 0, a.T);
  return Tokens{lo, max(hi - lo, 0)};
}
// The group that problem p belongs to, or -1.  (uniform)
__device__ __forceinline__ int group_of(const AttendArgs& a, int p) {
  if (a.groups == 0) return -1;
  const int g = count_not_above(a.group_starts, a.groups + 1, p) - 1;
  return g >= 0 && g < a.groups ? g : -1;
}
__device__ __forceinline__ int prefix_of(const AttendArgs& a, int g) { return g < 0 ? 0 : clampi(a.prefix_len[g], 0, a.N); }

// What the token at row r of its problem may see: rows c < hi with c >= lo or c < sinks.  r is -2^24 at least (a token before the first
// row), and the window n_tokens at most, 2^24, so that nothing here passes 32 bits.
struct Sight { int lo, hi; };
__device__ __forceinline__ Sight sight(const AttendArgs& a, int r) {
  return Sight{a.window > 0 ? max(r - a.window + 1, 0) : 0, max(r + 1, 0)};
}

// The rows of [base, lim) that a block of queries reads, in tiles of TK that start at multiples of 16 (16 rows from there on lie in one
// page): those before `sinks` and those from the lowest lo on.  No row lies in both.
template <int TK>
struct Span {
  int start_a, end_a, tiles_a, start_b, end_b, tiles;
  __device__ __forceinline__ Span(int base, int lim, int lo_min, int hi_max, int sinks) {
    end_b = min(hi_max, lim);
    start_b = max(base, lo_min) & ~15;
    start_a = base & ~15;
    end_a = min(min(sinks, lim), hi_max);
    if (end_a >= start_b) { start_b = start_a; end_a = start_a; }
    tiles_a = end_a > start_a ? (end_a - start_a + TK - 1) / TK : 0;
    tiles = tiles_a + (end_b > start_b ? (end_b - start_b + TK - 1) / TK : 0);
  }
  __device__ __forceinline__ int start(int i) const { return i < tiles_a ? start_a + i * TK : start_b + (i - tiles_a) * TK; }
  __device__ __forceinline__ int end(int i) const { return i < tiles_a ? end_a : end_b; }
};

// --------------------------------------------------------------------------------------------- where rows lie
// Rows of one problem and head, copied to LDS 16 at a time (four copies of four rows, 16 bytes a lane), keys and values.  The address of
// the 16 rows is the same in all lanes, a lane adds its offset among four rows.  Paged: the ids of 64 consecutive pages lie in the
// lanes of the wave (1024 rows and more); reload() is called with wave-uniform rows before rows are copied.
//
// Places in LDS of 16-byte piece `chunk` of row `row`: keys are read 16 rows at one chunk (the four low bits of the row spread
// them over all banks), values four rows at two neighbouring chunks, transposed (pairs of chunks are spread by three bits of the row).
__device__ __forceinline__ int key_chunk(int row, int chunk) { return chunk ^ (row & 15); }
__device__ __forceinline__ int value_chunk(int row, int chunk) { return chunk ^ ((row & 7) << 1); }

template <bool PAGED, int FOURS>
struct Rows {
  const unsigned char* k;
  const unsigned char* v;
  const int32_t* table;
  int N, shift, pages, num_pages, first, ids;
  uint32_t kst, vst;             // bytes
  int64_t kspage, vspage;        // bytes
  uint32_t koff[FOURS], voff[FOURS];     // of this lane: its row of four, and the chunk that belongs at its place
  int c0;
  // This wave copies FOURS times four rows of 16, from row 4 c0 on.
  __device__ __forceinline__ Rows(const AttendArgs& a, int p, int h, int c0) : c0(c0) {
    k = reinterpret_cast<const unsigned char*>(a.k + h * a.kl.sh);
    v = reinterpret_cast<const unsigned char*>(a.v + h * a.vl.sh);
    N = a.N;
    kst = (uint32_t)a.kl.st * 2; vst = (uint32_t)a.vl.st * 2;
    if constexpr (PAGED) {
      shift = a.kl.page_shift;
      pages = (a.N + (1 << shift) - 1) >> shift;
      num_pages = a.num_pages;
      table = a.kl.table + (int64_t)p * a.kl.table_stride;
      kspage = a.kl.spage * 2; vspage = a.vl.spage * 2;
      first = -64;
      ids = 0;
    } else {
      k += p * a.kl.sp * 2;
      v += p * a.vl.sp * 2;
    }
#pragma unroll
    for (int c = 0; c < FOURS; ++c) offsets(c, 15, &koff[c], &voff[c]);
  }
  // Offsets of copy c of this lane; rows past `last` of the 16 are that one.
  __device__ __forceinline__ void offsets(int c, int last, uint32_t* ko, uint32_t* vo) const {
    const int lane = threadIdx.x & 63, row = 4 * (c0 + c) + (lane >> 4), from = min(row, last);
    *ko = from * kst + (key_chunk(row, lane & 15) << 4);
    *vo = from * vst + (value_chunk(row, lane & 15) << 4);
  }
  __device__ __forceinline__ void reload(int row_lo, int row_hi) {
    if constexpr (PAGED) {
      const int lo = row_lo >> shift, hi = min(row_hi, N - 1) >> shift;
      if (lo < first || hi >= first + 64) {
        first = lo;
        ids = clampi(table[min(lo + (int)(threadIdx.x & 63), pages - 1)], 0, num_pages - 1);
      }
    }
  }
  // Where 16 rows lie that start at a multiple of 16.  Rows past the cache's last one are the last 16 again.
  struct Place { int at, page; };
  __device__ __forceinline__ Place place(int row16) const {
    const int at = __builtin_amdgcn_readfirstlane(min(row16, (N - 1) & ~15));
    if constexpr (PAGED) return Place{at, __builtin_amdgcn_readlane(ids, ((at >> shift) - first) & 63)};
    return Place{at, 0};
  }
  // Its keys and values to LDS, all keys before the values (who waits for the keys alone counts on it).  Past the end of a contiguous cache a
  // lane pulls its row back to the last one, in a page there is room: the caller hides what is past the end.
  __device__ __forceinline__ void copy(Place w, uint32_t k_to, uint32_t v_to) const {
    const unsigned char *kb, *vb;
    if constexpr (PAGED) {
      const uint32_t slot = w.at & ((1 << shift) - 1);
      kb = k + w.page * kspage + slot * kst;
      vb = v + w.page * vspage + slot * vst;
    } else {
      kb = k + (uint64_t)(uint32_t)w.at * kst;
      vb = v + (uint64_t)(uint32_t)w.at * vst;
      if (__builtin_expect(w.at + 16 > N, 0)) {
        uint32_t ko[FOURS], vo[FOURS];
#pragma unroll
        for (int c = 0; c < FOURS; ++c) offsets(c, N - 1 - w.at, &ko[c], &vo[c]);
#pragma unroll
        for (int c = 0; c < FOURS; ++c) dma16(kb, ko[c], k_to + c * 1024);
#pragma unroll
        for (int c = 0; c < FOURS; ++c) dma16(vb, vo[c], v_to + c * 1024);
        return;
      }
    }
#pragma unroll
    for (int c = 0; c < FOURS; ++c) dma16(kb, koff[c], k_to + c * 1024);
#pragma unroll
    for (int c = 0; c < FOURS; ++c) dma16(vb, voff[c], v_to + c * 1024);
  }
};

// Four rows of one channel: lane i of 16 gets channel i of the 16 channels whose four rows the lanes address, lane 4 m + n the
// 8 bytes of row m, channels 4 n .. 4 n + 3.
__device__ __forceinline__ s16x4 read_transposed(uint32_t lds_address) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)lds_address);
}
__device__ __forceinline__ bf16x8 read16(uint32_t lds_address) {
  return *(__attribute__((address_space(3))) const bf16x8*)(uintptr_t)lds_address;
}

// ------------------------------------------------------------------------------------------ infinities and NaN
// A hidden row's weight is 0, and 0 times infinity is NaN: where some query does not see a row of a tile, values that are not finite
// are taken out of the product, and the queries that give them weight get them added afterwards.
union Frag {
  bf16x8 b;
  uint32_t u[4];
  s16x4 s[2];
};
// The largest magnitudes, as bits, of the elements of f and of what came before, in both halves of a word (bf16 is ordered as its bits are).
__device__ __forceinline__ uint32_t largest_magnitudes(uint32_t so_far, const Frag& f) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  union { uint32_t u; u16x2 v; } a, b;
  a.u = so_far;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    b.u = f.u[i] & 0x7fff7fffu;
    a.v = __builtin_elementwise_max(a.v, b.v);
  }
  return a.u;
}
__device__ __forceinline__ bool not_finite(uint32_t largest) { return (largest & 0xffffu) >= 0x7f80u || (largest >> 16) >= 0x7f80u; }

// Bits n and above (n may be negative, or past 31), and a score where its row's bit is set, else -infinity.
__device__ __forceinline__ uint32_t bits_from(int n) { return n >= 32 ? 0u : 0xffffffffu << max(n, 0); }
__device__ __forceinline__ float seen_or(float score, uint32_t seen, int bit) {
  const uint32_t all = (uint32_t)((int32_t)(seen << (31 - bit)) >> 31);
  return __uint_as_float((__float_as_uint(score) & all) | (0xff800000u & ~all));
}
// f without what is not finite, and what that was: 1 for +inf, -256 for -inf, both (-255) for NaN.  A product with ones where there is
// weight, over 64 rows at most, says what a channel has met.
__device__ __forceinline__ Frag take_not_finite(Frag& f) {
  Frag met;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t keep = 0, m = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t x = (f.u[i] >> (16 * half)) & 0xffffu;
      const bool bad = (x & 0x7f80u) == 0x7f80u;
      keep |= (bad ? 0u : x) << (16 * half);
      m |= (bad ? ((x & 0x7fu) ? 0xc37fu : (x < 0x8000u ? 0x3f80u : 0xc380u)) : 0u) << (16 * half);
    }
    f.u[i] = keep; met.u[i] = m;
  }
  return met;
}
__device__ __forceinline__ float met_value(float met) {                   // (both make NaN)
  const float r = met > 0.f ? INFINITY : (truncf(met * 0.00390625f) * 256.f == met ? -INFINITY : NAN);
  return met == 0.f ? 0.f : r;
}
__device__ __forceinline__ Frag given_weight(const Frag& p) {        // 1 where the weight is not 0
  Frag r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.u[i] = ((p.u[i] & 0x7fffu) ? 0x3f80u : 0u) | ((p.u[i] & 0x7fff0000u) ? 0x3f800000u : 0u);
  return r;
}

__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }
// Subtrahend of the exponents: 0 as long as nothing is visible, so that 2^(-inf - M) is 0 and not NaN.
__device__ __forceinline__ float safe_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float lse_of(float m, float l) { return l > 0.f ? (m + __log2f(l)) * 0.69314718055994531f : (l == 0.f ? -INFINITY : l); }

// Four values as bf16, rounded to nearest even: the outputs' type.
__device__ __forceinline__ uint2 pack4(float x, float y, float z, float w) {
  typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
  union { bf16x4 b; uint2 u; } r;
  r.b = bf16x4{(__bf16)x, (__bf16)y, (__bf16)z, (__bf16)w};
  return r.u;
}

hipError_t launch_attend_small(const AttendArgs& a, bool paged, hipStream_t stream);
hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool prefix, hipStream_t stream);
// Tiles (of prefixes, or of problems' own rows) and few-rows units in one launch.
hipError_t launch_attend_beside(const AttendArgs& a, bool paged, bool prefix, hipStream_t stream);
hipError_t launch_attend_join(const AttendArgs& a, hipStream_t stream);

struct RotaryArgs {
  uint16_t* k_cache;
  uint16_t* v_cache;
  uint16_t* q_cache;           // or nullptr
  const uint16_t* k_new;
  const uint16_t* v_new;
  const uint16_t* q_new;
  uint16_t* q_out;
  const float* cos;
  const float* sin;
  const int32_t* starts;
  const int32_t* held;
  const int32_t* seen;
  int P, H, Hq, N, T, alpha, rotary, interleaved, table_rows, num_pages;
  KvLayout kl, vl;
  int64_t qsp, qsh, qst;       // query cache: problem, head, slot
  int64_t knt, knh, vnt, vnh, qnt, qnh, qot, qoh;
};
hipError_t launch_append_rotary(const RotaryArgs& a, hipStream_t stream);

}  // namespace rkv
