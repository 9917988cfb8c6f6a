// C ABI of rkv_attend.h: argument validation, how the work is cut, workspace carve-up and kernel sequencing.
#include <math.h>

#include <algorithm>

#include "attend_internal.h"

namespace rkv {

int64_t attend_tile_bound(int64_t T, int G, int64_t owners);

namespace {

constexpr int kMaxTokens = 1 << 24;
constexpr int64_t kMaxBlocks = 1 << 23;
constexpr int64_t kSlots = 512;             // workgroups of the many-rows kernel that the chip's 256 compute units hold
constexpr int64_t kSmallSlots = 512;        // and of the few-rows kernel
constexpr int64_t kMaxSplits = 128;         // (the join takes 256 parts)

bool row_stride(int64_t s) { return s >= kHeadDim && s <= 32768 && s % 8 == 0; }
bool wide_stride(int64_t s, bool several) { return s >= 0 && s % 8 == 0 && (s > 0 || !several); }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The caches as rkv_params describes them, checked as the compression step checks them.
struct Caches {
  int P, H, G, N;
  bool paged;
  KvLayout kl, vl;
};

rkv_status read_caches(const rkv_params& q, int num_pages, Caches* c) {
  if (q.num_problems < 0 || q.kv_heads < 1 || q.q_heads < 1 || q.n_tokens < 1 || q.q_heads % q.kv_heads != 0) return RKV_ERR_SHAPE;
  if (q.head_dim != kHeadDim || q.n_tokens > kMaxTokens || q.q_heads > 4096 || (int64_t)q.num_problems * q.kv_heads > (1 << 22)) return RKV_ERR_UNSUPPORTED;
  c->P = q.num_problems; c->H = q.kv_heads; c->G = q.q_heads / q.kv_heads; c->N = q.n_tokens;
  c->paged = q.page_size != 0;
  int shift = 0;
  if (c->paged) {
    if (q.page_size != 16 && q.page_size != 32 && q.page_size != 64 && q.page_size != 128) return RKV_ERR_UNSUPPORTED;
    while ((1 << shift) < q.page_size) ++shift;
    if (q.num_problems > 0 && q.block_table == nullptr) return RKV_ERR_NULL;
    if ((int64_t)q.table_stride * q.page_size < q.n_tokens || num_pages < 1) return RKV_ERR_SHAPE;
  }
  auto layout = [&](int64_t sp, int64_t sh, int64_t st, int64_t spage, KvLayout* l) {
    if (!c->paged && sp == 0 && sh == 0 && st == 0) {
      st = kHeadDim; sh = (int64_t)q.n_tokens * kHeadDim; sp = sh * q.kv_heads;
    }
    *l = KvLayout{c->paged ? q.block_table : nullptr, shift, q.table_stride, sp, sh, st, spage};
    return row_stride(st) && wide_stride(sh, q.kv_heads > 1) && (c->paged ? spage > 0 && spage % 8 == 0 : wide_stride(sp, q.num_problems > 1));
  };
  if (!layout(q.k_stride_problem, q.k_stride_head, q.k_stride_token, q.k_stride_page, &c->kl) ||
      !layout(q.v_stride_problem, q.v_stride_head, q.v_stride_token, q.v_stride_page, &c->vl))
    return RKV_ERR_SHAPE;
  return RKV_OK;
}

// Strides of an array [T, heads, d]; 0, 0 = dense.  Rows that are written must not lie in each other: one kind of stride is at least a
// row, the other one at least all of its rows.
bool token_strides(int64_t st, int64_t sh, int heads, int64_t tokens, int64_t* ot, int64_t* oh, bool written) {
  if (st == 0 && sh == 0) { *oh = kHeadDim; *ot = (int64_t)heads * kHeadDim; return true; }
  *ot = st; *oh = sh;
  if (!wide_stride(st, tokens > 1) || !wide_stride(sh, heads > 1) || st > (int64_t)1 << 40 || sh > (int64_t)1 << 40) return false;
  if (!written) return true;
  if ((heads > 1 && sh < kHeadDim) || (tokens > 1 && st < kHeadDim)) return false;
  // (divided, for the product of the second could pass 64 bits)
  return heads <= 1 || tokens <= 1 || st >= (heads - 1) * sh + kHeadDim || (sh - kHeadDim) / (tokens - 1) >= st;
}

struct AttendPlan {
  AttendArgs a;
  bool paged;
  size_t off_small_o, off_small_ml, off_tile_o, off_tile_ml, off_prefix_o, off_prefix_ml, total;
};

// Into how many workgroups the rows of a few-rows unit are dealt, at most, and how many rows are worth one: as many as the chip takes at once,
// with 64 rows each, then more where a unit still has 1024 rows for each, so that units of different lengths even out (not behind shared
// prefixes: what is left of the rows there is not known here, and workgroups that find nothing to do are not free: 64 samples of one prompt 4
// us), and one workgroup where the join would cost more than the rows: 101 rows of one sequence, 8 KV heads, 6.3 us whole and 8.1 in two
// parts, 501 rows 13.3 and 8.3; 301 rows of 16 sequences 10.1 and 11.5.  48
// ragged caches of up to 8320 rows under a window of 4096: 174 us with one workgroup a unit, 150 with four.
void split_small(int64_t units, int64_t reach, AttendArgs* a) {
  const int64_t fill = std::min((kSmallSlots + units - 1) / units, (reach + 63) / 64);
  const int64_t even = a->groups > 0 ? 0 : std::min((4 * kSmallSlots + units - 1) / units, reach / 1024);
  a->small_splits = a->groups == 0 && reach <= 192 + units ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(std::max(fill, even), kMaxSplits));
  a->small_share = fill >= even ? 64 : 512;
}

// Into how many parts the rows of the many-rows kernel's tiles are dealt where there are too few tiles to fill the chip: rounds of
// workgroups times steps of each (about 1.1 us, with four of them for its start), and what it takes to write the parts and read them
// again (4 TB/s).  511 tokens of seven heads behind 7681 rows, 112 tiles: 4 parts 75 us, 9 parts (two full rounds) 102 us, 5 parts (one round
// and a little) 112 us.
int split_tiles(int64_t tiles, int64_t rows, int64_t reach) {
  if (tiles >= kSlots) return 1;
  const int64_t steps = (reach + 31) / 32;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 32 && (s == 1 || s * 4 <= steps); ++s) {
    const double cost = 1.1 * (double)((tiles * s + kSlots - 1) / kSlots) * (double)((steps + s - 1) / s + 4) +
                        (s > 1 ? 3.0 + (double)rows * s * (2 * kHeadDim * 4) / 4e6 : 0.0);
    if (s == 1 || cost < least) { best = s; least = cost; }
  }
  return best;
}
// (no more under a window than without one, so that a workspace sized without it does)
int split_tiles(int64_t tiles, int64_t rows, int64_t reach, int64_t all) {
  const int s = split_tiles(tiles, rows, reach);
  return reach == all ? s : std::min(s, split_tiles(tiles, rows, all));
}

// Shared prefixes in one launch with the few-rows units behind them: a prefix's workgroup is a chain of dependent steps (0.55 us each, 5 for the
// start), which costs nothing as long as the units (10 us for 512 of them) and the steps of all workgroups keep the chip busy (0.4 us for
// 512 of them, and eight for each start); every part is written and read again (0.45 us for 1000 rows of queries).  Fitted to 17 sizes, where
// it picks what is 3 % slower than the best on average.  64 samples of 8 KV heads behind 4099 rows: 6 parts 32.6 us, 2 parts 56.5, 16
// parts 36.6; behind 16000 rows 13 parts 46, 6 parts 71, 32 parts 55; 32 times 2 samples behind 1000 rows 1 part 35, 4 parts 43; 16
// samples behind 8000 rows 32 parts 22.1, 6 parts 40.
int split_prefix(int64_t tiles, int64_t rows, int64_t reach, int64_t units) {
  const int64_t steps = (reach + 31) / 32;
  const double busy = 5.0 + 10.0 * (double)std::min(units, kSlots) / (double)kSlots;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 32 && (s == 1 || s * 4 <= steps); ++s) {
    const double chain = 5.0 + 0.55 * (double)((steps + s - 1) / s), work = 0.4 * (double)tiles * (double)(steps + 8 * s) / (double)kSlots;
    const double cost = std::max(chain, busy + work) + 0.45e-3 * (double)rows * s;
    if (s == 1 || cost < least) { best = s; least = cost; }
  }
  return best;
}
int split_prefix(int64_t tiles, int64_t rows, int64_t reach, int64_t units, int64_t all) {
  const int s = split_prefix(tiles, rows, reach, units);
  return reach == all ? s : std::min(s, split_prefix(tiles, rows, all, units));
}

rkv_status plan_attend(const rkv_params* prm, const rkv_attend_params* att, bool shared, AttendPlan* pl) {
  if (prm == nullptr || att == nullptr) return RKV_ERR_NULL;
  const rkv_attend_params& t = *att;
  Caches c;
  const rkv_status s = read_caches(*prm, t.num_pages, &c);
  if (s != RKV_OK) return s;
  if (t.tokens < 0 || (t.tokens > 0 && (t.max_new < 1 || t.max_new > t.tokens))) return RKV_ERR_SHAPE;
  if (t.groups < 0 || t.groups > c.P || (!shared && t.groups != 0)) return RKV_ERR_SHAPE;
  if (t.tokens > kMaxTokens || (int64_t)t.tokens * c.H * c.G > 0x7fffffff) return RKV_ERR_UNSUPPORTED;
  if (t.window < 0 || t.sinks < 0 || !(t.scale > 0.f) || !isfinite(t.scale)) return RKV_ERR_PARAM;
  AttendArgs& a = pl->a;
  a = AttendArgs{};
  if (!token_strides(t.q_stride_token, t.q_stride_head, c.H * c.G, t.tokens, &a.qst, &a.qsh, false) ||
      !token_strides(t.o_stride_token, t.o_stride_head, c.H * c.G, t.tokens, &a.ost, &a.osh, true))
    return RKV_ERR_SHAPE;
  a.starts = t.starts; a.kv_len = t.kv_len; a.group_starts = t.group_starts; a.prefix_len = t.prefix_len;
  a.P = c.P; a.H = c.H; a.G = c.G; a.N = c.N; a.T = t.tokens; a.groups = t.groups;
  // (a window of N rows hides nothing, and a larger one would take the lowest row that a token before the first one sees past 32 bits)
  a.window = std::min(t.window, c.N); a.sinks = t.sinks; a.num_pages = t.num_pages;
  a.kl = c.kl; a.vl = c.vl;
  a.scale2 = t.scale * 1.4426950408889634f;
  pl->paged = c.paged;
  pl->total = 0;
  if (c.P == 0 || t.tokens == 0) return RKV_OK;

  // Which kernels run.  Up to 32 rows of queries per KV head (new tokens * G) the few-rows kernel has them; where a problem may have
  // more, the many-rows kernel has those problems, and the few-rows kernel the others if there are any, in the same launch.  (A few-rows
  // kernel for up to 64 rows lost: 16 tokens of 4 heads behind 1000 rows 17.1 us, in tiles 12.8, behind 8000 rows of 4 sequences 45.6 and
  // 37.3; only many sequences of very different lengths were 4 to 13 % faster with it.)
  const int64_t most_rows = (int64_t)t.max_new * c.G, rows = (int64_t)t.tokens * c.H * c.G;
  // 17 to 32 rows over caches that keep the chip busy are the many-rows kernel's too (whatever the window, so that its workspace does for
  // all): three tokens of 8 heads behind 20 000 rows of 8 sequences 154 us, in tiles 127, 32 heads behind 4000 of 32 sequences 129 and 116;
  // behind 1000 rows of 64 sequences 46 and 47, behind prefixes 33 and 46.
  const bool heavy = most_rows > 16 && t.groups == 0 && (int64_t)c.P * c.H * c.N >= 900000;
  const bool large = most_rows > kSmallRows || heavy;
  // Rows of queries that the few-rows kernel takes of a problem, if it runs; and whether a problem may have so few (where one would leave the
  // others more than max_new each there is none, unless tokens are padding: the many-rows kernel has it then).
  const int small_rows = most_rows <= 16 || (heavy && most_rows <= kSmallRows) ? 16 : kSmallRows;
  const bool small = !large || (c.P > 1 && c.G <= small_rows && (int64_t)t.tokens * c.G - (int64_t)(c.P - 1) * most_rows <= small_rows);
  // rows that the queries of a unit or a tile, which have so many tokens, may see
  auto reach = [&](int64_t tokens) {
    return t.window > 0 ? std::min<int64_t>(c.N, (int64_t)t.window + t.sinks + std::min<int64_t>(tokens, t.max_new)) : (int64_t)c.N;
  };
  if (small) {
    a.small_rows = small_rows;
    split_small((int64_t)c.P * c.H, reach(a.small_rows / c.G), &a);
    // (a workgroup a row, which the join takes for more than 32 parts, would be more threads than a launch has)
    if (rows > (1 << 22)) a.small_splits = std::min(a.small_splits, 30);
    // (a token array that is mostly padding would make for large parts by token)
    a.small_by_token = !large && rows <= (int64_t)c.P * c.H * a.small_rows;
  }
  if (large) a.tile_splits = split_tiles(attend_tile_bound(t.tokens, c.G, c.P) * c.H, rows, reach(kTileRows / c.G + 2), c.N);
  if (t.groups > 0) {
    const int64_t tiles = attend_tile_bound(t.tokens, c.G, t.groups) * c.H;
    a.prefix_splits = !large ? split_prefix(tiles, rows, reach(t.max_new), (int64_t)c.P * c.H, c.N) : split_tiles(tiles, rows, reach(t.max_new), c.N);
  }
  if ((int64_t)c.P * c.H * std::max(a.small_splits, 1) > kMaxBlocks ||
      attend_tile_bound(t.tokens, c.G, c.P) * c.H * std::max(std::max(a.tile_splits, a.prefix_splits), 1) > kMaxBlocks ||
      (int64_t)t.tokens * ((c.H * c.G + 7) / 8) >= kMaxBlocks * 2 || (int64_t)c.P * c.H * 8 > kMaxBlocks * 4)
    return RKV_ERR_UNSUPPORTED;

  auto take = [&](int64_t bytes) {
    const size_t o = pl->total;
    pl->total = (o + (size_t)bytes + 255) & ~(size_t)255;
    return o;
  };
  const int64_t small_parts = a.small_splits > 1 || (small && t.groups > 0) ? (a.small_by_token ? rows : (int64_t)c.P * c.H * a.small_rows) * a.small_splits : 0;
  const int64_t tile_parts = a.tile_splits > 1 || (large && t.groups > 0) ? rows * a.tile_splits : 0;
  const int64_t prefix_parts = rows * a.prefix_splits;
  pl->off_small_o = take(small_parts * kHeadDim * 4);
  pl->off_small_ml = take(small_parts * 8);
  pl->off_tile_o = take(tile_parts * kHeadDim * 4);
  pl->off_tile_ml = take(tile_parts * 8);
  pl->off_prefix_o = take(prefix_parts * kHeadDim * 4);
  pl->off_prefix_ml = take(prefix_parts * 8);
  return RKV_OK;
}

rkv_status attend(const rkv_params* prm, const rkv_attend_params* att, bool shared, const void* q, const void* k, const void* v,
                  void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  AttendPlan pl;
  const rkv_status s = plan_attend(prm, att, shared, &pl);
  if (s != RKV_OK) return s;
  AttendArgs& a = pl.a;
  if (a.P == 0 || a.T == 0) return RKV_OK;
  if (q == nullptr || k == nullptr || v == nullptr || out == nullptr || a.starts == nullptr || a.kv_len == nullptr ||
      (a.groups > 0 && (a.group_starts == nullptr || a.prefix_len == nullptr)))
    return RKV_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return RKV_ERR_SHAPE;
  if (pl.total > 0 && (ws == nullptr || ((uintptr_t)ws & 255) != 0 || ws_bytes < pl.total)) return RKV_ERR_WORKSPACE;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  char* w = static_cast<char*>(ws);
  a.small_o = reinterpret_cast<float*>(w + pl.off_small_o);
  a.small_ml = reinterpret_cast<float2*>(w + pl.off_small_ml);
  a.tile_o = reinterpret_cast<float*>(w + pl.off_tile_o);
  a.tile_ml = reinterpret_cast<float2*>(w + pl.off_tile_ml);
  a.prefix_o = reinterpret_cast<float*>(w + pl.off_prefix_o);
  a.prefix_ml = reinterpret_cast<float2*>(w + pl.off_prefix_ml);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool prefix_beside = a.prefix_splits > 0 && a.tile_splits == 0;      // (there are few-rows units then)
  if (a.prefix_splits > 0 && !prefix_beside && launch_attend_tiles(a, pl.paged, true, st) != hipSuccess) return RKV_ERR_HIP;
  const hipError_t own = prefix_beside ? launch_attend_beside(a, pl.paged, true, st) :
                         a.tile_splits == 0 ? launch_attend_small(a, pl.paged, st) :
                         a.small_splits == 0 ? launch_attend_tiles(a, pl.paged, false, st) : launch_attend_beside(a, pl.paged, false, st);
  if (own != hipSuccess) return RKV_ERR_HIP;
  if ((a.prefix_splits > 0 || a.tile_splits > 1 || a.small_splits > 1) && launch_attend_join(a, st) != hipSuccess) return RKV_ERR_HIP;
  return RKV_OK;
}

}  // namespace
}  // namespace rkv

using namespace rkv;

extern "C" {

rkv_status rkv_attend_workspace_size(const rkv_params* prm, const rkv_attend_params* att, size_t* bytes) {
  if (bytes == nullptr) return RKV_ERR_NULL;
  AttendPlan pl;
  const rkv_status s = plan_attend(prm, att, true, &pl);
  if (s == RKV_OK) *bytes = pl.total;
  return s;
}

rkv_status rkv_attend(const rkv_params* prm, const rkv_attend_params* att, const void* q, const void* k, const void* v,
                      void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return attend(prm, att, false, q, k, v, out, lse, ws, ws_bytes, stream);
}

rkv_status rkv_attend_shared(const rkv_params* prm, const rkv_attend_params* att, const void* q, const void* k, const void* v,
                             void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return attend(prm, att, true, q, k, v, out, lse, ws, ws_bytes, stream);
}

rkv_status rkv_cache_append_rotary(const rkv_params* prm, const rkv_rotary_params* rot, void* k_cache, void* v_cache, void* q_cache,
                                   const void* k_new, const void* v_new, const void* q_new, void* q_out, void* stream) {
  if (prm == nullptr || rot == nullptr) return RKV_ERR_NULL;
  const rkv_rotary_params& r = *rot;
  Caches c;
  const rkv_status s = read_caches(*prm, r.num_pages, &c);
  if (s != RKV_OK) return s;
  const int Hq = c.H * c.G;
  if (r.tokens < 0 || r.table_rows < 1) return RKV_ERR_SHAPE;
  if (r.tokens > kMaxTokens / 2 || r.rotary_dim < 16 || r.rotary_dim > kHeadDim || r.rotary_dim % 16 != 0) return RKV_ERR_UNSUPPORTED;
  if (r.interleaved != 0 && r.interleaved != 1) return RKV_ERR_PARAM;
  RotaryArgs a = {};
  if (!token_strides(r.k_stride_token, r.k_stride_head, c.H, r.tokens, &a.knt, &a.knh, false) ||
      !token_strides(r.v_stride_token, r.v_stride_head, c.H, r.tokens, &a.vnt, &a.vnh, false) ||
      !token_strides(r.q_stride_token, r.q_stride_head, Hq, r.tokens, &a.qnt, &a.qnh, false) ||
      !token_strides(r.o_stride_token, r.o_stride_head, Hq, r.tokens, &a.qot, &a.qoh, true))
    return RKV_ERR_SHAPE;
  a.alpha = 1;
  if (q_cache != nullptr) {
    if (prm->alpha < 1) return RKV_ERR_SHAPE;
    a.alpha = prm->alpha;
    a.qsp = prm->q_stride_problem; a.qsh = prm->q_stride_head; a.qst = prm->q_stride_token;
    if (a.qsp == 0 && a.qsh == 0 && a.qst == 0) {
      a.qst = kHeadDim; a.qsh = (int64_t)a.alpha * kHeadDim; a.qsp = a.qsh * Hq;
    }
    if (a.qst < kHeadDim || a.qst % 8 != 0 || !wide_stride(a.qsh, Hq > 1) || !wide_stride(a.qsp, c.P > 1)) return RKV_ERR_SHAPE;
  }
  if (c.P == 0 || r.tokens == 0) return RKV_OK;
  if (k_cache == nullptr || v_cache == nullptr || k_new == nullptr || v_new == nullptr || q_new == nullptr || q_out == nullptr ||
      r.cos == nullptr || r.sin == nullptr || r.starts == nullptr || r.held == nullptr || r.seen == nullptr)
    return RKV_ERR_NULL;
  for (const void* x : {(const void*)k_cache, (const void*)v_cache, (const void*)q_cache, k_new, v_new, q_new, (const void*)q_out,
                        (const void*)r.cos, (const void*)r.sin})
    if (!aligned16(x)) return RKV_ERR_SHAPE;
  // in place only where every row stays where it lies: a workgroup would write over a row that another one still has to read
  if (q_out == q_new && ((r.tokens > 1 && a.qot != a.qnt) || (Hq > 1 && a.qoh != a.qnh))) return RKV_ERR_SHAPE;
  a.k_cache = static_cast<uint16_t*>(k_cache);
  a.v_cache = static_cast<uint16_t*>(v_cache);
  a.q_cache = static_cast<uint16_t*>(q_cache);
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.q_new = static_cast<const uint16_t*>(q_new);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.cos = r.cos; a.sin = r.sin; a.starts = r.starts; a.held = r.held; a.seen = r.seen;
  a.P = c.P; a.H = c.H; a.Hq = Hq; a.N = c.N; a.T = r.tokens;
  a.rotary = r.rotary_dim; a.interleaved = r.interleaved; a.table_rows = r.table_rows; a.num_pages = r.num_pages;
  a.kl = c.kl; a.vl = c.vl;
  return launch_append_rotary(a, static_cast<hipStream_t>(stream)) == hipSuccess ? RKV_OK : RKV_ERR_HIP;
}

}  // extern "C"
