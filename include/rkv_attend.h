/*
 * rkv_attend.h — C ABI of the decode loop around the compression step (rkv.h): new tokens appended with
 * their position rotation, attention over the cache, and attention of sequences that share a prompt.
 *
 * Everything rkv.h says about its entry points holds here: device pointers owned by the caller, work enqueued on `stream`
 * without synchronising, arguments validated before the first launch, the same status values, workspaces whose
 * contents need not be preserved.  `rkv_params` describes the caches as it does there; of its fields these
 * calls read num_problems, kv_heads, q_heads, n_tokens, head_dim (128), the strides of k and v, and the paging fields (plus alpha
 * and the q_stride_* for the query cache).  What the compression step asks beyond that (budget, G * alpha <= 64, N <= 32768, ...) is
 * not asked: n_tokens may be up to 2^24, q_heads up to 4096, in groups of any size, num_problems * kv_heads up to 2^22.  Of new tokens the
 * append takes T <= 2^23, attention T * ceil(q_heads / 8) < 2^24.  More is RKV_ERR_UNSUPPORTED.
 *
 * Strides of token arrays that are 0, 0 say dense; of others the one of a dimension with several entries is positive (arrays that are
 * broadcast are refused), and rows lie on 16 bytes.
 *
 * A batch is ragged: `starts` [P + 1] (int32, device, ascending) cuts the T new tokens into those of problem 0, 1, ...; a
 * problem may have none.  Rows of the token arrays behind starts[P] are neither read nor written.  Values that lie in
 * device memory cannot be refused: lengths are clamped into [0, n_tokens], tokens into [0, T), positions into the
 * rotation table, and pages into the pool, so nothing is accessed out of bounds whatever they hold.
 */
#ifndef RKV_ATTEND_H
#define RKV_ATTEND_H

#include "rkv.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * rkv_cache_append_rotary: token j of problem p (row t = starts[p] + j of k_new, v_new [T, kv_heads, d], q_new [T, q_heads, d])
 * has position seen[p] + j.  Its key and its queries are rotated by that position, its key and value are written at row
 * held[p] + j of the caches (contiguous or paged), its rotated queries to q_out [T, q_heads, d] and, for the last alpha tokens
 * of a problem, to slot (seen[p] + j) % alpha of the query cache (NULL: none), which is what rkv_compress takes as q_obs.  A cache
 * that has been compressed holds fewer rows than its sequence has positions, hence the two counts.
 *
 * Of a row's 128 channels the first rotary_dim are rotated in pairs, channel i with i + rotary_dim / 2, or 2 i with
 * 2 i + 1 if `interleaved`: (a, b) -> (a cos - b sin, b cos + a sin) with cos[position][i], sin[position][i] from tables
 * [table_rows, rotary_dim / 2] (fp32), in fp32 and rounded once.  A position past the table takes its last row; a token whose row is
 * not in [0, n_tokens), or whose page is not in [0, num_pages), is left out of the caches of keys and values.  q_out may be q_new, with
 * the same strides (others are refused).
 */
typedef struct {
  int32_t tokens;            /* T >= 0 */
  int32_t rotary_dim;        /* multiple of 16, 16 .. 128 */
  int32_t interleaved;       /* 0 or 1 */
  int32_t table_rows;        /* rows of cos and sin, >= 1 */
  int32_t num_pages;         /* pages of the pools (paged caches), >= 1 */
  const float* cos;          /* device, [table_rows, rotary_dim / 2], 16-byte aligned */
  const float* sin;
  const int32_t* starts;     /* device, [P + 1] */
  const int32_t* held;       /* device, [P]: rows in the cache before the call */
  const int32_t* seen;       /* device, [P]: position of the first new token */
  int64_t k_stride_token, k_stride_head;   /* of k_new, in elements; 0, 0 = dense [T, kv_heads, d]; likewise below */
  int64_t v_stride_token, v_stride_head;
  int64_t q_stride_token, q_stride_head;
  int64_t o_stride_token, o_stride_head;   /* of q_out */
} rkv_rotary_params;

rkv_status rkv_cache_append_rotary(const rkv_params* prm, const rkv_rotary_params* rot, void* k_cache, void* v_cache, void* q_cache,
                                   const void* k_new, const void* v_new, const void* q_new, void* q_out, void* stream);

/*
 * rkv_attend: attention of the new tokens over their problems' caches, which hold them already.  With n new tokens and
 * L = kv_len[p] rows, token j is row r = L - n + j and sees the rows c <= r; with window > 0 of those only
 * c > r - window or c < sinks.  out[t, hq] = sum_c w_c v_c, w = softmax over the visible rows of scale * q . k_c;
 * lse[t, hq] (fp32, dense, NULL: not wanted) = log sum_c exp(scale * q . k_c).  A token without a visible row (r < 0) gets zeros and
 * -infinity.  What a token does not see has no influence on it, infinities and NaN included.  Sums and the softmax are held in fp32; the
 * weights are rounded to bf16 before they are multiplied with v.
 *
 * max_new bounds the new tokens of one problem; the outputs of a problem that has more are unspecified.  The closer it is the better: which
 * kernels run, and in how many parts, goes by it.  T is always a valid bound.
 *
 * rkv_attend_shared: the problems group_starts[g] .. group_starts[g + 1] - 1 (device, int32 [groups + 1], ascending) hold the same values in
 * rows 0 .. prefix_len[g] - 1 (a prompt that they share: copies, or the same pages).  Those rows are read once for the whole group, from its
 * first problem's cache; the result is rkv_attend's.  Problems in no group are attended by themselves.
 *
 * Both need a workspace of rkv_attend_workspace_size() bytes (0 for calls that need none), 256-byte aligned; the size for a window of 0 does for
 * any window.  out must not overlap the other arrays, nor (refused) its rows each other.  groups is 0 for rkv_attend.
 */
typedef struct {
  int32_t tokens;            /* T >= 0 */
  int32_t max_new;           /* 1 .. T */
  int32_t window;            /* 0: no window */
  int32_t sinks;             /* >= 0; of interest with a window only */
  int32_t groups;            /* rkv_attend_shared: 0 .. P */
  int32_t num_pages;         /* pages of the pools (paged caches), >= 1 */
  float scale;               /* > 0, finite */
  const int32_t* starts;     /* device, [P + 1] */
  const int32_t* kv_len;     /* device, [P]: rows in the cache, the new tokens' included */
  const int32_t* group_starts;   /* device, [groups + 1] */
  const int32_t* prefix_len;     /* device, [groups] */
  int64_t q_stride_token, q_stride_head;   /* in elements; 0, 0 = dense [T, q_heads, d] */
  int64_t o_stride_token, o_stride_head;   /* of out */
} rkv_attend_params;

rkv_status rkv_attend_workspace_size(const rkv_params* prm, const rkv_attend_params* att, size_t* bytes);
rkv_status rkv_attend(const rkv_params* prm, const rkv_attend_params* att, const void* q, const void* k, const void* v,
                      void* out, float* lse, void* ws, size_t ws_bytes, void* stream);
rkv_status rkv_attend_shared(const rkv_params* prm, const rkv_attend_params* att, const void* q, const void* k, const void* v,
                             void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RKV_ATTEND_H */
