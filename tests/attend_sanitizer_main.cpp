// Host-side validation and planning of rkv_attend.h under AddressSanitizer and UndefinedBehaviorSanitizer (host code only): the size query
// over a grid of shapes, and every entry point with arguments that are refused before anything is launched.  Prints "ok <calls>".
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "rkv_attend.h"

static long calls = 0;
#define EXPECT(expr, want)                                                                   \
  do {                                                                                       \
    const int got_ = (int)(expr);                                                            \
    ++calls;                                                                                 \
    if (got_ != (int)(want)) {                                                               \
      std::printf("line %d: %s = %d (%s), expected %d\n", __LINE__, #expr, got_, rkv_status_string((rkv_status)got_), (int)(want)); \
      std::exit(1);                                                                          \
    }                                                                                        \
  } while (0)

int main() {
  void* fake = reinterpret_cast<void*>(0x1000);          // never dereferenced: validation fails first
  const int32_t* list = reinterpret_cast<const int32_t*>(fake);
  rkv_params p;
  std::memset(&p, 0, sizeof p);
  p.num_problems = 2; p.kv_heads = 8; p.q_heads = 32; p.n_tokens = 1152; p.head_dim = 128; p.alpha = 8;
  rkv_attend_params a;
  std::memset(&a, 0, sizeof a);
  a.tokens = 2; a.max_new = 1; a.scale = 0.1f; a.starts = a.kv_len = list;
  size_t bytes = 0;
  EXPECT(rkv_attend_workspace_size(&p, &a, &bytes), RKV_OK);
  EXPECT(rkv_attend_workspace_size(nullptr, &a, &bytes), RKV_ERR_NULL);
  EXPECT(rkv_attend_workspace_size(&p, nullptr, &bytes), RKV_ERR_NULL);
  EXPECT(rkv_attend_workspace_size(&p, &a, nullptr), RKV_ERR_NULL);
  for (int P : {-1, 0, 1, 2, 64, 1000, 1 << 20, INT32_MAX}) for (int H : {0, 1, 8, 1 << 20}) for (int G : {0, 1, 5, 64, 100, 4096})
    for (int N : {0, 1, 31, 1152, 32768, 1 << 24, INT32_MAX}) for (int T : {-1, 0, 1, 63, 4096, 1 << 24, INT32_MAX}) for (int most : {0, 1, 7, 300, INT32_MAX})
      for (int window : {0, 1, 4096, INT32_MAX}) for (int groups : {0, 1, 64}) {
        rkv_params q = p;
        q.num_problems = P; q.kv_heads = H; q.q_heads = (int32_t)((int64_t)H * G > INT32_MAX ? INT32_MAX : H * G); q.n_tokens = N;
        rkv_attend_params b = a;
        b.tokens = T; b.max_new = most; b.window = window; b.sinks = window; b.groups = groups;
        size_t all = 0;
        bytes = 0;
        const int s = rkv_attend_workspace_size(&q, &b, &bytes);
        ++calls;
        if (s > 0 || s < RKV_ERR_HIP) { std::printf("unexpected status %d\n", s); return 1; }
        b.window = 0;
        if (s == RKV_OK && (rkv_attend_workspace_size(&q, &b, &all) != RKV_OK || bytes > all)) { std::printf("a window needs more\n"); return 1; }
      }
  // refused before any launch
  EXPECT(rkv_attend(&p, &a, nullptr, fake, fake, fake, nullptr, fake, SIZE_MAX, nullptr), RKV_ERR_NULL);
  EXPECT(rkv_attend(&p, &a, fake, fake, fake, fake, nullptr, nullptr, 0, nullptr), RKV_ERR_WORKSPACE);
  EXPECT(rkv_attend(&p, &a, fake, fake, fake, reinterpret_cast<void*>(0x1008), nullptr, fake, SIZE_MAX, nullptr), RKV_ERR_SHAPE);
  a.groups = 1;
  EXPECT(rkv_attend(&p, &a, fake, fake, fake, fake, nullptr, fake, SIZE_MAX, nullptr), RKV_ERR_SHAPE);
  EXPECT(rkv_attend_shared(&p, &a, fake, fake, fake, fake, nullptr, fake, SIZE_MAX, nullptr), RKV_ERR_NULL);
  a.groups = 0;
  a.q_stride_token = INT64_MAX - 7; a.q_stride_head = 128;
  EXPECT(rkv_attend_workspace_size(&p, &a, &bytes), RKV_ERR_SHAPE);
  p.page_size = 16; p.table_stride = INT32_MAX; p.block_table = list;
  p.k_stride_page = p.v_stride_page = INT64_MAX - 7; p.k_stride_head = p.v_stride_head = 2048; p.k_stride_token = p.v_stride_token = 128;
  a.q_stride_token = a.q_stride_head = 0; a.num_pages = INT32_MAX;
  EXPECT(rkv_attend_workspace_size(&p, &a, &bytes), RKV_OK);
  rkv_rotary_params r;
  std::memset(&r, 0, sizeof r);
  r.tokens = 2; r.rotary_dim = 128; r.table_rows = 1; r.num_pages = 1;
  r.cos = r.sin = reinterpret_cast<const float*>(fake); r.starts = r.held = r.seen = list;
  EXPECT(rkv_cache_append_rotary(&p, &r, fake, fake, fake, fake, fake, nullptr, fake, nullptr), RKV_ERR_NULL);
  EXPECT(rkv_cache_append_rotary(&p, nullptr, fake, fake, fake, fake, fake, fake, fake, nullptr), RKV_ERR_NULL);
  r.rotary_dim = 24;
  EXPECT(rkv_cache_append_rotary(&p, &r, fake, fake, fake, fake, fake, fake, fake, nullptr), RKV_ERR_UNSUPPORTED);
  r.rotary_dim = 64; r.interleaved = 2;
  EXPECT(rkv_cache_append_rotary(&p, &r, fake, fake, fake, fake, fake, fake, fake, nullptr), RKV_ERR_PARAM);
  r.interleaved = 1; r.tokens = INT32_MAX;
  EXPECT(rkv_cache_append_rotary(&p, &r, fake, fake, fake, fake, fake, fake, fake, nullptr), RKV_ERR_UNSUPPORTED);
  r.tokens = 0;
  EXPECT(rkv_cache_append_rotary(&p, &r, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr), RKV_OK);
  std::printf("ok %ld\n", calls);
  return 0;
}
