// The launches that calls of rkv_attend.h ask for, recorded instead of made: this program defines the runtime's launch entry itself, so that
// the library's calls end here and no GPU is needed.  A launch holds at least one and fewer than 2^32 work items.  Goes through sizes up to
// the largest that are taken; prints a line for every call that is accepted and then not launched, and at the end how many were taken.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstring>

#include "rkv_attend.h"

static bool refused = false;
static long long launches = 0, largest = 0;
static dim3 grid_of, block_of;

extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  grid_of = grid; block_of = block;
  return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = grid_of; *block = block_of; *shared = 0; *stream = nullptr;
  return hipSuccess;
}
extern "C" hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  ++launches;
  const unsigned long long items = (unsigned long long)grid.x * block.x;
  if (items >= 1ull << 32 || grid.x == 0 || grid.y != 1 || grid.z != 1) refused = true;
  if ((long long)items > largest) largest = (long long)items;
  return hipSuccess;
}
extern "C" hipError_t hipGetLastError() {
  const bool r = refused;
  refused = false;
  return r ? hipErrorInvalidConfiguration : hipSuccess;
}

int main() {
  void* fake = reinterpret_cast<void*>(0x1000);
  const int32_t* list = static_cast<const int32_t*>(fake);
  long long taken = 0, bad = 0;
  for (int P : {1, 2, 3, 64, 4096, 1 << 20, 1 << 22})
    for (int H : {1, 2, 8})
      for (int G : {1, 5, 8, 63, 64, 65, 512})
        for (int N : {1, 1000, 40000, 1 << 24})
          for (int T : {1, 2, 100, 70000, 1 << 20, 1 << 21, 1 << 24})
            for (int bound = 0; bound < 3; ++bound)
              for (int groups : {0, 1, P})
                for (int window : {0, 100}) {
                  rkv_params p;
                  rkv_attend_params a;
                  std::memset(&p, 0, sizeof p);
                  std::memset(&a, 0, sizeof a);
                  p.num_problems = P; p.kv_heads = H; p.q_heads = H * G; p.n_tokens = N; p.head_dim = 128; p.alpha = 8;
                  a.tokens = T; a.max_new = bound == 0 ? 1 : (bound == 1 ? T : T / 2 + 1); a.window = window; a.sinks = 4; a.groups = groups; a.scale = 0.1f;
                  a.starts = a.kv_len = a.group_starts = a.prefix_len = list;
                  const rkv_status s = rkv_attend_shared(&p, &a, fake, fake, fake, fake, nullptr, fake, ~(size_t)0, nullptr);
                  if (s == RKV_OK) ++taken;
                  else if (s != RKV_ERR_UNSUPPORTED) {
                    ++bad;
                    std::printf("status %d: P %d H %d G %d N %d T %d max_new %d groups %d window %d\n", (int)s, P, H, G, N, T, a.max_new, groups, window);
                  }
                }
  for (int P : {1, 1 << 20})
    for (int T : {1, 1 << 23}) {
      rkv_params p;
      rkv_rotary_params r;
      std::memset(&p, 0, sizeof p);
      std::memset(&r, 0, sizeof r);
      p.num_problems = P; p.kv_heads = 2; p.q_heads = 4; p.n_tokens = 100; p.head_dim = 128; p.alpha = 8;
      r.tokens = T; r.rotary_dim = 128; r.table_rows = 10; r.cos = r.sin = static_cast<const float*>(fake);
      r.starts = r.held = r.seen = list;
      const rkv_status s = rkv_cache_append_rotary(&p, &r, fake, fake, fake, fake, fake, fake, fake, nullptr);
      if (s == RKV_OK) ++taken;
      else { ++bad; std::printf("append status %d: P %d T %d\n", (int)s, P, T); }
    }
  std::printf("taken %lld bad %lld launches %lld largest %lld\n", taken, bad, launches, largest);
  return 0;
}
