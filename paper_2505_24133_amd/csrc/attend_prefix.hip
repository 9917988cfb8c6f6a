// Shared prefixes and the problems' own rows behind them in one launch: the first workgroups take the prefixes (attend_tiles.h, bound by
// their start and by the matrix pipe), the others the own rows of single tokens (attend_small.h, bound by reading the cache), two
// waves of four; neither waits for the other.  64 samples of one prompt of 4099 rows and up to 400 of their own, 8 KV heads of 4: 27 us and 5 of
// the join, 24 + 24 + 8 in launches one after the other; 79 MB, most of them own rows, at 2.5 TB/s, held up by the chain of 21 steps that
// a sixth of a prefix is.  Eight times eight samples behind 8192 rows, four new tokens each: 59 us and 6.
#include "attend_small.h"
#include "attend_tiles.h"

namespace rkv {

int64_t attend_tile_bound(int64_t T, int G, int64_t owners);

namespace {

template <int MT, bool PAGED>
__global__ __launch_bounds__(tiles::kThreads, 2) void attend_prefix_kernel(AttendArgs a, int prefix_blocks) {
  __shared__ __attribute__((aligned(256))) union {
    tiles::Lds tiles;
    small::Lds<MT> small;
  } lds;
  if ((int)blockIdx.x < prefix_blocks) {
    tiles::attend<PAGED, true>(a, a.prefix_splits, blockIdx.x, lds.tiles);
  } else if (threadIdx.x < small::kThreads) {            // (barriers wait for the waves that are left)
    small::attend<MT, PAGED>(a, blockIdx.x - prefix_blocks, lds.small);
  }
}

}  // namespace

hipError_t launch_attend_prefix(const AttendArgs& a, bool paged, hipStream_t stream) {
  const int64_t prefix = attend_tile_bound(a.T, a.G, a.groups) * a.H * a.prefix_splits;
  const dim3 grid((unsigned)(prefix + (int64_t)a.P * a.H * a.small_splits));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(tiles::kThreads), 0, stream, a, (int)prefix); };
  if (a.small_rows <= 16) paged ? go(attend_prefix_kernel<1, true>) : go(attend_prefix_kernel<1, false>);
  else paged ? go(attend_prefix_kernel<2, true>) : go(attend_prefix_kernel<2, false>);
  return hipGetLastError();
}

}  // namespace rkv
