// The many-rows attention (attend_tiles.h) of problems' own rows and of shared prefixes, each in a launch of its own.
#include "attend_tiles.h"

namespace rkv {

namespace {

template <bool PAGED, bool PREFIX>
__global__ __launch_bounds__(tiles::kThreads, 2) void attend_tiles_kernel(AttendArgs a, int splits) {
  __shared__ __attribute__((aligned(256))) tiles::Lds lds;
  tiles::attend<PAGED, PREFIX>(a, splits, blockIdx.x, lds);
}

}  // namespace

// The most tiles that T tokens of `owners` problems or groups can make.
int64_t attend_tile_bound(int64_t T, int G, int64_t owners) { return T * G / kTileRows + (owners < T ? owners : T); }

hipError_t launch_attend_tiles(const AttendArgs& a, bool paged, bool prefix, hipStream_t stream) {
  const int splits = prefix ? a.prefix_splits : a.tile_splits;
  const dim3 grid((unsigned)(attend_tile_bound(a.T, a.G, prefix ? a.groups : a.P) * a.H * splits));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(tiles::kThreads), 0, stream, a, splits); };
  if (prefix) paged ? go(attend_tiles_kernel<true, true>) : go(attend_tiles_kernel<false, true>);
  else paged ? go(attend_tiles_kernel<true, false>) : go(attend_tiles_kernel<false, false>);
  return hipGetLastError();
}

}  // namespace rkv
