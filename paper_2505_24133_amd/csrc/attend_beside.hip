// Both attention kernels in one launch: the first workgroups take tiles of many rows (attend_tiles.h: shared prefixes, or the prompts of a
// batch), the others the units of few (attend_small.h: what lies behind the prefixes, or the batch's single tokens), two waves of four;
// neither waits for the other.
// 64 samples of one prompt of 4099 rows and up to 400 of their own, 8 KV heads of 4: 27 us and 5 of the join, 24 + 24 + 8 in launches one
// after the other; 79 MB, most of them own rows, at 2.5 TB/s, held up by the chain of 21 steps that a sixth of a prefix is.  Eight times
// eight samples behind 8192 rows, four new tokens each: 59 us and 6.
#include "attend_small.h"
#include "attend_tiles.h"

namespace rkv {

int64_t attend_tile_bound(int64_t T, int G, int64_t owners);

namespace {

template <int MT, bool PAGED, bool PREFIX>
__global__ __launch_bounds__(tiles::kThreads, 2) void attend_beside_kernel(AttendArgs a, int splits, int tile_blocks) {
  __shared__ __attribute__((aligned(256))) union {
    tiles::Lds tiles;
    small::Lds<MT> small;
  } lds;
  if ((int)blockIdx.x < tile_blocks) {
    tiles::attend<PAGED, PREFIX>(a, splits, blockIdx.x, lds.tiles);
  } else if (threadIdx.x < small::kThreads) {            // (barriers wait for the waves that are left)
    small::attend<MT, PAGED>(a, blockIdx.x - tile_blocks, lds.small);
  }
}

}  // namespace

hipError_t launch_attend_beside(const AttendArgs& a, bool paged, bool prefix, hipStream_t stream) {
  const int splits = prefix ? a.prefix_splits : a.tile_splits;
  const int64_t first = attend_tile_bound(a.T, a.G, prefix ? a.groups : a.P) * a.H * splits;
  const dim3 grid((unsigned)(first + (int64_t)a.P * a.H * a.small_splits));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(tiles::kThreads), 0, stream, a, splits, (int)first); };
  if (!prefix && a.small_rows <= 16) paged ? go(attend_beside_kernel<1, true, false>) : go(attend_beside_kernel<1, false, false>);
  else if (!prefix) paged ? go(attend_beside_kernel<2, true, false>) : go(attend_beside_kernel<2, false, false>);
  else if (a.small_rows <= 16) paged ? go(attend_beside_kernel<1, true, true>) : go(attend_beside_kernel<1, false, true>);
  else paged ? go(attend_beside_kernel<2, true, true>) : go(attend_beside_kernel<2, false, true>);
  return hipGetLastError();
}

}  // namespace rkv
