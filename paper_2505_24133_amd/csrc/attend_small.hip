// The few-rows attention (attend_small.h) in a launch of its own.
#include "attend_small.h"

namespace rkv {

namespace {

template <int MT, bool PAGED>
__global__ __launch_bounds__(small::kThreads) void attend_small_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(256))) small::Lds<MT> lds;
  small::attend<MT, PAGED>(a, blockIdx.x, lds);
}

}  // namespace

hipError_t launch_attend_small(const AttendArgs& a, bool paged, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)a.P * a.H * a.small_splits));
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(small::kThreads), 0, stream, a); };
  if (a.small_rows <= 16) paged ? go(attend_small_kernel<1, true>) : go(attend_small_kernel<1, false>);
  else paged ? go(attend_small_kernel<2, true>) : go(attend_small_kernel<2, false>);
  return hipGetLastError();
}

}  // namespace rkv
