// What operators report of numbers that no kernel of theirs looks at, because the result has no elements.
#include "operators/common.cuh"

namespace acc {
namespace ops {
namespace {

__global__ void __launch_bounds__(256) k_look_over(Report report, const int* x, int64_t n, int bound) {
  follow();
  bool bad = false;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) bad = bad || x[i] >= bound;
  if (bad) raise_index(report);
}

}  // namespace

int report_beyond(const ClusterLaunch& L, const int* x, int64_t n, int bound) {
  if (n == 0) return ACC_OK;
  ++L.extra_launches;
  const int grid = (int)std::min<int64_t>((n + 255) / 256, (int64_t)sm_count() * 8);
  return launch_following(k_look_over, dim3(grid), 256, 0, L.stream, report_of(L), x, n, bound);
}

}  // namespace ops
}  // namespace acc
