// The norm kernels of f32 blocks.
#include "adacons_norm_run.cuh"

namespace adacons {

bool norm_run_f32(const NormParams& p, const NormPlan& n, bool, bool vec, bool back, cudaStream_t st) {
  return norm_launch<float, float>(p, n, vec, back, st);
}
bool norm_run_sum_f32(const NormParams& p, dim3 grid, LaunchKind kind, cudaStream_t st) {
  return launch(&norm_sum_kernel<float>, grid, dim3(kNormSumThreads), 0, st, kind, 1, p);
}

}  // namespace adacons
