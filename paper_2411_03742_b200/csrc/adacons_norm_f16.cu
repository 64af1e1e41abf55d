// The norm kernels of f16 blocks.
#include "adacons_norm_run.cuh"

namespace adacons {

bool norm_run_f16(const NormParams& p, const NormPlan& n, bool same, bool vec, bool back, cudaStream_t st) {
  return same ? norm_launch<__half, __half>(p, n, vec, back, st) : norm_launch<float, __half>(p, n, vec, back, st);
}
bool norm_run_sum_f16(const NormParams& p, dim3 grid, LaunchKind kind, cudaStream_t st) {
  return launch(&norm_sum_kernel<__half>, grid, dim3(kNormSumThreads), 0, st, kind, 1, p);
}

}  // namespace adacons
