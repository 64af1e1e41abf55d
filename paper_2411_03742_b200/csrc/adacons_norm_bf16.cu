// The norm kernels of bf16 blocks.
#include "adacons_norm_run.cuh"

namespace adacons {

bool norm_run_bf16(const NormParams& p, const NormPlan& n, bool same, bool vec, bool back, cudaStream_t st) {
  return same ? norm_launch<__nv_bfloat16, __nv_bfloat16>(p, n, vec, back, st) : norm_launch<float, __nv_bfloat16>(p, n, vec, back, st);
}
bool norm_run_sum_bf16(const NormParams& p, dim3 grid, LaunchKind kind, cudaStream_t st) {
  return launch(&norm_sum_kernel<__nv_bfloat16>, grid, dim3(kNormSumThreads), 0, st, kind, 1, p);
}

}  // namespace adacons
