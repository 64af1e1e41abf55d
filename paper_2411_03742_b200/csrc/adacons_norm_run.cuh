// Launches of the norm kernels by type; one translation unit for each block type, so that they compile side by side.
#pragma once

#include "adacons_host.cuh"
#include "adacons_norm.cuh"

namespace adacons {

// How a shape is laid out on the device: threads of a row and of a block, groups of a thread, blocks.
struct NormPlan { int tpr, threads, groups, parts, forward_blocks, backward_blocks, c; };

template <typename X, typename F, int C, bool VEC>
bool norm_launch(const NormParams& p, const NormPlan& n, bool back, cudaStream_t st) {
  if (!back) return launch(&norm_forward_kernel<X, F, C, VEC>, dim3(n.forward_blocks), dim3(n.threads), 0, st, kLaunchPlain, 1, p);
  const size_t fold = n.threads > n.tpr ? static_cast<size_t>(n.threads) * kNormN * sizeof(float) : 0;
  return launch(&norm_backward_kernel<X, F, C, VEC>, dim3(n.backward_blocks), dim3(n.threads), fold, st, kLaunchPlain, 1, p);
}
template <typename X, typename F>
bool norm_launch(const NormParams& p, const NormPlan& n, bool vec, bool back, cudaStream_t st) {
  if (vec) return n.c == 1 ? norm_launch<X, F, 1, true>(p, n, back, st) : n.c == 2 ? norm_launch<X, F, 2, true>(p, n, back, st) : norm_launch<X, F, 4, true>(p, n, back, st);
  return n.c == 1 ? norm_launch<X, F, 1, false>(p, n, back, st) : n.c == 2 ? norm_launch<X, F, 2, false>(p, n, back, st) : norm_launch<X, F, 4, false>(p, n, back, st);
}

// same: the stream is of the block's type, else fp32
bool norm_run_f32(const NormParams& p, const NormPlan& n, bool same, bool vec, bool back, cudaStream_t st);
bool norm_run_bf16(const NormParams& p, const NormPlan& n, bool same, bool vec, bool back, cudaStream_t st);
bool norm_run_f16(const NormParams& p, const NormPlan& n, bool same, bool vec, bool back, cudaStream_t st);
bool norm_run_sum_f32(const NormParams& p, dim3 grid, LaunchKind kind, cudaStream_t st);
bool norm_run_sum_bf16(const NormParams& p, dim3 grid, LaunchKind kind, cudaStream_t st);
bool norm_run_sum_f16(const NormParams& p, dim3 grid, LaunchKind kind, cudaStream_t st);

}  // namespace adacons
