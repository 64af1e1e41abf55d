// Launches of the norm kernels by type; one translation unit for each block type, so that they compile side by side.
#pragma once

#include <algorithm>

#include "adacons_host.cuh"
#include "adacons_norm.cuh"

namespace adacons {

// How a shape is laid out on the device: threads of a row, groups of a thread, blocks.
struct NormPlan { int tpr, groups, parts, forward_blocks, backward_blocks, c; };

constexpr int kNormShared = 226 * 1024;          // of an SM: gains and ring


// Rows that a row's threads have under way: as many as fit, four at most (one means that nothing is ahead).
template <typename X, typename F, int C, bool VEC>
bool norm_launch(NormParams p, const NormPlan& n, bool back, cudaStream_t st) {
  const auto kernel = back ? &norm_backward_kernel<X, F, C, VEC> : &norm_forward_kernel<X, F, C, VEC>;
  p.ring = 2 * C * n.tpr * kNormN * static_cast<int>(sizeof(float));
  int shared = p.ring;
  p.depth = 1;
  if (VEC && C <= 2) {
    const int x = static_cast<int>(sizeof(X)) / 2, f = static_cast<int>(sizeof(F)) / 2, gate = p.gate_kind != kGateToken ? 0 : p.gate_as.wide ? 2 : f;
    p.vectors = C * (back ? 2 * x + 2 * f + gate : x + (p.f.data != nullptr ? f : 0) + gate);
    const int row = p.vectors * 16 * kNormThreads;
    const long long turns = back ? (p.tokens / p.groups + p.parts - 1) / p.parts : (p.tokens + n.forward_blocks - 1) / n.forward_blocks;       // tokens of a block
    p.depth = static_cast<int>(std::max(1ll, std::min<long long>({4, (kNormShared - p.ring) / row, (turns * n.tpr + kNormThreads - 1) / kNormThreads})));
    shared += p.depth * row;
  }
  if (back && kNormThreads > n.tpr) shared = std::max(shared, p.ring + C * kNormThreads * kNormN * static_cast<int>(sizeof(float)));
  // Beyond what a kernel has without asking, its static part aside.  The same limit at every launch, whichever thread or device: it costs little beside one.
  if (shared > 40 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormShared) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return launch(kernel, dim3(back ? n.backward_blocks : n.forward_blocks), dim3(kNormThreads), static_cast<size_t>(shared), st, kLaunchPlain, 1, p);
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
