// Host side of rotary positions (include/adacons_ops.h).
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "adacons_host.cuh"
#include "adacons_rope.cuh"

using namespace adacons;

struct adacons_rope {
  int device = 0, sms = 0;
  int rot = 0, interleaved = 0;
  float gain = 1.f;
  double* turns = nullptr;      // device: f_i / (2 pi)
};

namespace {

RopeDivisor divisor(int64_t d) {
  RopeDivisor r;
  r.s = 0;
  while ((1ll << r.s) < d) ++r.s;
  r.m = static_cast<unsigned>(((1ull << (31 + r.s)) + static_cast<unsigned long long>(d) - 1) / static_cast<unsigned long long>(d));
  return r;
}

template <int DT, bool IL>
bool launch_rope(const RopeParams& p, bool vec, unsigned blocks, cudaStream_t st) {
  return vec ? launch(&rope_kernel<DT, IL, true>, dim3(blocks), dim3(kRopeThreads), 0, st, kLaunchPlain, 1, p)
             : launch(&rope_kernel<DT, IL, false>, dim3(blocks), dim3(kRopeThreads), 0, st, kLaunchPlain, 1, p);
}

}  // namespace

extern "C" {

int adacons_rope_create(adacons_rope** out, int rot, const double* frequencies, double gain, int interleaved) {
  if (out == nullptr || frequencies == nullptr || rot < 2 || rot % 2 != 0 || (interleaved != 0 && interleaved != 1) || !std::isfinite(gain)) return ADACONS_EINVAL;
  if (rot > 2 * kRopeMaxTable) return ADACONS_ELIMIT;
  for (int k = 0; k < rot / 2; ++k)
    if (!std::isfinite(frequencies[k])) return ADACONS_EINVAL;
  DeviceInfo info;
  const int rc = query_device(&info);
  if (rc != ADACONS_OK) return rc;
  try {
    std::vector<double> turns(frequencies, frequencies + rot / 2);
    for (double& t : turns) t /= 2.0 * 3.14159265358979323846;
    adacons_rope* c = new adacons_rope();
    c->device = info.device;
    c->sms = info.sms;
    c->rot = rot;
    c->interleaved = interleaved;
    c->gain = static_cast<float>(gain);
    if (cudaMalloc(&c->turns, turns.size() * sizeof(double)) != cudaSuccess) { cudaGetLastError(); delete c; return ADACONS_ENOMEM; }
    if (cudaMemcpy(c->turns, turns.data(), turns.size() * sizeof(double), cudaMemcpyHostToDevice) != cudaSuccess) {
      cudaGetLastError();
      cudaFree(c->turns);
      delete c;
      return ADACONS_ECUDA;
    }
    *out = c;
    return ADACONS_OK;
  } catch (const std::bad_alloc&) {
    return ADACONS_ENOMEM;
  } catch (...) {
    return ADACONS_EINVAL;
  }
}

int adacons_rope_apply(adacons_rope* c, const adacons_rope_shape* s, const void* x, const int64_t* x_strides, void* y, const int64_t* y_strides,
                       const int32_t* positions, int64_t first, int inverse, void* cuda_stream) {
  if (c == nullptr || s == nullptr || x_strides == nullptr || y_strides == nullptr || (inverse != 0 && inverse != 1)) return ADACONS_EINVAL;
  if (s->dtype != ADACONS_F32 && s->dtype != ADACONS_BF16) return ADACONS_EINVAL;
  if (s->batch < 0 || s->len < 0 || s->heads < 0 || s->head_dim < c->rot) return ADACONS_EINVAL;
  if (s->head_dim > (1 << 20) || s->heads > (1 << 20) || s->batch > (1 << 30) || s->len > (1 << 30)) return ADACONS_ELIMIT;
  if (static_cast<int64_t>(s->heads) * s->head_dim > (1 << 26)) return ADACONS_ELIMIT;
  if (s->batch == 0 || s->len == 0 || s->heads == 0) return ADACONS_OK;
  const size_t elem = s->dtype == ADACONS_F32 ? 4 : 2;
  if (x == nullptr || y == nullptr || reinterpret_cast<uintptr_t>(x) % elem != 0 || reinterpret_cast<uintptr_t>(y) % elem != 0) return ADACONS_EINVAL;
  RopeParams p = {};
  p.x = x;
  p.y = y;
  p.positions = positions;
  p.turns = c->turns;
  p.first = first;
  p.tokens = static_cast<long long>(s->batch) * s->len;
  p.seq = s->len;
  p.heads = s->heads;
  p.dim = s->head_dim;
  p.rot = c->rot;
  p.xb = x_strides[0]; p.xs = x_strides[1]; p.xh = x_strides[2];
  p.yb = y_strides[0]; p.ys = y_strides[1]; p.yh = y_strides[2];
  p.gain = c->gain;
  p.inverse = inverse;
  // whole vectors: everything that moves a pointer is a multiple of 16 bytes, and so are the parts of a head
  const int n = static_cast<int>(16 / elem);
  bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(y) % 16 == 0 && p.rot % (2 * n) == 0 && p.dim % n == 0;
  const int sizes[3] = {s->batch, s->len, s->heads};
  for (int k = 0; k < 3; ++k)
    if (sizes[k] > 1 && (x_strides[k] % n != 0 || y_strides[k] % n != 0)) vec = false;
  // Tokens per block: about four vectors' worth of work a thread, but no fewer blocks than fill the device, and a table that fits.
  const int64_t per_token = static_cast<int64_t>(p.heads) * (p.rot / 2 + p.dim - p.rot) / (vec ? n : 1);
  int64_t tpb = std::max<int64_t>(1, (4 * kRopeThreads + per_token - 1) / std::max<int64_t>(1, per_token));
  tpb = std::min<int64_t>(tpb, std::max<int64_t>(1, p.tokens / (4 * c->sms)));
  tpb = std::min<int64_t>(tpb, std::max(1, kRopeMaxTable / (p.rot / 2)));
  tpb = std::min<int64_t>(tpb, kRopeMaxTokens);
  p.tokens_per_block = static_cast<int>(tpb);
  // as the kernel counts them
  const int64_t rest = x == y ? 0 : (p.dim - p.rot) / (vec ? n : 1), per_head = p.rot / 2 / (vec ? n : 1) + (vec ? (rest + 1) / 2 : rest);
  p.per_head = divisor(per_head);
  p.per_token = divisor(per_head * p.heads);
  const int64_t blocks = (p.tokens + tpb - 1) / tpb;
  if (blocks > 0x7fffffff) return ADACONS_ELIMIT;
  DeviceGuard guard(c->device);
  if (!guard.ok) return ADACONS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  bool ok;
  if (s->dtype == ADACONS_F32) ok = c->interleaved ? launch_rope<0, true>(p, vec, static_cast<unsigned>(blocks), st) : launch_rope<0, false>(p, vec, static_cast<unsigned>(blocks), st);
  else ok = c->interleaved ? launch_rope<1, true>(p, vec, static_cast<unsigned>(blocks), st) : launch_rope<1, false>(p, vec, static_cast<unsigned>(blocks), st);
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

int adacons_rope_destroy(adacons_rope* c) {
  if (c == nullptr) return ADACONS_OK;
  DeviceGuard guard(c->device);
  cudaFree(c->turns);
  cudaGetLastError();
  delete c;
  return ADACONS_OK;
}

}  // extern "C"
