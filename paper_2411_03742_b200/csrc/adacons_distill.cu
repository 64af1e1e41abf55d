// Host side of distillation from top logits (include/adacons_ops.h): checks and launches.
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>

#include "adacons_distill.cuh"
#include "adacons_host.cuh"

using namespace adacons;

namespace {

int size_of(int dtype) { return dtype == ADACONS_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == ADACONS_F32 || dtype == ADACONS_BF16 || dtype == ADACONS_F16; }

int check_shape(const adacons_distill_shape* s) {
  if (s == nullptr || !known(s->dtype) || !known(s->teacher_dtype)) return ADACONS_EINVAL;
  if ((s->ids_bits != 32 && s->ids_bits != 64) || (s->labels_bits != 0 && s->labels_bits != 32 && s->labels_bits != 64)) return ADACONS_EINVAL;
  if (s->tokens < 0 || s->vocab < 1 || s->top < 1) return ADACONS_EINVAL;
  // 1 / tau and tau^2 stay in fp32's range
  if (!(s->temperature >= 0x1p-60f && s->temperature <= 0x1p60f) || !(s->mix >= 0.f && s->mix <= 1.f)) return ADACONS_EINVAL;
  if (s->top > kDistillMaxK || s->vocab > (1 << 30) || s->tokens > (1 << 27)) return ADACONS_ELIMIT;
  return ADACONS_OK;
}

int check_matrix(const adacons_distill_matrix* m, int size, const adacons_distill_shape* s) {
  if (m == nullptr || (s->tokens > 0 && m->data == nullptr)) return ADACONS_EINVAL;
  return reinterpret_cast<uintptr_t>(m->data) % size == 0 ? ADACONS_OK : ADACONS_EALIGN;
}

int check_inputs(const adacons_distill_shape* s, const adacons_distill_matrix* z, const adacons_distill_matrix* ids, const adacons_distill_matrix* teacher, const void* labels) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  if ((rc = check_matrix(z, size_of(s->dtype), s)) != ADACONS_OK || (rc = check_matrix(ids, s->ids_bits / 8, s)) != ADACONS_OK ||
      (rc = check_matrix(teacher, size_of(s->teacher_dtype), s)) != ADACONS_OK)
    return rc;
  if (s->labels_bits == 0) return ADACONS_OK;
  if (s->tokens > 0 && labels == nullptr) return ADACONS_EINVAL;
  return reinterpret_cast<uintptr_t>(labels) % (s->labels_bits / 8) == 0 ? ADACONS_OK : ADACONS_EALIGN;
}

DistillParams base_params(const adacons_distill_shape* s, const adacons_distill_matrix* z, const adacons_distill_matrix* ids, const adacons_distill_matrix* teacher, const void* labels) {
  DistillParams p = {};
  p.z = z->data;
  p.ids = ids->data;
  p.teacher = teacher->data;
  p.labels = s->labels_bits == 0 ? nullptr : labels;
  p.z_row = z->row_stride;
  p.ids_row = ids->row_stride;
  p.teacher_row = teacher->row_stride;
  p.vocab = s->vocab;
  p.top = s->top;
  p.ids_wide = s->ids_bits == 64;
  p.labels_wide = s->labels_bits == 64;
  p.teacher_type = s->teacher_dtype;
  p.tau = s->temperature;
  p.mix = s->mix;
  p.tokens = s->tokens;
  return p;
}
// which exponentials a call takes: see DistillState
int mode_of(const DistillParams& p) { return p.labels == nullptr || p.tau == 1.f ? 0 : p.tau == 2.f || p.tau == 3.f || p.tau == 4.f ? static_cast<int>(p.tau) : 1; }

// A warp for a short vocabulary, sixteen for a long one: a block's start and joins cost about 2 us, and that many more blocks run at once.
int threads_of(int elements) { return elements <= 1024 ? 32 : elements <= 8192 ? 128 : 512; }

// Blocks of a token: twice as many while all of them run at once and each has 4096 logits or more.
int shares_of(int64_t tokens, int vocab, int resident, int most) {
  int shares = 1;
  while (shares < most && tokens * shares * 2 <= resident && vocab / (shares * 2) >= 4096) shares *= 2;
  return shares;
}

template <typename T, int MODE>
bool run(const DistillParams& p, bool back, int threads, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(p.tokens * p.shares)), block(threads);
  return back ? launch(&distill_backward_kernel<T, MODE>, grid, block, 0, st, kLaunchPlain, 1, p) : launch(&distill_forward_kernel<T, MODE>, grid, block, 0, st, kLaunchPlain, p.shares, p);
}
template <typename T>
bool run(const DistillParams& p, bool back, int threads, cudaStream_t st) {
  switch (mode_of(p)) {
    case 0: return run<T, 0>(p, back, threads, st);
    case 1: return run<T, 1>(p, back, threads, st);
    case 2: return run<T, 2>(p, back, threads, st);
    case 3: return run<T, 3>(p, back, threads, st);
    default: return run<T, 4>(p, back, threads, st);
  }
}
bool run(const adacons_distill_shape* s, const DistillParams& p, bool back, cudaStream_t st) {
  const int threads = threads_of(p.vocab / p.shares);
  if (s->dtype == ADACONS_F32) return run<float>(p, back, threads, st);
  return s->dtype == ADACONS_BF16 ? run<__nv_bfloat16>(p, back, threads, st) : run<__half>(p, back, threads, st);
}

}  // namespace

extern "C" {

int adacons_distill_forward(const adacons_distill_shape* s, const adacons_distill_matrix* logits, const adacons_distill_matrix* ids, const adacons_distill_matrix* teacher,
                            const void* labels, float* loss, float* rows, void* cuda_stream) {
  int rc = check_inputs(s, logits, ids, teacher, labels);
  if (rc != ADACONS_OK) return rc;
  if (s->tokens == 0) return ADACONS_OK;
  if (loss == nullptr || rows == nullptr || reinterpret_cast<uintptr_t>(loss) % 4 != 0 || reinterpret_cast<uintptr_t>(rows) % 4 != 0 || loss == rows) return ADACONS_EINVAL;
  for (const void* r : {static_cast<const void*>(loss), static_cast<const void*>(rows)})
    if (r == logits->data || r == ids->data || r == teacher->data || (s->labels_bits != 0 && r == labels)) return ADACONS_EINVAL;
  int sms = 0;
  if ((rc = device_sms(&sms)) != ADACONS_OK) return rc;
  DistillParams p = base_params(s, logits, ids, teacher, labels);
  p.loss = loss;
  p.rows = rows;
  p.shares = shares_of(p.tokens, p.vocab, 2 * sms, 8);
  return run(s, p, false, static_cast<cudaStream_t>(cuda_stream)) ? ADACONS_OK : ADACONS_ECUDA;
}

int adacons_distill_backward(const adacons_distill_shape* s, const float* dloss, int64_t dloss_stride, const adacons_distill_matrix* logits, const adacons_distill_matrix* ids,
                             const adacons_distill_matrix* teacher, const void* labels, const float* rows, const adacons_distill_matrix* dlogits, void* cuda_stream) {
  int rc = check_inputs(s, logits, ids, teacher, labels);
  if (rc != ADACONS_OK) return rc;
  const int size = size_of(s->dtype);
  if ((rc = check_matrix(dlogits, size, s)) != ADACONS_OK) return rc;
  if (s->tokens == 0) return ADACONS_OK;
  if (dloss == nullptr || rows == nullptr || reinterpret_cast<uintptr_t>(dloss) % 4 != 0 || reinterpret_cast<uintptr_t>(rows) % 4 != 0) return ADACONS_EINVAL;
  const void* to = dlogits->data;
  if (to == ids->data || to == teacher->data || to == rows || to == dloss || (s->labels_bits != 0 && to == labels)) return ADACONS_EINVAL;
  if (to == logits->data && s->tokens > 1 && dlogits->row_stride != logits->row_stride) return ADACONS_EINVAL;      // dlogits may take logits' place
  int sms = 0;
  if ((rc = device_sms(&sms)) != ADACONS_OK) return rc;
  DistillParams p = base_params(s, logits, ids, teacher, labels);
  p.dloss = dloss;
  p.dloss_step = dloss_stride;
  p.rows = const_cast<float*>(rows);
  p.dz = dlogits->data;
  p.dz_row = dlogits->row_stride;
  p.vectors = (reinterpret_cast<uintptr_t>(p.dz) - reinterpret_cast<uintptr_t>(p.z)) % 16 == 0 && (p.tokens == 1 || (p.dz_row - p.z_row) * size % 16 == 0);
  p.shares = shares_of(p.tokens, p.vocab, 2 * sms, 64);
  return run(s, p, true, static_cast<cudaStream_t>(cuda_stream)) ? ADACONS_OK : ADACONS_ECUDA;
}

}  // extern "C"
