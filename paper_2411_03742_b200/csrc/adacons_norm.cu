// Host side of the norms around a block (include/adacons_ops.h): checks and launches.
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>

#include "adacons_host.cuh"
#include "adacons_norm_run.cuh"

using namespace adacons;

namespace {

NormDivisor divisor(int d) {
  NormDivisor r;
  r.s = 0;
  while ((1ll << r.s) < d) ++r.s;
  r.m = static_cast<unsigned>(((1ull << (31 + r.s)) + static_cast<unsigned long long>(d) - 1) / static_cast<unsigned long long>(d));
  return r;
}

int size_of(int dtype) { return dtype == ADACONS_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == ADACONS_F32 || dtype == ADACONS_BF16 || dtype == ADACONS_F16; }

int check_shape(const adacons_norm_shape* s) {
  if (s == nullptr || !known(s->stream_dtype) || !known(s->dtype)) return ADACONS_EINVAL;
  if (s->stream_dtype != s->dtype && s->stream_dtype != ADACONS_F32) return ADACONS_EINVAL;
  if (s->batch < 0 || s->len < 0 || s->dim < 1) return ADACONS_EINVAL;
  if (s->gate < ADACONS_NORM_GATE_NONE || s->gate > ADACONS_NORM_GATE_TOKEN || s->gate_by < ADACONS_NORM_BY_ITSELF || s->gate_by > ADACONS_NORM_BY_TANH) return ADACONS_EINVAL;
  for (int t : {s->gate_dtype, s->post_dtype, s->pre_dtype})
    if (t != ADACONS_F32 && t != s->dtype) return ADACONS_EINVAL;
  if (!std::isfinite(s->scale) || !(s->eps > 0.f) || !std::isfinite(s->eps)) return ADACONS_EINVAL;
  if (s->dim > kNormMaxDim || static_cast<int64_t>(s->batch) * s->len > 0x7fffffff) return ADACONS_ELIMIT;
  return ADACONS_OK;
}

// Two groups a thread for rows that are moved in vectors; one where single elements are, whose loads otherwise wait for one another.
NormPlan plan_of(const adacons_norm_shape* s, int sms, bool vec) {
  NormPlan n = {};
  n.c = s->dim <= (vec ? 256 : 4096) ? 1 : s->dim <= 8192 ? 2 : 4;
  const int wanted = (s->dim + kNormN * n.c - 1) / (kNormN * n.c);
  n.tpr = 32;
  while (n.tpr < wanted) n.tpr *= 2;
  const int64_t tokens = static_cast<int64_t>(s->batch) * s->len;
  const int per_block = kNormThreads / n.tpr;
  n.forward_blocks = static_cast<int>(std::min<int64_t>((tokens + per_block - 1) / per_block, sms));
  // Backward: a share of a group has a row for each of a block's, or more, and there are no more shares than blocks at once.
  n.groups = s->gate == ADACONS_NORM_GATE_SEQUENCE ? std::max(1, s->batch) : 1;
  const int64_t of_group = tokens / n.groups;
  n.parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((of_group + per_block - 1) / per_block, sms / n.groups)));
  n.backward_blocks = static_cast<int>(std::min<int64_t>(static_cast<int64_t>(n.groups) * n.parts, sms));
  return n;
}

// Records of the sums over tokens: one row of `dim` for each item, and one for each block where `pre` has a gradient.
int64_t item_records(const NormPlan& n) { return static_cast<int64_t>(n.groups) * n.parts; }
int64_t workspace_bytes(const adacons_norm_shape* s, int sms) {
  int64_t records = 0;
  for (bool vec : {false, true}) {
    const NormPlan n = plan_of(s, sms, vec);
    records = std::max(records, item_records(n) + n.backward_blocks);
  }
  return records * s->dim * static_cast<int64_t>(sizeof(float));
}

// Strides of dimensions of size one are never used, whatever the caller has there.
int check_rows(const adacons_norm_rows* t, int dtype, const adacons_norm_shape* s, bool optional) {
  if (t == nullptr) return optional ? ADACONS_OK : ADACONS_EINVAL;
  if (s->batch == 0 || s->len == 0) return ADACONS_OK;
  if (t->data == nullptr) return optional ? ADACONS_OK : ADACONS_EINVAL;
  return reinterpret_cast<uintptr_t>(t->data) % size_of(dtype) == 0 ? ADACONS_OK : ADACONS_EALIGN;
}

NormRows as_rows(const adacons_norm_rows* t) {
  if (t == nullptr || t->data == nullptr) return {nullptr, 0, 0};
  return {t->data, t->batch_stride, t->row_stride};
}

bool same_place(const adacons_norm_rows* a, const adacons_norm_rows* b) { return a != nullptr && b != nullptr && a->data != nullptr && a->data == b->data; }
bool same_rows(const adacons_norm_rows* a, const adacons_norm_rows* b, const adacons_norm_shape* s) {
  return same_place(a, b) && (s->batch == 1 || a->batch_stride == b->batch_stride) && (s->len == 1 || a->row_stride == b->row_stride);
}

// Whole vectors of 16 bytes: every address that a row or a gain starts at is a multiple of them.
struct Vectors {
  bool ok;
  explicit Vectors(const adacons_norm_shape* s) : ok(s->dim % kNormN == 0) {}
  void gain(const void* p) { ok = ok && reinterpret_cast<uintptr_t>(p) % 16 == 0; }
  void rows(const adacons_norm_rows* t, int dtype, int batch, int len) {
    if (t == nullptr || t->data == nullptr) return;
    const int n = 16 / size_of(dtype);
    gain(t->data);
    ok = ok && (batch <= 1 || t->batch_stride % n == 0) && (len <= 1 || t->row_stride % n == 0);
  }
};

NormParams base_params(const adacons_norm_shape* s, const NormPlan& n, const adacons_norm_rows* f, const adacons_norm_rows* gate, const void* post, const void* pre) {
  NormParams p = {};
  p.f = as_rows(f);
  p.gate_kind = p.f.data != nullptr ? s->gate : kGateNone;
  if (p.gate_kind != kGateNone) p.gate = as_rows(gate);
  if (p.gate_kind == kGateSequence) p.gate.row = 0;
  p.gate_as = {nullptr, s->gate_dtype == ADACONS_F32};
  p.post = {p.f.data != nullptr ? post : nullptr, s->post_dtype == ADACONS_F32};
  p.pre = {pre, s->pre_dtype == ADACONS_F32};
  p.by = s->gate_by;
  p.tokens = static_cast<int64_t>(s->batch) * s->len;
  p.len = s->len;
  p.dim = s->dim;
  p.tpr = n.tpr;
  p.scale = s->scale;
  p.eps = s->eps;
  p.share = static_cast<float>(1.0 / s->dim);
  p.by_len = divisor(std::max(1, s->len));
  return p;
}

bool go(const adacons_norm_shape* s, const NormParams& p, const NormPlan& n, bool vec, bool back, cudaStream_t st) {
  const bool same = s->stream_dtype == s->dtype;
  if (s->dtype == ADACONS_F32) return norm_run_f32(p, n, same, vec, back, st);
  return s->dtype == ADACONS_BF16 ? norm_run_bf16(p, n, same, vec, back, st) : norm_run_f16(p, n, same, vec, back, st);
}

int check_gains(const adacons_norm_shape* s, const void* post, const void* pre) {
  if (reinterpret_cast<uintptr_t>(post) % size_of(s->post_dtype) != 0 || reinterpret_cast<uintptr_t>(pre) % size_of(s->pre_dtype) != 0) return ADACONS_EALIGN;
  return ADACONS_OK;
}
// A gate's rows: none, one, one for each sequence, one for each token.
int check_gate(const adacons_norm_shape* s, const adacons_norm_rows* gate) {
  if (s->gate == ADACONS_NORM_GATE_NONE) return ADACONS_OK;
  if (gate == nullptr || (s->batch > 0 && (s->len > 0 || s->gate == ADACONS_NORM_GATE_SEQUENCE) && gate->data == nullptr)) return ADACONS_EINVAL;
  if (s->gate == ADACONS_NORM_GATE_CHANNEL && gate->data == nullptr) return ADACONS_EINVAL;
  return reinterpret_cast<uintptr_t>(gate->data) % size_of(s->gate_dtype) == 0 ? ADACONS_OK : ADACONS_EALIGN;
}
int gate_batch(const adacons_norm_shape* s) { return s->gate >= ADACONS_NORM_GATE_SEQUENCE ? s->batch : 1; }
int gate_len(const adacons_norm_shape* s) { return s->gate == ADACONS_NORM_GATE_TOKEN ? s->len : 1; }

}  // namespace

extern "C" {

int adacons_norm_forward(const adacons_norm_shape* s, const adacons_norm_rows* x, const adacons_norm_rows* f, const adacons_norm_rows* gate, const void* post,
                         const void* pre, const adacons_norm_rows* out, const adacons_norm_rows* normed, float* rows, void* cuda_stream) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  const bool has_f = f != nullptr && f->data != nullptr;
  if ((rc = check_rows(x, s->stream_dtype, s, false)) != ADACONS_OK || (rc = check_rows(f, s->dtype, s, true)) != ADACONS_OK ||
      (rc = check_rows(out, s->stream_dtype, s, !has_f)) != ADACONS_OK || (rc = check_rows(normed, s->dtype, s, pre == nullptr)) != ADACONS_OK ||
      (rc = check_gains(s, post, pre)) != ADACONS_OK)
    return rc;
  if (has_f && (rc = check_gate(s, gate)) != ADACONS_OK) return rc;
  if (s->batch == 0 || s->len == 0) return ADACONS_OK;
  if (!has_f && pre == nullptr) return ADACONS_OK;
  if (rows == nullptr || reinterpret_cast<uintptr_t>(rows) % 4 != 0) return ADACONS_EINVAL;
  const adacons_norm_rows* gate_rows = has_f && s->gate != ADACONS_NORM_GATE_NONE ? gate : nullptr;
  const adacons_norm_rows* to_normed = pre != nullptr ? normed : nullptr;
  const adacons_norm_rows* to_out = has_f ? out : nullptr;
  // results in the place of what is read, or of one another; x' may take x's place
  if ((same_place(to_out, x) && !same_rows(to_out, x, s)) || same_place(to_out, f) || same_place(to_out, gate_rows) || same_place(to_normed, x) || same_place(to_normed, f) ||
      same_place(to_normed, gate_rows) || same_place(to_normed, to_out))
    return ADACONS_EINVAL;
  int sms = 0;
  if ((rc = device_sms(&sms)) != ADACONS_OK) return rc;
  Vectors v(s);
  v.rows(x, s->stream_dtype, s->batch, s->len);
  v.rows(f, s->dtype, s->batch, s->len);
  v.rows(to_out, s->stream_dtype, s->batch, s->len);
  v.rows(to_normed, s->dtype, s->batch, s->len);
  v.rows(gate_rows, s->gate_dtype, gate_batch(s), gate_len(s));
  if (has_f) v.gain(post);
  v.gain(pre);
  const NormPlan n = plan_of(s, sms, v.ok);
  NormParams p = base_params(s, n, f, gate, post, pre);
  p.x = as_rows(x);
  p.out = as_rows(to_out);
  p.normed = as_rows(to_normed);
  p.rows = rows;
  return go(s, p, n, v.ok, false, static_cast<cudaStream_t>(cuda_stream)) ? ADACONS_OK : ADACONS_ECUDA;
}

int adacons_norm_workspace_bytes(const adacons_norm_shape* s, int64_t* bytes) {
  if (bytes == nullptr) return ADACONS_EINVAL;
  int rc = check_shape(s), sms = 0;
  if (rc != ADACONS_OK || (rc = device_sms(&sms)) != ADACONS_OK) return rc;
  *bytes = workspace_bytes(s, sms);
  return ADACONS_OK;
}

int adacons_norm_backward(const adacons_norm_shape* s, const adacons_norm_rows* dout, const adacons_norm_rows* dnormed, const adacons_norm_rows* out, const adacons_norm_rows* f,
                          const adacons_norm_rows* gate, const void* post, const void* pre, const float* rows, const adacons_norm_rows* dx, const adacons_norm_rows* df,
                          const adacons_norm_rows* dgate, void* dpost, void* dpre, void* workspace, int64_t bytes, void* cuda_stream) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  const bool has_f = f != nullptr && f->data != nullptr, has_pre = pre != nullptr && dnormed != nullptr && dnormed->data != nullptr;
  if ((rc = check_rows(dout, s->stream_dtype, s, true)) != ADACONS_OK || (rc = check_rows(dnormed, s->dtype, s, true)) != ADACONS_OK ||
      (rc = check_rows(out, s->stream_dtype, s, !has_pre)) != ADACONS_OK || (rc = check_rows(f, s->dtype, s, true)) != ADACONS_OK ||
      (rc = check_rows(dx, s->stream_dtype, s, false)) != ADACONS_OK || (rc = check_rows(df, s->dtype, s, !has_f)) != ADACONS_OK ||
      (rc = check_gains(s, post, pre)) != ADACONS_OK || (rc = check_gains(s, dpost, dpre)) != ADACONS_OK)
    return rc;
  const bool has_post = has_f && post != nullptr, has_gate = has_f && s->gate != ADACONS_NORM_GATE_NONE;
  if (has_gate && ((rc = check_gate(s, gate)) != ADACONS_OK || (rc = check_gate(s, dgate)) != ADACONS_OK)) return rc;
  if ((has_post && dpost == nullptr) || (pre != nullptr && dpre == nullptr)) return ADACONS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool empty = s->batch == 0 || s->len == 0;
  if (empty) {                                   // sums over no tokens; tensors without elements may all be at address 0
    bool ok = true;
    if (dpost != nullptr) ok = ok && cudaMemsetAsync(dpost, 0, static_cast<size_t>(s->dim) * size_of(s->post_dtype), st) == cudaSuccess;
    if (dpre != nullptr) ok = ok && cudaMemsetAsync(dpre, 0, static_cast<size_t>(s->dim) * size_of(s->pre_dtype), st) == cudaSuccess;
    const bool summed = dgate != nullptr && dgate->data != nullptr;
    const int rows = !summed ? 0 : s->gate == ADACONS_NORM_GATE_CHANNEL ? 1 : s->gate == ADACONS_NORM_GATE_SEQUENCE ? s->batch : 0;
    const size_t size = size_of(s->gate_dtype), width = s->dim * size, pitch = rows > 1 ? static_cast<size_t>(dgate->batch_stride) * size : width;
    if (rows > 0) ok = ok && cudaMemset2DAsync(dgate->data, pitch, 0, width, rows, st) == cudaSuccess;
    if (!ok) cudaGetLastError();
    return ok ? ADACONS_OK : ADACONS_ECUDA;
  }
  if ((has_post || has_pre) && (rows == nullptr || reinterpret_cast<uintptr_t>(rows) % 4 != 0)) return ADACONS_EINVAL;
  const adacons_norm_rows *gate_rows = has_gate ? gate : nullptr, *to_gate = has_gate ? dgate : nullptr, *to_f = has_f ? df : nullptr;
  const adacons_norm_rows* reads[] = {has_pre ? out : nullptr, has_pre ? dnormed : nullptr, has_f ? f : nullptr, gate_rows};
  const adacons_norm_rows* writes[] = {dx, to_f, to_gate};
  for (const adacons_norm_rows* w : writes) {
    for (const adacons_norm_rows* r : reads)
      if (same_place(w, r)) return ADACONS_EINVAL;
    for (const adacons_norm_rows* other : writes)
      if (w != other && same_place(w, other)) return ADACONS_EINVAL;
  }
  if (same_place(dx, dout) && !same_rows(dx, dout, s)) return ADACONS_EINVAL;      // dx may take dout's place
  if (same_place(to_f, dout) || same_place(to_gate, dout)) return ADACONS_EINVAL;
  int sms = 0;
  if ((rc = device_sms(&sms)) != ADACONS_OK) return rc;
  Vectors v(s);
  v.rows(dout, s->stream_dtype, s->batch, s->len);
  v.rows(dx, s->stream_dtype, s->batch, s->len);
  if (has_pre) {
    v.rows(out, s->stream_dtype, s->batch, s->len);
    v.rows(dnormed, s->dtype, s->batch, s->len);
  }
  v.rows(has_f ? f : nullptr, s->dtype, s->batch, s->len);
  v.rows(to_f, s->dtype, s->batch, s->len);
  v.rows(gate_rows, s->gate_dtype, gate_batch(s), gate_len(s));
  v.rows(to_gate, s->gate_dtype, gate_batch(s), gate_len(s));
  if (has_f) v.gain(post);
  v.gain(pre);
  const NormPlan n = plan_of(s, sms, v.ok);
  const bool wants_sum = has_post || (has_gate && s->gate != ADACONS_NORM_GATE_TOKEN);
  if (wants_sum || pre != nullptr) {
    if (workspace == nullptr || bytes < workspace_bytes(s, sms)) return ADACONS_EINVAL;
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return ADACONS_EALIGN;
  }
  NormParams p = base_params(s, n, f, gate, post, pre);
  p.dout = as_rows(dout);
  if (has_pre) {
    p.dnormed = as_rows(dnormed);
    p.out = as_rows(out);
  }
  p.dx = as_rows(dx);
  p.df = as_rows(to_f);
  p.dgate = as_rows(to_gate);
  p.rows = const_cast<float*>(rows);
  p.dpost = has_post ? dpost : nullptr;
  p.dpre = pre != nullptr ? dpre : nullptr;
  p.groups = n.groups;
  p.parts = n.parts;
  p.blocks = n.backward_blocks;
  if (wants_sum) p.sums = static_cast<float*>(workspace);
  if (has_pre) p.pre_sums = static_cast<float*>(workspace) + item_records(n) * s->dim;
  if (!go(s, p, n, v.ok, true, st)) return ADACONS_ECUDA;
  if (!wants_sum && pre == nullptr) return ADACONS_OK;
  const dim3 grid(static_cast<unsigned>((s->dim + 31) / 32));
  const LaunchKind kind = kLaunchOverlap;
  bool ok;
  if (s->dtype == ADACONS_F32) ok = norm_run_sum_f32(p, grid, kind, st);
  else if (s->dtype == ADACONS_BF16) ok = norm_run_sum_bf16(p, grid, kind, st);
  else ok = norm_run_sum_f16(p, grid, kind, st);
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

}  // extern "C"
