// Host side of attention and its gradient (include/adacons_ops.h): checks, tensor maps and launches.
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>
#include <mutex>

#include "adacons_attn.cuh"
#include "adacons_host.cuh"

using namespace adacons;

static __device__ uint32_t g_attn_flags;

namespace {

constexpr int kMaxDevices = 64;

struct AttnDevice {
  bool ready = false;
  DeviceInfo info;
  uint32_t* flags = nullptr;
};

template <typename K>
bool raise(K kernel, uint32_t bytes) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) == cudaSuccess) return true;
  cudaGetLastError();
  return false;
}
template <int D, bool BF16, bool STARVE = false>
bool raise_all() {
  static_assert(AttnFwdSmem<D>::kBytes <= 112 * 1024 && attn_backward_smem<D>() <= (AttnBwd<D>::kBlocks == 2 ? 112 : 227) * 1024, "shared memory of a block");
  return raise(attn_forward_kernel<D, BF16, STARVE>, AttnFwdSmem<D>::kBytes) && raise(attn_backward_kernel<D, BF16, STARVE>, attn_backward_smem<D>());
}

// The first call on a device sets the kernels' shared-memory limits; later ones only look the entry up.
int attn_device(AttnDevice** out) {
  static std::mutex mutex;
  static AttnDevice devices[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
  if (dev < 0 || dev >= kMaxDevices) return ADACONS_ELIMIT;
  std::lock_guard<std::mutex> lock(mutex);
  AttnDevice& d = devices[dev];
  if (!d.ready) {
    const int rc = query_device(&d.info);
    if (rc != ADACONS_OK) return rc;
    void* flags = nullptr;
    if (!raise_all<64, true>() || !raise_all<64, false>() || !raise_all<128, true>() || !raise_all<128, false>() ||
        cudaGetSymbolAddress(&flags, g_attn_flags) != cudaSuccess) {
      cudaGetLastError();
      return ADACONS_ECUDA;
    }
    d.flags = static_cast<uint32_t*>(flags);
    d.ready = true;
  }
  *out = &d;
  return ADACONS_OK;
}

int check_shape(const adacons_attn_shape* s) {
  if (s == nullptr) return ADACONS_EINVAL;
  if (s->dtype != ADACONS_BF16 && s->dtype != ADACONS_F16) return ADACONS_EINVAL;
  if (s->batch < 0 || s->q_heads < 1 || s->kv_heads < 1 || s->q_heads % s->kv_heads != 0 || s->q_len < 0 || s->kv_len < 0) return ADACONS_EINVAL;
  if (s->head_dim < 8 || s->head_dim % 8 != 0) return ADACONS_EINVAL;
  if (!(s->scale > 0.f) || !std::isfinite(s->scale) || (s->causal != 0 && s->causal != 1)) return ADACONS_EINVAL;
  if (s->head_dim > 128 || s->batch > 65535 || s->q_heads > 65535 || s->q_len > (1 << 30) || s->kv_len > (1 << 30)) return ADACONS_ELIMIT;
  return ADACONS_OK;
}

// Strides of dimensions of size one are never used, whatever the caller has there.
int check_tensor(const adacons_attn_tensor* t, int batch, int len, int heads) {
  if (t == nullptr) return ADACONS_EINVAL;
  if (batch == 0 || len == 0) return ADACONS_OK;
  if (t->data == nullptr) return ADACONS_EINVAL;
  const int64_t strides[3] = {t->batch_stride, t->seq_stride, t->head_stride};
  const int sizes[3] = {batch, len, heads};
  if (reinterpret_cast<uintptr_t>(t->data) % 16 != 0) return ADACONS_EALIGN;
  for (int k = 0; k < 3; ++k) {
    if (sizes[k] == 1) continue;
    if (strides[k] <= 0 || strides[k] >= (1ll << 38)) return ADACONS_EINVAL;
    if (strides[k] % 8 != 0) return ADACONS_EALIGN;
  }
  return ADACONS_OK;
}

int64_t peak_blocks(int kv_len) { return (static_cast<int64_t>(kv_len) + kAttnPeakRows - 1) / kAttnPeakRows; }

// Whether two tensors with elements start at the same place: a result there would be written while other blocks still read.
bool same_place(const adacons_attn_tensor* a, int a_len, const adacons_attn_tensor* b, int b_len) { return a_len > 0 && b_len > 0 && a->data == b->data; }

bool make_map(const AttnDevice& d, CUtensorMap* map, const adacons_attn_shape* s, const adacons_attn_tensor* t, int len, int heads, const void* spare, int rows) {
  // a tensor without tokens is never read, but its map has to exist
  const void* base = len > 0 ? t->data : spare;
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(s->head_dim), static_cast<cuuint64_t>(len > 0 ? len : 1), static_cast<cuuint64_t>(heads),
                              static_cast<cuuint64_t>(s->batch)};
  const cuuint64_t one = static_cast<cuuint64_t>(s->head_dim) * 2;
  const cuuint64_t strides[3] = {len > 1 ? static_cast<cuuint64_t>(t->seq_stride) * 2 : one, heads > 1 && len > 0 ? static_cast<cuuint64_t>(t->head_stride) * 2 : one,
                                 s->batch > 1 && len > 0 ? static_cast<cuuint64_t>(t->batch_stride) * 2 : one};
  const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(rows), 1, 1};
  return encode_map(d.info, map, s->dtype == ADACONS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides, box);
}

AttnOut as_out(const adacons_attn_tensor* t) { return {t->data, t->batch_stride, t->seq_stride, t->head_stride}; }

AttnParams base_params(const AttnDevice& d, const adacons_attn_shape* s) {
  AttnParams p = {};
  p.B = s->batch;
  p.Hq = s->q_heads;
  p.Hkv = s->kv_heads;
  p.Sq = s->q_len;
  p.Sk = s->kv_len;
  p.D = s->head_dim;
  p.causal = s->causal;
  p.sq_pad = (s->q_len + kAttnTile - 1) / kAttnTile * kAttnTile;
  p.scale = s->scale;
  p.scale_log2 = s->scale * kLog2e;
  p.kv_lens = s->kv_lens;
  p.flags = d.flags;
  return p;
}

// Blocks that share one tile's walk over the `tiles` of the other side: twice as many while all of them still run at once and
// each has two tiles or more.  Forward, one query over 4000 keys of 4 heads: 57 us alone, 33, 20 and 14 us shared by 2, 4 and 8; 2000 x 2000 causal of
// 4 heads 30, 21, 18 us, and 28 us by 8, more than run at once; 300 x 300 11.1 us alone and 13.3 by 2, with a tile or two each.
int key_shares(int64_t blocks, int64_t tiles, int resident) {
  int shares = 1;
  while (shares < 8 && blocks * shares * 2 <= resident && tiles >= 4 * shares) shares *= 2;
  return shares;
}

// The gradient's two kinds of block, with walks of `queries` and `keys` tiles: the sharing with the shortest of what bounds it, the longest
// block or the work of all.  In tiles: a block's start and end cost about three, a join two; the work is spread unevenly, hence the 1.3.
// 4000 queries on 200 keys of 8 / 2 heads (64 elements): 281 us alone, 147, 80 and 47 us with a key tile's walk shared by 2, 4, 8; 200 on 3000 causal 44 -> 15 us;
// 2000 x 2000 of 4 / 2 heads (128) 64 us, 41 with the key tiles' walks shared by 2, 56 by 4, 60 with both kinds' by 4; 300 x 300 13.7 us alone, 14.9 by 2.
void share_walks(AttnParams* p, int64_t key_blocks, int64_t queries, int64_t query_blocks, int64_t keys, int resident) {
  double best = 0.0;
  for (int split = 1; split <= 8; split *= 2)
    for (int which = split > 1 ? 1 : 3; which <= 3; ++which) {
      const int k = which & 1 ? split : 1, q = which & 2 ? split : 1;
      const double by_key = static_cast<double>((queries + k - 1) / k) + 3.0 + (k > 1 ? 2.0 : 0.0);
      const double by_query = static_cast<double>((keys + q - 1) / q) + 3.0 + (q > 1 ? 2.0 : 0.0);
      const double time = std::max(std::max(by_key, by_query), 1.3 * (key_blocks * k * by_key + query_blocks * q * by_query) / resident);
      if (split > 1 && time >= best) continue;
      best = time;
      p->split = split;
      p->key_split = k;
      p->query_split = q;
    }
}

template <int D, bool BF16, bool STARVE = false>
bool run_forward(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, AttnParams p, int sms, cudaStream_t st) {
  const int q_tiles = (p.Sq + kAttnTile - 1) / kAttnTile;
  p.split = key_shares(static_cast<int64_t>(q_tiles) * p.Hq * p.B, (p.Sk + kAttnTile - 1) / kAttnTile, 2 * sms);
  return launch(&attn_forward_kernel<D, BF16, STARVE>, dim3(q_tiles * p.split, p.Hq, p.B), dim3(kFwdThreads), AttnFwdSmem<D>::kBytes, st, kLaunchPlain, p.split,
                mq, mk, mv, p);
}

template <int D, bool BF16, bool STARVE = false>
bool run_backward(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mdo, AttnParams p, const adacons_attn_tensor* dout,
                  const adacons_attn_tensor* v, const adacons_attn_tensor* out, const float* lse, AttnOut dq, AttnOut dk, AttnOut dv, float* lse2, float* delta, float* peaks,
                  int sms, cudaStream_t st) {
  p.dout = {dout->data, dout->batch_stride, dout->seq_stride, dout->head_stride};
  p.o = {out->data, out->batch_stride, out->seq_stride, out->head_stride};
  p.v = {v->data, v->batch_stride, v->seq_stride, v->head_stride};
  p.lse_in = lse;
  p.lse2 = lse2;
  p.delta = delta;
  const bool separate = delta != nullptr && p.sq_pad > 0;
  if (separate) {
    const int q_blocks = p.sq_pad / kAttnStatRows<D>, k_blocks = BF16 ? 0 : static_cast<int>((peak_blocks(p.Sk) * p.Hkv + p.Hq - 1) / p.Hq);
    if (!launch(&attn_delta_kernel<D, BF16>, dim3(q_blocks + k_blocks, p.Hq, p.B), dim3(256), 0, st, kLaunchPlain, 1, p, lse2, delta, peaks)) return false;
    if (!BF16) p.peaks = peaks;
  }
  p.out = dq;
  p.dk = dk;
  p.dv = dv;
  const int64_t q_tiles = p.sq_pad / kAttnTile, k_tiles = (static_cast<int64_t>(p.Sk) + kAttnTile - 1) / kAttnTile;
  int64_t key_blocks = k_tiles * p.Hkv * p.B, query_blocks = q_tiles * p.Hq * p.B;
  share_walks(&p, key_blocks, p.Hq / p.Hkv * q_tiles, query_blocks, k_tiles, sms * AttnBwd<D>::kBlocks);
  key_blocks = (key_blocks * p.key_split + p.split - 1) / p.split * p.split;
  query_blocks = (query_blocks * p.query_split + p.split - 1) / p.split * p.split;
  return key_blocks + query_blocks <= 0x7fffffff &&
         launch(&attn_backward_kernel<D, BF16, STARVE>, dim3(static_cast<unsigned>(key_blocks + query_blocks)), dim3(AttnBwd<D>::kThreads), attn_backward_smem<D>(), st,
                separate ? kLaunchOverlap : kLaunchPlain, p.split, mq, mk, mv, mdo, p, static_cast<int>(key_blocks), static_cast<int>(q_tiles));
}

// lse2 and delta of every padded row; fp16: a maximum for each block of the kernel that makes them, of q's rows and of v's
int64_t workspace_bytes(const adacons_attn_shape* s) {
  const int64_t pad = (static_cast<int64_t>(s->q_len) + kAttnTile - 1) / kAttnTile * kAttnTile;
  int64_t words = 2 * pad * s->q_heads;
  if (s->dtype == ADACONS_F16) {
    const int64_t rows = s->head_dim <= 64 ? kAttnStatRows<64> : kAttnStatRows<128>;
    words += pad / rows * s->q_heads + peak_blocks(s->kv_len) * s->kv_heads;
  }
  return static_cast<int64_t>(sizeof(float)) * words * s->batch;
}

}  // namespace

namespace {

int forward(const adacons_attn_shape* s, const adacons_attn_tensor* q, const adacons_attn_tensor* k, const adacons_attn_tensor* v,
            const adacons_attn_tensor* out, float* lse, void* cuda_stream, bool starve) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  if ((rc = check_tensor(q, s->batch, s->q_len, s->q_heads)) != ADACONS_OK || (rc = check_tensor(out, s->batch, s->q_len, s->q_heads)) != ADACONS_OK ||
      (rc = check_tensor(k, s->batch, s->kv_len, s->kv_heads)) != ADACONS_OK || (rc = check_tensor(v, s->batch, s->kv_len, s->kv_heads)) != ADACONS_OK)
    return rc;
  if (s->batch == 0 || s->q_len == 0) return ADACONS_OK;
  if (same_place(out, s->q_len, k, s->kv_len) || same_place(out, s->q_len, v, s->kv_len)) return ADACONS_EINVAL;
  if (lse == nullptr || reinterpret_cast<uintptr_t>(lse) % 4 != 0) return ADACONS_EINVAL;
  AttnDevice* d = nullptr;
  if ((rc = attn_device(&d)) != ADACONS_OK) return rc;
  CUtensorMap mq, mk, mv;
  if (!make_map(*d, &mq, s, q, s->q_len, s->q_heads, q->data, kAttnTile) || !make_map(*d, &mk, s, k, s->kv_len, s->kv_heads, q->data, kAttnTile) ||
      !make_map(*d, &mv, s, v, s->kv_len, s->kv_heads, q->data, kAttnTile))
    return ADACONS_ECUDA;
  AttnParams p = base_params(*d, s);
  p.out = as_out(out);
  p.lse = lse;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  bool ok;
  if (starve) ok = run_forward<64, true, true>(mq, mk, mv, p, d->info.sms, st);
  else if (s->head_dim <= 64) ok = s->dtype == ADACONS_BF16 ? run_forward<64, true>(mq, mk, mv, p, d->info.sms, st) : run_forward<64, false>(mq, mk, mv, p, d->info.sms, st);
  else ok = s->dtype == ADACONS_BF16 ? run_forward<128, true>(mq, mk, mv, p, d->info.sms, st) : run_forward<128, false>(mq, mk, mv, p, d->info.sms, st);
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

int backward(const adacons_attn_shape* s, const adacons_attn_tensor* dout, const adacons_attn_tensor* q, const adacons_attn_tensor* k,
             const adacons_attn_tensor* v, const adacons_attn_tensor* out, const float* lse, const adacons_attn_tensor* dq,
             const adacons_attn_tensor* dk, const adacons_attn_tensor* dv, void* workspace, int64_t bytes, void* cuda_stream, bool starve) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  const adacons_attn_tensor* by_q[] = {dout, q, out, dq};
  const adacons_attn_tensor* by_k[] = {k, v, dk, dv};
  for (const adacons_attn_tensor* t : by_q)
    if ((rc = check_tensor(t, s->batch, s->q_len, s->q_heads)) != ADACONS_OK) return rc;
  for (const adacons_attn_tensor* t : by_k)
    if ((rc = check_tensor(t, s->batch, s->kv_len, s->kv_heads)) != ADACONS_OK) return rc;
  if (s->batch == 0 || (s->q_len == 0 && s->kv_len == 0)) return ADACONS_OK;
  const adacons_attn_tensor* all[] = {dout, q, out, k, v, dq, dk, dv};
  auto len_of = [&](int t) { return t < 3 || t == 5 ? s->q_len : s->kv_len; };
  for (int r = 5; r < 8; ++r)
    for (int t = 0; t < r; ++t)
      if (same_place(all[r], len_of(r), all[t], len_of(t))) return ADACONS_EINVAL;
  if (s->q_len > 0) {
    const int64_t pad = (static_cast<int64_t>(s->q_len) + kAttnTile - 1) / kAttnTile * kAttnTile;
    if (lse == nullptr || reinterpret_cast<uintptr_t>(lse) % 4 != 0) return ADACONS_EINVAL;
    const bool is_short = s->q_heads / s->kv_heads * pad <= ADACONS_ATTN_SHORT_ROWS && (s->dtype == ADACONS_BF16 || s->kv_len <= ADACONS_ATTN_SHORT_KEYS);
    if (workspace == nullptr ? !is_short : bytes < workspace_bytes(s)) return ADACONS_EINVAL;
  }
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return ADACONS_EALIGN;
  AttnDevice* d = nullptr;
  if ((rc = attn_device(&d)) != ADACONS_OK) return rc;
  const void* spare = s->q_len > 0 ? q->data : k->data;
  const int rows = s->head_dim <= 64 ? AttnBwd<64>::kTok : AttnBwd<128>::kTok;
  CUtensorMap mq, mk, mv, mdo;
  if (!make_map(*d, &mq, s, q, s->q_len, s->q_heads, spare, rows) || !make_map(*d, &mk, s, k, s->kv_len, s->kv_heads, spare, rows) ||
      !make_map(*d, &mv, s, v, s->kv_len, s->kv_heads, spare, rows) || !make_map(*d, &mdo, s, dout, s->q_len, s->q_heads, spare, rows))
    return ADACONS_ECUDA;
  const AttnParams p = base_params(*d, s);
  float* lse2 = static_cast<float*>(workspace);
  float* delta = lse2 == nullptr ? nullptr : lse2 + static_cast<int64_t>(p.B) * p.Hq * p.sq_pad;
  float* peaks = delta == nullptr ? nullptr : delta + static_cast<int64_t>(p.B) * p.Hq * p.sq_pad;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  auto go = [&](auto run) { return run(mq, mk, mv, mdo, p, dout, v, out, lse, as_out(dq), as_out(dk), as_out(dv), lse2, delta, peaks, d->info.sms, st); };
  bool ok;
  if (starve) ok = go(run_backward<64, true, true>);
  else if (s->head_dim <= 64) ok = s->dtype == ADACONS_BF16 ? go(run_backward<64, true>) : go(run_backward<64, false>);
  else ok = s->dtype == ADACONS_BF16 ? go(run_backward<128, true>) : go(run_backward<128, false>);
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

}  // namespace

extern "C" {

int adacons_attn_forward(const adacons_attn_shape* s, const adacons_attn_tensor* q, const adacons_attn_tensor* k, const adacons_attn_tensor* v,
                         const adacons_attn_tensor* out, float* lse, void* cuda_stream) {
  return forward(s, q, k, v, out, lse, cuda_stream, false);
}

int adacons_attn_workspace_bytes(const adacons_attn_shape* s, int64_t* bytes) {
  if (bytes == nullptr) return ADACONS_EINVAL;
  const int rc = check_shape(s);
  if (rc == ADACONS_OK) *bytes = workspace_bytes(s);
  return rc;
}

int adacons_attn_backward(const adacons_attn_shape* s, const adacons_attn_tensor* dout, const adacons_attn_tensor* q, const adacons_attn_tensor* k,
                          const adacons_attn_tensor* v, const adacons_attn_tensor* out, const float* lse, const adacons_attn_tensor* dq,
                          const adacons_attn_tensor* dk, const adacons_attn_tensor* dv, void* workspace, int64_t bytes, void* cuda_stream) {
  return backward(s, dout, q, k, v, out, lse, dq, dk, dv, workspace, bytes, cuda_stream, false);
}

int adacons_selftest_attention(const adacons_attn_shape* s, const adacons_attn_tensor* q, const adacons_attn_tensor* k, const adacons_attn_tensor* v,
                               const adacons_attn_tensor* out, float* lse, const adacons_attn_tensor* dq, const adacons_attn_tensor* dk,
                               const adacons_attn_tensor* dv, void* workspace, int64_t bytes, void* cuda_stream) {
  if (s == nullptr || s->dtype != ADACONS_BF16 || s->head_dim > 64) return ADACONS_EINVAL;
  AttnDevice* d = nullptr;
  int rc = attn_device(&d);
  if (rc != ADACONS_OK) return rc;
  if (!raise_all<64, true, true>()) return ADACONS_ECUDA;
  if (dq == nullptr) return forward(s, q, k, v, out, lse, cuda_stream, true);
  return backward(s, out, q, k, v, out, lse, dq, dk, dv, workspace, bytes, cuda_stream, true);
}

int adacons_attn_get_status(uint32_t* flags, void* cuda_stream) {
  if (flags == nullptr) return ADACONS_EINVAL;
  AttnDevice* d = nullptr;
  const int rc = attn_device(&d);
  if (rc != ADACONS_OK) return rc;
  return take_status(d->flags, flags, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
