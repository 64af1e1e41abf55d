// Host side of the gated feed-forward block (include/adacons_ops.h): checks, tensor maps, plans and launches.
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>

#include "adacons_ffn.cuh"
#include "adacons_host.cuh"

using namespace adacons;

static __device__ uint32_t g_ffn_flags;

namespace {

constexpr int kMaxDevices = 64;

struct FfnDevice {
  bool ready = false;
  DeviceInfo info;
  int pairs = 0;                                 // pairs of blocks that run at once
  uint32_t* flags = nullptr;
};

template <int KIND, bool BF16, int CG, bool STARVE = false>
bool raise() {
  if (cudaFuncSetAttribute(ffn_kernel<KIND, BF16, CG, STARVE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(FfnTiling<CG>::bytes(CG == 2 ? kFfnPairStages : kFfnLoneStages))) == cudaSuccess) return true;
  cudaGetLastError();
  return false;
}
template <int KIND> bool raise_kind() { return raise<KIND, true, 1>() && raise<KIND, true, 2>() && raise<KIND, false, 1>() && raise<KIND, false, 2>(); }

// The first call on a device sets the kernels' shared-memory limits; later ones only look the entry up.
int ffn_device(FfnDevice** out) {
  static std::mutex mutex;
  static FfnDevice devices[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
  if (dev < 0 || dev >= kMaxDevices) return ADACONS_ELIMIT;
  std::lock_guard<std::mutex> lock(mutex);
  FfnDevice& d = devices[dev];
  if (!d.ready) {
    const int rc = query_device(&d.info);
    if (rc != ADACONS_OK) return rc;
    void* flags = nullptr;
    if (!raise_kind<kFfnUp>() || !raise_kind<kFfnBack>() || !raise_kind<kFfnPlain>() || cudaGetSymbolAddress(&flags, g_ffn_flags) != cudaSuccess) {
      cudaGetLastError();
      return ADACONS_ECUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(2 * d.info.sms);
    cfg.blockDim = dim3(kFfnThreads);
    cfg.dynamicSmemBytes = FfnTiling<2>::bytes(kFfnPairStages);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int pairs = 0;
    if (cudaOccupancyMaxActiveClusters(&pairs, ffn_kernel<kFfnPlain, true, 2>, &cfg) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
    d.pairs = std::max(1, std::min(pairs, d.info.sms / 2));
    d.flags = static_cast<uint32_t*>(flags);
    d.ready = true;
  }
  *out = &d;
  return ADACONS_OK;
}

int check_shape(const adacons_ffn_shape* s) {
  if (s == nullptr || (s->dtype != ADACONS_BF16 && s->dtype != ADACONS_F16)) return ADACONS_EINVAL;
  if (s->tokens < 0 || s->dim < 8 || s->dim % 8 != 0 || s->hidden < 8 || s->hidden % 8 != 0) return ADACONS_EINVAL;
  if (s->act < ADACONS_FFN_SILU || s->act > ADACONS_FFN_RELU) return ADACONS_EINVAL;
  if (s->tokens > (1 << 24) || s->dim > (1 << 18) || s->hidden > (1 << 18)) return ADACONS_ELIMIT;
  return ADACONS_OK;
}

int check_matrix(const adacons_ffn_matrix* m, int rows, int cols, bool optional) {
  if (m == nullptr) return ADACONS_EINVAL;
  if (m->data == nullptr) return optional || rows == 0 ? ADACONS_OK : ADACONS_EINVAL;
  if (rows == 0) return ADACONS_OK;
  if (reinterpret_cast<uintptr_t>(m->data) % 16 != 0) return ADACONS_EALIGN;
  if (rows > 1) {
    if (m->row_stride < cols || m->row_stride >= (1ll << 38)) return ADACONS_EINVAL;
    if (m->row_stride % 8 != 0) return ADACONS_EALIGN;
  }
  return ADACONS_OK;
}

bool make_map(const FfnDevice& d, CUtensorMap* map, const adacons_ffn_shape* s, const void* data, int64_t row_stride, int rows, int cols) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(rows > 1 ? row_stride : cols) * 2};
  const cuuint32_t box[2] = {64, 64};
  return encode_map(d.info, map, s->dtype == ADACONS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, data, dims, strides, box);
}

// results, for stores of 32 x 32
bool make_out(const FfnDevice& d, CUtensorMap* map, const adacons_ffn_shape* s, const FfnRows& r, int rows, int cols) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(r.row) * 2};
  const cuuint32_t box[2] = {32, 32}, ones[2] = {1, 1};
  return d.info.encode(map, s->dtype == ADACONS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, static_cast<cuuint32_t>(2), r.data, dims, strides, box, ones,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

FfnRows as_rows(const void* data, int64_t row_stride, int cols, int rows) {
  FfnRows r;
  r.data = const_cast<void*>(data);
  r.row = rows > 1 ? row_stride : cols;
  r.wide = reinterpret_cast<uintptr_t>(data) % 32 == 0 && r.row % 16 == 0;
  return r;
}
FfnRows as_rows(const adacons_ffn_matrix* m, int cols, int rows) { return as_rows(m->data, m->row_stride, cols, rows); }

int64_t up_to(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }
// A matrix (tokens x hidden) of the workspace
int64_t hidden_bytes(const adacons_ffn_shape* s) { return up_to(static_cast<int64_t>(s->tokens) * s->hidden * 2, 256); }
int64_t workspace_bytes(const adacons_ffn_shape* s, bool back) {
  return back ? 3 * hidden_bytes(s) + (s->dtype == ADACONS_F16 ? static_cast<int64_t>(kFfnWords) * 4 : 0) : hidden_bytes(s);
}

struct FfnPlan { int cg, shares; double time; };

// Tiles by pairs of blocks or by lone ones, and how many share one's K: the quickest by a count of cycles.  A stage of half a pair's tile takes 540 cycles where both halves
// of a tile share the left operand, 720 where pairs have one each; one of a lone block's 1000 (its operands, from L2; 128 tiles of 86 stages: 97,000), two beside one another
// twice that.  A launch costs 8000 cycles from the first operand to the last store, a join 2500.
FfnPlan plan_of(const FfnDevice& d, const FfnProblem* q, int n, int columns_by) {
  double work = 0.0;                             // stages of halves
  int64_t lone_tiles = 0, halves = 0;
  int steps = 1;
  for (int k = 0; k < n; ++k) {
    const int all = q[k].steps * q[k].segments, half = 256 / columns_by, lone = 128 / columns_by;
    const int64_t of_this = static_cast<int64_t>((q[k].m + 255) / 256) * ((q[k].n + half - 1) / half);
    halves += of_this;
    work += static_cast<double>(of_this) * all;
    lone_tiles += static_cast<int64_t>((q[k].m + 127) / 128) * ((q[k].n + lone - 1) / lone);
    steps = std::max(steps, all);
  }
  FfnPlan best = {2, 1, 8000.0 + (halves <= d.pairs ? steps * 720.0 : std::max(std::ceil(work / steps / d.pairs) * steps, work / d.pairs) * 540.0)};
  for (int shares = 1; shares <= 8; shares *= 2) {
    if (shares > 1 && (steps < 2 * shares || n > 1)) break;
    const int64_t per_sm = (lone_tiles * shares + d.info.sms - 1) / d.info.sms;
    const double time = per_sm * ((steps + shares - 1) / shares) * 1000.0 + ((per_sm + 1) / 2) * (8000.0 + (shares > 1 ? 2500.0 : 0.0));
    if (time < best.time) best = {1, shares, time};
  }
  return best;
}

template <int KIND, bool BF16, int CG>
bool run(const FfnParams& p, int blocks, int cluster, bool overlap, cudaStream_t st) {
  return launch(&ffn_kernel<KIND, BF16, CG>, dim3(blocks), dim3(kFfnThreads), FfnTiling<CG>::bytes(CG == 2 ? kFfnPairStages : p.stages), st, overlap ? kLaunchOverlap : kLaunchPlain, cluster, p);
}

// Whether all tiles of pairs go as halves by themselves, whose two accumulators take turns, so that one half's ending runs beside the next one's products; a whole tile's two
// endings have little beside them, but it shares a stage's left operand (540 cycles for 720).  A half's ending takes about 12,500 cycles (Back: two matrices read, three written;
// 14,500 with gelu), 8000 (Up) or 5000.  Gradient of 8192 x 512 x 2048 (8 stages) 145 -> 139 us, 4096 x 1024 x 4096 (16) 200 -> 190.5, 2048 x 2048 x 8192 (32) 375 -> 364; with 64
// stages, 4096 x 4096 x 10944, 1527 -> 1543.
bool by_halves(int kind, int problems, const FfnProblem& q) {
  const double ending = kind == kFfnBack ? 12500.0 : kind == kFfnUp ? 8000.0 : 5000.0, steps = static_cast<double>(q.steps) * q.segments;
  return problems == 1 && 2 * std::max(720.0 * steps, ending) < 1080.0 * steps + 2 * ending - 4000.0;
}

// Numbers the problems' tiles and launches.
template <int KIND>
bool run(const FfnDevice& d, const adacons_ffn_shape* s, FfnParams* p, int n, const FfnPlan& plan, bool overlap, cudaStream_t st) {
  const int tm = 128 * plan.cg, tn = KIND == kFfnUp ? tm / 2 : tm;       // of half a tile
  for (int k = 0; KIND == kFfnPlain && k < n; ++k)
    if (!make_out(d, &p->outs[k], s, p->problem[k].out, p->problem[k].m, p->problem[k].n)) return false;
  p->problems = n;
  p->wholes = 0;
  p->shares = plan.shares;
  p->act = s->act;
  p->flags = d.flags;
  for (int k = 0; k < n; ++k) {
    FfnProblem& q = p->problem[k];
    q.tiles_m = (q.m + tm - 1) / tm;
    q.tiles_n = (q.n + tn - 1) / tn;
    q.first = p->wholes;
    p->wholes += q.tiles_m * ((q.tiles_n + plan.cg - 1) / plan.cg);
  }
  p->tiles = p->wholes;
  const bool bf16 = s->dtype == ADACONS_BF16;
  if (plan.cg == 2) {
    // a last round in which at most half of the pairs would have a tile: halves, for all
    const bool all = by_halves(KIND, n, p->problem[0]);
    const int rest = all ? p->wholes : p->wholes % d.pairs;
    if (all || 2 * rest <= d.pairs) {
      p->wholes -= rest;
      p->tiles += rest;
    }
    const int blocks = 2 * std::min(p->tiles, d.pairs);
    return bf16 ? run<KIND, true, 2>(*p, blocks, 2, overlap, st) : run<KIND, false, 2>(*p, blocks, 2, overlap, st);
  }
  const int blocks = p->tiles * plan.shares;
  p->stages = blocks <= d.info.sms ? kFfnLoneStages : kFfnCrowdStages;
  return bf16 ? run<KIND, true, 1>(*p, blocks, plan.shares, overlap, st) : run<KIND, false, 1>(*p, blocks, plan.shares, overlap, st);
}

int steps_of(int k) { return (k + kFfnTK - 1) / kFfnTK; }

// Whether the forward pass goes by the kernel for a few tokens: where the weights stay in L2 it is the quicker one up to 32 tokens, elsewhere up to 4; the figures stand there.
bool few_tokens(const adacons_ffn_shape* s) {
  return s->tokens <= (6 * static_cast<int64_t>(s->dim) * s->hidden <= kFfnL2 ? kFfnFew : kFfnFewLong);
}

// Sixteen warps a block where there are few blocks and K leaves each of the warps eight stages of 32 or more, eight elsewhere, whose blocks end and begin beside one another
// (1 x 1024 x 4096, 512 blocks and 128: 10.1 us, by eight alone 11.8, by sixteen 13.5; 1 x 4096 x 10944, 1368 blocks and 512: by eight 61.6 to 63.4, by sixteen 70.0).
template <int KIND, bool BF16>
bool run_few(const FfnDevice& d, const FfnFewParams& p, bool overlap, cudaStream_t st) {
  const int warps = p.k >= 8 * 16 * 32 && (p.n + 7) / 8 <= 4 * d.info.sms ? 16 : 8, sixteens = p.tokens <= 16 ? 1 : 2;
  const size_t bytes = static_cast<size_t>(warps) * (KIND == kFfnUp ? 2 : 1) * sixteens * 16 * 8 * sizeof(float);
  const dim3 grid((p.n + 7) / 8), block(32 * warps);
  const LaunchKind kind = overlap ? kLaunchOverlap : kLaunchPlain;
  return sixteens == 1 ? launch(&ffn_few_kernel<KIND, BF16, 1>, grid, block, bytes, st, kind, 1, p) : launch(&ffn_few_kernel<KIND, BF16, 2>, grid, block, bytes, st, kind, 1, p);
}

// Whether two matrices start at the same place: a result there would be written while other blocks still read.
bool same_place(const adacons_ffn_matrix* a, const adacons_ffn_matrix* b) { return a != b && a->data != nullptr && a->data == b->data; }

bool any_same(const adacons_ffn_matrix* const* results, int n, const adacons_ffn_matrix* const* reads, int m) {
  for (int r = 0; r < n; ++r) {
    for (int k = 0; k < m; ++k)
      if (same_place(results[r], reads[k])) return true;
    for (int k = 0; k < r; ++k)
      if (same_place(results[r], results[k])) return true;
  }
  return false;
}

// y's product: x through both projections; `gate` and `up` may have no data.
FfnProblem up_problem(const adacons_ffn_shape* s, void* h) {
  FfnProblem q = {};
  q.a[0] = 0;
  q.b[0] = 1;
  q.b[1] = 2;
  q.m = s->tokens;
  q.n = s->hidden;
  q.steps = steps_of(s->dim);
  q.segments = 1;
  q.early = 1;
  q.out = as_rows(h, s->hidden, s->hidden, s->tokens);
  return q;
}

}  // namespace

extern "C" {

int adacons_ffn_workspace_bytes(const adacons_ffn_shape* s, int backward, int64_t* bytes) {
  if (bytes == nullptr) return ADACONS_EINVAL;
  const int rc = check_shape(s);
  if (rc == ADACONS_OK) *bytes = workspace_bytes(s, backward != 0);
  return rc;
}

int adacons_ffn_forward(const adacons_ffn_shape* s, const adacons_ffn_matrix* x, const adacons_ffn_matrix* wg, const adacons_ffn_matrix* wu, const adacons_ffn_matrix* wd,
                        const adacons_ffn_matrix* out, const adacons_ffn_matrix* gate, const adacons_ffn_matrix* up, void* workspace, int64_t bytes, void* cuda_stream) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  if ((rc = check_matrix(x, s->tokens, s->dim, false)) != ADACONS_OK || (rc = check_matrix(wg, s->hidden, s->dim, false)) != ADACONS_OK ||
      (rc = check_matrix(wu, s->hidden, s->dim, false)) != ADACONS_OK || (rc = check_matrix(wd, s->dim, s->hidden, false)) != ADACONS_OK ||
      (rc = check_matrix(out, s->tokens, s->dim, false)) != ADACONS_OK || (rc = check_matrix(gate, s->tokens, s->hidden, true)) != ADACONS_OK ||
      (rc = check_matrix(up, s->tokens, s->hidden, true)) != ADACONS_OK)
    return rc;
  if (s->tokens == 0) return ADACONS_OK;
  if ((gate->data == nullptr) != (up->data == nullptr)) return ADACONS_EINVAL;
  const adacons_ffn_matrix *results[] = {out, gate, up}, *reads[] = {x, wg, wu, wd};
  if (any_same(results, 3, reads, 4)) return ADACONS_EINVAL;
  if (workspace == nullptr || bytes < workspace_bytes(s, false)) return ADACONS_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return ADACONS_EALIGN;
  FfnDevice* d = nullptr;
  if ((rc = ffn_device(&d)) != ADACONS_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (few_tokens(s)) {
    FfnFewParams few = {};
    few.x = as_rows(x, s->dim, s->tokens);
    few.w[0] = as_rows(wg, s->dim, s->hidden);
    few.w[1] = as_rows(wu, s->dim, s->hidden);
    few.gate = as_rows(gate, s->hidden, s->tokens);
    few.up = as_rows(up, s->hidden, s->tokens);
    few.out = as_rows(workspace, s->hidden, s->hidden, s->tokens);
    few.tokens = s->tokens;
    few.n = s->hidden;
    few.k = s->dim;
    few.act = s->act;
    FfnFewParams down = few;
    down.x = few.out;
    down.w[0] = as_rows(wd, s->hidden, s->dim);
    down.out = as_rows(out, s->dim, s->tokens);
    down.n = s->dim;
    down.k = s->hidden;
    const bool ok = s->dtype == ADACONS_BF16 ? run_few<kFfnUp, true>(*d, few, false, st) && run_few<kFfnPlain, true>(*d, down, true, st)
                                             : run_few<kFfnUp, false>(*d, few, false, st) && run_few<kFfnPlain, false>(*d, down, true, st);
    return ok ? ADACONS_OK : ADACONS_ECUDA;
  }
  FfnParams p;
  std::memset(&p, 0, sizeof(p));
  if (!make_map(*d, &p.maps[0], s, x->data, x->row_stride, s->tokens, s->dim) || !make_map(*d, &p.maps[1], s, wg->data, wg->row_stride, s->hidden, s->dim) ||
      !make_map(*d, &p.maps[2], s, wu->data, wu->row_stride, s->hidden, s->dim))
    return ADACONS_ECUDA;
  p.problem[0] = up_problem(s, workspace);
  p.gate = as_rows(gate, s->hidden, s->tokens);
  p.up = as_rows(up, s->hidden, s->tokens);
  if ((p.gate.data != nullptr && (!make_out(*d, &p.outs[0], s, p.gate, s->tokens, s->hidden) || !make_out(*d, &p.outs[1], s, p.up, s->tokens, s->hidden))) ||
      !make_out(*d, &p.outs[2], s, p.problem[0].out, s->tokens, s->hidden) || !run<kFfnUp>(*d, s, &p, 1, plan_of(*d, p.problem, 1, 2), false, st))
    return ADACONS_ECUDA;
  if (!make_map(*d, &p.maps[0], s, workspace, s->hidden, s->tokens, s->hidden) || !make_map(*d, &p.maps[1], s, wd->data, wd->row_stride, s->dim, s->hidden)) return ADACONS_ECUDA;
  FfnProblem q = {};
  q.b[0] = 1;
  q.m = s->tokens;
  q.n = s->dim;
  q.steps = steps_of(s->hidden);
  q.segments = 1;
  q.early = 1;
  q.out = as_rows(out, s->dim, s->tokens);
  p.problem[0] = q;
  return run<kFfnPlain>(*d, s, &p, 1, plan_of(*d, p.problem, 1, 1), true, st) ? ADACONS_OK : ADACONS_ECUDA;
}

int adacons_ffn_backward(const adacons_ffn_shape* s, const adacons_ffn_matrix* dout, const adacons_ffn_matrix* x, const adacons_ffn_matrix* wg, const adacons_ffn_matrix* wu,
                         const adacons_ffn_matrix* wd, const adacons_ffn_matrix* gate, const adacons_ffn_matrix* up, const adacons_ffn_matrix* dx, const adacons_ffn_matrix* dwg,
                         const adacons_ffn_matrix* dwu, const adacons_ffn_matrix* dwd, void* workspace, int64_t bytes, void* cuda_stream) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  if ((rc = check_matrix(dout, s->tokens, s->dim, false)) != ADACONS_OK || (rc = check_matrix(x, s->tokens, s->dim, false)) != ADACONS_OK ||
      (rc = check_matrix(wg, s->hidden, s->dim, false)) != ADACONS_OK || (rc = check_matrix(wu, s->hidden, s->dim, false)) != ADACONS_OK ||
      (rc = check_matrix(wd, s->dim, s->hidden, false)) != ADACONS_OK || (rc = check_matrix(gate, s->tokens, s->hidden, false)) != ADACONS_OK ||
      (rc = check_matrix(up, s->tokens, s->hidden, false)) != ADACONS_OK || (rc = check_matrix(dx, s->tokens, s->dim, true)) != ADACONS_OK ||
      (rc = check_matrix(dwg, s->hidden, s->dim, true)) != ADACONS_OK || (rc = check_matrix(dwu, s->hidden, s->dim, true)) != ADACONS_OK ||
      (rc = check_matrix(dwd, s->dim, s->hidden, true)) != ADACONS_OK)
    return rc;
  const adacons_ffn_matrix *results[] = {dx, dwg, dwu, dwd}, *reads[] = {dout, x, wg, wu, wd, gate, up};
  if (any_same(results + (s->tokens == 0), 4 - (s->tokens == 0), reads, 7)) return ADACONS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  FfnDevice* d = nullptr;
  if (s->tokens == 0) {                          // sums over no tokens
    if ((rc = ffn_device(&d)) != ADACONS_OK) return rc;
    const int rows[] = {s->hidden, s->hidden, s->dim}, cols[] = {s->dim, s->dim, s->hidden};
    for (int k = 0; k < 3; ++k)
      if (results[k + 1]->data != nullptr &&
          cudaMemset2DAsync(results[k + 1]->data, static_cast<size_t>(results[k + 1]->row_stride) * 2, 0, static_cast<size_t>(cols[k]) * 2, rows[k], st) != cudaSuccess) {
        cudaGetLastError();
        return ADACONS_ECUDA;
      }
    return ADACONS_OK;
  }
  if (workspace == nullptr || bytes < workspace_bytes(s, true)) return ADACONS_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return ADACONS_EALIGN;
  if ((rc = ffn_device(&d)) != ADACONS_OK) return rc;
  unsigned char* work = static_cast<unsigned char*>(workspace);
  void *dg = work, *du = work + hidden_bytes(s), *h = work + 2 * hidden_bytes(s);
  unsigned* peaks = s->dtype == ADACONS_F16 ? reinterpret_cast<unsigned*>(work + 3 * hidden_bytes(s)) : nullptr;
  const FfnRows dy = as_rows(dout, s->dim, s->tokens);
  if (peaks != nullptr && !launch(&ffn_peak_kernel, dim3(kFfnPeaks), dim3(256), 0, st, kLaunchPlain, 1, static_cast<const void*>(dy.data), dy.row, s->tokens, s->dim, peaks)) return ADACONS_ECUDA;
  enum { kDy, kWd, kDg, kDu, kWg, kWu, kX, kH };
  FfnParams p;
  std::memset(&p, 0, sizeof(p));
  if (!make_map(*d, &p.maps[kDy], s, dout->data, dout->row_stride, s->tokens, s->dim) || !make_map(*d, &p.maps[kWd], s, wd->data, wd->row_stride, s->dim, s->hidden) ||
      !make_map(*d, &p.maps[kDg], s, dg, s->hidden, s->tokens, s->hidden) || !make_map(*d, &p.maps[kDu], s, du, s->hidden, s->tokens, s->hidden) ||
      !make_map(*d, &p.maps[kWg], s, wg->data, wg->row_stride, s->hidden, s->dim) || !make_map(*d, &p.maps[kWu], s, wu->data, wu->row_stride, s->hidden, s->dim) ||
      !make_map(*d, &p.maps[kX], s, x->data, x->row_stride, s->tokens, s->dim) || !make_map(*d, &p.maps[kH], s, h, s->hidden, s->tokens, s->hidden))
    return ADACONS_ECUDA;
  p.peaks = peaks;
  p.beyond = peaks == nullptr ? nullptr : peaks + kFfnPeaks;
  p.gate = as_rows(gate, s->hidden, s->tokens);
  p.up = as_rows(up, s->hidden, s->tokens);
  p.dgate = as_rows(dg, s->hidden, s->hidden, s->tokens);
  p.dup = as_rows(du, s->hidden, s->hidden, s->tokens);
  FfnProblem q = {};
  q.a[0] = kDy;
  q.b[0] = kWd;
  q.b_across = 1;
  q.m = s->tokens;
  q.n = s->hidden;
  q.steps = steps_of(s->dim);
  q.segments = 1;
  q.early = 1;
  q.out = as_rows(h, s->hidden, s->hidden, s->tokens);
  p.problem[0] = q;
  if (!make_out(*d, &p.outs[0], s, p.dgate, s->tokens, s->hidden) || !make_out(*d, &p.outs[1], s, p.dup, s->tokens, s->hidden) ||
      !make_out(*d, &p.outs[2], s, q.out, s->tokens, s->hidden) || !run<kFfnBack>(*d, s, &p, 1, plan_of(*d, p.problem, 1, 1), peaks != nullptr, st))
    return ADACONS_ECUDA;
  if (peaks != nullptr) {                        // once more where dg or du do not fit, with a factor that makes them
    p.beyond = nullptr;
    p.again = 1;
    if (!run<kFfnBack>(*d, s, &p, 1, plan_of(*d, p.problem, 1, 1), true, st)) return ADACONS_ECUDA;
  }
  // dx, and the weights' gradients
  FfnProblem by_x = {}, by_w[3];
  int weights = 0;
  const bool has_x = dx->data != nullptr;
  by_x.a[0] = kDg; by_x.a[1] = kDu;
  by_x.b[0] = kWg; by_x.b[1] = kWu;
  by_x.b_across = 1;
  by_x.m = s->tokens;
  by_x.n = s->dim;
  by_x.steps = steps_of(s->hidden);
  by_x.segments = 2;
  by_x.early = 1;
  by_x.scaled = peaks != nullptr;
  by_x.out = as_rows(dx, s->dim, s->tokens);
  auto weight = [&](const adacons_ffn_matrix* to, int a, int b, int m, int n, bool scaled) {
    FfnProblem w = {};
    w.a[0] = a;
    w.b[0] = b;
    w.a_across = w.b_across = 1;
    w.m = m;
    w.n = n;
    w.steps = steps_of(s->tokens);
    w.segments = 1;
    w.scaled = scaled;
    w.out = as_rows(to, n, m);
    by_w[weights++] = w;
  };
  weight(dwg, kDg, kX, s->hidden, s->dim, peaks != nullptr);
  weight(dwu, kDu, kX, s->hidden, s->dim, peaks != nullptr);
  weight(dwd, kDy, kH, s->dim, s->hidden, false);
  // whichever are wanted, each comes from the plan for all: the same bits
  const FfnPlan x_plan = plan_of(*d, &by_x, 1, 1), w_plan = plan_of(*d, by_w, weights, 1);
  weights = 0;
  for (int k = 0; k < 3; ++k)
    if (results[k + 1]->data != nullptr) by_w[weights++] = by_w[k];
  if (has_x && weights > 0 && x_plan.cg == 2 && w_plan.cg == 2) {      // one launch, the longer tiles first
    const bool x_first = by_x.steps * 2 >= by_w[0].steps;
    for (int k = 0; k < weights; ++k) p.problem[k + x_first] = by_w[k];
    p.problem[x_first ? 0 : weights] = by_x;
    return run<kFfnPlain>(*d, s, &p, weights + 1, x_plan, true, st) ? ADACONS_OK : ADACONS_ECUDA;
  }
  if (has_x) {
    p.problem[0] = by_x;
    if (!run<kFfnPlain>(*d, s, &p, 1, x_plan, true, st)) return ADACONS_ECUDA;
  }
  if (weights > 0) {
    for (int k = 0; k < weights; ++k) p.problem[k] = by_w[k];
    if (!run<kFfnPlain>(*d, s, &p, weights, w_plan, true, st)) return ADACONS_ECUDA;
  }
  return ADACONS_OK;
}

int adacons_ffn_get_status(uint32_t* flags, void* cuda_stream) {
  if (flags == nullptr) return ADACONS_EINVAL;
  FfnDevice* d = nullptr;
  const int rc = ffn_device(&d);
  if (rc != ADACONS_OK) return rc;
  return take_status(d->flags, flags, static_cast<cudaStream_t>(cuda_stream));
}

int adacons_selftest_ffn(const adacons_ffn_shape* s, int paired, const adacons_ffn_matrix* x, const adacons_ffn_matrix* wg, const adacons_ffn_matrix* wu, void* workspace,
                         int64_t bytes, void* cuda_stream) {
  int rc = check_shape(s);
  if (rc != ADACONS_OK) return rc;
  const int rows = paired ? 256 : 128;
  if (s->dtype != ADACONS_BF16 || s->tokens < 1 || s->tokens > rows || s->hidden > rows / 2 || (paired != 0 && paired != 1)) return ADACONS_EINVAL;
  if ((rc = check_matrix(x, s->tokens, s->dim, false)) != ADACONS_OK || (rc = check_matrix(wg, s->hidden, s->dim, false)) != ADACONS_OK ||
      (rc = check_matrix(wu, s->hidden, s->dim, false)) != ADACONS_OK)
    return rc;
  if (workspace == nullptr || bytes < workspace_bytes(s, false)) return ADACONS_EINVAL;
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return ADACONS_EALIGN;
  FfnDevice* d = nullptr;
  if ((rc = ffn_device(&d)) != ADACONS_OK) return rc;
  if (!raise<kFfnUp, true, 1, true>() || !raise<kFfnUp, true, 2, true>()) return ADACONS_ECUDA;
  FfnParams p;
  std::memset(&p, 0, sizeof(p));
  if (!make_map(*d, &p.maps[0], s, x->data, x->row_stride, s->tokens, s->dim) || !make_map(*d, &p.maps[1], s, wg->data, wg->row_stride, s->hidden, s->dim) ||
      !make_map(*d, &p.maps[2], s, wu->data, wu->row_stride, s->hidden, s->dim))
    return ADACONS_ECUDA;
  p.problem[0] = up_problem(s, workspace);
  p.problem[0].tiles_m = p.problem[0].tiles_n = 1;
  p.problems = p.tiles = p.wholes = p.shares = 1;
  p.stages = kFfnCrowdStages;
  p.act = s->act;
  p.flags = d->flags;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool ok = paired ? launch(&ffn_kernel<kFfnUp, true, 2, true>, dim3(2), dim3(kFfnThreads), FfnTiling<2>::bytes(kFfnPairStages), st, kLaunchPlain, 2, p)
                         : launch(&ffn_kernel<kFfnUp, true, 1, true>, dim3(1), dim3(kFfnThreads), FfnTiling<1>::bytes(kFfnCrowdStages), st, kLaunchPlain, 1, p);
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

}  // extern "C"
