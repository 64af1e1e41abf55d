// Host side of the orthogonalisation of a flat update vector (include/adacons_ops.h): layout, plan and launches.
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "adacons_host.cuh"
#include "adacons_orth.cuh"

using namespace adacons;

struct adacons_orth {
  DeviceInfo dev;
  int dtype = 0, steps = 0;
  int64_t d = 0;
  double eps = 0;
  std::vector<double> coeffs;         // [steps][a, b, c]
  unsigned char* memory = nullptr;    // one allocation: descriptors, lists, partial sums, iterates
  size_t bytes = 0;
  const OrthMat* mats = nullptr;
  const CUtensorMap* maps = nullptr;
  const OrthTile* load_tiles = nullptr;
  const OrthTile* tiles[3] = {};      // by OrthKind
  int num_tiles[3] = {}, cg[3] = {};
  const OrthChunk* chunks = nullptr;
  double* partial = nullptr;
  uint32_t* flags = nullptr;
  int num_load = 0, num_chunks = 0;
  int64_t launches = 0;
};

namespace {

// A side is the K of a product; the tensor cores' rounding toward zero makes a sum over it low by up to
// 4e-8 per 16 elements, 6.5e-4 at this limit: below the rounding of the fp16 operands.
constexpr int64_t kMaxSide = 1 << 18;

struct Arena {                        // offsets first, pointers once the allocation exists
  size_t used = 0;
  size_t take(size_t bytes) {
    const size_t at = used;
    used += (bytes + 255) / 256 * 256;
    return at;
  }
};

// The tiles of one product for a tiling with CG blocks per tile, longest first, as the persistent
// blocks (or pairs) take them in turn, and the modelled time of the busiest one in cycles.  The model:
// a stage's products take 64 (128) cycles per 16 K elements and fp16 pass, a lone block about 1.3 times that (its operand
// traffic from L2 per product is twice a pair's), an epilogue overlaps with the next tile's products.
double plan_tiles(const std::vector<OrthMat>& mats, int kind, bool split, int cg, int sms, std::vector<OrthTile>* tiles) {
  const int tm = 128 * cg, tn = split ? 128 : 128 * cg;
  tiles->clear();
  std::vector<int> order(mats.size());
  for (size_t k = 0; k < mats.size(); ++k) order[k] = static_cast<int>(k);
  auto depth = [&](int k) { return kind == kOrthGram ? mats[k].l : mats[k].r; };
  std::sort(order.begin(), order.end(), [&](int x, int y) { return depth(x) != depth(y) ? depth(x) > depth(y) : x < y; });
  const int workers = sms / cg;
  std::vector<double> busy(workers, 0.0);
  for (int k : order) {
    const int cols = kind == kOrthApply ? mats[k].l : mats[k].r;
    const double stages = (depth(k) + kOrthTK - 1) / kOrthTK;
    const double products = stages * 4 * (tn / 2) * (split ? 3 : 1) * (cg == 1 ? 1.3 : 1.0);
    const double cost = std::max(products, 16.0 * tn) + 500.0;
    for (int64_t j = 0; j * tn < cols; ++j)
      for (int64_t i = 0; i * tm < mats[k].r; ++i) {
        if (kind != kOrthApply && i * tm + tm - 1 < j * tn) continue;
        busy[tiles->size() % workers] += cost;
        tiles->push_back({k, static_cast<int>(i), static_cast<int>(j), 0});
      }
  }
  return *std::max_element(busy.begin(), busy.end()) + 16.0 * tn;
}

template <int KIND, bool SPLIT, int CG>
bool launch_product(const adacons_orth* c, const OrthParams& p, cudaStream_t st) {
  static_assert(OrthTiling<SPLIT, CG>::kBytes <= 227 * 1024, "shared memory of a block");
  const int blocks = std::min(p.num_tiles, c->dev.sms / CG) * CG;
  return launch(&orth_product_kernel<KIND, SPLIT, CG>, dim3(blocks), dim3(kOrthThreads), OrthTiling<SPLIT, CG>::kBytes, st, true, CG, p);
}

template <int KIND>
bool launch_kind(const adacons_orth* c, OrthParams p, cudaStream_t st) {
  p.tiles = c->tiles[KIND];
  p.num_tiles = c->num_tiles[KIND];
  if (c->dtype == ADACONS_F32) return c->cg[KIND] == 2 ? launch_product<KIND, true, 2>(c, p, st) : launch_product<KIND, true, 1>(c, p, st);
  return c->cg[KIND] == 2 ? launch_product<KIND, false, 2>(c, p, st) : launch_product<KIND, false, 1>(c, p, st);
}

template <int KIND, bool SPLIT, int CG>
bool raise_smem() {
  if (cudaFuncSetAttribute(orth_product_kernel<KIND, SPLIT, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, OrthTiling<SPLIT, CG>::kBytes) == cudaSuccess) return true;
  cudaGetLastError();
  return false;
}
template <int KIND>
bool raise_smem_kind() { return raise_smem<KIND, false, 1>() && raise_smem<KIND, false, 2>() && raise_smem<KIND, true, 1>() && raise_smem<KIND, true, 2>(); }

int create(adacons_orth** out, int dtype, int64_t d, int num, const int64_t* rows, const int64_t* cols, const int64_t* offsets, int scaling,
           int steps, const double* coeffs, double eps) {
  std::vector<std::pair<int64_t, int64_t>> spans;
  for (int k = 0; k < num; ++k) {
    if (rows[k] < 1 || cols[k] < 1 || offsets[k] < 0) return ADACONS_EINVAL;
    if (rows[k] > kMaxSide || cols[k] > kMaxSide) return ADACONS_ELIMIT;
    if (rows[k] * cols[k] > d || offsets[k] > d - rows[k] * cols[k]) return ADACONS_EINVAL;
    spans.emplace_back(offsets[k], offsets[k] + rows[k] * cols[k]);
  }
  std::sort(spans.begin(), spans.end());
  for (size_t k = 1; k < spans.size(); ++k)
    if (spans[k].first < spans[k - 1].second) return ADACONS_EINVAL;
  for (int k = 0; k < 3 * steps; ++k)
    if (!std::isfinite(coeffs[k])) return ADACONS_EINVAL;

  DeviceInfo dev;
  int rc = query_device(&dev);
  if (rc != ADACONS_OK) return rc;
  if (!raise_smem_kind<kOrthGram>() || !raise_smem_kind<kOrthPoly>() || !raise_smem_kind<kOrthApply>()) return ADACONS_ECUDA;

  adacons_orth* c = new adacons_orth();
  c->dev = dev;
  c->dtype = dtype;
  c->d = d;
  c->steps = steps;
  c->eps = eps;
  c->coeffs.assign(coeffs, coeffs + 3 * steps);
  const bool split = dtype == ADACONS_F32;

  std::vector<OrthMat> mats(num);
  std::vector<OrthChunk> chunks;
  std::vector<OrthTile> load, lists[3];
  for (int k = 0; k < num; ++k) {
    OrthMat& m = mats[k];
    std::memset(&m, 0, sizeof(m));
    m.transposed = rows[k] > cols[k];
    m.r = static_cast<int>(std::min(rows[k], cols[k]));
    m.l = static_cast<int>(std::max(rows[k], cols[k]));
    m.ldx = (m.l + 7) / 8 * 8;
    m.lds = (m.r + 7) / 8 * 8;
    m.offset = offsets[k];
    m.vec_out = m.l % 8 == 0 && offsets[k] % 8 == 0;
    m.scale = scaling ? static_cast<float>(std::sqrt(std::max(1.0, static_cast<double>(rows[k]) / static_cast<double>(cols[k])))) : 1.f;
    m.norm_first = static_cast<int>(chunks.size());
    m.norm_count = static_cast<int>((rows[k] * cols[k] + kOrthNormChunk - 1) / kOrthNormChunk);
    for (int q = 0; q < m.norm_count; ++q) chunks.push_back({k, q});
    for (int i = 0; i < (m.r + kOrthLoadTile - 1) / kOrthLoadTile; ++i)
      for (int j = 0; j < (m.l + kOrthLoadTile - 1) / kOrthLoadTile; ++j) load.push_back({k, i, j, 0});
  }
  for (int kind = 0; kind < 3; ++kind) {
    std::vector<OrthTile> one, two;
    const double t1 = plan_tiles(mats, kind, split, 1, dev.sms, &one), t2 = plan_tiles(mats, kind, split, 2, dev.sms, &two);
    c->cg[kind] = t2 < t1 ? 2 : 1;
    lists[kind] = t2 < t1 ? two : one;
    c->num_tiles[kind] = static_cast<int>(lists[kind].size());
  }
  c->num_chunks = static_cast<int>(chunks.size());
  c->num_load = static_cast<int>(load.size());

  Arena a;
  const size_t at_mats = a.take(num * sizeof(OrthMat)), at_maps = a.take(static_cast<size_t>(num) * kMapCount * sizeof(CUtensorMap));
  size_t at_tiles[3];
  for (int kind = 0; kind < 3; ++kind) at_tiles[kind] = a.take(lists[kind].size() * sizeof(OrthTile));
  const size_t at_load = a.take(load.size() * sizeof(OrthTile)), at_chunks = a.take(chunks.size() * sizeof(OrthChunk));
  const size_t at_partial = a.take(chunks.size() * sizeof(double)), at_flags = a.take(sizeof(uint32_t));
  const size_t head = a.used;
  std::vector<size_t> at(static_cast<size_t>(num) * kMapCount, 0);
  for (int k = 0; k < num; ++k)
    for (int q = 0; q < kMapCount; ++q) {
      const bool is_x = q < kMapS;
      if (!is_x && (q & 1) && !split) continue;                  // S and B are pairs only in an fp32 context
      at[k * kMapCount + q] = a.take(static_cast<size_t>(mats[k].r) * (is_x ? mats[k].ldx : mats[k].lds) * sizeof(__half));
    }
  c->bytes = a.used;
  if (cudaMalloc(&c->memory, c->bytes) != cudaSuccess) { cudaGetLastError(); delete c; return ADACONS_ENOMEM; }
  std::vector<unsigned char> host(head, 0);
  std::vector<CUtensorMap> maps(static_cast<size_t>(num) * kMapCount);
  for (int k = 0; k < num; ++k) {
    OrthMat& m = mats[k];
    __half** fields[kMapCount] = {&m.x[0][0], &m.x[0][1], &m.x[1][0], &m.x[1][1], &m.s[0], &m.s[1], &m.b[0], &m.b[1]};
    for (int q = 0; q < kMapCount; ++q) {
      const size_t where = at[k * kMapCount + q];
      if (where == 0) continue;
      *fields[q] = reinterpret_cast<__half*>(c->memory + where);
      const bool is_x = q < kMapS;
      const cuuint64_t dims[2] = {static_cast<cuuint64_t>(is_x ? m.l : m.r), static_cast<cuuint64_t>(m.r)};
      const cuuint64_t strides[1] = {static_cast<cuuint64_t>(is_x ? m.ldx : m.lds) * sizeof(__half)};
      const cuuint32_t box[2] = {64, 64};
      if (!encode_map(dev, &maps[k * kMapCount + q], CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, c->memory + where, dims, strides, box)) {
        cudaFree(c->memory);
        delete c;
        return ADACONS_ECUDA;
      }
    }
  }
  std::memcpy(host.data() + at_mats, mats.data(), num * sizeof(OrthMat));
  std::memcpy(host.data() + at_maps, maps.data(), maps.size() * sizeof(CUtensorMap));
  for (int kind = 0; kind < 3; ++kind) {
    std::memcpy(host.data() + at_tiles[kind], lists[kind].data(), lists[kind].size() * sizeof(OrthTile));
    c->tiles[kind] = reinterpret_cast<const OrthTile*>(c->memory + at_tiles[kind]);
  }
  std::memcpy(host.data() + at_load, load.data(), load.size() * sizeof(OrthTile));
  std::memcpy(host.data() + at_chunks, chunks.data(), chunks.size() * sizeof(OrthChunk));
  // the padding of the iterates is read by the epilogues (never by a product): zero it once
  if (cudaMemset(c->memory + head, 0, c->bytes - head) != cudaSuccess ||
      cudaMemcpy(c->memory, host.data(), head, cudaMemcpyHostToDevice) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    cudaGetLastError();
    cudaFree(c->memory);
    delete c;
    return ADACONS_ECUDA;
  }
  c->mats = reinterpret_cast<const OrthMat*>(c->memory + at_mats);
  c->maps = reinterpret_cast<const CUtensorMap*>(c->memory + at_maps);
  c->load_tiles = reinterpret_cast<const OrthTile*>(c->memory + at_load);
  c->chunks = reinterpret_cast<const OrthChunk*>(c->memory + at_chunks);
  c->partial = reinterpret_cast<double*>(c->memory + at_partial);
  c->flags = reinterpret_cast<uint32_t*>(c->memory + at_flags);
  *out = c;
  return ADACONS_OK;
}

}  // namespace

extern "C" {

int adacons_orth_create(adacons_orth** out, int dtype, int64_t d, int num_matrices, const int64_t* rows, const int64_t* cols,
                        const int64_t* offsets, int scaling, int steps, const double* coeffs, double eps) {
  if (out == nullptr || rows == nullptr || cols == nullptr || offsets == nullptr || coeffs == nullptr) return ADACONS_EINVAL;
  if (dtype != ADACONS_F32 && dtype != ADACONS_BF16) return ADACONS_EINVAL;
  if (d < 1 || num_matrices < 1 || num_matrices > (1 << 20) || (scaling != 0 && scaling != 1)) return ADACONS_EINVAL;
  if (steps < 1 || steps > 64 || !(eps >= 0.0) || !std::isfinite(eps)) return ADACONS_EINVAL;
  try {
    return create(out, dtype, d, num_matrices, rows, cols, offsets, scaling, steps, coeffs, eps);
  } catch (const std::bad_alloc&) {
    return ADACONS_ENOMEM;
  } catch (...) {
    return ADACONS_EINVAL;
  }
}

int adacons_orth_apply(adacons_orth* c, const void* update, void* out, void* cuda_stream) {
  if (c == nullptr || update == nullptr || out == nullptr) return ADACONS_EINVAL;
  const size_t elem = c->dtype == ADACONS_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(update) % elem != 0 || reinterpret_cast<uintptr_t>(out) % elem != 0) return ADACONS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  bool ok;
  if (c->dtype == ADACONS_F32) {
    ok = launch(&orth_norm_kernel<0>, dim3(c->num_chunks), dim3(256), 0, st, false, 1, update, c->mats, c->chunks, c->partial) &&
         launch(&orth_load_kernel<0>, dim3(c->num_load), dim3(256), 0, st, true, 1, update, c->mats, c->load_tiles, static_cast<const double*>(c->partial), c->eps);
  } else {
    ok = launch(&orth_norm_kernel<1>, dim3(c->num_chunks), dim3(256), 0, st, false, 1, update, c->mats, c->chunks, c->partial) &&
         launch(&orth_load_kernel<1>, dim3(c->num_load), dim3(256), 0, st, true, 1, update, c->mats, c->load_tiles, static_cast<const double*>(c->partial), c->eps);
  }
  OrthParams p = {};
  p.mats = c->mats;
  p.maps = c->maps;
  p.flags = c->flags;
  p.out = out;
  p.out_aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0;
  for (int s = 0; ok && s < c->steps; ++s) {
    const double* k = &c->coeffs[3 * s];
    p.src = s & 1;
    p.a = static_cast<float>(k[0]);
    p.b = static_cast<float>(k[1]);
    p.c = static_cast<float>(k[2]);
    p.t = s >= 3 ? static_cast<float>(-0.75 * (k[1] + k[2])) : 0.f;
    p.last = s == c->steps - 1;
    ok = launch_kind<kOrthGram>(c, p, st) && launch_kind<kOrthPoly>(c, p, st) && launch_kind<kOrthApply>(c, p, st);
  }
  c->launches = 2 + 3 * c->steps;
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

int adacons_orth_get_status(adacons_orth* c, uint32_t* flags, void* cuda_stream) {
  if (c == nullptr || flags == nullptr) return ADACONS_EINVAL;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (cudaMemcpyAsync(flags, c->flags, sizeof(uint32_t), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaMemsetAsync(c->flags, 0, sizeof(uint32_t), st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) {
    cudaGetLastError();
    return ADACONS_ECUDA;
  }
  return ADACONS_OK;
}

int adacons_orth_get_info(adacons_orth* c, int key, int64_t* value) {
  if (c == nullptr || value == nullptr) return ADACONS_EINVAL;
  if (key == ADACONS_ORTH_INFO_BYTES) *value = static_cast<int64_t>(c->bytes);
  else if (key == ADACONS_ORTH_INFO_LAUNCHES) *value = c->launches;
  else return ADACONS_EINVAL;
  return ADACONS_OK;
}

int adacons_orth_destroy(adacons_orth* c) {
  if (c == nullptr) return ADACONS_OK;
  int now = 0;
  const bool moved = cudaGetDevice(&now) == cudaSuccess && now != c->dev.device && cudaSetDevice(c->dev.device) == cudaSuccess;
  cudaFree(c->memory);
  if (moved) cudaSetDevice(now);
  cudaGetLastError();
  delete c;
  return ADACONS_OK;
}

}  // extern "C"
