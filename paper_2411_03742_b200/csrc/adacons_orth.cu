// Host side of the orthogonalisation of a flat update vector (include/adacons_ops.h): layout, plan and launches.
#include "adacons_ops.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <memory>
#include <new>
#include <utility>
#include <vector>

#include "adacons_host.cuh"
#include "adacons_orth.cuh"

using namespace adacons;

struct adacons_orth {
  DeviceInfo dev;
  int dtype = 0, steps = 0;
  int64_t d = 0;
  double eps = 0;
  unsigned char* memory = nullptr;    // one allocation: descriptors, lists, partial sums, iterates
  size_t bytes = 0;
  const OrthSpot* load_tiles = nullptr;
  const OrthChunk* chunks = nullptr;
  double* partial = nullptr;
  OrthParams params = {};             // all but the result's address
  const int* starved = nullptr;       // the self-test's params.begin
  int cg = 1, tn = 128, blocks = 0;
  bool small = false;                 // all matrices fit the one-block kernel
  int num_load = 0, num_chunks = 0, num_mats = 0;
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

// Who computes which tile when: one list of tiles per worker (a block, or a pair of them).
struct OrthPlan {
  int cg = 1, tn = 128, workers = 1, mirrored = 1;
  std::vector<std::vector<OrthTile>> lists;
  double cycles = 0;                  // modelled time
  int slots = 0;                      // partial sums of split products
};

// The simulation's costs, in cycles, measured on the kernel.  A stage (64 K elements): what a block's operands take to
// arrive, about 60 bytes a cycle, 40 when all blocks load at once, or its products.  From the last product of a tile to where
// others may read it: the strips' arithmetic (a pair's tile has four of them), the store, the fence, the counter, the look.
// An fp32 context's mirror image is written from registers.
struct OrthCosts {
  double stage, strip, mirror, tail, add, crowd;      // crowd: of the workers' mean busy time, what they take from one another where all load
  OrthCosts(bool split, int cg, int tn) : stage((split ? 1300 : cg == 2 ? 800 : 600) * (tn == 64 ? 0.75 : 1.0)), strip(split ? 1500 : 1300), mirror(split ? 6000 : 600), tail(6500), add(900), crowd(cg == 2 ? 0.1 : 0.3) {}
};
constexpr int kPartStages = 4;        // the fewest stages of a part: below, adding it costs what it saves
// Split products move more bytes, which the model does not see where every block loads: a plan with them has to be better by this.
constexpr double kSplitGain = 0.96;

// The matrices' turns.  Of what is ready, the product with the longest way to go comes first, so that all matrices advance
// side by side; their iterates (8 bytes an element: a pair read, a pair written) then go through HBM in every product once
// they are several times the 126 MB of L2.  From four times kTurnBytes on they are therefore taken in turns of that size,
// those with the longest way first, a later turn's products only filling what the earlier leave idle: twelve
// encoder layers 3.69 -> 3.60 ms, twenty-four 8.06 -> 7.33 ms.  Smaller vectors are better off side by side
// (24 ragged matrices of 200 MB 0.99 against 1.02 ms).
constexpr double kTurnBytes = 100e6;
std::vector<int> turns(const std::vector<OrthMat>& mats, const std::vector<double>& way) {
  std::vector<int> order(mats.size()), turn(mats.size(), 0);
  double all = 0, before = 0;
  for (size_t k = 0; k < mats.size(); ++k) {
    order[k] = static_cast<int>(k);
    all += 8.0 * mats[k].r * mats[k].l;
  }
  if (all < 4 * kTurnBytes) return turn;
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return way[x] > way[y]; });
  for (int k : order) {
    turn[k] = static_cast<int>(before / kTurnBytes);
    before += 8.0 * mats[k].r * mats[k].l;
  }
  return turn;
}

// Plans that cannot be shorter than `limit` are given up before their lists are made.
OrthPlan simulate(const std::vector<OrthMat>& mats, bool split, int steps, int cg, int tn, bool mirrored, int most_parts, int workers, double limit) {
  OrthPlan plan;
  plan.cg = cg;
  plan.tn = tn;
  plan.mirrored = mirrored;
  const OrthCosts cost(split, cg, tn);
  const int tm = 128 * cg, num = static_cast<int>(mats.size());
  struct Spot { int i, j; };
  // after: from the last stage to readable; way: all of it.  A product split over K hands out, before its own tiles, those of
  // the parts 1 .. parts - 1: `helpers` tiles stored, `handed` their way from last stage to readable, `adding` what adding them costs.
  struct Product {
    std::vector<Spot> spots;
    unsigned stored = 0, helpers = 0, before = 0;
    int depth = 0, parts = 1, part_depth = 0, slot = 0;
    double busy = 0, after = 0, way = 0, handed = 0, adding = 0;
    size_t tiles() const { return spots.size() * parts; }
  };
  std::vector<Product> products(static_cast<size_t>(num) * 3);
  size_t most = 1;
  // what depends on the number of parts: how long a part, and the way of all of it
  auto cut = [&](Product& pr, int kind, int rows, int cols, int parts) {
    const int live = std::min((cols + 63) / 64, tn / 64), stages = (pr.depth + kOrthTK - 1) / kOrthTK, part_stages = (stages + parts - 1) / parts;
    pr.parts = (stages + part_stages - 1) / part_stages;
    pr.part_depth = part_stages * kOrthTK;
    pr.adding = (pr.parts - 1) * live * cost.add;
    pr.busy = std::max(part_stages * cost.stage, tn / 64 * cost.strip + pr.adding);
    pr.after = cost.tail + live * cost.strip + (kind != kOrthApply && mirrored && rows > tm ? cost.mirror : 0.0) + pr.adding;
    pr.handed = cost.tail + live * cost.strip;
    pr.way = pr.busy + pr.after + (pr.parts > 1 ? pr.handed : 0.0);
  };
  for (int k = 0; k < num; ++k)
    for (int kind = 0; kind < 3; ++kind) {
      Product& pr = products[3 * k + kind];
      const int rows = mats[k].r, cols = kind == kOrthApply ? mats[k].l : mats[k].r;
      pr.depth = kind == kOrthGram ? mats[k].l : mats[k].r;
      for (int64_t j = 0; j * tn < cols; ++j)
        for (int64_t i = 0; i * tm < rows; ++i) {
          if (kind != kOrthApply && mirrored && i < j) continue;
          pr.spots.push_back({static_cast<int>(i), static_cast<int>(j)});
          for (int rank = 0; rank < cg; ++rank) pr.stored += i * tm + rank * 128 < rows;
        }
      cut(pr, kind, rows, cols, 1);
    }
  // A Gram product is split no further than the longest matrix's step calls for, at its own best.
  auto step = [&](int k) { return products[3 * k].way + products[3 * k + 1].way + products[3 * k + 2].way; };
  auto most_of = [&](int k) {
    const Product& pr = products[3 * k];
    return std::min(most_parts, std::min(workers / static_cast<int>(pr.spots.size()), (pr.depth + kOrthTK - 1) / kOrthTK / kPartStages));
  };
  double longest = 0.0;
  for (int k = 0; k < num; ++k) {
    double best = step(k);
    for (int parts = 2; parts <= most_of(k); ++parts) {
      cut(products[3 * k], kOrthGram, mats[k].r, mats[k].r, parts);
      best = std::min(best, step(k));
    }
    longest = std::max(longest, best);
  }
  std::vector<double> step_way(num, 0.0);
  for (int k = 0; k < num; ++k) {
    int parts = 1;
    do cut(products[3 * k], kOrthGram, mats[k].r, mats[k].r, parts);
    while (step(k) > longest && ++parts <= most_of(k));
    step_way[k] = step(k);
    unsigned before = 0;
    for (int kind = 0; kind < 3; ++kind) {
      Product& pr = products[3 * k + kind];
      pr.helpers = pr.stored * (pr.parts - 1);
      pr.slot = plan.slots;
      plan.slots += static_cast<int>(pr.spots.size()) * (pr.parts - 1);
      pr.before = before;
      before += pr.stored + pr.helpers;
      most = std::max(most, pr.tiles() * static_cast<size_t>(num));
    }
  }
  plan.workers = static_cast<int>(std::min<size_t>(workers, most));
  double busy = 0.0;                                       // of all workers: no plan is shorter than their even share
  for (const Product& pr : products) busy += pr.busy * pr.tiles();
  const double share = steps * busy / plan.workers, crowd = cost.crowd * share;
  plan.cycles = share + crowd;
  if (plan.cycles >= limit) return plan;
  plan.cycles = crowd;
  plan.lists.resize(plan.workers);
  struct Open { double at, way; int mat, step, kind; size_t next; double end, handed; };       // a product that may start at `at`; handed: when its parts are there
  auto sooner = [](const Open& x, const Open& y) { return x.at != y.at ? x.at > y.at : x.mat > y.mat; };
  const std::vector<int> turn = turns(mats, step_way);
  auto shorter = [&](const Open& x, const Open& y) {
    return turn[x.mat] != turn[y.mat] ? turn[x.mat] > turn[y.mat] : x.way != y.way ? x.way < y.way : x.mat > y.mat;
  };
  std::vector<Open> future, ready;     // heaps: the soonest, the one with the longest way to go
  for (int k = 0; k < num; ++k) future.push_back({0.0, step_way[k] * steps, k, 0, 0, 0, 0.0, 0.0});
  std::make_heap(future.begin(), future.end(), sooner);
  typedef std::pair<double, int> Free;                                                 // when, who
  std::vector<Free> idle;
  for (int w = 0; w < plan.workers; ++w) idle.emplace_back(0.0, w);
  std::make_heap(idle.begin(), idle.end(), std::greater<Free>());
  while (!future.empty() || !ready.empty()) {
    std::pop_heap(idle.begin(), idle.end(), std::greater<Free>());
    Free& who = idle.back();
    if (ready.empty()) who.first = std::max(who.first, future.front().at);
    while (!future.empty() && future.front().at <= who.first) {
      std::pop_heap(future.begin(), future.end(), sooner);
      ready.push_back(future.back());
      std::push_heap(ready.begin(), ready.end(), shorter);
      future.pop_back();
    }
    Open& open = ready.front();
    const Product& pr = products[3 * open.mat + open.kind];
    const int number = static_cast<int>(open.next % pr.spots.size()), part = (static_cast<int>(open.next / pr.spots.size()) + 1) % pr.parts;      // part 0, the tiles themselves, last
    const Spot spot = pr.spots[number];
    ++open.next;
    const OrthMat& m = mats[open.mat];
    const unsigned per_step = products[3 * open.mat + 2].before + products[3 * open.mat + 2].stored;
    OrthTile tile = {};
    tile.mat = open.mat;
    tile.i = spot.i;
    tile.j = spot.j;
    tile.first = part * pr.part_depth;
    tile.depth = std::min(pr.part_depth, pr.depth - tile.first);
    tile.rows = m.r;
    tile.cols = open.kind == kOrthApply ? m.l : m.r;
    tile.needs = open.step * per_step + pr.before;
    tile.ready = tile.needs + (part == 0 ? pr.helpers : 0);
    tile.step_kind = open.step * 4 + (part == 0 ? open.kind : kOrthPart);
    tile.adds = part == 0 ? pr.parts - 1 : 0;
    tile.slot = pr.slot + number * (pr.parts - 1) + (part == 0 ? 0 : part - 1);
    plan.lists[who.second].push_back(tile);
    who.first = std::max(who.first, open.at) + pr.busy;      // idle since before the product could start
    if (part != 0) open.handed = std::max(open.handed, who.first + pr.handed);
    else open.end = std::max(open.end, std::max(who.first, open.handed) + pr.after);
    std::push_heap(idle.begin(), idle.end(), std::greater<Free>());
    if (open.next == pr.tiles()) {
      Open then = open;
      std::pop_heap(ready.begin(), ready.end(), shorter);
      ready.pop_back();
      plan.cycles = std::max(plan.cycles, then.end + crowd);
      then.at = then.end;
      then.way -= pr.way;
      then.next = 0;
      then.handed = 0.0;
      if (++then.kind == 3) { then.kind = 0; ++then.step; }
      if (then.step < steps) {
        future.push_back(then);
        std::push_heap(future.begin(), future.end(), sooner);
      }
    }
  }
  return plan;
}

// The plan with the shortest simulated time: pairs or lone blocks, Gram products whole or split over K, symmetric products
// mirrored or, where blocks would idle, computed in full.  For vectors of many tiles only the first choice is tried.
OrthPlan choose_plan(const std::vector<OrthMat>& mats, bool split, int steps, int singles, int pairs) {
  double tiles = 0;
  for (const OrthMat& m : mats) tiles += 3.0 * ((m.r + 255) / 256) * ((m.l + 255) / 256);
  const bool many = tiles * steps > 40000;
  struct Tiling { int cg, tn; bool mirrored; };
  std::vector<Tiling> tilings = {{1, 128, true}, {1, 128, false}, {1, 64, false}};
  if (!split) tilings.insert(tilings.begin(), {{2, 256, true}, {2, 256, false}});
  if (many) tilings.resize(1);
  OrthPlan best;
  best.cycles = 1e300;
  for (int parts = 1; parts <= (many ? 1 : 8); parts *= 2)
    for (const Tiling& t : tilings) {
      const double limit = (parts > 1 && best.slots == 0 ? kSplitGain : 1.0) * best.cycles;
      OrthPlan plan = simulate(mats, split, steps, t.cg, t.tn, t.mirrored, parts, t.cg == 2 ? pairs : singles, limit);
      if (plan.cycles < limit) best = std::move(plan);
    }
  return best;
}

template <bool SPLIT, int CG, int TN>
int prepare_kernel(int sms, int* workers) {
  using T = OrthTiling<SPLIT, CG, TN>;
  static_assert(T::kBytes <= 227 * 1024, "shared memory of a block");
  auto* kernel = &orth_steps_kernel<SPLIT, CG, TN>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kBytes) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
  if (CG == 1) {
    *workers = sms;                   // one block an SM fits: its shared memory is checked above
    return ADACONS_OK;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sms / CG * CG);
  cfg.blockDim = dim3(kOrthThreads);
  cfg.dynamicSmemBytes = T::kBytes;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int pairs = 0;
  if (cudaOccupancyMaxActiveClusters(&pairs, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); return ADACONS_ECUDA; }
  *workers = std::min(pairs, sms / CG);
  return *workers > 0 ? ADACONS_OK : ADACONS_ECUDA;
}

template <bool SPLIT>
int prepare_small() {
  static_assert(kSmallBytes <= 227 * 1024, "shared memory of a block");
  if (cudaFuncSetAttribute(orth_small_kernel<SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallBytes) == cudaSuccess) return ADACONS_OK;
  cudaGetLastError();
  return ADACONS_ECUDA;
}

template <bool SPLIT, int CG, int TN>
bool launch_steps(const adacons_orth* c, const OrthParams& p, cudaStream_t st) {
  return launch(&orth_steps_kernel<SPLIT, CG, TN>, dim3(c->blocks), dim3(kOrthThreads), OrthTiling<SPLIT, CG, TN>::kBytes, st, kLaunchCooperative, CG, p);
}

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
  const bool split = dtype == ADACONS_F32;
  int singles = 0, pairs = 0;
  rc = split ? prepare_kernel<true, 1, 128>(dev.sms, &singles) : prepare_kernel<false, 1, 128>(dev.sms, &singles);
  if (rc == ADACONS_OK) rc = split ? prepare_kernel<true, 1, 64>(dev.sms, &singles) : prepare_kernel<false, 1, 64>(dev.sms, &singles);
  if (rc == ADACONS_OK && !split) rc = prepare_kernel<false, 2, 256>(dev.sms, &pairs);
  if (rc == ADACONS_OK) rc = split ? prepare_small<true>() : prepare_small<false>();
  if (rc != ADACONS_OK) return rc;

  std::unique_ptr<adacons_orth> holder(new adacons_orth());      // released at the end: nothing leaks if a list runs out of memory
  adacons_orth* c = holder.get();
  c->dev = dev;
  c->dtype = dtype;
  c->d = d;
  c->steps = steps;
  c->eps = eps;

  std::vector<OrthMat> mats(num);
  std::vector<OrthChunk> chunks;
  std::vector<OrthSpot> load;
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
    m.vec_in = offsets[k] % 8 == 0 && rows[k] * cols[k] % 8 == 0;
    m.scale = scaling ? static_cast<float>(std::sqrt(std::max(1.0, static_cast<double>(rows[k]) / static_cast<double>(cols[k])))) : 1.f;
    m.norm_first = static_cast<int>(chunks.size());
    m.norm_count = static_cast<int>((rows[k] * cols[k] + kOrthNormChunk - 1) / kOrthNormChunk);
    for (int q = 0; q < m.norm_count; ++q) chunks.push_back({k, q});
    for (int i = 0; i < (m.r + kOrthLoadTile - 1) / kOrthLoadTile; ++i)
      for (int j = 0; j < (m.l + kOrthLoadCols - 1) / kOrthLoadCols; ++j) load.push_back({k, i, j});
  }
  // The one-block kernel only where every matrix fits it: beside larger ones the small ones cost the general kernel
  // next to nothing (their chain is the shorter), and a second launch would come on top.
  c->small = true;
  for (const OrthMat& m : mats) c->small = c->small && m.r <= kOrthSmallR && m.l <= kOrthSmallL;
  const OrthPlan plan = c->small ? OrthPlan() : choose_plan(mats, split, steps, singles, pairs);
  c->cg = plan.cg;
  c->tn = plan.tn;
  c->blocks = plan.workers * plan.cg;
  std::vector<OrthTile> tiles;
  std::vector<int> begin(1, 0);
  for (const auto& list : plan.lists) {
    tiles.insert(tiles.end(), list.begin(), list.end());
    begin.push_back(static_cast<int>(tiles.size()));
  }
  c->num_mats = num;
  std::vector<OrthStep> step_coeffs(steps);
  for (int s = 0; s < steps; ++s) {
    const double* q = coeffs + 3 * s;
    step_coeffs[s] = {static_cast<float>(q[0]), static_cast<float>(q[1]), static_cast<float>(q[2]),
                      static_cast<float>(!split && !c->small ? q[0] : s >= 3 ? -0.75 * (q[1] + q[2]) : 0.0)};
  }
  c->num_chunks = static_cast<int>(chunks.size());
  c->num_load = static_cast<int>(load.size());

  Arena a;
  const size_t at_mats = a.take(num * sizeof(OrthMat)), at_maps = a.take(static_cast<size_t>(num) * kMapCount * sizeof(CUtensorMap));
  const size_t at_tiles = a.take(tiles.size() * sizeof(OrthTile)), at_begin = a.take(begin.size() * sizeof(int)), at_starved = a.take(begin.size() * sizeof(int));
  const size_t at_coeffs = a.take(step_coeffs.size() * sizeof(OrthStep)), at_done = a.take(num * sizeof(unsigned));
  const size_t at_load = a.take(load.size() * sizeof(OrthSpot)), at_chunks = a.take(chunks.size() * sizeof(OrthChunk));
  const size_t at_partial = a.take(chunks.size() * sizeof(double)), at_flags = a.take(sizeof(uint32_t));
  const size_t head = a.used;
  const size_t at_sums = a.take(static_cast<size_t>(plan.slots) * plan.cg * (plan.tn / 64) * 2 * kOrthStripPart);     // the strips of each of cg blocks
  std::vector<size_t> at(static_cast<size_t>(num) * kMapCount, 0);
  for (int k = 0; k < num && !c->small; ++k)
    for (int q = 0; q < kMapCount; ++q) {
      const bool is_x = q < kMapS;
      if (!is_x && (q & 1) && !split) continue;                  // S and B are pairs only in an fp32 context
      at[k * kMapCount + q] = a.take(static_cast<size_t>(mats[k].r) * (is_x ? mats[k].ldx : mats[k].lds) * sizeof(__half));
    }
  c->bytes = a.used;
  std::vector<unsigned char> host(head, 0);
  std::vector<CUtensorMap> maps(static_cast<size_t>(num) * kMapCount);
  if (cudaMalloc(&c->memory, c->bytes) != cudaSuccess) { cudaGetLastError(); return ADACONS_ENOMEM; }
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
        return ADACONS_ECUDA;
      }
    }
  }
  std::memcpy(host.data() + at_mats, mats.data(), num * sizeof(OrthMat));
  std::memcpy(host.data() + at_maps, maps.data(), maps.size() * sizeof(CUtensorMap));
  OrthParams& p = c->params;
  std::memcpy(host.data() + at_tiles, tiles.data(), tiles.size() * sizeof(OrthTile));
  std::memcpy(host.data() + at_begin, begin.data(), begin.size() * sizeof(int));
  begin[0] = 1;                                              // the first worker's first tile is nobody's, which its matrix waits for
  std::memcpy(host.data() + at_starved, begin.data(), begin.size() * sizeof(int));
  c->starved = reinterpret_cast<const int*>(c->memory + at_starved);
  p.tiles = reinterpret_cast<const OrthTile*>(c->memory + at_tiles);
  p.begin = reinterpret_cast<const int*>(c->memory + at_begin);
  p.mirrored = plan.mirrored;
  std::memcpy(host.data() + at_coeffs, step_coeffs.data(), step_coeffs.size() * sizeof(OrthStep));
  std::memcpy(host.data() + at_load, load.data(), load.size() * sizeof(OrthSpot));
  std::memcpy(host.data() + at_chunks, chunks.data(), chunks.size() * sizeof(OrthChunk));
  // the padding of the iterates is read by the epilogues (never by a product): zero it once
  if (cudaMemset(c->memory + head, 0, c->bytes - head) != cudaSuccess ||
      cudaMemcpy(c->memory, host.data(), head, cudaMemcpyHostToDevice) != cudaSuccess || cudaDeviceSynchronize() != cudaSuccess) {
    cudaGetLastError();
    cudaFree(c->memory);
    return ADACONS_ECUDA;
  }
  p.mats = reinterpret_cast<const OrthMat*>(c->memory + at_mats);
  p.maps = reinterpret_cast<const CUtensorMap*>(c->memory + at_maps);
  p.coeffs = reinterpret_cast<const OrthStep*>(c->memory + at_coeffs);
  p.done = reinterpret_cast<unsigned*>(c->memory + at_done);
  p.flags = reinterpret_cast<uint32_t*>(c->memory + at_flags);
  p.sums = c->memory + at_sums;
  p.steps = steps;
  c->load_tiles = reinterpret_cast<const OrthSpot*>(c->memory + at_load);
  c->chunks = reinterpret_cast<const OrthChunk*>(c->memory + at_chunks);
  c->partial = reinterpret_cast<double*>(c->memory + at_partial);
  *out = holder.release();
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

}  // extern "C"

namespace {

int apply(adacons_orth* c, const void* update, void* out, void* cuda_stream, bool starve) {
  if (c == nullptr || update == nullptr || out == nullptr) return ADACONS_EINVAL;
  const size_t elem = c->dtype == ADACONS_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(update) % elem != 0 || reinterpret_cast<uintptr_t>(out) % elem != 0) return ADACONS_EINVAL;
  DeviceGuard guard(c->dev.device);
  if (!guard.ok) return ADACONS_ECUDA;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  OrthParams p = c->params;
  p.out = out;
  p.out_aligned = reinterpret_cast<uintptr_t>(out) % 16 == 0;
  if (starve) p.begin = c->starved;
  const double* partial = c->partial;
  const int aligned = reinterpret_cast<uintptr_t>(update) % 16 == 0;
  c->launches = c->small ? 1 : 3;
  bool ok;
  if (c->small) {
    if (c->dtype == ADACONS_F32) ok = launch(&orth_small_kernel<true>, dim3(c->num_mats), dim3(kOrthSmallThreads), kSmallBytes, st, kLaunchPlain, 1, p, update, aligned, c->eps);
    else ok = launch(&orth_small_kernel<false>, dim3(c->num_mats), dim3(kOrthSmallThreads), kSmallBytes, st, kLaunchPlain, 1, p, update, aligned, c->eps);
  } else if (c->dtype == ADACONS_F32) {
    ok = launch(&orth_norm_kernel<0>, dim3(c->num_chunks), dim3(256), 0, st, kLaunchPlain, 1, update, aligned, p.mats, c->chunks, c->partial) &&
         launch(&orth_load_kernel<0>, dim3(c->num_load), dim3(256), 0, st, kLaunchOverlap, 1, update, aligned, p.mats, c->load_tiles, partial, c->eps, p.done, c->num_mats) &&
         (c->tn == 128 ? launch_steps<true, 1, 128>(c, p, st) : launch_steps<true, 1, 64>(c, p, st));
  } else {
    ok = launch(&orth_norm_kernel<1>, dim3(c->num_chunks), dim3(256), 0, st, kLaunchPlain, 1, update, aligned, p.mats, c->chunks, c->partial) &&
         launch(&orth_load_kernel<1>, dim3(c->num_load), dim3(256), 0, st, kLaunchOverlap, 1, update, aligned, p.mats, c->load_tiles, partial, c->eps, p.done, c->num_mats) &&
         (c->cg == 2 ? launch_steps<false, 2, 256>(c, p, st) : c->tn == 128 ? launch_steps<false, 1, 128>(c, p, st) : launch_steps<false, 1, 64>(c, p, st));
  }
  return ok ? ADACONS_OK : ADACONS_ECUDA;
}

}  // namespace

extern "C" {

int adacons_orth_apply(adacons_orth* c, const void* update, void* out, void* cuda_stream) { return apply(c, update, out, cuda_stream, false); }

int adacons_selftest_orth(adacons_orth* c, const void* update, void* out, void* cuda_stream) {
  if (c == nullptr || c->small) return ADACONS_EINVAL;
  return apply(c, update, out, cuda_stream, true);
}

int adacons_orth_get_status(adacons_orth* c, uint32_t* flags, void* cuda_stream) {
  if (c == nullptr || flags == nullptr) return ADACONS_EINVAL;
  DeviceGuard guard(c->dev.device);
  if (!guard.ok) return ADACONS_ECUDA;
  return take_status(c->params.flags, flags, static_cast<cudaStream_t>(cuda_stream));
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
  DeviceGuard guard(c->dev.device);
  cudaFree(c->memory);
  cudaGetLastError();
  delete c;
  return ADACONS_OK;
}

}  // extern "C"
