// Gated feed-forward block and its gradient: kernels (sm_100a).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "adacons_tc.cuh"

namespace adacons {

// ----------------------------------------------------------------------------------------------
//     g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T
// and back, from dy and the saved g and u:
//     dh = dy Wd,  dg = dh u act'(g),  du = dh act(g),  dx = dg Wg + du Wu,
//     dWg = dg^T x,  dWu = du^T x,  dWd = dy^T h
// All of it is matrix products with something done to a tile of the result, so there is one kernel with three endings:
//   Up     a tile of g and the same tile of u side by side in one accumulator (the right operand's rows are half Wg's, half Wu's):
//          the ending has both and writes g, u and h
//   Back   a tile of dh, with g and u read where they are: writes dg, du and h, which is not kept between the passes
//   Plain  y; dx, whose two products are one with twice the K; the weights' gradients, three products in one launch
// The operands lie as the caller has them: every tensor is a matrix of 64 x 64 boxes, taken K-major where its rows run along K and MN-major
// where they run across it, and no transposed copy is made.
//
// Tiles.  CG = 2: a pair of blocks (two SMs) shares a tile of 256 x 256; each holds 128 rows of the left operand, half of the right one
// and 128 rows of the result, 64 bytes from L2 a cycle and SM at the tensor pipe's full rate where a block alone would need 96.
// One pair per two SMs walks through the tiles; one warp of each block copies operand stages by TMA, one thread of the even block issues the products
// into one of two accumulators, eight warps work off the other.  CG = 1: tiles of 128 x 128, one block each, for problems whose
// larger tiles would leave SMs idle; the blocks of a cluster may share one tile's K and add up their sums, in order, through one another's
// shared memory.  Sums are fp32 throughout; g, u, h, dg and du are rounded to the tensors' type once, as operands.
// fp16 holds dg and du times 2^k, with 2^k from dy's largest element, so that small or large gradients do not leave its range; the products
// that they go into are divided by it again.
// ----------------------------------------------------------------------------------------------
constexpr int kFfnTK = 64;                       // K elements per stage: one 128-byte swizzled row
constexpr int kFfnStages = 6;
constexpr uint32_t kFfnOperand = 128 * kFfnTK * 2, kFfnStage = 2 * kFfnOperand;      // of a block: 128 rows of either operand
constexpr uint32_t kFfnBars = kFfnStages * kFfnStage;
constexpr uint32_t kFfnBytes = kFfnBars + 256 + 1024;          // + alignment of the base
constexpr int kFfnThreads = 320;                 // warps 0-7 endings, 8 operand copies, 9 products
constexpr int kFfnGroup = 8;                     // rows of tiles that are walked through together: their operands stay in L2
constexpr int kFfnSumRow = 132;                  // floats of a row of partial sums
constexpr int kFfnPeaks = 128;                   // blocks that look for dy's largest element
static_assert(128 * kFfnSumRow * 4 <= kFfnBars, "partial sums take the stages' place");

enum FfnKind { kFfnUp = 0, kFfnBack = 1, kFfnPlain = 2 };
enum FfnAct { kActSilu = 0, kActGelu = 1, kActGeluTanh = 2, kActRelu = 3 };

struct FfnRows {                                 // rows of 16-bit elements; null: not there
  void* data;
  long long row;
  int wide;                                      // rows start on 32 bytes
};
// One product: C (m x n) = sum over segments of A B^T.
struct FfnProblem {
  int a[2], b[2];                                // tensor maps: of each segment (Plain, Back), b: of Wg and Wu (Up)
  int m, n, steps, segments;                     // steps of kFfnTK of a segment
  int a_across, b_across;                        // the operand's rows are the K index
  int tiles_m, tiles_n, first;                   // first: number of its first tile
  int scaled;                                    // the operands hold 2^k times
  FfnRows out;
};
struct FfnParams {
  CUtensorMap maps[8];
  FfnProblem problem[4];
  int problems, tiles, act, shares;
  FfnRows gate, up;                              // Up: written; Back: read
  FfnRows dgate, dup;                            // Back
  const unsigned* peaks;                         // of dy, kFfnPeaks of them (fp16), or null
  uint32_t* flags;
};

template <bool BF16>
__device__ __forceinline__ float2 ffn_unpack(uint32_t v) {
  if (BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
template <bool BF16>
__device__ __forceinline__ uint32_t ffn_pack(float a, float b) {
  if (BF16) return pack_bf16x2_rn(a, b);
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// act(g) and its derivative.  gelu: g Phi(g) with Phi from the error function's approximation by Abramowitz and Stegun, 7.1.26 (absolute error
// 1.5e-7 of a value that is rounded to 11 bits at most), whose exponential is the derivative's as well.
template <bool SLOPE>
__device__ __forceinline__ void ffn_act(int act, float g, float& a, float& slope) {
  if (act == kActSilu) {
    const float s = __fdividef(1.f, 1.f + __expf(-g));
    a = g * s;
    if (SLOPE) slope = fmaf(a, 1.f - s, s);
  } else if (act == kActGelu) {
    const float e = __expf(-0.5f * g * g);
    const float t = __fdividef(1.f, fmaf(0.3275911f * 0.70710678118654752f, fabsf(g), 1.f));
    const float q = 0.5f * e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float phi = g < 0.f ? q : 1.f - q;
    a = g * phi;
    if (SLOPE) slope = fmaf(g * 0.39894228040143268f, e, phi);
  } else if (act == kActGeluTanh) {
    const float k = 0.79788456080286536f, in = k * fmaf(0.044715f * g * g, g, g);
    const float s = __fdividef(1.f, 1.f + __expf(-2.f * in));        // (1 + tanh in) / 2
    a = g * s;
    if (SLOPE) slope = fmaf(2.f * a * (1.f - s), k * fmaf(3.f * 0.044715f * g, g, 1.f), s);
  } else {
    a = fmaxf(g, 0.f);
    if (g != g) a = g;
    if (SLOPE) slope = g > 0.f ? 1.f : 0.f;
  }
}

// The power of two that dg and du are held with (fp16): dy's largest element comes to lie in [1/2, 1).
__device__ __forceinline__ int ffn_exponent(const unsigned* peaks) {
  const int lane = threadIdx.x & 31;
  unsigned top = 0;
  for (int k = lane; k < kFfnPeaks; k += 32) top = max(top, peaks[k]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const int e = static_cast<int>(top >> 23);      // of a finite positive fp32 value; fp16 has none below 2^-24
  return e == 0 ? 0 : 126 - e;
}
__device__ __forceinline__ float ffn_power(int e) { return __int_as_float((127 + e) << 23); }

// Eight values of a row, 16 bytes; `full`: sixteen, 32 bytes.
template <bool BF16>
__device__ __forceinline__ uint4 ffn_round8(const float* v) {
  return make_uint4(ffn_pack<BF16>(v[0], v[1]), ffn_pack<BF16>(v[2], v[3]), ffn_pack<BF16>(v[4], v[5]), ffn_pack<BF16>(v[6], v[7]));
}
template <bool BF16, int N>
__device__ __forceinline__ void ffn_put(const FfnRows& to, int row, int col, int cols, const float (&v)[N]) {
  unsigned char* at = static_cast<unsigned char*>(to.data) + (row * to.row + col) * 2;
  const uint4 a = ffn_round8<BF16>(v);
  if constexpr (N == 16) {
    const uint4 b = ffn_round8<BF16>(v + 8);
    if (to.wide && col + 16 <= cols) {
      st_global_v8(at, a, b, 0ull);
      return;
    }
    if (col + 16 <= cols) *reinterpret_cast<uint4*>(at + 16) = b;
  }
  *reinterpret_cast<uint4*>(at) = a;
}
template <int N>
__device__ __forceinline__ void ffn_get(uint4 (&v)[N / 8], const FfnRows& from, int row, int col, int cols, bool there) {
#pragma unroll
  for (int k = 0; k < N / 8; ++k) {
    v[k] = make_uint4(0u, 0u, 0u, 0u);
    if (there && col + 8 * k < cols) v[k] = *reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(from.data) + (row * from.row + col + 8 * k) * 2);
  }
}

// What becomes of N neighbouring results of a row inside the matrix.  v: the sums (Up: of g), w: Up: of u; gate, up: Back: g and u there.
template <int KIND, bool BF16, int N>
__device__ __forceinline__ void ffn_end(const FfnParams& p, const FfnProblem& q, float factor, int row, int col, float (&v)[N], float (&w)[N], const uint4 (&gate)[N / 8],
                                        const uint4 (&up)[N / 8]) {
  if constexpr (KIND == kFfnPlain) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= factor;
    ffn_put<BF16>(q.out, row, col, q.n, v);
  } else if constexpr (KIND == kFfnUp) {
    if (p.gate.data != nullptr) {
      ffn_put<BF16>(p.gate, row, col, q.n, v);
      ffn_put<BF16>(p.up, row, col, q.n, w);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float a, unused;
      ffn_act<false>(p.act, v[e], a, unused);
      w[e] *= a;
    }
    ffn_put<BF16>(q.out, row, col, q.n, w);
  } else {
    float h[N];
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
      const uint32_t gs[4] = {gate[k].x, gate[k].y, gate[k].z, gate[k].w}, us[4] = {up[k].x, up[k].y, up[k].z, up[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 g2 = ffn_unpack<BF16>(gs[i]), u2 = ffn_unpack<BF16>(us[i]);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int e = 8 * k + 2 * i + s;
          const float u = s ? u2.y : u2.x, dh = v[e] * factor;
          float a, slope;
          ffn_act<true>(p.act, s ? g2.y : g2.x, a, slope);
          h[e] = a * u;
          v[e] = dh * u * slope;
          w[e] = dh * a;
        }
      }
    }
    ffn_put<BF16>(p.dgate, row, col, q.n, v);
    ffn_put<BF16>(p.dup, row, col, q.n, w);
    ffn_put<BF16>(q.out, row, col, q.n, h);
  }
}

// Tile t: its problem, and which one of it; kFfnGroup rows of tiles at a time, along the columns.
struct FfnSpot { int problem, i, j; };
__device__ __forceinline__ FfnSpot ffn_spot(const FfnParams& p, int t) {
  FfnSpot s;
  s.problem = 0;
  while (s.problem + 1 < p.problems && t >= p.problem[s.problem + 1].first) ++s.problem;
  const FfnProblem& q = p.problem[s.problem];
  const int at = t - q.first, group = at / (kFfnGroup * q.tiles_n), in = at - group * kFfnGroup * q.tiles_n;
  const int rows = min(kFfnGroup, q.tiles_m - group * kFfnGroup);
  s.j = in / rows;
  s.i = group * kFfnGroup + in - s.j * rows;
  return s;
}

template <int KIND, bool BF16, int CG, bool STARVE = false>
__global__ void __launch_bounds__(kFfnThreads, 1) ffn_kernel(const __grid_constant__ FfnParams p) {
  extern __shared__ unsigned char smem_dyn[];
  constexpr int kTM = 128 * CG, kTN = 128 * CG, kCols = KIND == kFfnUp ? kTN / 2 : kTN;      // kCols: columns of the result in a tile
  constexpr int kBuffers = CG;                   // a lone block has one tile
  constexpr uint32_t kTmemCols = kBuffers * kTN;
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + kFfnBars);
  uint64_t* empty = full + kFfnStages;
  uint64_t* acc_full = empty + kFfnStages;       // [2]
  uint64_t* acc_free = acc_full + 2;             // [2]
  uint64_t* drain = acc_free + 2;
  __shared__ uint32_t s_tmem;
  __shared__ int s_issued;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int shares = CG == 2 ? 1 : p.shares;
  const int rank = CG == 2 || shares > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int half = CG == 2 ? rank : 0;           // of a pair
  const int worker = CG == 2 ? blockIdx.x / 2 : blockIdx.x / shares, workers = CG == 2 ? gridDim.x / 2 : p.tiles;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kFfnStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_free[s], 8 * CG); }
    mbar_init(drain, 1);
    s_abort = 0;
    s_issued = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == 9) tmem_alloc<CG>(&s_tmem, kTmemCols);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_launch_dependents();
  pdl_wait();

  // K steps of a tile that are this block's
  auto steps_of = [&](const FfnProblem& q, int& begin, int& end) {
    const int all = q.steps * q.segments;
    begin = CG == 2 ? 0 : static_cast<int>(static_cast<long long>(all) * rank / shares);
    end = CG == 2 ? all : static_cast<int>(static_cast<long long>(all) * (rank + 1) / shares);
  };

  if (warp == 8) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t parity = 1;                       // the stages start out empty
      bool ok = true;
      for (int t = worker; ok && t < p.tiles; t += workers) {
        const FfnSpot s = ffn_spot(p, t);
        const FfnProblem& q = p.problem[s.problem];
        int begin, end;
        steps_of(q, begin, end);
        const int arow = s.i * kTM + half * 128;
        for (int k = begin; k < end; ++k) {
          if (STARVE && k == end - 1) break;
          if (s_abort || !mbar_wait_bounded(&empty[stage], parity)) { s_abort = 1; ok = false; break; }
          const int segment = k >= q.steps ? 1 : 0, k0 = (k - segment * q.steps) * kFfnTK;
          unsigned char* at = smem + stage * kFfnStage;
          if (half == 0) mbar_expect_tx(&full[stage], CG * kFfnStage);      // a pair's bytes all count on the even block's barrier
          auto load = [&](unsigned char* dst, int map, int x, int y) {
            if (CG == 2) tma_load_2d_pair(dst, &p.maps[map], &full[stage], x, y);
            else tma_load_2d(dst, &p.maps[map], &full[stage], x, y);
          };
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = arow + h * 64;
            load(at + h * 8192, q.a[segment], q.a_across ? r : k0, q.a_across ? k0 : r);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            int map, r;
            if (KIND == kFfnUp) {
              map = q.b[CG == 2 ? half : h];
              r = s.j * kCols + (CG == 2 ? h * 64 : 0);
            } else {
              map = q.b[segment];
              r = s.j * kCols + half * 128 + h * 64;
            }
            load(at + kFfnOperand + h * 8192, map, q.b_across ? r : k0, q.b_across ? k0 : r);
          }
          ++issued;
          if (++stage == kFfnStages) { stage = 0; parity ^= 1u; }
        }
      }
      s_issued = issued;
    }
  } else if (warp == 9) {
    if (half == 0) {
      // The whole warp goes through the loop, so that addresses and descriptors are uniform values; one lane issues.
      const bool issuer = elect_one();
      const uint32_t base = (smem_addr(smem) & 0x3ffffu) >> 4;             // descriptors count 16-byte units; above are a cluster block's number and their other fields
      int stage = 0, buf = 0;
      uint32_t parity = 0, acc_parity = 1;
      bool ok = true;
      for (int t = worker; ok && t < p.tiles; t += workers) {
        const FfnSpot s = ffn_spot(p, t);
        const FfnProblem& q = p.problem[s.problem];
        int begin, end;
        steps_of(q, begin, end);
        const uint32_t idesc = mma_idesc(kTM, kTN, BF16, false, false) | (q.a_across ? 1u << 15 : 0u) | (q.b_across ? 1u << 16 : 0u);
        const uint64_t a_base = q.a_across ? desc_mnmajor(0, 8192) : desc_kmajor(0), b_base = q.b_across ? desc_mnmajor(0, 8192) : desc_kmajor(0);
        const uint32_t a_step = q.a_across ? 2048 / 16 : 32 / 16, b_step = q.b_across ? 2048 / 16 : 32 / 16;
        if (s_abort || !mbar_wait_bounded(&acc_free[buf], acc_parity)) ok = false;
        for (int k = begin; k < end; ++k) {
          ok = ok && !s_abort && mbar_wait_bounded(&full[stage], parity);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) { s_abort = 1; break; }
          tc_fence_after();
          const uint64_t a = a_base + (base + stage * (kFfnStage >> 4)), b = b_base + (base + stage * (kFfnStage >> 4) + (kFfnOperand >> 4));
          if (issuer) {
#pragma unroll
            for (int kk = 0; kk < kFfnTK / 16; ++kk) mma_ss<CG>(tmem + buf * kTN, a + kk * a_step, b + kk * b_step, idesc, kk != 0 ? 1u : k != begin);
            mma_commit<CG>(&empty[stage]);
          }
          __syncwarp();
          if (++stage == kFfnStages) { stage = 0; parity ^= 1u; }
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { s_abort = 1; break; }
        if (issuer) mma_commit<CG>(&acc_full[buf]);
        __syncwarp();
        if (++buf == kBuffers) { buf = 0; acc_parity ^= 1u; }
      }
      if (s_abort && issuer) { mma_commit<CG>(drain); mbar_wait_bounded(drain, 0); }
      __syncwarp();
    }
  } else {
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int side = warp >> 2;                  // this warp's half of the columns
    int buf = 0;
    uint32_t parity = 0;
    int exponent = 0;
    if (p.peaks != nullptr) exponent = ffn_exponent(p.peaks);
    for (int t = worker; t < p.tiles; t += workers) {
      const FfnSpot s = ffn_spot(p, t);
      const FfnProblem& q = p.problem[s.problem];
      const int row = s.i * kTM + half * 128 + (warp & 3) * 32 + lane, col0 = s.j * kCols + side * (kCols / 2);
      const float factor = KIND == kFfnBack ? ffn_power(exponent) : q.scaled ? ffn_power(-exponent) : 1.f;
      const bool there = row < q.m;
      uint4 gate[2], up[2];
      if (KIND == kFfnBack && shares == 1) {     // under way while the products are
        ffn_get<16>(gate, p.gate, row, col0, q.n, there);
        ffn_get<16>(up, p.up, row, col0, q.n, there);
      }
      const bool got = !s_abort && mbar_wait_bounded(&acc_full[buf], parity);
      if (!__all_sync(0xffffffffu, got)) { s_abort = 1; break; }
      tc_fence_after();
      const uint32_t acc = tmem + buf * kTN + side * (kCols / 2) + lanes;
      if (shares == 1) {
#pragma unroll 1
        for (int c = 0; c < kCols / 2; c += 16) {
          const int col = col0 + c;
          uint32_t raw[16], raw_up[16];
          tmem_ld16(acc + c, raw);
          if (KIND == kFfnUp) tmem_ld16(acc + kCols + c, raw_up);
          uint4 next_gate[2], next_up[2];
          if (KIND == kFfnBack && c + 16 < kCols / 2) {
            ffn_get<16>(next_gate, p.gate, row, col + 16, q.n, there);
            ffn_get<16>(next_up, p.up, row, col + 16, q.n, there);
          }
          tmem_wait_ld();
          if (there && col < q.n) {
            float v[16], w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              v[e] = __uint_as_float(raw[e]);
              w[e] = KIND == kFfnUp ? __uint_as_float(raw_up[e]) : 0.f;
            }
            ffn_end<KIND, BF16, 16>(p, q, factor, row, col, v, w, gate, up);
          }
          __syncwarp();
          if (KIND == kFfnBack) {
#pragma unroll
            for (int k = 0; k < 2; ++k) { gate[k] = next_gate[k]; up[k] = next_up[k]; }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) { if (CG == 2) mbar_arrive_leader(&acc_free[buf]); else mbar_arrive_one(&acc_free[buf]); }
        __syncwarp();
      } else {                                   // this block's sums, where the stages were: all products that read those are complete
        float* sums = reinterpret_cast<float*>(smem) + ((warp & 3) * 32 + lane) * kFfnSumRow + side * 64;
#pragma unroll 1
        for (int c = 0; c < 64; c += 16) {
          uint32_t raw[16];
          tmem_ld16(tmem + side * 64 + c + lanes, raw);
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(sums + c + 4 * k) = make_uint4(raw[4 * k], raw[4 * k + 1], raw[4 * k + 2], raw[4 * k + 3]);
        }
      }
      if (++buf == kBuffers) { buf = 0; parity ^= 1u; }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (CG == 1 && shares > 1) {
    cluster_sync_all();                          // every block's sums are in place
    const FfnSpot s = ffn_spot(p, worker);
    const FfnProblem& q = p.problem[s.problem];
    if (warp < 8 && !s_abort) {
      const float factor = KIND == kFfnBack ? ffn_power(p.peaks == nullptr ? 0 : ffn_exponent(p.peaks)) : q.scaled ? ffn_power(p.peaks == nullptr ? 0 : -ffn_exponent(p.peaks)) : 1.f;
      constexpr int kEights = kCols / 8;
      for (int unit = threadIdx.x; unit < 128 / shares * kEights; unit += 256) {
        const int r = unit / kEights * shares + rank, c = unit % kEights * 8;        // the blocks take the rows in turn
        const int row = s.i * kTM + r, col = s.j * kCols + c;
        if (row >= q.m || col >= q.n) continue;
        uint4 gate[1], up[1];
        if (KIND == kFfnBack) {
          ffn_get<8>(gate, p.gate, row, col, q.n, true);
          ffn_get<8>(up, p.up, row, col, q.n, true);
        }
        float v[8], w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = w[e] = 0.f;
        const float* at = reinterpret_cast<const float*>(smem) + r * kFfnSumRow + c;
        for (int b = 0; b < shares; ++b) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float4 f = ld_cluster_f32x4(at + 4 * k, b);
            v[4 * k] += f.x; v[4 * k + 1] += f.y; v[4 * k + 2] += f.z; v[4 * k + 3] += f.w;
            if (KIND == kFfnUp) {
              const float4 d = ld_cluster_f32x4(at + kCols + 4 * k, b);
              w[4 * k] += d.x; w[4 * k + 1] += d.y; w[4 * k + 2] += d.z; w[4 * k + 3] += d.w;
            }
          }
        }
        ffn_end<KIND, BF16, 8>(p, q, factor, row, col, v, w, gate, up);
      }
    }
    cluster_sync_all();                          // nobody leaves while its sums are read
  }
  if (CG == 2) cluster_sync_all();               // the pair's copies and arrivals are all in, unless a wait expired
  if (s_abort && threadIdx.x == 0) {             // no copy may land after the block has gone
    for (int s = 0; half == 0 && s < kFfnStages && s < s_issued; ++s) {
      const int uses = (s_issued - 1 - s) / kFfnStages;          // the stage's last copy is its use number `uses`
      mbar_wait_bounded(&full[s], uses & 1);
    }
    atomicOr(p.flags, kFlagTimeout);
  }
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc<CG>(tmem, kTmemCols);
  }
}

// fp16: the largest finite |element| of dy, as the bits of its fp32 value, one for each block.
__global__ void __launch_bounds__(256) ffn_peak_kernel(const void* dy, long long pitch, int rows, int cols, unsigned* peaks) {
  __shared__ unsigned s_top[8];
  pdl_launch_dependents();
  const int eights = cols / 8;
  unsigned top = 0;
  for (int r = blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += kFfnPeaks * 8) {
    const unsigned char* row = static_cast<const unsigned char*>(dy) + r * pitch * 2;
#pragma unroll 4
    for (int k = threadIdx.x & 31; k < eights; k += 32) {
      const uint4 v = *reinterpret_cast<const uint4*>(row + 16 * k);
      const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned half_bits = (u[e / 2] >> (16 * (e & 1))) & 0x7fffu;
        if (half_bits < 0x7c00u) top = max(top, half_bits);
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) top = max(top, s_top[w]);
    peaks[blockIdx.x] = __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(top))));
  }
}

}  // namespace adacons
