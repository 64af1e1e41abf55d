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
// Tiles.  CG = 2: a pair of blocks (two SMs) shares a tile of 256 x 512, in two halves of 256 columns; each block holds 128 rows of the left operand, half of
// the right one's and 128 rows of the result, all 512 columns of its tensor memory.  That takes 48 bytes from L2 a cycle and SM at the tensor
// pipe's full rate; L2 gives 40 to 50, and tiles of 256 x 256 in two buffers, which take 64, kept the pipe 69 to 74 % busy where these keep it 82 to 90 %.
// One pair per two SMs walks through the tiles; one warp of each block copies operand stages by TMA, one thread of the even block issues the products,
// eight warps work off what is complete, 32 rows x 32 columns at a time, which leave through shared memory by TMA (stored by the lanes, each at
// its own row, they took three times as long as what is computed for them).  The products of a tile's first and last stages run half by half, so that one half is worked off, or
// freed, beside the other's products.  The last tiles are halves where that evens out the pairs' work, and all are where K is short against the
// ending: then the two accumulators take turns.  CG = 1: tiles of 128 x 128, one block each and two blocks an SM,
// for problems whose larger tiles would leave SMs idle; the blocks of a cluster may share one tile's K and add up their sums, in order, through one another's
// shared memory.  Sums are fp32 throughout; g, u, h, dg and du are rounded to the tensors' type once, as operands (results 2.4e-3 from 64 bits instead of 1.7e-3 in bf16,
// 3e-4 instead of 2.1e-4 in fp16; operands of 32 bits would take three products for one).
// fp16 holds dg and du times 2^k; the products that they go into are divided by it again.  k is 0, or brings dy's largest element to [1/2, 1) where that is smaller, so that small
// gradients keep their bits.  How much larger than dy the products are is known once they are there: if dg or du round to infinity, the first product notes the largest of them and is
// made again with the k, possibly below 0, that just holds it; otherwise its second launch returns at once (231 x 520 x 1368 31.4 -> 32.8 us, 4096 x 1024 x 4096 195 -> 197.5;
// made again, 43 and 298).  So no token has fewer bits than without a factor, unless dg or du were infinite then (bringing the largest element down to 1 in any case left tokens with 1e-3 beside one with 3000 half of their dx).
// ----------------------------------------------------------------------------------------------
constexpr int kFfnTK = 64;                       // K elements per stage: one 128-byte swizzled row
constexpr uint32_t kFfnOperand = 128 * kFfnTK * 2;             // of a block: 128 rows of an operand
constexpr int kFfnSumRow = 132;                  // floats of a row of partial sums
constexpr int kFfnEndWarps = 8, kFfnThreads = 32 * (kFfnEndWarps + 2);      // endings, operand copies, products
constexpr uint32_t kFfnPatch = 32 * 64;          // bytes of 32 rows x 32 columns on their way out: two of them a warp
template <int CG> struct FfnTiling {
  static constexpr int kHalves = CG;             // of a tile's columns
  static constexpr uint32_t kStage = (1 + kHalves) * kFfnOperand;
  static constexpr uint32_t bytes(int stages) { return stages * kStage + 512 + (CG == 2 ? 2 * kFfnEndWarps * kFfnPatch : 0u) + 1024; }       // + alignment of the base
  static constexpr uint32_t kTmemCols = kHalves * 128 * CG;
};
// Stages: of a pair; of a lone block where one runs on an SM, and where two do
constexpr int kFfnPairStages = 4, kFfnLoneStages = 6, kFfnCrowdStages = 3;
static_assert(128 * kFfnSumRow * 4 <= kFfnCrowdStages * FfnTiling<1>::kStage, "partial sums take the stages' place");
static_assert(FfnTiling<2>::bytes(kFfnPairStages) <= 227 * 1024 && FfnTiling<1>::bytes(kFfnLoneStages) <= 227 * 1024 && FfnTiling<1>::bytes(kFfnCrowdStages) <= 112 * 1024,
              "shared memory of a block");
constexpr int kFfnGroup = 8;                     // rows of tiles that are walked through together: their operands stay in L2
constexpr int kFfnPeaks = 127;                   // blocks that look for dy's largest element
constexpr int kFfnWords = kFfnPeaks + 1;         // what they find, then the largest of dg and du that rounds to infinity as it is held (0: none)
constexpr float kFfnBeyond = 65520.f;            // rounds to infinity in fp16, as all above it

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
  int tiles_m, tiles_n, first;                   // tiles_n: counted in halves; first: number of its first whole tile
  int scaled;                                    // the operands hold 2^k times
  int early;                                     // the right operand is not the work of the kernel before
  FfnRows out;
};
struct FfnParams {
  CUtensorMap maps[8];                           // operands: boxes of 64 x 64
  CUtensorMap outs[4];                           // results: boxes of 32 x 32.  Up, Back: the two beside `out`, then out; Plain: each problem's
  FfnProblem problem[4];
  int problems, tiles, act, shares;
  int wholes;                                    // tiles from this number on are halves
  int stages;                                    // of a lone block
  FfnRows gate, up;                              // Up: written; Back: read
  FfnRows dgate, dup;                            // Back
  const unsigned* peaks;                         // kFfnWords of them (fp16), or null
  unsigned* beyond;                              // the last of them, where it is still to be found (Back)
  int again;                                     // Back: only if there is one
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

__device__ __forceinline__ float2 ffn_ex2(float2 x) {
  float2 y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(x.y));
  return y;
}
__device__ __forceinline__ float2 ffn_rcp(float2 x) {
  float2 y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(x.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(x.y));
  return y;
}
__device__ __forceinline__ float2 ffn_both(float v) { return make_float2(v, v); }
// act(g) and its derivative, of two values.  gelu: g Phi(g) with Phi from the error function's approximation by Abramowitz and Stegun, 7.1.26 (absolute error
// 1.5e-7 of a value that is rounded to 11 bits at most), whose exponential is the derivative's as well.
template <int ACT, bool SLOPE>
__device__ __forceinline__ void ffn_act(float2 g, float2& a, float2& slope) {
  constexpr float kLog2 = 1.4426950408889634f;
  const float2 one = ffn_both(1.f);
  if (ACT == kActSilu) {
    const float2 s = ffn_rcp(add2(ffn_ex2(mul2(g, ffn_both(-kLog2))), one));
    a = mul2(g, s);
    if (SLOPE) slope = fma2(a, fma2(s, ffn_both(-1.f), one), s);
  } else if (ACT == kActGelu) {
    const float2 e = ffn_ex2(mul2(mul2(g, ffn_both(-0.5f * kLog2)), g));
    const float2 t = ffn_rcp(fma2(make_float2(fabsf(g.x), fabsf(g.y)), ffn_both(0.3275911f * 0.70710678118654752f), one));
    float2 q = fma2(t, ffn_both(0.5f * 1.061405429f), ffn_both(0.5f * -1.453152027f));
    q = fma2(t, q, ffn_both(0.5f * 1.421413741f));
    q = fma2(t, q, ffn_both(0.5f * -0.284496736f));
    q = fma2(t, q, ffn_both(0.5f * 0.254829592f));
    q = mul2(mul2(e, t), q);
    const float2 rest = fma2(q, ffn_both(-1.f), one), phi = make_float2(g.x < 0.f ? q.x : rest.x, g.y < 0.f ? q.y : rest.y);
    a = mul2(g, phi);
    if (SLOPE) slope = fma2(mul2(g, ffn_both(0.39894228040143268f)), e, phi);
  } else if (ACT == kActGeluTanh) {
    constexpr float k = 0.79788456080286536f;
    const float2 g2 = mul2(g, g), in = mul2(g, fma2(g2, ffn_both(0.044715f * k), ffn_both(k)));
    const float2 s = ffn_rcp(add2(ffn_ex2(mul2(in, ffn_both(-2.f * kLog2))), one));        // (1 + tanh in) / 2
    a = mul2(g, s);
    if (SLOPE) slope = fma2(mul2(mul2(a, ffn_both(2.f)), fma2(s, ffn_both(-1.f), one)), fma2(g2, ffn_both(3.f * 0.044715f * k), ffn_both(k)), s);
  } else {
    a = make_float2(g.x < 0.f ? 0.f : g.x, g.y < 0.f ? 0.f : g.y);
    if (SLOPE) slope = make_float2(g.x > 0.f ? 1.f : 0.f, g.y > 0.f ? 1.f : 0.f);
  }
}
// of N pairs, the choice made once: the values' chains run beside one another (with a choice for each of them 512 columns took 35,000 cycles)
template <bool SLOPE, int N>
__device__ __forceinline__ void ffn_act_all(int act, const float2 (&g)[N], float2 (&a)[N], float2 (&slope)[N]) {
  switch (act) {
    case kActSilu:
#pragma unroll
      for (int e = 0; e < N; ++e) ffn_act<kActSilu, SLOPE>(g[e], a[e], slope[e]);
      break;
    case kActGelu:
#pragma unroll
      for (int e = 0; e < N; ++e) ffn_act<kActGelu, SLOPE>(g[e], a[e], slope[e]);
      break;
    case kActGeluTanh:
#pragma unroll
      for (int e = 0; e < N; ++e) ffn_act<kActGeluTanh, SLOPE>(g[e], a[e], slope[e]);
      break;
    default:
#pragma unroll
      for (int e = 0; e < N; ++e) ffn_act<kActRelu, SLOPE>(g[e], a[e], slope[e]);
  }
}

// The power of two that dg and du are held with (fp16).  `settled`: whether they are known to fit, or by how much they do not.
__device__ __forceinline__ int ffn_exponent(const unsigned* peaks, bool settled) {
  const int lane = threadIdx.x & 31;
  unsigned top = 0;
  for (int k = lane; k < kFfnPeaks; k += 32) top = max(top, peaks[k]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  int e = static_cast<int>(top >> 23);           // of a finite fp32 value that fp16 can have
  e = e == 0 ? 0 : max(0, 126 - e);
  if (settled && peaks[kFfnPeaks] != 0u) {       // down to the largest power that keeps it below kFfnBeyond, 2^15 (2 - 2^-11)
    const unsigned beyond = peaks[kFfnPeaks];
    e -= static_cast<int>(beyond >> 23) - (127 + 15) + ((beyond & 0x7fffffu) >= 0x7ff000u ? 1 : 0);
  }
  return e;
}
// The largest finite one of dg and du that does not fit.
template <int N>
__device__ __forceinline__ void ffn_note(const float2 (&v)[N], const float2 (&w)[N], unsigned* beyond) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) top = fmaxf(fmaxf(fmaxf(top, fabsf(v[e].x)), fmaxf(fabsf(v[e].y), fabsf(w[e].x))), fabsf(w[e].y));
  if (top < kFfnBeyond) return;
  top = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float all[4] = {fabsf(v[e].x), fabsf(v[e].y), fabsf(w[e].x), fabsf(w[e].y)};
#pragma unroll
    for (int k = 0; k < 4; ++k) top = all[k] < INFINITY ? fmaxf(top, all[k]) : top;
  }
  if (top >= kFfnBeyond) atomicMax(beyond, __float_as_uint(top));
}
__device__ __forceinline__ float ffn_power(int e) { return __int_as_float((127 + e) << 23); }

template <bool BF16, int N>
__device__ __forceinline__ void ffn_round(const float2 (&v)[N / 2], uint4* w) {
#pragma unroll
  for (int k = 0; k < N / 8; ++k)
    w[k] = make_uint4(ffn_pack<BF16>(v[4 * k].x, v[4 * k].y), ffn_pack<BF16>(v[4 * k + 1].x, v[4 * k + 1].y), ffn_pack<BF16>(v[4 * k + 2].x, v[4 * k + 2].y),
                      ffn_pack<BF16>(v[4 * k + 3].x, v[4 * k + 3].y));
}
// A warp's way out: 32 rows x 32 columns, a row a lane, into one of two places of shared memory, 16-byte units permuted as the tensor map's 64-byte swizzle
// has them, and from there by TMA, which clips the matrix's edges.  The place is free again once the copy before last has read it.
struct FfnWay {
  unsigned char* places;
  int next;
  __device__ __forceinline__ void put(const uint4 (&v)[4], const CUtensorMap* map, int row0, int col) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) bulk_wait_read<1>();
    __syncwarp();
    unsigned char* at = places + next * kFfnPatch;
#pragma unroll
    for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(at + lane * 64 + ((k ^ ((lane >> 1) & 3)) * 16)) = v[k];
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(map, at, col, row0);
      bulk_commit();
    }
    next ^= 1;
  }
};
__device__ __forceinline__ uint4* ffn_at(const FfnRows& t, int row, int col) {
  return reinterpret_cast<uint4*>(static_cast<unsigned char*>(t.data) + (row * t.row + col) * 2);
}
template <int N>
__device__ __forceinline__ void ffn_get(uint4 (&v)[N / 8], const FfnRows& from, int row, int col, int cols, bool there) {
  const uint4* at = ffn_at(from, row, col);
  if (from.wide && there && col + N <= cols) {
#pragma unroll
    for (int k = 0; k + 1 < N / 8; k += 2) ld_stream_v8(at + k, v[k], v[k + 1]);
    if (N / 8 % 2 != 0) v[N / 8 - 1] = at[N / 8 - 1];
    return;
  }
#pragma unroll
  for (int k = 0; k < N / 8; ++k) {
    v[k] = make_uint4(0u, 0u, 0u, 0u);
    if (there && col + 8 * k + 8 <= cols) v[k] = at[k];
  }
}

// What becomes of N neighbouring results of a row.  v: the sums (Up: of g), w: Up: of u; gate, up: Back: g and u there.  one, two: g and u (Up), dg and du (Back);
// result: h, or what Plain writes.
template <int KIND, bool BF16, int N>
__device__ __forceinline__ void ffn_end(int act, float factor, float2 (&v)[N / 2], float2 (&w)[N / 2], const uint4* gate, const uint4* up, uint4* one, uint4* two, uint4* result) {
  float2 a[N / 2];
  if constexpr (KIND == kFfnPlain) {
#pragma unroll
    for (int e = 0; e < N / 2; ++e) a[e] = mul2(v[e], ffn_both(factor));
  } else if constexpr (KIND == kFfnUp) {
    ffn_act_all<false>(act, v, a, a);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) a[e] = mul2(a[e], w[e]);
  } else {
    float2 g[N / 2], slope[N / 2];
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
      g[4 * k] = ffn_unpack<BF16>(gate[k].x);
      g[4 * k + 1] = ffn_unpack<BF16>(gate[k].y);
      g[4 * k + 2] = ffn_unpack<BF16>(gate[k].z);
      g[4 * k + 3] = ffn_unpack<BF16>(gate[k].w);
    }
    ffn_act_all<true>(act, g, a, slope);
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
      const uint32_t us[4] = {up[k].x, up[k].y, up[k].z, up[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 4 * k + i;
        const float2 u = ffn_unpack<BF16>(us[i]), dh = mul2(v[e], ffn_both(factor));
        v[e] = mul2(mul2(dh, u), slope[e]);
        w[e] = mul2(dh, a[e]);
        a[e] = mul2(a[e], u);
      }
    }
  }
  if (KIND != kFfnPlain) {
    ffn_round<BF16, N>(v, one);
    ffn_round<BF16, N>(w, two);
  }
  ffn_round<BF16, N>(a, result);
}

// Tile t: its problem, the row of tiles, its first half and how many of them.  kFfnGroup rows of tiles at a time, along the columns.
struct FfnSpot { int problem, i, j, halves; };
template <int CG>
__device__ __forceinline__ FfnSpot ffn_spot(const FfnParams& p, int t) {
  constexpr int kHalves = FfnTiling<CG>::kHalves;
  FfnSpot s;
  const int whole = t < p.wholes ? t : p.wholes + (t - p.wholes) / kHalves;
  s.problem = 0;
  while (s.problem + 1 < p.problems && whole >= p.problem[s.problem + 1].first) ++s.problem;
  const FfnProblem& q = p.problem[s.problem];
  const int columns = (q.tiles_n + kHalves - 1) / kHalves;
  const int at = whole - q.first, group = at / (kFfnGroup * columns), in = at - group * kFfnGroup * columns;
  const int rows = min(kFfnGroup, q.tiles_m - group * kFfnGroup);
  const int j = in / rows;
  s.i = group * kFfnGroup + in - j * rows;
  s.j = j * kHalves;
  s.halves = min(kHalves, q.tiles_n - s.j);
  if (t >= p.wholes) {
    const int half = (t - p.wholes) % kHalves;
    s.j += half;
    s.halves = half < s.halves ? 1 : 0;          // the second half of a tile that has one: nothing
  }
  return s;
}

template <int KIND, bool BF16, int CG, bool STARVE = false>
__global__ void __launch_bounds__(kFfnThreads, CG == 2 ? 1 : 2) ffn_kernel(const __grid_constant__ FfnParams p) {
  extern __shared__ unsigned char smem_dyn[];
  if (KIND == kFfnBack && !BF16 && p.again) {    // the same in all blocks
    pdl_launch_dependents();
    pdl_wait();
    if (p.peaks[kFfnPeaks] == 0u) return;
  }
  using T = FfnTiling<CG>;
  constexpr int kTM = 128 * CG, kTN = 128 * CG, kCols = KIND == kFfnUp ? kTN / 2 : kTN;      // of half a tile; kCols: columns of the result
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  const int stages = CG == 2 ? kFfnPairStages : p.stages;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + stages * T::kStage);
  uint64_t* empty = full + stages;
  uint64_t* acc_full = empty + stages;       // [2] half by half
  uint64_t* acc_free = acc_full + 2;             // [2]
  uint64_t* drain = acc_free + 2;
  __shared__ uint32_t s_tmem;
  __shared__ int s_issued;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int shares = CG == 2 ? 1 : p.shares;
  const int rank = CG == 2 || shares > 1 ? static_cast<int>(cluster_rank()) : 0;
  const int side_of_pair = CG == 2 ? rank : 0;
  const int worker = CG == 2 ? blockIdx.x / 2 : blockIdx.x / shares, workers = CG == 2 ? gridDim.x / 2 : p.tiles;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_free[s], kFfnEndWarps * CG); }
    mbar_init(drain, 1);
    s_abort = 0;
    s_issued = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == kFfnEndWarps + 1) tmem_alloc<CG>(&s_tmem, T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_launch_dependents();

  // K steps of a tile that are this block's
  auto steps_of = [&](const FfnProblem& q, int& begin, int& end) {
    const int all = q.steps * q.segments;
    begin = CG == 2 ? 0 : static_cast<int>(static_cast<long long>(all) * rank / shares);
    end = CG == 2 ? all : static_cast<int>(static_cast<long long>(all) * (rank + 1) / shares);
  };

  if (warp == kFfnEndWarps) {
    // The whole warp goes through the loop, so that maps and coordinates are uniform values; one lane issues.  With the loop inside one lane's branch a
    // copy took 220 cycles to issue, 890 a stage of four.
    const bool issuer = elect_one();
    int stage = 0, issued = 0, ahead = 0;
    uint32_t parity = 1;                         // the stages start out empty
    bool ok = true;
    auto copy = [&](unsigned char* dst, const CUtensorMap* map, int x, int y, int at) {
      if (CG == 2) tma_load_2d_pair(dst, map, &full[at], x, y);
      else tma_load_2d(dst, map, &full[at], x, y);
    };
    // Stages `from` to `to` of a tile, both operands, or as much as `left` and `right` say; `wait`: for each to be empty.
    auto stages_of = [&](const FfnSpot& s, const FfnProblem& q, int from, int to, bool left, int right_from, bool wait) {
      for (int segment = 0; segment < q.segments && ok; ++segment) {
        const CUtensorMap* a_map = &p.maps[q.a[segment]];
        const CUtensorMap* b_map[2] = {&p.maps[KIND == kFfnUp ? q.b[CG == 2 ? side_of_pair : 0] : q.b[segment]], &p.maps[KIND == kFfnUp ? q.b[CG == 2 ? side_of_pair : 1] : q.b[segment]]};
        const int first = max(from, segment * q.steps), last = min(to, (segment + 1) * q.steps);
        const int a_row = s.i * kTM + side_of_pair * 128;
        const int b_row = s.j * kCols + (KIND == kFfnUp ? 0 : side_of_pair * 128), b_box = KIND == kFfnUp && CG == 1 ? 0 : 64;       // to the operand's second box
        const int halves = s.halves, a_across = q.a_across, b_across = q.b_across;
        for (int k = first; k < last; ++k) {
          if (wait) {
            const bool got = !s_abort && mbar_wait_bounded(&empty[stage], parity);
            if (!__all_sync(0xffffffffu, got)) { s_abort = 1; ok = false; break; }
          }
          if (issuer) {
            const int k0 = (k - segment * q.steps) * kFfnTK;
            unsigned char* at = smem + stage * T::kStage;
            if (k >= right_from) {
              if (side_of_pair == 0) mbar_expect_tx(&full[stage], CG * (1 + halves) * kFfnOperand);      // a pair's bytes all count on the even block's barrier
#pragma unroll
              for (int n = 0; n < T::kHalves; ++n) {
                if (n >= halves) break;
                const int r = b_row + n * kCols;
                copy(at + (1 + n) * kFfnOperand, b_map[0], b_across ? r : k0, b_across ? k0 : r, stage);
                copy(at + (1 + n) * kFfnOperand + 8192, b_map[1], b_across ? r + b_box : k0, b_across ? k0 : r + b_box, stage);
              }
            }
            if (left) {
              copy(at, a_map, a_across ? a_row : k0, a_across ? k0 : a_row, stage);
              copy(at + 8192, a_map, a_across ? a_row + 64 : k0, a_across ? k0 : a_row + 64, stage);
            }
          }
          __syncwarp();
          if (left) ++issued;
          if (++stage == stages) { stage = 0; parity ^= 1u; }
        }
      }
    };
    // What does not come from the kernel before is on its way while that one ends.
    if (worker < p.tiles && !STARVE) {
      const FfnSpot s = ffn_spot<CG>(p, worker);
      const FfnProblem& q = p.problem[s.problem];
      int begin, end;
      steps_of(q, begin, end);
      if (q.early && s.halves > 0) {
        ahead = min(stages, end - begin);
        stages_of(s, q, begin, begin + ahead, false, 0, false);
        stage = 0;
        parity = 1;
      }
    }
    pdl_wait();
    for (int t = worker; ok && t < p.tiles; t += workers) {
      const FfnSpot s = ffn_spot<CG>(p, t);
      if (s.halves == 0) continue;
      const FfnProblem& q = p.problem[s.problem];
      int begin, end;
      steps_of(q, begin, end);
      stages_of(s, q, begin, STARVE ? end - 1 : end, true, t == worker ? begin + ahead : begin, true);
    }
    if (lane == 0) s_issued = max(issued, ahead);
  } else if (warp == kFfnEndWarps + 1) {
    if (side_of_pair == 0) {
      // The whole warp goes through the loop, so that addresses and descriptors are uniform values; one lane issues.
      const bool issuer = elect_one();
      const uint32_t base = (smem_addr(smem) & 0x3ffffu) >> 4;             // descriptors count 16-byte units; above are a cluster block's number and their other fields
      int stage = 0;
      uint32_t parity = 0, free_parity = 3u;     // of accumulator a: bit a
      int turn = 0;                              // the accumulator of the next half by itself: they take turns
      bool ok = true;
      for (int t = worker; ok && t < p.tiles; t += workers) {
        const FfnSpot s = ffn_spot<CG>(p, t);
        if (s.halves == 0) continue;
        const FfnProblem& q = p.problem[s.problem];
        int begin, end;
        steps_of(q, begin, end);
        const int steps = end - begin, acc0 = s.halves == 1 ? turn : 0;
        if (CG == 2 && s.halves == 1) turn ^= 1;
        const uint32_t idesc = mma_idesc(kTM, kTN, BF16, false, false) | (q.a_across ? 1u << 15 : 0u) | (q.b_across ? 1u << 16 : 0u);
        const uint64_t a_base = q.a_across ? desc_mnmajor(0, 8192) : desc_kmajor(0), b_base = q.b_across ? desc_mnmajor(0, 8192) : desc_kmajor(0);
        const uint32_t a_step = q.a_across ? 2048 / 16 : 32 / 16, b_step = q.b_across ? 2048 / 16 : 32 / 16;
        auto get = [&](uint64_t* bar, uint32_t phase) {
          const bool got = !s_abort && mbar_wait_bounded(bar, phase);
          if (!__all_sync(0xffffffffu, got)) { s_abort = 1; ok = false; }
          return ok;
        };
        auto products = [&](int at, int half, bool first) {
          const uint64_t a = a_base + (base + at * (T::kStage >> 4)), b = b_base + (base + at * (T::kStage >> 4) + (1 + half) * (kFfnOperand >> 4));
          if (issuer) {
#pragma unroll
            for (int kk = 0; kk < kFfnTK / 16; ++kk) mma_ss<CG>(tmem + (acc0 + half) * kTN, a + kk * a_step, b + kk * b_step, idesc, kk != 0 || !first ? 1u : 0u);
          }
          __syncwarp();
        };
        auto commit = [&](uint64_t* bar) {
          if (issuer) mma_commit<CG>(bar);
          __syncwarp();
        };
        // `count` stages from the present one on, half after half; `opens`: the tile's first, `closes`: its last
        auto by_halves = [&](int count, bool opens, bool closes) {
          for (int half = 0; half < s.halves; ++half) {
            if (opens) {
              if (!get(&acc_free[acc0 + half], (free_parity >> (acc0 + half)) & 1u)) return;
              free_parity ^= 1u << (acc0 + half);
            }
            int at = stage;
            uint32_t phase = parity;
            for (int k = 0; k < count; ++k) {
              if (half == 0 && !get(&full[at], phase)) return;
              tc_fence_after();
              products(at, half, opens && k == 0);
              if (half == s.halves - 1) commit(&empty[at]);
              if (++at == stages) { at = 0; phase ^= 1u; }
            }
            if (closes) commit(&acc_full[acc0 + half]);
            if (half == s.halves - 1) { stage = at; parity = phase; }
          }
        };
        const int first = min(steps, stages), last = min(steps - first, stages);
        by_halves(first, true, last == 0);
        for (int k = first; ok && k < steps - last; ++k) {
          if (!get(&full[stage], parity)) break;
          tc_fence_after();
          for (int half = 0; half < s.halves; ++half) products(stage, half, false);
          commit(&empty[stage]);
          if (++stage == stages) { stage = 0; parity ^= 1u; }
        }
        if (ok && last > 0) by_halves(last, false, true);
      }
      if (s_abort && issuer) { mma_commit<CG>(drain); mbar_wait_bounded(drain, 0); }
      __syncwarp();
    }
  } else {
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    constexpr int kShare = kCols / (kFfnEndWarps / 4);       // columns of a warp
    const int side = warp >> 2;                  // which of them
    uint32_t parity = 0u;                        // of accumulator a: bit a
    int turn = 0;
    // a lone block's products have all read their stages by the time anything is put there
    FfnWay way = {smem + (CG == 2 ? stages * T::kStage + 512 : 0u) + warp * 2 * kFfnPatch, 0};
    pdl_wait();
    int exponent = 0;
    if (p.peaks != nullptr) exponent = ffn_exponent(p.peaks, KIND == kFfnPlain || p.again);
    bool ok = true;
    for (int t = worker; ok && t < p.tiles; t += workers) {
      const FfnSpot s = ffn_spot<CG>(p, t);
      const FfnProblem& q = p.problem[s.problem];
      const int row0 = s.i * kTM + side_of_pair * 128 + (warp & 3) * 32, row = row0 + lane;
      const float factor = KIND == kFfnBack ? ffn_power(exponent) : q.scaled ? ffn_power(-exponent) : 1.f;
      const bool there = row < q.m;
      const int acc0 = s.halves == 1 ? turn : 0;
      if (CG == 2 && s.halves == 1) turn ^= 1;
#pragma unroll 1
      for (int half = 0; half < s.halves; ++half) {
        const int col0 = (s.j + half) * kCols + side * kShare;
        uint4 gate[4], up[4];
        if (KIND == kFfnBack && shares == 1) {   // under way while the products are
          ffn_get<32>(gate, p.gate, row, col0, q.n, there);
          ffn_get<32>(up, p.up, row, col0, q.n, there);
        }
        const bool got = !s_abort && mbar_wait_bounded(&acc_full[acc0 + half], (parity >> (acc0 + half)) & 1u);
        if (!__all_sync(0xffffffffu, got)) { s_abort = 1; ok = false; break; }
        parity ^= 1u << (acc0 + half);
        tc_fence_after();
        const uint32_t acc = tmem + (acc0 + half) * kTN + side * kShare + lanes;
        if (shares == 1) {
#pragma unroll 1
          for (int c = 0; c < kShare && row0 < q.m; c += 32) {
            const int col = col0 + c;
            if (col >= q.n) break;
            uint32_t raw[32], raw_up[32];
            tmem_ld32(acc + c, raw);
            if (KIND == kFfnUp) tmem_ld32(acc + kCols + c, raw_up);
            uint4 one[4], two[4], result[4], next_gate[4], next_up[4];
            if (KIND == kFfnBack && c + 32 < kShare) {
              ffn_get<32>(next_gate, p.gate, row, col + 32, q.n, there);
              ffn_get<32>(next_up, p.up, row, col + 32, q.n, there);
            }
            tmem_wait_ld();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float2 v[8], w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                v[e] = make_float2(__uint_as_float(raw[16 * h + 2 * e]), __uint_as_float(raw[16 * h + 2 * e + 1]));
                if (KIND == kFfnUp) w[e] = make_float2(__uint_as_float(raw_up[16 * h + 2 * e]), __uint_as_float(raw_up[16 * h + 2 * e + 1]));
              }
              ffn_end<KIND, BF16, 16>(p.act, factor, v, w, gate + 2 * h, up + 2 * h, one + 2 * h, two + 2 * h, result + 2 * h);
              if (KIND == kFfnBack && !BF16 && p.beyond != nullptr) ffn_note(v, w, p.beyond);
            }
            if (KIND == kFfnBack || (KIND == kFfnUp && p.gate.data != nullptr)) {
              way.put(one, &p.outs[0], row0, col);
              way.put(two, &p.outs[1], row0, col);
            }
            way.put(result, &p.outs[KIND == kFfnPlain ? s.problem : 2], row0, col);
            if (KIND == kFfnBack) {
#pragma unroll
              for (int k = 0; k < 4; ++k) { gate[k] = next_gate[k]; up[k] = next_up[k]; }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) { if (CG == 2) mbar_arrive_leader(&acc_free[acc0 + half]); else mbar_arrive_one(&acc_free[acc0 + half]); }
          __syncwarp();
        } else {                                 // this block's sums, where the stages were: all products that read those are complete
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
      }
    }
    if (lane == 0) bulk_wait<0>();
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (CG == 1 && shares > 1) {
    cluster_sync_all();                          // every block's sums are in place
    const FfnSpot s = ffn_spot<CG>(p, worker);
    const FfnProblem& q = p.problem[s.problem];
    if (warp < 8 && !s_abort) {
      const int exponent = p.peaks == nullptr ? 0 : ffn_exponent(p.peaks, KIND == kFfnPlain || p.again);
      const float factor = KIND == kFfnBack ? ffn_power(exponent) : q.scaled ? ffn_power(-exponent) : 1.f;
      // The blocks take the rows in turn.  First the sums, neighbouring lanes at neighbouring 16 bytes of the other blocks' memory and all blocks' under way at once, into this
      // block's own place for them, which nobody else reads (8 columns a lane straight into the ending took 9,000 to 12,000 cycles for 16 rows).
      float* mine = reinterpret_cast<float*>(smem);
      for (int unit = threadIdx.x; unit < 128 / shares * 32; unit += 32 * kFfnEndWarps) {
        const int r = unit / 32 * shares + rank;
        if (s.i * kTM + r >= q.m) continue;
        float* at = mine + r * kFfnSumRow + unit % 32 * 4;
        float4 f[8];
#pragma unroll
        for (int b = 0; b < 8; ++b) f[b] = b < shares ? ld_cluster_f32x4(at, b) : make_float4(0.f, 0.f, 0.f, 0.f);
        float2 lo = make_float2(f[0].x, f[0].y), hi = make_float2(f[0].z, f[0].w);
#pragma unroll
        for (int b = 1; b < 8; ++b) {
          lo = add2(lo, make_float2(f[b].x, f[b].y));
          hi = add2(hi, make_float2(f[b].z, f[b].w));
        }
        *reinterpret_cast<float4*>(at) = make_float4(lo.x, lo.y, hi.x, hi.y);
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kFfnEndWarps) : "memory");
      constexpr int kEights = kCols / 8;
      for (int unit = threadIdx.x; unit < 128 / shares * kEights; unit += 32 * kFfnEndWarps) {
        const int r = unit / kEights * shares + rank, c = unit % kEights * 8;
        const int row = s.i * kTM + r, col = s.j * kCols + c;
        if (row >= q.m || col >= q.n) continue;
        uint4 gate, up, one, two, result;
        if (KIND == kFfnBack) {
          gate = *ffn_at(p.gate, row, col);
          up = *ffn_at(p.up, row, col);
        }
        float2 v[4], w[4];
        const float* at = mine + r * kFfnSumRow + c;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = *reinterpret_cast<const float2*>(at + 2 * e);
          w[e] = KIND == kFfnUp ? *reinterpret_cast<const float2*>(at + kCols + 2 * e) : make_float2(0.f, 0.f);
        }
        ffn_end<KIND, BF16, 8>(p.act, factor, v, w, &gate, &up, &one, &two, &result);
        if (KIND == kFfnBack && !BF16 && p.beyond != nullptr) ffn_note(v, w, p.beyond);
        if (KIND == kFfnBack || (KIND == kFfnUp && p.gate.data != nullptr)) {
          *ffn_at(KIND == kFfnUp ? p.gate : p.dgate, row, col) = one;
          *ffn_at(KIND == kFfnUp ? p.up : p.dup, row, col) = two;
        }
        *ffn_at(q.out, row, col) = result;
      }
    }
    cluster_sync_all();                          // nobody leaves while its sums are read
  }
  if (CG == 2) cluster_sync_all();               // the pair's copies and arrivals are all in, unless a wait expired
  if (s_abort && threadIdx.x == 0) {             // no copy may land after the block has gone
    for (int s = 0; side_of_pair == 0 && s < stages && s < s_issued; ++s) {
      const int uses = (s_issued - 1 - s) / stages;          // the stage's last copy is its use number `uses`
      mbar_wait_bounded(&full[s], uses & 1);
    }
    atomicOr(p.flags, kFlagTimeout);
  }
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  if (warp == kFfnEndWarps + 1) {
    tc_fence_after();
    tmem_dealloc<CG>(tmem, T::kTmemCols);
  }
}

// ----------------------------------------------------------------------------------------------
// A few tokens (up to 32): the weights are what has to be read, 2 bytes for one or two products each, and what counts is how soon all of them are asked
// for.  A block takes eight rows of the weights (Up: of both projections), its warps divide K among them, up to 128 at a time in turn, and add up
// their sums through shared memory in order.  A lane's 16 bytes of a weight row and of a token's row are the same eight K; which of a product's sixteen
// places a K takes is the same on both sides, so they go into the warp's products as they were loaded, without a
// turn through shared memory.  What the kernel before does not make, the first weights, is asked for while that one ends.
// 1024 x 4096: one token 10.1 us, 16 11.8, 32 16.1 where tiles of 128 tokens take 19.5; 2048 x 8192, 101 MB of weights: 16 31.2, 32 42.1, tiles 42.6.  Weights that do not
// stay in L2 (4096 x 10944, 269 MB): one 63.4 (4.2 TB/s), eight 73.1, tiles 68.5.  Blocks that go on from tile to tile with the next tile's weights under way were slower
// (12.4 us, 15.1 and 77.0): a block's join then holds up its own next products, where now another block's go on.
// ----------------------------------------------------------------------------------------------
constexpr int kFfnFew = 32, kFfnFewLong = 4, kFfnFewWarps = 16;
constexpr long long kFfnL2 = 126ll << 20;
struct FfnFewParams {
  FfnRows x, w[2], out, gate, up;                // w: rows of weights; Plain: one
  int tokens, n, k, act;
};

template <bool BF16>
__device__ __forceinline__ void ffn_mma(float (&c)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3, const uint32_t b0, const uint32_t b1) {
  if (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// MT: sixteens of tokens
template <int KIND, bool BF16, int MT>
__global__ void __launch_bounds__(32 * kFfnFewWarps) ffn_few_kernel(const FfnFewParams p) {
  constexpr int kW = KIND == kFfnUp ? 2 : 1;
  constexpr int kDeep = MT == 1 ? 4 : 2;         // of a warp's K under way at once, and as many again of the weights
  extern __shared__ float s_sums[];              // [warp][kW][16 MT][8]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int row = lane >> 2, at = (lane & 3) * 8, col = blockIdx.x * 8 + row;
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  pdl_launch_dependents();
  float acc[kW][MT][4];
#pragma unroll
  for (int w = 0; w < kW; ++w)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[w][m][e] = 0.f;
  uint4 weights[kDeep][kW];
  auto ask = [&](int k0) {
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int k = k0 + d * 32 + at;
#pragma unroll
      for (int w = 0; w < kW; ++w) weights[d][w] = k < p.k && col < p.n ? ld_stream_v4(ffn_at(p.w[w], col, k)) : none;
    }
  };
  int k0 = warp * kDeep * 32;
  ask(k0);
  pdl_wait();
  for (; k0 < p.k; k0 += kDeep * warps * 32) {
    uint4 x[kDeep][MT][2], now[kDeep][kW];
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int k = k0 + d * 32 + at;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int token = m * 16 + h * 8 + row;
          x[d][m][h] = k < p.k && token < p.tokens ? *ffn_at(p.x, token, k) : none;
        }
#pragma unroll
      for (int w = 0; w < kW; ++w) now[d][w] = weights[d][w];
    }
    ask(k0 + kDeep * warps * 32);
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int w = 0; w < kW; ++w) {
          ffn_mma<BF16>(acc[w][m], x[d][m][0].x, x[d][m][1].x, x[d][m][0].y, x[d][m][1].y, now[d][w].x, now[d][w].y);
          ffn_mma<BF16>(acc[w][m], x[d][m][0].z, x[d][m][1].z, x[d][m][0].w, x[d][m][1].w, now[d][w].z, now[d][w].w);
        }
  }
  auto place = [&](int of_warp, int w, int token, int c) { return s_sums + ((of_warp * kW + w) * MT * 16 + token) * 8 + c; };
#pragma unroll
  for (int w = 0; w < kW; ++w)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) *reinterpret_cast<float2*>(place(warp, w, m * 16 + h * 8 + row, (lane & 3) * 2)) = make_float2(acc[w][m][2 * h], acc[w][m][2 * h + 1]);
  __syncthreads();
  for (int o = threadIdx.x; o < MT * 16 * 4; o += blockDim.x) {
    const int token = o >> 2, c = (o & 3) * 2, to = blockIdx.x * 8 + c;
    if (token >= p.tokens || to >= p.n) continue;
    float2 sum[kW][1];
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      sum[w][0] = make_float2(0.f, 0.f);
      for (int v = 0; v < warps; ++v) sum[w][0] = add2(sum[w][0], *reinterpret_cast<const float2*>(place(v, w, token, c)));
    }
    auto put = [&](const FfnRows& r, float2 v) { *reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(r.data) + (token * r.row + to) * 2) = ffn_pack<BF16>(v.x, v.y); };
    if constexpr (KIND == kFfnUp) {
      if (p.gate.data != nullptr) {
        put(p.gate, sum[0][0]);
        put(p.up, sum[kW - 1][0]);
      }
      float2 a[1];
      ffn_act_all<false>(p.act, sum[0], a, a);
      put(p.out, mul2(a[0], sum[kW - 1][0]));
    } else {
      put(p.out, sum[0][0]);
    }
  }
}

// fp16: the largest finite |element| of dy, as the bits of its fp32 value, one for each block; the word behind them is cleared.
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
    if (blockIdx.x == 0) peaks[kFfnPeaks] = 0u;
    for (int w = 1; w < 8; ++w) top = max(top, s_top[w]);
    peaks[blockIdx.x] = __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(top))));
  }
}

}  // namespace adacons
