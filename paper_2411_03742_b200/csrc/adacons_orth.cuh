// Newton-Schulz orthogonalisation of the matrices of a flat update vector: kernels (sm_100a).
#pragma once

#include <cuda_fp16.h>

#include "adacons_tc.cuh"

namespace adacons {

// ----------------------------------------------------------------------------------------------
// For every matrix G (m x n) of the vector, with r = min(m, n), l = max(m, n) and X = G or G^T so
// that X is r x l:
//     X <- X / (|X|_F + eps)
//     steps times:   S = X X^T     B = b S + c S S     X <- a X + B X
//     out = scale * X (transposed back)
// The polynomial a s + b s^3 + c s^5 acts on the singular values and drives them toward one.
//
// Number format.  The products run on the tensor cores from fp16 operands.  An iterate is kept as a
// pair hi + lo of fp16 values of 2^11 X (22 bits, range 2^-25 .. 2^16 after the power-of-two scale),
// S and B as 2^13 S and 2^11 B.  In a bf16 context the products take the hi parts only, and the term
// a X takes the pair; in an fp32 context S and B are pairs too and each product is the sum
// lo hi + hi lo + hi hi, smallest terms first, in one fp32 accumulator.
// Why not bf16 operands: rounding the iterates to 8 bits costs 1e-2 of the result's norm on a
// Gaussian matrix and 1e-1 on one with a few strong directions (the small singular values grow
// 3.4-fold per step and the rounding noise of the strong ones grows with them); 11 bits with the
// a X term exact stay below 1.8e-3, the size of one bf16 rounding of the result.
// The diagonal: near orthogonality B is close to (b + c) I, and rounding that diagonal is the largest
// single error.  From the fourth step on B + t I is stored with t = -3/4 (b + c) and a - t takes the
// place of a, an identity in exact arithmetic; it brings the error from 1.7e-3 to 1.1e-3 on Gaussian
// matrices (on a matrix of rank 8 plus noise 5e-4 instead of 1.5e-4, still a third of the rounding).
// ----------------------------------------------------------------------------------------------
constexpr int kOrthTM = 128;             // rows of an output tile
constexpr int kOrthTK = 64;              // K elements per stage: one 128-byte swizzled row
constexpr float kOrthXScale = 2048.f, kOrthSScale = 8192.f, kOrthBScale = 2048.f;
constexpr int kOrthThreads = 192;        // warps 0-3 epilogue, 4 TMA, 5 MMA
constexpr int kOrthNormChunk = 16384;    // elements per block of the norm kernel
constexpr int kOrthLoadTile = 64;

enum OrthKind { kOrthGram = 0, kOrthPoly = 1, kOrthApply = 2 };
enum OrthMap { kMapX0 = 0, kMapX1 = 2, kMapS = 4, kMapB = 6, kMapCount = 8 };   // + 1: the lo part

struct OrthMat {
  int r, l;                // X is r x l, r <= l
  int transposed;          // the matrix in the vector has l rows of r elements
  int ldx, lds;            // row pitch of X and of S, B (elements)
  int vec_out;             // output rows start on 8- (bf16) or 16-byte (fp32) boundaries relative to the vector's start
  int norm_first, norm_count;
  float scale;
  long long offset;        // of the matrix in the vector
  __half* x[2][2];         // [buffer][hi, lo]
  __half* s[2];
  __half* b[2];
};
struct OrthTile { int mat, i, j, pad; };
struct OrthChunk { int mat; int first; };      // norm kernel: chunk number within the matrix

struct OrthParams {
  const OrthMat* mats;
  const CUtensorMap* maps;       // [matrix][kMapCount]
  const OrthTile* tiles;
  int num_tiles;
  int src;                       // buffer of X that is read
  float a, b, c, t;              // t: what is added to B's diagonal
  void* out;                     // last step: the flat result
  int last, out_bf16, out_aligned;
  uint32_t* flags;
};

// ----------------------------------------------------------------------------------------------
// |G|_F^2 by chunks: fp64 throughout, so that no magnitude of the input over- or underflows; the
// blocks' sums are added in a fixed order by whoever needs the norm.
// ----------------------------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ float orth_in(const void* p, long long i) {
  return DT == 0 ? static_cast<const float*>(p)[i] : __uint_as_float(static_cast<uint32_t>(static_cast<const unsigned short*>(p)[i]) << 16);
}

template <int DT>
__global__ void __launch_bounds__(256) orth_norm_kernel(const void* in, const OrthMat* mats, const OrthChunk* chunks, double* partial) {
  __shared__ double s_sum[8];
  const OrthChunk ch = chunks[blockIdx.x];
  const long long size = static_cast<long long>(mats[ch.mat].r) * mats[ch.mat].l;
  const long long begin = static_cast<long long>(ch.first) * kOrthNormChunk;
  const long long end = begin + kOrthNormChunk < size ? begin + kOrthNormChunk : size;
  const long long base = mats[ch.mat].offset;
  double sum = 0.0;
#pragma unroll 8
  for (long long i = begin + threadIdx.x; i < end; i += 256) {
    const double v = orth_in<DT>(in, base + i);
    sum = fma(v, v, sum);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double v = 0.0;
    for (int w = 0; w < 8; ++w) v += s_sum[w];
    partial[blockIdx.x] = v;
  }
}

__device__ __forceinline__ void orth_split(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}

// X_0 = G / (|G|_F + eps) as pairs, transposed where the matrix is taller than wide.
template <int DT>
__global__ void __launch_bounds__(256) orth_load_kernel(const void* in, const OrthMat* mats, const OrthTile* tiles, const double* partial, double eps) {
  __shared__ float s_tile[kOrthLoadTile][kOrthLoadTile + 1];
  __shared__ double s_sum[8];
  pdl_launch_dependents();
  pdl_wait();
  const OrthTile t = tiles[blockIdx.x];
  const OrthMat& m = mats[t.mat];
  const int tid = threadIdx.x;
  double sum = 0.0;
  for (int k = tid; k < m.norm_count; k += 256) sum += partial[m.norm_first + k];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((tid & 31) == 0) s_sum[tid >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < 8; ++w) sum += s_sum[w];
  const float mul = static_cast<float>(static_cast<double>(kOrthXScale) / (sqrt(sum) + eps));
  // one tile of the matrix as it lies in the vector: `rows` x `cols`, row-major
  const int rows = m.transposed ? m.l : m.r, cols = m.transposed ? m.r : m.l;
  const int r0 = (m.transposed ? t.j : t.i) * kOrthLoadTile, c0 = (m.transposed ? t.i : t.j) * kOrthLoadTile;
  const int tx = tid & 63, ty = tid >> 6;
#pragma unroll 4
  for (int y = ty; y < kOrthLoadTile; y += 4) {
    const int row = r0 + y, col = c0 + tx;
    s_tile[y][tx] = row < rows && col < cols ? orth_in<DT>(in, m.offset + static_cast<long long>(row) * cols + col) * mul : 0.f;
  }
  __syncthreads();
  const int pair = tid & 31;
#pragma unroll 4
  for (int y = tid >> 5; y < kOrthLoadTile; y += 8) {
    const int row = t.i * kOrthLoadTile + y, col = t.j * kOrthLoadTile + 2 * pair;
    if (row >= m.r || col >= m.ldx) continue;           // the pitch is even: a pair never straddles it
    const float v0 = m.transposed ? s_tile[2 * pair][y] : s_tile[y][2 * pair];
    const float v1 = m.transposed ? s_tile[2 * pair + 1][y] : s_tile[y][2 * pair + 1];
    __half h0, l0, h1, l1;
    orth_split(v0, h0, l0);
    orth_split(v1, h1, l1);
    const long long at = static_cast<long long>(row) * m.ldx + col;
    *reinterpret_cast<__half2*>(m.x[0][0] + at) = __halves2half2(h0, h1);
    *reinterpret_cast<__half2*>(m.x[0][1] + at) = __halves2half2(l0, l1);
  }
}

// ----------------------------------------------------------------------------------------------
// The three products of a step, all matrices of the vector in one persistent launch.
// Output tiles of 128 x TN; one warp copies operand stages (128 + TN rows of 64 K elements) by TMA,
// one thread issues the tcgen05 products into one of two TMEM accumulators, four warps drain the
// other.  S and S S are symmetric: only tiles that reach the lower triangle are computed, and each
// writes its mirror image where no tile does.
//   Gram   S = X X^T        both operands K-major, straight from X's rows
//   Poly   B = b S + c S S + t I
//   Apply  X' = (a - t) X + B X    the right operand is X again, MN-major: no transposed copy exists
// The epilogue turns each 32 x 32 block of the accumulator in shared memory so that global reads and
// writes run along rows; mirror images and transposed results are written from the accumulator's own
// orientation, where the lanes of a warp are neighbours.
// ----------------------------------------------------------------------------------------------
template <int TN> struct OrthSmem {
  static constexpr uint32_t kA = kOrthTM * kOrthTK * 2, kB = TN * kOrthTK * 2, kStage = kA + kB;
  static constexpr int kStages = TN == 256 ? 4 : 6;
  static constexpr uint32_t kTurn = kStages * kStage;                // 4 warps x 32 x 32 fp32
  static constexpr uint32_t kBars = kTurn + 4 * 4096;
  static constexpr uint32_t kBytes = kBars + 256;
};

template <int KIND, bool SPLIT, int TN>
__device__ __forceinline__ void orth_epilogue_tile(const OrthParams& p, const OrthTile t, uint32_t tmem, float* turn, uint64_t* drained) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const OrthMat& m = p.mats[t.mat];
  const int r = m.r, ncols = KIND == kOrthApply ? m.l : m.r, ld = KIND == kOrthApply ? m.ldx : m.lds;
  const int row0 = t.i * kOrthTM + warp * 32;
  const int q = lane & 7, sub = lane >> 3;
  const __half* add_hi = KIND == kOrthApply ? m.x[p.src][0] : m.s[0];
  const __half* add_lo = KIND == kOrthApply ? m.x[p.src][1] : m.s[1];
  __half* dst_hi = KIND == kOrthGram ? m.s[0] : KIND == kOrthPoly ? m.b[0] : m.x[p.src ^ 1][0];
  __half* dst_lo = KIND == kOrthGram ? m.s[1] : KIND == kOrthPoly ? m.b[1] : m.x[p.src ^ 1][1];
  const bool last = KIND == kOrthApply && p.last;
  constexpr bool kAddLo = KIND == kOrthApply || SPLIT;      // X is always a pair, S only in an fp32 context
  constexpr bool kStoreLo = KIND == kOrthApply || SPLIT;
#pragma unroll 1
  for (int ch = 0; ch < TN / 32; ++ch) {
    const int col0 = t.j * TN + ch * 32;
    const bool live = col0 < ncols && row0 < r;
    uint2 ah[8], al[8];
    if (KIND != kOrthGram && live) {
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int row = row0 + it * 4 + sub, col = col0 + q * 4;
        ah[it] = al[it] = make_uint2(0u, 0u);
        if (row < r && col < ld) {
          const long long at = static_cast<long long>(row) * ld + col;
          ah[it] = *reinterpret_cast<const uint2*>(add_hi + at);
          if (kAddLo) al[it] = *reinterpret_cast<const uint2*>(add_lo + at);
        }
      }
    }
    uint32_t acc[32];
    tmem_ld32(tmem + ch * 32 + (static_cast<uint32_t>(warp * 32) << 16), acc);
    tmem_wait_ld();
    if (ch == TN / 32 - 1) {                     // the accumulator is free for the tile after next
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_one(drained);
    }
    if (!live) continue;
#pragma unroll
    for (int g = 0; g < 8; ++g)
      *reinterpret_cast<uint4*>(turn + lane * 32 + ((g ^ (lane & 7)) * 4)) = make_uint4(acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
    __syncwarp();
    // a tile above the diagonal that is not computed gets its mirror image from here
    const bool mirror = KIND != kOrthApply && !((col0 / kOrthTM) * kOrthTM + kOrthTM - 1 >= (row0 / TN) * TN);
    const bool keep = mirror || (last && m.transposed);
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int lrow = it * 4 + sub, row = row0 + lrow, col = col0 + q * 4;
      float* cell = turn + lrow * 32 + ((q ^ (lrow & 7)) * 4);
      const float4 v4 = *reinterpret_cast<const float4*>(cell);
      float v[4] = {v4.x, v4.y, v4.z, v4.w};
      float add[4] = {0.f, 0.f, 0.f, 0.f};
      if (KIND != kOrthGram) {
        const float2 h0 = __half22float2(*reinterpret_cast<const __half2*>(&ah[it].x)), h1 = __half22float2(*reinterpret_cast<const __half2*>(&ah[it].y));
        add[0] = h0.x; add[1] = h0.y; add[2] = h1.x; add[3] = h1.y;
        if (kAddLo) {
          const float2 l0 = __half22float2(*reinterpret_cast<const __half2*>(&al[it].x)), l1 = __half22float2(*reinterpret_cast<const __half2*>(&al[it].y));
          add[0] += l0.x; add[1] += l0.y; add[2] += l1.x; add[3] += l1.y;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (KIND == kOrthGram) v[e] *= kOrthSScale / (kOrthXScale * kOrthXScale);
        if (KIND == kOrthPoly) {
          v[e] = (p.c * (kOrthBScale / (kOrthSScale * kOrthSScale))) * v[e] + (p.b * (kOrthBScale / kOrthSScale)) * add[e];
          if (row == col + e) v[e] += p.t * kOrthBScale;
        }
        if (KIND == kOrthApply) v[e] = (p.a - p.t) * add[e] + v[e] * (1.f / kOrthBScale);
        if (last) v[e] *= m.scale / kOrthXScale;
      }
      if (keep) *reinterpret_cast<float4*>(cell) = make_float4(v[0], v[1], v[2], v[3]);
      if (row >= r || col >= ncols) continue;
      if (!last) {
        const long long at = static_cast<long long>(row) * ld + col;
        __half h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) orth_split(v[e], h[e], l[e]);
        *reinterpret_cast<uint2*>(dst_hi + at) = *reinterpret_cast<const uint2*>(h);
        if (kStoreLo) *reinterpret_cast<uint2*>(dst_lo + at) = *reinterpret_cast<const uint2*>(l);
      } else if (!m.transposed) {
        const long long at = m.offset + static_cast<long long>(row) * m.l + col;
        if (m.vec_out && p.out_aligned && col + 3 < ncols) {
          if (p.out_bf16) *reinterpret_cast<uint2*>(static_cast<unsigned short*>(p.out) + at) = make_uint2(pack_bf16x2_rn(v[0], v[1]), pack_bf16x2_rn(v[2], v[3]));
          else *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < ncols) {
              if (p.out_bf16) static_cast<unsigned short*>(p.out)[at + e] = static_cast<unsigned short>(pack_bf16x2_rn(v[e], 0.f) & 0xffffu);
              else static_cast<float*>(p.out)[at + e] = v[e];
            }
        }
      }
    }
    if (keep) {
      __syncwarp();
      const int row = row0 + lane;
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        const float4 v4 = *reinterpret_cast<const float4*>(turn + lane * 32 + ((g ^ (lane & 7)) * 4));
        const float v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = col0 + 4 * g + e;
          if (row >= r || col >= ncols) continue;
          if (KIND != kOrthApply) {
            const long long at = static_cast<long long>(col) * ld + row;
            __half h, l;
            orth_split(v[e], h, l);
            dst_hi[at] = h;
            if (kStoreLo) dst_lo[at] = l;
          } else {
            const long long at = m.offset + static_cast<long long>(col) * m.r + row;
            if (p.out_bf16) static_cast<unsigned short*>(p.out)[at] = static_cast<unsigned short>(pack_bf16x2_rn(v[e], 0.f) & 0xffffu);
            else static_cast<float*>(p.out)[at] = v[e];
          }
        }
      }
    }
    __syncwarp();
  }
}

template <int KIND, bool SPLIT, int TN>
__global__ void __launch_bounds__(kOrthThreads, 1) orth_product_kernel(const OrthParams p) {
  extern __shared__ unsigned char smem_dyn[];
  using L = OrthSmem<TN>;
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  float* turn = reinterpret_cast<float*>(smem + L::kTurn);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* empty = full + L::kStages;
  uint64_t* acc_full = empty + L::kStages;       // [2]
  uint64_t* acc_free = acc_full + 2;             // [2]
  uint64_t* drain = acc_free + 2;
  __shared__ uint32_t s_tmem;
  __shared__ int s_issued;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_free[s], 4); }
    mbar_init(drain, 1);
    s_abort = 0;
    s_issued = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == 5) tmem_alloc(&s_tmem, 2 * TN);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_launch_dependents();
  pdl_wait();

  constexpr int kPasses = SPLIT ? 3 : 1;         // lo hi, hi lo, hi hi
  if (warp == 4) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t parity = 1;                       // the stages start out empty
      bool ok = true;
      for (int k = blockIdx.x; ok && k < p.num_tiles; k += gridDim.x) {
        const OrthTile t = p.tiles[k];
        const CUtensorMap* maps = p.maps + static_cast<long long>(t.mat) * kMapCount;
        const int K = KIND == kOrthGram ? p.mats[t.mat].l : p.mats[t.mat].r;
        const int a_map = KIND == kOrthGram ? kMapX0 + 2 * p.src : KIND == kOrthPoly ? kMapS : kMapB;
        const int b_map = KIND == kOrthPoly ? kMapS : kMapX0 + 2 * p.src;
        for (int pass = 0; ok && pass < kPasses; ++pass) {
          const CUtensorMap* ma = maps + a_map + (SPLIT && pass == 0 ? 1 : 0);
          const CUtensorMap* mb = maps + b_map + (SPLIT && pass == 1 ? 1 : 0);
          for (int k0 = 0; k0 < K; k0 += kOrthTK) {
            if (s_abort || !mbar_wait_bounded(&empty[stage], parity)) { s_abort = 1; ok = false; break; }
            unsigned char* sa = smem + stage * L::kStage;
            unsigned char* sb = sa + L::kA;
            mbar_expect_tx(&full[stage], L::kStage);
#pragma unroll
            for (int h = 0; h < kOrthTM / 64; ++h) tma_load_2d(sa + h * 8192, ma, &full[stage], k0, t.i * kOrthTM + h * 64);
#pragma unroll
            for (int h = 0; h < TN / 64; ++h) {
              if (KIND == kOrthApply) tma_load_2d(sb + h * 8192, mb, &full[stage], t.j * TN + h * 64, k0);
              else tma_load_2d(sb + h * 8192, mb, &full[stage], k0, t.j * TN + h * 64);
            }
            ++issued;
            if (++stage == L::kStages) { stage = 0; parity ^= 1u; }
          }
        }
      }
      s_issued = issued;
    }
  } else if (warp == 5) {
    if (lane == 0) {
      constexpr uint32_t idesc = mma_idesc(kOrthTM, TN, false, false, KIND == kOrthApply);
      int stage = 0, buf = 0;
      uint32_t parity = 0, acc_parity = 1;
      bool ok = true;
      for (int k = blockIdx.x; ok && k < p.num_tiles; k += gridDim.x) {
        const OrthTile t = p.tiles[k];
        const int K = KIND == kOrthGram ? p.mats[t.mat].l : p.mats[t.mat].r;
        const int steps = kPasses * ((K + kOrthTK - 1) / kOrthTK);
        if (s_abort || !mbar_wait_bounded(&acc_free[buf], acc_parity)) { s_abort = 1; break; }
        tc_fence_after();
        const uint32_t d = tmem + buf * TN;
        for (int s = 0; s < steps; ++s) {
          if (s_abort || !mbar_wait_bounded(&full[stage], parity)) { s_abort = 1; ok = false; break; }
          tc_fence_after();
          const uint32_t sa = smem_addr(smem + stage * L::kStage), sb = sa + L::kA;
#pragma unroll
          for (int kk = 0; kk < kOrthTK / 16; ++kk)
            mma_ss(d, desc_kmajor(sa + kk * 32), KIND == kOrthApply ? desc_mnmajor(sb + kk * 2048, 8192) : desc_kmajor(sb + kk * 32), idesc,
                   (s | kk) != 0);
          mma_commit(&empty[stage]);
          if (++stage == L::kStages) { stage = 0; parity ^= 1u; }
        }
        if (ok) mma_commit(&acc_full[buf]);
        buf ^= 1;
        if (buf == 0) acc_parity ^= 1u;
      }
      if (s_abort) { mma_commit(drain); mbar_wait_bounded(drain, 0); }
    }
  } else {
    int buf = 0;
    uint32_t parity = 0;
    for (int k = blockIdx.x; k < p.num_tiles; k += gridDim.x) {
      const bool got = !s_abort && mbar_wait_bounded(&acc_full[buf], parity);
      if (!__all_sync(0xffffffffu, got)) { s_abort = 1; break; }
      tc_fence_after();
      orth_epilogue_tile<KIND, SPLIT, TN>(p, p.tiles[k], tmem + buf * TN, turn + warp * 1024, &acc_free[buf]);
      buf ^= 1;
      if (buf == 0) parity ^= 1u;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (s_abort && threadIdx.x == 0) {             // no copy may land after the block has gone
    for (int s = 0; s < L::kStages && s < s_issued; ++s) {
      const int uses = (s_issued - 1 - s) / L::kStages;          // the stage's last copy is its use number `uses`
      mbar_wait_bounded(&full[s], uses & 1);
    }
    atomicOr(p.flags, kFlagTimeout);
  }
  __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    tmem_dealloc(tmem, 2 * TN);
  }
}

}  // namespace adacons
