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
// S and B as 2^13 S and 2^11 B.  In a bf16 context the products take the hi parts only, and B is stored as
// B + a I, so that X <- (B + a I) X_hi + a X_lo: the epilogue reads the lo part alone, and in the last step, whose
// errors no further step enlarges, nothing.  (With a X added from the pair the steps moved an eighth more bytes, and
// bytes between L2 and the SMs are what bounds them: twelve encoder layers 3.76 -> 3.60 ms.)  In an fp32 context S and B are pairs too
// and each product is the sum (lo hi + hi lo) + hi hi.  The tensor cores round a running sum toward zero, low by up to 4e-8 of it
// per chained product: harmless beside an 11-bit operand, but 4e-5 of an fp32 result after five steps
// on sides of 1024.  There the hi hi terms are chained over 64 K elements at most and the chunks'
// sums added by the epilogue, round to nearest (the small terms, 2^-11 of the sum, in one accumulator).
// Why not bf16 operands: rounding the iterates to 8 bits costs 1e-2 of the result's norm on a
// Gaussian matrix and 1e-1 on one with a few strong directions (the small singular values grow
// 3.4-fold per step and the rounding noise of the strong ones grows with them); 11 bits with the
// a X term from the pair stay below 1.5e-3 before the result's own rounding, 1.7e-3 (Gaussian, rank 8 plus noise,
// singular values over four decades).
// The diagonal in an fp32 context, and where a matrix stays in one block: near orthogonality B is close to (b + c) I, and rounding that diagonal is the
// largest single error.  From the fourth step on B + t I is stored with t = -3/4 (b + c) and a - t takes the
// place of a, an identity in exact arithmetic.
// ----------------------------------------------------------------------------------------------
constexpr int kOrthTK = 64;              // K elements per stage: one 128-byte swizzled row
constexpr int kOrthChunk = 1;            // fp32 contexts: stages (64 K elements) per hi hi accumulator
constexpr float kOrthXScale = 2048.f, kOrthSScale = 8192.f, kOrthBScale = 2048.f;
constexpr int kOrthThreads = 352;        // warps 0-7 epilogue, 8 operand copies, 9 products, 10 epilogue copies
constexpr int kOrthNormChunk = 16384;    // elements per block of the norm kernel
constexpr int kOrthLoadTile = 64, kOrthLoadCols = 256;

enum OrthKind { kOrthGram = 0, kOrthPoly = 1, kOrthApply = 2, kOrthPart = 3 };     // part: of a Gram product split over K
enum OrthMap { kMapX0 = 0, kMapX1 = 2, kMapS = 4, kMapB = 6, kMapCount = 8 };   // + 1: the lo part

struct OrthMat {
  int r, l;                // X is r x l, r <= l
  int transposed;          // the matrix in the vector has l rows of r elements
  int ldx, lds;            // row pitch of X and of S, B (elements)
  int vec_out;             // rows of the result are whole groups of 8 elements, aligned relative to the vector's start
  int vec_in;              // the matrix starts on, and is a multiple of, 8 elements
  int norm_first, norm_count;
  float scale;
  long long offset;        // of the matrix in the vector
  __half* x[2][2];         // [buffer][hi, lo]
  __half* s[2];
  __half* b[2];
};
struct OrthSpot { int mat, i, j; };           // load kernel: a tile of a matrix
// One tile of one product, with all that the warps other than the epilogue's need to know of its matrix.
struct __align__(16) OrthTile {
  int mat, i, j, depth;    // depth: K elements, from `first` on
  int rows, cols;          // of the product: r x l or r x r
  unsigned needs;          // tiles of the matrix that the blocks must have stored before
  int step_kind;           // step * 4 + OrthKind
  int first, adds;         // adds: partial sums that other tiles have of this one
  int slot;                // where those are, one after the other, or where this part goes
  unsigned ready;          // tiles that must have been stored before what the epilogue adds is there
};
struct OrthStep { float a, b, c, t; };         // t: what is added to B's diagonal
struct OrthChunk { int mat; int first; };      // norm kernel: chunk number within the matrix

struct OrthParams {
  const OrthMat* mats;
  const CUtensorMap* maps;       // [matrix][kMapCount]
  const OrthTile* tiles;         // each worker's after the other's
  const int* begin;              // [workers + 1]
  const OrthStep* coeffs;        // [steps]
  unsigned* done;                // [matrix] blocks' tiles stored so far
  unsigned char* sums;           // partial sums: [slot][block of a pair][strip], each strip as it lies in shared memory
  int mirrored;                  // symmetric products are computed on and below the diagonal only
  int steps;
  void* out;                     // the flat result
  int out_aligned;
  uint32_t* flags;
};

// ----------------------------------------------------------------------------------------------
// |G|_F^2 by chunks: fp64 throughout, so that no magnitude of the input over- or underflows; the
// blocks' sums are added in a fixed order by whoever needs the norm.  What it multiplies by, 2^11 / (|G|_F + eps), can lie
// outside fp32 where G does not (norms below 6e-36): then it goes in two steps, the first an exact power of two.
// ----------------------------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ float orth_in(const void* p, long long i) {
  return DT == 0 ? static_cast<const float*>(p)[i] : __uint_as_float(static_cast<uint32_t>(static_cast<const unsigned short*>(p)[i]) << 16);
}

// eight consecutive elements from a 16-byte boundary (fp32: 32 bytes of it)
template <int DT>
__device__ __forceinline__ void orth_in8(const void* p, long long i, float (&v)[8]) {
  if (DT == 0) {
    const uint4 a = ld_stream_v4(static_cast<const float*>(p) + i), b = ld_stream_v4(static_cast<const float*>(p) + i + 4);
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
  } else {
    const uint4 a = ld_stream_v4(static_cast<const unsigned short*>(p) + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = unpack_pair<1>(a, k);
      v[2 * k] = f.x;
      v[2 * k + 1] = f.y;
    }
  }
}

struct OrthFactor {
  float first, then;                               // first: 1 unless the factor is outside 2^-100 .. 2^100
  __device__ __forceinline__ OrthFactor(double square, double eps) {
    const double norm = sqrt(square) + eps;
    double by = static_cast<double>(kOrthXScale) / (norm > 0.0 ? fmax(norm, 0x1p-189) : norm);     // the smallest fp32 number is 2^-149: below it is eps, of a matrix of zeros
    first = 1.f;
    if (by > 0x1p100 && by < INFINITY) { first = 0x1p100f; by *= 0x1p-100; }
    else if (by < 0x1p-100 && by > 0.0) { first = 0x1p-100f; by *= 0x1p100; }
    then = static_cast<float>(by);
  }
};

template <int DT>
__global__ void __launch_bounds__(256) orth_norm_kernel(const void* in, int aligned, const OrthMat* mats, const OrthChunk* chunks, double* partial) {
  __shared__ double s_sum[8];
  const OrthChunk ch = chunks[blockIdx.x];
  const OrthMat& m = mats[ch.mat];
  const long long size = static_cast<long long>(m.r) * m.l;
  const long long begin = static_cast<long long>(ch.first) * kOrthNormChunk;
  const long long end = begin + kOrthNormChunk < size ? begin + kOrthNormChunk : size;
  const long long base = m.offset;
  double sum = 0.0;
  if (aligned && m.vec_in) {                       // the matrix is whole groups of eight
#pragma unroll 4
    for (long long i = begin + 8 * threadIdx.x; i < end; i += 8 * 256) {
      float v[8];
      orth_in8<DT>(in, base + i, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), sum);
    }
  } else {
#pragma unroll 8
    for (long long i = begin + threadIdx.x; i < end; i += 256) {
      const double v = orth_in<DT>(in, base + i);
      sum = fma(v, v, sum);
    }
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

// X_0 = G / (|G|_F + eps) as pairs, transposed where the matrix is taller than wide.  A block makes 64 rows x
// 256 columns of X, 64 x 64 at a time.
template <int DT>
__global__ void __launch_bounds__(256) orth_load_kernel(const void* in, int aligned, const OrthMat* mats, const OrthSpot* tiles, const double* partial, double eps, unsigned* done, int counters) {
  __shared__ float s_tile[kOrthLoadTile][kOrthLoadTile + 1];
  __shared__ double s_sum[8];
  pdl_launch_dependents();
  pdl_wait();
  const OrthSpot t = tiles[blockIdx.x];
  const OrthMat& m = mats[t.mat];
  const int tid = threadIdx.x;
  if (blockIdx.x == 0)
    for (int k = tid; k < counters; k += 256) done[k] = 0u;
  double sum = 0.0;
  for (int k = tid; k < m.norm_count; k += 256) sum += partial[m.norm_first + k];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((tid & 31) == 0) s_sum[tid >> 5] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < 8; ++w) sum += s_sum[w];
  const OrthFactor by(sum, eps);
  const int rows = m.transposed ? m.l : m.r, cols = m.transposed ? m.r : m.l;      // as it lies in the vector, row-major
  const bool vec = aligned && m.vec_in && cols % 8 == 0;
  const int r = m.r, ldx = m.ldx, transposed = m.transposed;
  const long long offset = m.offset;
  __half *hi = m.x[0][0], *lo = m.x[0][1];
  const int row_base = t.i * kOrthLoadTile;
  if (vec && !transposed) {                        // straight through: 8 columns a thread, 8 threads a row of 64, 32 rows at a time
#pragma unroll 4
    for (int n = 0; n < 8; ++n) {
      const int row = row_base + (n & 1) * 32 + (tid >> 3), col = t.j * kOrthLoadCols + (n >> 1) * kOrthLoadTile + (tid & 7) * 8;
      if (row >= r || col >= cols) continue;
      float v[8];
      orth_in8<DT>(in, offset + static_cast<long long>(row) * cols + col, v);
      __half h[8], l[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) orth_split(v[e] * by.first * by.then, h[e], l[e]);
      const long long at = static_cast<long long>(row) * ldx + col;
      *reinterpret_cast<uint4*>(hi + at) = *reinterpret_cast<const uint4*>(h);
      *reinterpret_cast<uint4*>(lo + at) = *reinterpret_cast<const uint4*>(l);
    }
    return;
  }
  for (int n = 0; n < kOrthLoadCols / kOrthLoadTile; ++n) {
    const int col_base = t.j * kOrthLoadCols + n * kOrthLoadTile;
    if (col_base >= ldx) return;
    const int r0 = transposed ? col_base : row_base, c0 = transposed ? row_base : col_base;
    if (vec) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int y = q * 32 + (tid >> 3), x = (tid & 7) * 8;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r0 + y < rows && c0 + x < cols) orth_in8<DT>(in, offset + static_cast<long long>(r0 + y) * cols + c0 + x, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s_tile[y][x + e] = v[e] * by.first * by.then;
      }
    } else {
      const int tx = tid & 63, ty = tid >> 6;
#pragma unroll 8
      for (int y = ty; y < kOrthLoadTile; y += 4) {
        const int row = r0 + y, col = c0 + tx;
        s_tile[y][tx] = row < rows && col < cols ? orth_in<DT>(in, offset + static_cast<long long>(row) * cols + col) * by.first * by.then : 0.f;
      }
    }
    __syncthreads();
    const int pair = tid & 31;
#pragma unroll 4
    for (int y = tid >> 5; y < kOrthLoadTile; y += 8) {
      const int row = row_base + y, col = col_base + 2 * pair;
      if (row >= r || col >= ldx) continue;             // the pitch is even: a pair never straddles it
      const float v0 = transposed ? s_tile[2 * pair][y] : s_tile[y][2 * pair];
      const float v1 = transposed ? s_tile[2 * pair + 1][y] : s_tile[y][2 * pair + 1];
      __half h0, l0, h1, l1;
      orth_split(v0, h0, l0);
      orth_split(v1, h1, l1);
      const long long at = static_cast<long long>(row) * ldx + col;
      *reinterpret_cast<__half2*>(hi + at) = __halves2half2(h0, h1);
      *reinterpret_cast<__half2*>(lo + at) = __halves2half2(l0, l1);
    }
    __syncthreads();
  }
}

// ----------------------------------------------------------------------------------------------
// All steps of all matrices in one persistent launch, one block per SM.
//
// Every block (or pair) goes through its own list of tiles, which the host has laid out by simulating the
// steps with measured costs: whoever is free takes the tile whose matrix has the longest way to go.  A
// matrix's next product starts when all tiles of its last one are stored, which a counter per matrix says;
// while one is completed elsewhere the others keep the block busy.  A tile never waits for one that comes
// later in the simulated time, so the lists cannot lock.  One launch per product instead (three a step) left the
// device idle at every boundary, half of the time of one encoder layer.
// The blocks wait for one another, so the launch is cooperative; each wait is bounded.
//
//   Gram   S = X X^T        both operands K-major, straight from X's rows; on long rows of few tiles split over K: other
//                           blocks bring the partial sums, in fp32, which the tile's epilogue adds in the parts' order
//                           (64 x 4096 fp32 283 -> 135 us, eight of 16 x 4096 bf16 156 -> 115 us)
//   Poly   B = b S + c S S + t I
//   Apply  X' = (a - t) X + B X    the right operand is X again, MN-major: no transposed copy exists
// S and S S are symmetric: where there is work for all, only tiles that reach the lower triangle are computed,
// and each writes its mirror image where no tile does.
//
// Tiles.  CG = 2: a pair of blocks (two SMs) shares a tile of 256 x TN; each holds 128 rows of the left
// operand, half of the right one and 128 rows of the result, so that an operand byte from L2 feeds
// twice the products of a single block's tile.  CG = 1: 128 x 128, for problems with too few tiles to occupy the device, and
// for fp32 contexts, whose three products a stage need no more of the operands than arrives (pairs were no faster there);
// or 128 x 64, where blocks would idle all the same: what bounds such a matrix is its chain of products, three quarters of
// the operands to wait for and one strip instead of two (256 x 512 bf16 91 -> 78 us, fp32 136 -> 110 us).
// In each block one warp copies operand stages by TMA, one thread (of the even block) issues the
// tcgen05 products into one of two TMEM accumulators, and eight warps drain the other.
//
// The epilogue works on strips of 128 rows x 64 columns in shared memory: a further warp brings what is
// added (X, S) by TMA two or three strips ahead, the eight warps put the result in its place, and the
// strip leaves by TMA, which also clips the matrix's edges.  With plain loads and stores of 8 bytes a
// lane instead, the epilogue of a 256 x 256 tile took 25,000 cycles where its products take 8,000 (K = 1024).
// Mirror images go the same way, turned in the half of the strip that single values leave free (from an fp32
// context's pairs, and for transposed results, straight to global memory from the accumulator's own orientation,
// where the lanes of a warp are neighbours).  Written to global memory two bytes a lane, they cost a phase 13,000 cycles.
// ----------------------------------------------------------------------------------------------
constexpr uint32_t kOrthStripPart = 128 * 128;   // 128 rows x 64 fp16 values: two boxes of 64 swizzled rows
template <bool SPLIT, int CG, int TN> struct OrthTiling {
  static_assert(!SPLIT || CG == 1, "fp32 contexts use lone blocks");
  static constexpr int kTM = 128 * CG, kTN = TN;
  static constexpr int kParts = SPLIT ? 2 : 1;
  static constexpr int kBRows = kTN / CG;                            // of the right operand, in each block
  static constexpr uint32_t kA = 128 * kOrthTK * 2, kB = kBRows * kOrthTK * 2;
  static constexpr uint32_t kStage = kParts * (kA + kB);             // A hi (lo), B hi (lo)
  static constexpr int kRing = SPLIT ? 2 : 3;                        // strips
  static constexpr int kStages = (224 * 1024 - kRing * 2 * kOrthStripPart) / kStage;
  static constexpr uint32_t kStrips = kStages * kStage;
  static constexpr uint32_t kBars = kStrips + kRing * 2 * kOrthStripPart;
  static constexpr uint32_t kBytes = kBars + 256 + 1024;             // + alignment of the base
  static constexpr int kBlocks = kTN / 64;                           // strips of a tile
  static constexpr uint32_t kTmemCols = (SPLIT ? 4 : 2) * kTN;       // big[2] (small[2])
};

// What of a tile exists: strips with columns inside the matrix, none for a block without rows.
template <bool SPLIT, int CG, int TN>
__device__ __forceinline__ int orth_live_strips(const OrthTile& t, int rank) {
  using T = OrthTiling<SPLIT, CG, TN>;
  if (t.i * T::kTM + rank * 128 >= t.rows) return 0;
  const int left = (t.cols - t.j * T::kTN + 63) / 64;
  return left < T::kBlocks ? left : T::kBlocks;
}

// Eight elements: v <- by_v v + by_x (hi + lo), two at a time.
__device__ __forceinline__ void orth_scale8(float2 (&v)[4], float by_v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], make_float2(by_v, by_v));
}
__device__ __forceinline__ void orth_add8(float2 (&v)[4], float by_x, const unsigned char* at) {
  const uint4 x = *reinterpret_cast<const uint4*>(at);
  const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = fma2(make_float2(by_x, by_x), __half22float2(*reinterpret_cast<const __half2*>(&u[k])), v[k]);
}
__device__ __forceinline__ void orth_diagonal8(float2 (&v)[4], int at, float t) {        // element `at` of the eight, if it is one
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k].x += at == 2 * k ? t : 0.f;
    v[k].y += at == 2 * k + 1 ? t : 0.f;
  }
}
// hi and (in h and l) the rest, each rounded to fp16
template <bool PAIR>
__device__ __forceinline__ void orth_round8(const float2 (&v)[4], uint4& h, uint4& l) {
  uint32_t a[4], b[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __half2 q = __float22half2_rn(v[k]);
    a[k] = *reinterpret_cast<const uint32_t*>(&q);
    if (PAIR) {
      const float2 f = __half22float2(q);
      const __half2 rest = __float22half2_rn(add2(v[k], make_float2(-f.x, -f.y)));
      b[k] = *reinterpret_cast<const uint32_t*>(&rest);
    }
  }
  h = make_uint4(a[0], a[1], a[2], a[3]);
  if (PAIR) l = make_uint4(b[0], b[1], b[2], b[3]);
}
// fp32 words as their upper and lower halves, in the two parts of a place
__device__ __forceinline__ void orth_halves8(const float2 (&v)[4], uint4& upper, uint4& lower) {
  uint32_t u[4], d[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    u[k] = __byte_perm(__float_as_uint(v[k].x), __float_as_uint(v[k].y), 0x7632);
    d[k] = __byte_perm(__float_as_uint(v[k].x), __float_as_uint(v[k].y), 0x5410);
  }
  upper = make_uint4(u[0], u[1], u[2], u[3]);
  lower = make_uint4(d[0], d[1], d[2], d[3]);
}
__device__ __forceinline__ uint4 orth_bf16x8(const float2 (&v)[4]) {
  return make_uint4(pack_bf16x2_rn(v[0].x, v[0].y), pack_bf16x2_rn(v[1].x, v[1].y), pack_bf16x2_rn(v[2].x, v[2].y), pack_bf16x2_rn(v[3].x, v[3].y));
}
__device__ __forceinline__ uint32_t orth_word(const uint4& v, int k) { return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w; }

// What the epilogue needs of a matrix, fetched once per tile and before its products are there: read where it
// is used, it comes from global memory again at every strip, 700 of the 1000 cycles of one.
struct OrthView {
  int r, cols, lds, l, transposed, vec;
  float scale;
  long long offset;
  unsigned short *hi, *lo;                         // where mirror images go
  __device__ __forceinline__ OrthView(const OrthParams& p, const OrthTile& t) {
    const OrthMat& m = p.mats[t.mat];
    const int kind = t.step_kind & 3;
    r = t.rows;
    cols = t.cols;
    l = m.l;
    lds = m.lds;
    transposed = m.transposed;
    vec = m.vec_out && p.out_aligned;
    scale = m.scale / kOrthXScale;
    offset = m.offset;
    hi = reinterpret_cast<unsigned short*>(kind == kOrthGram ? m.s[0] : m.b[0]);
    lo = reinterpret_cast<unsigned short*>(kind == kOrthGram ? m.s[1] : m.b[1]);
  }
};

// One 32 x 32 block of the product: row0 + lane is this thread's row; its 32 columns from col0 on are read from
// tensor memory at `acc`.  hi / lo: the block's place in the strip, `half` selecting its 64 bytes of each 128-byte row.
// A loop of 16 columns and not unrolled code for 32: every product of a small matrix runs this once, and
// fetching the longer code took 3000 to 6000 cycles of it.  (With 8 columns a turn large matrices lose a tenth to the waits.)
template <int KIND, bool SPLIT, int CG, int TN>
__device__ __forceinline__ void orth_finish_block(const OrthParams& p, const OrthStep& step, bool last_step, const OrthView& m, int row0, int col0, uint32_t acc,
                                                  unsigned char* hi, unsigned char* lo, int half) {
  using T = OrthTiling<SPLIT, CG, TN>;
  const int lane = threadIdx.x & 31;
  const int r = m.r, ncols = m.cols, row = row0 + lane;
  const bool last = KIND == kOrthApply && last_step;
  constexpr bool kPair = KIND == kOrthApply || SPLIT;      // X is always a pair, S and B only in an fp32 context
  // where no tile above the diagonal is computed, its image comes from here
  const bool mirror = KIND != kOrthApply && p.mirrored && row0 / T::kTM > col0 / T::kTN;
  const bool turned = last && m.transposed;
  unsigned char* hrow = hi + lane * 128;
  unsigned char* lrow = lo + lane * 128;
  const float by_x = KIND == kOrthPoly ? step.b * (kOrthBScale / kOrthSScale) : SPLIT ? step.a - step.t : step.a;
  const float by_v = KIND == kOrthGram ? kOrthSScale / (kOrthXScale * kOrthXScale) : KIND == kOrthPoly ? step.c * (kOrthBScale / (kOrthSScale * kOrthSScale)) : 1.f / kOrthBScale;
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
   uint32_t a[16];
   tmem_ld16(acc + turn * 16, a);
   tmem_wait_ld();
#pragma unroll
   for (int sub = 0; sub < 2; ++sub) {
    const int g = 2 * turn + sub;
    const int at = ((4 * half + g) ^ (lane & 7)) * 16;
    float2 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(a[8 * sub + 2 * k]), __uint_as_float(a[8 * sub + 2 * k + 1]));
    orth_scale8(v, by_v);
    if constexpr (KIND == kOrthPoly || SPLIT && KIND == kOrthApply) {
      orth_add8(v, by_x, hrow + at);
      if (SPLIT) orth_add8(v, by_x, lrow + at);
      if (KIND == kOrthPoly && row0 == col0) orth_diagonal8(v, lane - 8 * g, step.t * kOrthBScale);
    }
    if (!SPLIT && KIND == kOrthApply && !last) orth_add8(v, by_x, lrow + at);      // t = a: the hi part's share is in the product
    if (!last) {
      uint4 h, l;
      orth_round8<kPair>(v, h, l);
      *reinterpret_cast<uint4*>(hrow + at) = h;
      if (kPair) *reinterpret_cast<uint4*>(lrow + at) = l;
      if (!SPLIT && mirror) {                        // turned into the strip's free part: 64 rows, the strip's columns, of two boxes
        const int r64 = row & 63;
        unsigned char* turned_at = lo - static_cast<int>(row & 32) * 128 + (half * 32 + 8 * g) * 128 + (r64 & 7) * 2;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          *reinterpret_cast<unsigned short*>(turned_at + e * 128 + (((r64 >> 3) ^ e) * 16)) = static_cast<unsigned short>(orth_word(h, e / 2) >> (16 * (e & 1)));
      }
      if (SPLIT && mirror && row < r) {
        const int col = col0 + 8 * g;
        unsigned short* to_hi = m.hi + static_cast<long long>(col) * m.lds + row;
        unsigned short* to_lo = m.lo + static_cast<long long>(col) * m.lds + row;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (col + e < ncols) {
            to_hi[static_cast<long long>(e) * m.lds] = static_cast<unsigned short>(orth_word(h, e / 2) >> (16 * (e & 1)));
            to_lo[static_cast<long long>(e) * m.lds] = static_cast<unsigned short>(orth_word(l, e / 2) >> (16 * (e & 1)));
          }
        }
      }
      continue;
    }
    orth_scale8(v, m.scale);
    if (turned) {
      const int col = col0 + 8 * g;
      const long long to = m.offset + static_cast<long long>(col) * r + row;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = e & 1 ? v[e / 2].y : v[e / 2].x;
        if (row < r && col + e < ncols) {
          if (SPLIT) static_cast<float*>(p.out)[to + static_cast<long long>(e) * r] = f;
          else static_cast<unsigned short*>(p.out)[to + static_cast<long long>(e) * r] = static_cast<unsigned short>(pack_bf16x2_rn(f, 0.f) & 0xffffu);
        }
      }
    } else if (SPLIT) {                            // the strip's two parts hold the upper and the lower halves of the fp32 words
      uint4 u, d;
      orth_halves8(v, u, d);
      *reinterpret_cast<uint4*>(hrow + at) = u;
      *reinterpret_cast<uint4*>(lrow + at) = d;
    } else {
      *reinterpret_cast<uint4*>(hrow + at) = orth_bf16x8(v);
    }
   }
  }
  if (last && !turned) {                           // to the vector, along rows
    __syncwarp();
    if (m.vec) {                                     // 8 columns a lane, 8 rows at a time
      const int q = lane & 3;
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const int lr = it * 8 + (lane >> 2), col = col0 + 8 * q;
        const int at = lr * 128 + ((4 * half + q) ^ (lr & 7)) * 16;
        if (row0 + lr >= r || col >= ncols) continue;
        const long long to = m.offset + static_cast<long long>(row0 + lr) * m.l + col;
        const uint4 u = *reinterpret_cast<const uint4*>(hi + at);
        if (SPLIT) {
          const uint4 d = *reinterpret_cast<const uint4*>(lo + at);
          uint4* dst = reinterpret_cast<uint4*>(static_cast<float*>(p.out) + to);
          dst[0] = make_uint4(__byte_perm(d.x, u.x, 0x5410), __byte_perm(d.x, u.x, 0x7632), __byte_perm(d.y, u.y, 0x5410), __byte_perm(d.y, u.y, 0x7632));
          dst[1] = make_uint4(__byte_perm(d.z, u.z, 0x5410), __byte_perm(d.z, u.z, 0x7632), __byte_perm(d.w, u.w, 0x5410), __byte_perm(d.w, u.w, 0x7632));
        } else {
          *reinterpret_cast<uint4*>(static_cast<unsigned short*>(p.out) + to) = u;
        }
      }
    } else {                                       // one column a lane
      const int col = col0 + lane;
      for (int lr = 0; lr < 32 && row0 + lr < r; ++lr) {
        const int at = lr * 128 + ((4 * half + (lane >> 3)) ^ (lr & 7)) * 16 + (lane & 7) * 2;
        if (col >= ncols) continue;
        const long long to = m.offset + static_cast<long long>(row0 + lr) * m.l + col;
        const uint32_t u = *reinterpret_cast<const unsigned short*>(hi + at);
        if (SPLIT) static_cast<uint32_t*>(p.out)[to] = u << 16 | *reinterpret_cast<const unsigned short*>(lo + at);
        else static_cast<unsigned short*>(p.out)[to] = static_cast<unsigned short>(u);
      }
    }
  }
}

// Partial sums travel as strips of fp32 words, their upper and lower halves in the two parts of a place, so
// that each thread reads what its own place in the product is.
__device__ __forceinline__ void orth_part_out(uint32_t acc, unsigned char* hi, unsigned char* lo, int half) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int turn = 0; turn < 2; ++turn) {
    uint32_t a[16];
    tmem_ld16(acc + turn * 16, a);
    tmem_wait_ld();
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const int at = lane * 128 + ((4 * half + 2 * turn + sub) ^ (lane & 7)) * 16;
      float2 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = make_float2(__uint_as_float(a[8 * sub + 2 * k]), __uint_as_float(a[8 * sub + 2 * k + 1]));
      uint4 u, d;
      orth_halves8(v, u, d);
      *reinterpret_cast<uint4*>(hi + at) = u;
      *reinterpret_cast<uint4*>(lo + at) = d;
    }
  }
}
__device__ __forceinline__ void orth_part_in(uint32_t acc, const unsigned char* hi, const unsigned char* lo, int half) {
  const int lane = threadIdx.x & 31;
  uint32_t a[32];
  tmem_ld32(acc, a);
  tmem_wait_ld();
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int at = lane * 128 + ((4 * half + g) ^ (lane & 7)) * 16;
    const uint4 u = *reinterpret_cast<const uint4*>(hi + at), d = *reinterpret_cast<const uint4*>(lo + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 s = add2(make_float2(__uint_as_float(a[8 * g + 2 * k]), __uint_as_float(a[8 * g + 2 * k + 1])),
                            make_float2(__uint_as_float(__byte_perm(orth_word(d, k), orth_word(u, k), 0x5410)),
                                        __uint_as_float(__byte_perm(orth_word(d, k), orth_word(u, k), 0x7632))));
      a[8 * g + 2 * k] = __float_as_uint(s.x);
      a[8 * g + 2 * k + 1] = __float_as_uint(s.y);
    }
  }
  tmem_st32(acc, a);
  tmem_wait_st();
}

// The tiles of one block in the order in which all of its warps go through them.  The next tile's record
// is on its way while a tile is worked on.
struct OrthWalk {
  const OrthParams& p;
  int k, end;
  OrthTile t, next_t;
  __device__ __forceinline__ OrthWalk(const OrthParams& params, int worker) : p(params), k(p.begin[worker]), end(p.begin[worker + 1]) {
    if (k < end) t = p.tiles[k];
    if (k + 1 < end) next_t = p.tiles[k + 1];
  }
  __device__ __forceinline__ bool more() const { return k < end; }
  __device__ __forceinline__ void next() {
    ++k;
    t = next_t;
    if (k + 1 < end) next_t = p.tiles[k + 1];
  }
  __device__ __forceinline__ int kind() const { return t.step_kind & 3; }
  __device__ __forceinline__ int step() const { return t.step_kind >> 2; }
};

__device__ __forceinline__ unsigned orth_load_acquire(const unsigned* p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// Whether what a product reads is there; the copies that follow are ordered behind the look.
__device__ __forceinline__ bool orth_ready(const OrthWalk& w, unsigned tiles) {
  if (orth_load_acquire(w.p.done + w.t.mat) < tiles) return false;
  asm volatile("fence.proxy.async.global;" ::: "memory");
  return true;
}
__device__ __forceinline__ bool orth_wait_ready(const OrthWalk& w, unsigned tiles, volatile int* s_abort) {
  if (orth_ready(w, tiles)) return true;
  const unsigned long long t0 = global_timer_ns();
  while (!*s_abort) {
    if (orth_ready(w, tiles)) return true;
    __nanosleep(40);
    if (global_timer_ns() - t0 > kWaitLimitNs) return false;
  }
  return false;
}

template <bool SPLIT, int CG, int TN>
__global__ void __launch_bounds__(kOrthThreads, 1) orth_steps_kernel(const OrthParams p) {
  extern __shared__ unsigned char smem_dyn[];
  using T = OrthTiling<SPLIT, CG, TN>;
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + T::kBars);
  uint64_t* empty = full + T::kStages;
  uint64_t* acc_full = empty + T::kStages;       // [2]
  uint64_t* acc_free = acc_full + 2;             // [2]
  uint64_t* strip_full = acc_free + 2;           // [kRing] what is added has arrived (or, with nothing to add, the place is free)
  uint64_t* strip_done = strip_full + T::kRing;  // [kRing] the eight warps have put the result there
  uint64_t* drain = strip_done + T::kRing;
  __shared__ uint32_t s_tmem;
  __shared__ int s_issued, s_strips;
  __shared__ volatile int s_abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CG == 2 ? static_cast<int>(cluster_rank()) : 0;
  const int worker = blockIdx.x / CG;

  if (threadIdx.x == 0) {
    for (int s = 0; s < T::kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_free[s], 8 * CG); }
    for (int s = 0; s < T::kRing; ++s) { mbar_init(&strip_full[s], 1); mbar_init(&strip_done[s], 8); }
    mbar_init(drain, 1);
    s_abort = 0;
    s_issued = 0;
    s_strips = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == 9) tmem_alloc<CG>(&s_tmem, T::kTmemCols);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = s_tmem;

  if (warp == 8) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t parity = 1;                       // the stages start out empty
      bool ok = true;
      for (OrthWalk w(p, worker); ok && w.more(); w.next()) {
        const CUtensorMap* maps = p.maps + static_cast<long long>(w.t.mat) * kMapCount;
        const CUtensorMap* x_map = maps + kMapX0 + 2 * (w.step() & 1);
        const CUtensorMap* ma = w.kind() == kOrthPoly ? maps + kMapS : w.kind() == kOrthApply ? maps + kMapB : x_map;
        const CUtensorMap* mb = w.kind() == kOrthPoly ? maps + kMapS : x_map;
        const bool across = w.kind() == kOrthApply;                           // the right operand's K runs along its rows
        const int arow = w.t.i * T::kTM + rank * 128, brow = w.t.j * T::kTN + rank * T::kBRows;
        if (!orth_wait_ready(w, w.t.needs, &s_abort)) { s_abort = 1; break; }
        for (int k0 = w.t.first; k0 < w.t.first + w.t.depth; k0 += kOrthTK) {
          if (s_abort || !mbar_wait_bounded(&empty[stage], parity)) { s_abort = 1; ok = false; break; }
          unsigned char* at = smem + stage * T::kStage;
          if (rank == 0) mbar_expect_tx(&full[stage], CG * T::kStage);      // the pair's bytes all count on the even block's barrier
          auto load = [&](unsigned char* dst, const CUtensorMap* map, int x, int y) {
            if (CG == 2) tma_load_2d_pair(dst, map, &full[stage], x, y);
            else tma_load_2d(dst, map, &full[stage], x, y);
          };
#pragma unroll
          for (int part = 0; part < T::kParts; ++part) {
#pragma unroll
            for (int h = 0; h < 2; ++h) load(at + part * T::kA + h * 8192, ma + part, k0, arow + h * 64);
#pragma unroll
            for (int h = 0; h < T::kBRows / 64; ++h)
              load(at + T::kParts * T::kA + part * T::kB + h * 8192, mb + part, across ? brow + h * 64 : k0, across ? k0 : brow + h * 64);
          }
          ++issued;
          if (++stage == T::kStages) { stage = 0; parity ^= 1u; }
        }
      }
      s_issued = issued;
    }
  } else if (warp == 9) {
    if (rank == 0) {
      // The whole warp goes through the loop, so that addresses and descriptors are uniform values; one
      // lane issues.  With the loop itself inside one lane's branch, a product of 64 cycles took 150 to issue.
      const bool issuer = elect_one();
      const uint32_t base = smem_addr(smem) >> 4;                          // descriptors count 16-byte units
      int stage = 0, buf = 0, small = 0;
      uint32_t parity = 0, acc_parity = 1;
      bool ok = true;
      for (OrthWalk w(p, worker); ok && w.more(); w.next()) {
        const bool across = w.kind() == kOrthApply;
        const uint32_t idesc = across ? mma_idesc(T::kTM, T::kTN, false, false, true) : mma_idesc(T::kTM, T::kTN, false, false, false);
        const uint64_t b_base = across ? desc_mnmajor(0, 8192) : desc_kmajor(0);
        const uint32_t b_step = across ? 2048 / 16 : 32 / 16;
        const int steps = (w.t.depth + kOrthTK - 1) / kOrthTK;
        int in_acc = 0;
        for (int s = 0; s < steps; ++s) {
          if (in_acc == 0) {
            if (s_abort || !mbar_wait_bounded(&acc_free[buf], acc_parity)) ok = false;
          }
          ok = ok && !s_abort && mbar_wait_bounded(&full[stage], parity);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) { s_abort = 1; break; }
          tc_fence_after();
          const uint32_t big = tmem + buf * T::kTN, low = tmem + (2 + small) * T::kTN;
          const uint64_t a_hi = desc_kmajor(0) + (base + stage * (T::kStage >> 4)), a_lo = a_hi + (T::kA >> 4);
          const uint64_t b_hi = b_base + (base + stage * (T::kStage >> 4) + ((T::kParts * T::kA) >> 4)), b_lo = b_hi + (T::kB >> 4);
          if (issuer) {
#pragma unroll
            for (int kk = 0; kk < kOrthTK / 16; ++kk) {
              if (SPLIT) {
                mma_ss<CG>(low, a_lo + kk * 2, b_hi + kk * b_step, idesc, kk != 0 ? 1u : s != 0);
                mma_ss<CG>(low, a_hi + kk * 2, b_lo + kk * b_step, idesc, 1u);
              }
              mma_ss<CG>(big, a_hi + kk * 2, b_hi + kk * b_step, idesc, kk != 0 ? 1u : in_acc != 0);
            }
            mma_commit<CG>(&empty[stage]);
          }
          __syncwarp();
          if (++stage == T::kStages) { stage = 0; parity ^= 1u; }
          ++in_acc;
          if (s == steps - 1 || (SPLIT && in_acc == kOrthChunk)) {
            if (issuer) mma_commit<CG>(&acc_full[buf]);
            in_acc = 0;
            buf ^= 1;
            if (buf == 0) acc_parity ^= 1u;
          }
        }
        small ^= 1;
      }
      if (s_abort && issuer) { mma_commit<CG>(drain); mbar_wait_bounded(drain, 0); }
      __syncwarp();
    }
  } else if (warp == 10) {
    if (lane == 0) {
      // `ask` brings strips, at most kRing of them ahead of `give`, which sends them off.  A strip with partial sums to
      // add takes a turn for each of them before its own.
      struct Strips {
        OrthWalk w;
        int strip, live, turn = 0;
        __device__ __forceinline__ Strips(const OrthParams& p, int worker, int rank) : w(p, worker) { open(rank); }
        __device__ __forceinline__ void open(int rank) {                   // the next tile that has strips here
          for (; w.more(); w.next()) {
            live = orth_live_strips<SPLIT, CG, TN>(w.t, rank);
            strip = 0;
            if (live > 0) return;
          }
        }
        __device__ __forceinline__ void next(int rank) {
          if (turn++ < w.t.adds) return;
          turn = 0;
          if (++strip == live) { w.next(); open(rank); }
        }
        __device__ __forceinline__ bool adds() const { return turn < w.t.adds; }
        __device__ __forceinline__ unsigned char* sum(int slot, int rank) const {
          return w.p.sums + (static_cast<size_t>(slot * CG + rank) * T::kBlocks + strip) * (2 * kOrthStripPart);
        }
      };
      Strips ask(p, worker, rank), give(p, worker, rank);
      int loads = 0, stored = 0, b = 0;
      uint32_t parity = 0;
      while (give.w.more() && !s_abort) {
        const int ahead = loads - stored;
        if (ask.w.more() && ahead < T::kRing) {
          // the strip that was here has been sent: every strip is a group, and `pending` of them left after it
          const int to = loads % T::kRing, pending = T::kRing - 1 - ahead;
          if (pending == 0) bulk_wait_read<0>();
          else if (pending == 1) bulk_wait_read<1>();
          else bulk_wait_read<2>();
          unsigned char* at = smem + T::kStrips + to * 2 * kOrthStripPart;
          const bool apply = ask.w.kind() == kOrthApply;
          if (((ask.w.kind() == kOrthGram || ask.w.kind() == kOrthPart) && !ask.adds()) || (!SPLIT && apply && ask.w.step() == p.steps - 1)) {
            mbar_arrive_one(&strip_full[to]);
            ++loads;
            ask.next(rank);
            continue;
          }
          // nothing of this block may stay unsent while it waits for what others compute from it
          const bool there = ahead > 0 ? orth_ready(ask.w, ask.w.t.ready) : orth_wait_ready(ask.w, ask.w.t.ready, &s_abort);
          if (there && ask.adds()) {
            mbar_expect_tx(&strip_full[to], 2 * kOrthStripPart);
            bulk_load(at, ask.sum(ask.w.t.slot + ask.turn, rank), 2 * kOrthStripPart, &strip_full[to]);
            ++loads;
            ask.next(rank);
            continue;
          }
          if (there) {
            // in a bf16 context S, and the lo part of X; in an fp32 context both parts of either
            const int first = !SPLIT && apply ? 1 : 0, parts = SPLIT || apply ? 2 : 1;
            const CUtensorMap* map = p.maps + static_cast<long long>(ask.w.t.mat) * kMapCount + (apply ? kMapX0 + 2 * (ask.w.step() & 1) : kMapS);
            const int row = ask.w.t.i * T::kTM + rank * 128, col = ask.w.t.j * T::kTN + ask.strip * 64;
            mbar_expect_tx(&strip_full[to], (parts - first) * kOrthStripPart);
            for (int part = first; part < parts; ++part)
#pragma unroll
              for (int h = 0; h < 2; ++h) tma_load_2d(at + part * kOrthStripPart + h * 8192, map + part, &strip_full[to], col, row + h * 64);
            ++loads;
            ask.next(rank);
            continue;
          }
          if (ahead == 0) { s_abort = 1; break; }
        }
        if (!mbar_wait_bounded(&strip_done[b], parity)) { s_abort = 1; break; }
        const bool last = give.w.kind() == kOrthApply && give.w.step() == p.steps - 1;     // written to the result by the warps themselves
        if (!last && !give.adds()) {
          // in a bf16 context the last step does without X's lo part
          const int parts = SPLIT || (give.w.kind() == kOrthApply && give.w.step() < p.steps - 2) ? 2 : 1;
          const CUtensorMap* map = p.maps + static_cast<long long>(give.w.t.mat) * kMapCount +
                                   (give.w.kind() == kOrthGram ? kMapS : give.w.kind() == kOrthPoly ? kMapB : kMapX0 + 2 * ((give.w.step() & 1) ^ 1));
          const unsigned char* at = smem + T::kStrips + b * 2 * kOrthStripPart;
          const int row = give.w.t.i * T::kTM + rank * 128, col = give.w.t.j * T::kTN + give.strip * 64;
          if (give.w.kind() == kOrthPart) {
            bulk_store(give.sum(give.w.t.slot, rank), at, 2 * kOrthStripPart);
          } else {
            for (int part = 0; part < parts; ++part)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (row + h * 64 < give.w.t.rows) tma_store_2d(map + part, at + part * kOrthStripPart + h * 8192, col, row + h * 64);
          }
          if (!SPLIT && p.mirrored && (give.w.kind() == kOrthGram || give.w.kind() == kOrthPoly) && give.w.t.i > give.w.t.j) {      // the mirror image
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (row + h * 64 < give.w.t.rows) tma_store_2d(map, at + kOrthStripPart + h * 8192, row + h * 64, col);
          }
        }
        bulk_commit();
        if (!last && !give.adds() && give.strip == give.live - 1) {      // the tile is complete: say so once its bytes are
          bulk_wait<0>();
          asm volatile("fence.proxy.async.global;" ::: "memory");
          asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p.done + give.w.t.mat) : "memory");
        }
        ++stored;
        give.next(rank);
        if (++b == T::kRing) { b = 0; parity ^= 1u; }
      }
      bulk_wait<0>();
      s_strips = loads;
    }
  } else {
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const int half = warp >> 2;                            // this warp's 32 columns of each strip
    int buf = 0, small = 0, place = 0;
    uint32_t parity = 0, strip_parity = 0;
    auto wait_for = [&](uint64_t* bar, uint32_t phase) {
      const bool got = !s_abort && mbar_wait_bounded(bar, phase);
      if (!__all_sync(0xffffffffu, got)) { s_abort = 1; return false; }
      return true;
    };
    auto release = [&]() {                                 // this warp has read all it needs of the accumulator
      tc_fence_before();
      __syncwarp();
      if (lane == 0) { if (CG == 2) mbar_arrive_leader(&acc_free[buf]); else mbar_arrive_one(&acc_free[buf]); }
      __syncwarp();                                        // an fp32 context writes tensor memory next, as a whole warp
      buf ^= 1;
      if (buf == 0) parity ^= 1u;
    };
    auto used = [&]() {                                    // this warp is through with a place
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive_one(&strip_done[place]);
      if (++place == T::kRing) { place = 0; strip_parity ^= 1u; }
    };
    auto finish = [&](const OrthWalk& w, const OrthStep& step, const OrthView& m, int strip, uint32_t acc) {
      if (!wait_for(&strip_full[place], strip_parity)) return false;
      unsigned char* at = smem + T::kStrips + place * 2 * kOrthStripPart + (warp & 3) * 32 * 128;
      const int row0 = w.t.i * T::kTM + rank * 128 + (warp & 3) * 32, col0 = w.t.j * T::kTN + strip * 64 + half * 32;
      const bool last = w.step() == p.steps - 1;
      if (w.kind() == kOrthPart) orth_part_out(acc, at, at + kOrthStripPart, half);
      else if (w.kind() == kOrthGram) orth_finish_block<kOrthGram, SPLIT, CG, TN>(p, step, last, m, row0, col0, acc, at, at + kOrthStripPart, half);
      else if (w.kind() == kOrthPoly) orth_finish_block<kOrthPoly, SPLIT, CG, TN>(p, step, last, m, row0, col0, acc, at, at + kOrthStripPart, half);
      else orth_finish_block<kOrthApply, SPLIT, CG, TN>(p, step, last, m, row0, col0, acc, at, at + kOrthStripPart, half);
      used();
      return true;
    };
    auto finish_tile = [&](const OrthWalk& w, const OrthStep& step, const OrthView& m, int live, uint32_t base) {
#pragma unroll 1
      for (int s = 0; s < live; ++s) {
#pragma unroll 1
        for (int n = 0; n < w.t.adds; ++n) {               // in the parts' order, whoever is first
          if (!wait_for(&strip_full[place], strip_parity)) return false;
          const unsigned char* at = smem + T::kStrips + place * 2 * kOrthStripPart + (warp & 3) * 32 * 128;
          orth_part_in(base + s * 64, at, at + kOrthStripPart, half);
          used();
        }
        if (!finish(w, step, m, s, base + s * 64)) return false;
      }
      return true;
    };
    bool ok = true;
    for (OrthWalk w(p, worker); ok && w.more(); w.next()) {
      const OrthView m(p, w.t);
      const OrthStep step = p.coeffs[w.step()];
      const int live = orth_live_strips<SPLIT, CG, TN>(w.t, rank);
      if (!SPLIT) {
        if (!wait_for(&acc_full[buf], parity)) break;
        tc_fence_after();
        const uint32_t base = tmem + buf * T::kTN + half * 32 + lanes;
        ok = finish_tile(w, step, m, live, base);
        release();
      } else {
        const int chunks = ((w.t.depth + kOrthTK - 1) / kOrthTK + kOrthChunk - 1) / kOrthChunk;
        float2 sum[T::kBlocks][16];
#pragma unroll
        for (int s = 0; s < T::kBlocks; ++s)
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[s][e] = make_float2(0.f, 0.f);
        auto drain_into_sum = [&](uint32_t from) {
#pragma unroll
          for (int s = 0; s < T::kBlocks; ++s) {
            uint32_t acc[32];
            tmem_ld32(from + s * 64, acc);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[s][e] = add2(sum[s][e], make_float2(__uint_as_float(acc[2 * e]), __uint_as_float(acc[2 * e + 1])));
          }
        };
        for (int q = 0; q < chunks; ++q) {
          if (!wait_for(&acc_full[buf], parity)) { ok = false; break; }
          tc_fence_after();
          drain_into_sum(tmem + buf * T::kTN + half * 32 + lanes);
          if (q < chunks - 1) release();
        }
        if (ok) drain_into_sum(tmem + (2 + small) * T::kTN + half * 32 + lanes);       // the last chunk's commit covers the small terms too
        if (!ok) break;
        // The small terms' accumulator is written again by the tile after next, which waits for a chunk of the next tile
        // to be drained here if that has two or more: then this chunk need not be held any longer.
        const bool early = w.k + 1 >= w.end || w.next_t.depth > kOrthChunk * kOrthTK;
        if (early) release();
        // the sums go back to where the small terms were, so that one loop serves either kind of context
#pragma unroll
        for (int s = 0; s < T::kBlocks; ++s) {
          uint32_t acc[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[e] = __float_as_uint(e & 1 ? sum[s][e / 2].y : sum[s][e / 2].x);
          tmem_st32(tmem + (2 + small) * T::kTN + half * 32 + lanes + s * 64, acc);
        }
        tmem_wait_st();
        const uint32_t base = tmem + (2 + small) * T::kTN + half * 32 + lanes;
        ok = finish_tile(w, step, m, live, base);
        if (!early) release();
        small ^= 1;
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();               // the pair's copies and arrivals are all in, unless a wait expired
  if (s_abort && threadIdx.x == 0) {             // no copy may land after the block has gone
    for (int s = 0; rank == 0 && s < T::kStages && s < s_issued; ++s) {
      const int uses = (s_issued - 1 - s) / T::kStages;          // the stage's last copy is its use number `uses`
      mbar_wait_bounded(&full[s], uses & 1);
    }
    for (int s = 0; s < T::kRing && s < s_strips; ++s) mbar_wait_bounded(&strip_full[s], ((s_strips - 1 - s) / T::kRing) & 1);
    atomicOr(p.flags, kFlagTimeout);
  }
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc<CG>(tmem, T::kTmemCols);
  }
}

// ----------------------------------------------------------------------------------------------
// Vectors of small matrices only (short side up to 128, long side up to 256): one block takes a matrix through
// everything, norm to result, with X, S and B in shared memory and the accumulators in tensor memory; nothing but the
// matrix itself crosses global memory.  What bounds it is the chain of a step's three products and epilogues,
// 7 to 14 us a step; through the general kernel the same chain is 12 to 17 us, most of it stores, fences and
// looks at counters (96 x 200 fp32 64 us here and 86 there, 400 of them in bf16 144 and 284, 128 x 256 bf16 57 and 62).
//
// X is held as up to four blocks of 128 rows x 64 columns (swizzled 128-byte rows, as TMA would leave them):
// K-major operand of the Gram product, MN-major right operand of the Apply product.  S and B share a place: B
// replaces S element by element once the product that reads S is complete.
// ----------------------------------------------------------------------------------------------
constexpr int kOrthSmallR = 128, kOrthSmallL = 256;
constexpr int kOrthSmallThreads = 544;           // warps 0-15 elementwise, 16 products
constexpr uint32_t kSmallBlock = 128 * 128, kSmallXLo = 4 * kSmallBlock, kSmallS = 8 * kSmallBlock, kSmallSLo = 10 * kSmallBlock, kSmallBytes = 12 * kSmallBlock + 1024;

template <bool SPLIT>
__global__ void __launch_bounds__(kOrthSmallThreads, 1) orth_small_kernel(const OrthParams p, const void* in, int aligned, double eps) {
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  __shared__ uint64_t s_done;
  __shared__ uint32_t s_tmem;
  __shared__ double s_sum[16];
  __shared__ volatile int s_abort;
  constexpr int DT = SPLIT ? 0 : 1;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const OrthMat m = p.mats[blockIdx.x];
  if (tid == 0) { mbar_init(&s_done, 1); s_abort = 0; mbar_init_fence(); }
  if (warp == 16) tmem_alloc(&s_tmem, 512);
  // X_0, transposed where the matrix is taller than wide; everything outside it stays zero
  for (int k = tid; k < static_cast<int>(12 * kSmallBlock / 16); k += kOrthSmallThreads) reinterpret_cast<uint4*>(smem)[k] = make_uint4(0u, 0u, 0u, 0u);
  const int size = m.r * m.l;
  double sum = 0.0;
  const int width = m.transposed ? m.r : m.l;     // of a row in the vector
  const int step_y = kOrthSmallThreads / width, step_x = kOrthSmallThreads - step_y * width;
  // element (y, x) of the matrix in X's blocks
  auto place_of = [&](int y, int x) {
    const int row = m.transposed ? x : y, col = m.transposed ? y : x;
    return (col >> 6) * kSmallBlock + row * 128 + ((((col >> 3) & 7) ^ (row & 7)) << 4) + (col & 7) * 2;
  };
  __syncthreads();                                 // the zeros
  // Rows of whole groups of eight: all of a thread's elements in flight at once, kept until the norm is known.
  constexpr int kHeld = kOrthSmallR * kOrthSmallL / 8 / kOrthSmallThreads + 1;
  const bool vec = aligned && m.vec_in && width % 8 == 0;
  float held[kHeld][8];
  if (vec) {
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
      const int k = tid + q * kOrthSmallThreads;
      if (8 * k < size) {
        orth_in8<DT>(in, m.offset + 8 * k, held[q]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) held[q][e] = 0.f;
      }
    }
#pragma unroll
    for (int q = 0; q < kHeld; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fma(static_cast<double>(held[q][e]), static_cast<double>(held[q][e]), sum);
  } else {
    // As it comes first: bf16 where the hi parts will be, fp32 as upper and lower halves.
    for (int k0 = tid, y = tid / width, x = tid - y * width; k0 < size;) {       // eight loads on their way at a time
      float v[8];
  #pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = k0 + e * kOrthSmallThreads < size ? orth_in<DT>(in, m.offset + k0 + e * kOrthSmallThreads) : 0.f;
  #pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), sum);
        if (k0 < size) {
          const uint32_t at = place_of(y, x), bits = __float_as_uint(v[e]);
          *reinterpret_cast<unsigned short*>(smem + at) = static_cast<unsigned short>(bits >> 16);
          if (SPLIT) *reinterpret_cast<unsigned short*>(smem + kSmallXLo + at) = static_cast<unsigned short>(bits);
        }
        k0 += kOrthSmallThreads;
        y += step_y;
        x += step_x;
        if (x >= width) { x -= width; ++y; }
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (warp < 16 && lane == 0) s_sum[warp] = sum;
  __shared__ double s_last;
  if (warp == 16 && lane == 0) s_last = sum;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  sum = s_last;
  for (int w = 0; w < 16; ++w) sum += s_sum[w];
  const OrthFactor by(sum, eps);
  if (vec) {
#pragma unroll
    for (int q = 0; q < kHeld; ++q) {
      const int k = 8 * (tid + q * kOrthSmallThreads);
      if (k >= size) continue;
      const int y = k / width, x = k - y * width;
      float2 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = make_float2(held[q][2 * e], held[q][2 * e + 1]);
      orth_scale8(v, by.first);
      orth_scale8(v, by.then);
      uint4 h, l;
      orth_round8<true>(v, h, l);
      if (!m.transposed) {
        const uint32_t at = place_of(y, x);
        *reinterpret_cast<uint4*>(smem + at) = h;
        *reinterpret_cast<uint4*>(smem + kSmallXLo + at) = l;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t at = place_of(y, x + e);
          *reinterpret_cast<unsigned short*>(smem + at) = static_cast<unsigned short>(orth_word(h, e / 2) >> (16 * (e & 1)));
          *reinterpret_cast<unsigned short*>(smem + kSmallXLo + at) = static_cast<unsigned short>(orth_word(l, e / 2) >> (16 * (e & 1)));
        }
      }
    }
  } else {
    for (int k = tid; k < 8 * ((m.l + 63) / 64) * m.r; k += kOrthSmallThreads) {       // then pairs of 2^11 X_0, eight elements at a time
      const int group = k / m.r;
      unsigned char* at = smem + (group >> 3) * kSmallBlock + (k - group * m.r) * 128 + (group & 7) * 16;
      const uint4 u = *reinterpret_cast<const uint4*>(at), d = *reinterpret_cast<const uint4*>(at + kSmallXLo);
      float2 v[4];
  #pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t a = orth_word(u, q), b = SPLIT ? orth_word(d, q) : 0u;
        v[q] = make_float2(__uint_as_float(__byte_perm(b, a, 0x5410)), __uint_as_float(__byte_perm(b, a, 0x7632)));
      }
      orth_scale8(v, by.first);
      orth_scale8(v, by.then);
      uint4 h, l;
      orth_round8<true>(v, h, l);
      *reinterpret_cast<uint4*>(at) = h;
      *reinterpret_cast<uint4*>(at + kSmallXLo) = l;
    }
  }
  fence_proxy_async_smem();
  __syncthreads();

  bool issuer = false;
  if (warp == 16) issuer = elect_one();
  const int row = (warp & 3) * 32 + lane, part = warp >> 2;
  const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
  const uint32_t base = smem_addr(smem);
  const int r16 = (m.r + 15) / 16, l16 = (m.l + 15) / 16;
  uint32_t parity = 0;
  // Tensor memory: one accumulator of 128 columns (Apply: 256) for each 64 of K.
  for (int s = 0; s < p.steps; ++s) {
    const OrthStep step = p.coeffs[s];
    const bool last = s == p.steps - 1;
    for (int kind = 0; kind < 3; ++kind) {
      if (warp == 16) {
        const uint64_t x_rows = desc_kmajor(0) + (base >> 4), x_cols = desc_mnmajor(0, kSmallBlock) + (base >> 4), s_rows = desc_kmajor(0) + ((base + kSmallS) >> 4);
        const uint64_t a0 = kind == kOrthGram ? x_rows : s_rows, b0 = kind == kOrthPoly ? s_rows : kind == kOrthGram ? x_rows : x_cols;
        const uint32_t a_lo = (kind == kOrthGram ? kSmallXLo : kSmallSLo - kSmallS) >> 4, b_lo = (kind == kOrthPoly ? kSmallSLo - kSmallS : kSmallXLo) >> 4;
        const uint32_t idesc = kind == kOrthApply ? mma_idesc(128, 0, false, false, true) | (static_cast<uint32_t>(l16 * 16) >> 3 << 17) : mma_idesc(128, 128, false, false, false);
        const int steps_k = kind == kOrthGram ? l16 : r16;
        const uint32_t b_step = kind == kOrthApply ? 2048 >> 4 : 32 >> 4, wide = kind == kOrthApply ? 256 : 128;
        // The small terms first, then the hi hi ones: on top of them, and from K = 64 (Apply: 64) on in accumulators of
        // their own, chained four products at most.  The whole warp loops, so that the descriptors are uniform values; one lane issues.
        for (int pass = SPLIT ? 0 : 1; pass < 2; ++pass)
          for (int k0 = 0; k0 < steps_k; k0 += 4) {
            const uint32_t block = (k0 >> 2) * (kSmallBlock >> 4);
            const uint64_t a = a0 + block, b = b0 + (kind == kOrthApply ? static_cast<uint32_t>(k0) * (2048 >> 4) : block);
            const uint32_t d = tmem + (pass == 0 ? 0u : static_cast<uint32_t>(k0 >> 2) * wide), more = pass == 0 ? k0 != 0 : SPLIT && k0 == 0;
            if (issuer) {
#pragma unroll
              for (int kk = 0; kk < 4; ++kk) {
                if (k0 + kk >= steps_k) continue;
                if (pass == 0) {
                  mma_ss(d, a + a_lo + kk * 2, b + kk * b_step, idesc, kk != 0 ? 1u : more);
                  mma_ss(d, a + kk * 2, b + b_lo + kk * b_step, idesc, 1u);
                } else {
                  mma_ss(d, a + kk * 2, b + kk * b_step, idesc, kk != 0 ? 1u : more);
                }
              }
            }
            __syncwarp();
          }
        if (issuer) mma_commit(&s_done);
        __syncwarp();
      }
      if (!mbar_wait_bounded(&s_done, parity)) s_abort = 1;
      parity ^= 1u;
      tc_fence_after();
      if (warp < 16 && (warp & 3) * 32 < m.r) {    // rows beyond the matrix are zero and stay so
        const int chains = ((kind == kOrthGram ? l16 : r16) + 3) / 4;
        const uint32_t wide = kind == kOrthApply ? 256 : 128;
        const int col0 = part * (kind == kOrthApply ? 64 : 32), cols = kind == kOrthApply ? m.l : m.r;
        unsigned char* place = smem + (kind == kOrthApply ? 0u : kSmallS) + (col0 >> 6) * kSmallBlock + row * 128;
        const uint32_t place_lo = kind == kOrthApply ? kSmallXLo : kSmallSLo - kSmallS;
        const float by_x = kind == kOrthPoly ? step.b * (kOrthBScale / kOrthSScale) : step.a - step.t;
        const float by_v = kind == kOrthGram ? kOrthSScale / (kOrthXScale * kOrthXScale)
                                             : kind == kOrthPoly ? step.c * (kOrthBScale / (kOrthSScale * kOrthSScale)) : 1.f / kOrthBScale;
        const int turns = kind == kOrthApply ? 4 : 2;
#pragma unroll 1
        for (int turn = 0; turn < turns; ++turn) {
          const int col = col0 + turn * 16;
          if (col >= cols) break;                  // warp-uniform; what lies beyond is zero and stays so
          float2 v[8];
          {
            uint32_t a[16], b[16];
            tmem_ld16(tmem + lanes + col, a);
            if (chains > 1) tmem_ld16(tmem + wide + lanes + col, b);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              v[k] = make_float2(__uint_as_float(a[2 * k]), __uint_as_float(a[2 * k + 1]));
              if (chains > 1) v[k] = add2(v[k], make_float2(__uint_as_float(b[2 * k]), __uint_as_float(b[2 * k + 1])));
            }
            if (chains > 2) {                      // the Gram product of more than 128 columns
              tmem_ld16(tmem + 2 * wide + lanes + col, a);
              if (chains > 3) tmem_ld16(tmem + 3 * wide + lanes + col, b);
              tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                v[k] = add2(v[k], make_float2(__uint_as_float(a[2 * k]), __uint_as_float(a[2 * k + 1])));
                if (chains > 3) v[k] = add2(v[k], make_float2(__uint_as_float(b[2 * k]), __uint_as_float(b[2 * k + 1])));
              }
            }
          }
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
            unsigned char* at = place + (((((col & 63) >> 3) + sub) ^ (row & 7)) << 4);
            float2 w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = v[4 * sub + k];
            orth_scale8(w, by_v);
            if (kind != kOrthGram) {
              orth_add8(w, by_x, at);
              if (SPLIT || kind == kOrthApply) orth_add8(w, by_x, at + place_lo);
              if (kind == kOrthPoly && part == (warp & 3)) orth_diagonal8(w, row - col - 8 * sub, step.t * kOrthBScale);
            }
            uint4 h, l;
            if (kind == kOrthApply && last) {      // the result in X's place: bf16, or the upper and lower halves of fp32 words
              orth_scale8(w, m.scale / kOrthXScale);
              if (SPLIT) orth_halves8(w, h, l);
              else h = orth_bf16x8(w);
            } else {
              orth_round8<true>(w, h, l);
            }
            *reinterpret_cast<uint4*>(at) = h;
            if (SPLIT || (kind == kOrthApply && !last)) *reinterpret_cast<uint4*>(at + place_lo) = l;
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
      }
      __syncthreads();
      tc_fence_after();
      if (s_abort) break;                          // set before the barrier: the whole block agrees
    }
    if (s_abort) break;
  }
  if (!s_abort) {                                  // to the vector, as it lies there
#pragma unroll 4
    for (int k = tid, y = tid / width, x = tid - y * width; k < size; k += kOrthSmallThreads) {
      const uint32_t at = place_of(y, x);
      const uint32_t u = *reinterpret_cast<const unsigned short*>(smem + at);
      if (SPLIT) static_cast<uint32_t*>(p.out)[m.offset + k] = u << 16 | *reinterpret_cast<const unsigned short*>(smem + kSmallXLo + at);
      else static_cast<unsigned short*>(p.out)[m.offset + k] = static_cast<unsigned short>(u);
      y += step_y;
      x += step_x;
      if (x >= width) { x -= width; ++y; }
    }
  }
  if (s_abort && tid == 0) atomicOr(p.flags, kFlagTimeout);
  __syncthreads();
  if (warp == 16) tmem_dealloc(tmem, 512);
}

}  // namespace adacons
