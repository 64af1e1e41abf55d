// Attention and its gradient on the tensor cores: kernels (sm_100a).
#pragma once

#include <cuda_fp16.h>

#include "adacons_ops.h"
#include "adacons_tc.cuh"

namespace adacons {

// ----------------------------------------------------------------------------------------------
// For one query head:  S = scale Q K^T with -inf where a query does not see a key,
//     lse_i = log sum_j exp S_ij     P = exp(S - lse)     O = P V
// and from dO, with Delta_i = sum_d dO_id O_id:
//     dV = P^T dO     dP = dO V^T     dS = P o (dP - Delta)     dQ = scale dS K     dK = scale dS^T Q
// Key j is visible to query i when j < kv_len and, with a causal mask, j <= i + Sk - Sq.  A query
// that sees no key has O = 0, lse = -inf and no part in any gradient.
//
// Operand tiles are 128 rows (queries or keys) of 64 or 128 head elements, fetched by TMA from 4-D
// tensors (element, token, head, batch): whatever lies past the last token or the head's last element
// arrives as zero, so that odd lengths and head sizes need no other code.  A tile is one or two blocks
// of 128 swizzled 128-byte rows; read along its rows it is the K-major operand of a product over head
// elements, read across them the MN-major operand of a product over tokens, from the same bytes.
// Keys from kv_len on may hold anything, Inf and NaN included: their rows are zeroed in shared
// memory before any product over keys (0 x NaN would spread to every query).
// So are the rows of queries that see no key, of q and dO in the gradient.
// S, the statistics, the accumulators and dS up to its rounding are fp32; P and dS are rounded to the
// inputs' 16-bit type as operands of the second products, an error of the size of the results' own rounding.
// fp16 has that error only between 2^-14 and 2^16, and the gradient's P and dS lie far below on long rows or under small dO (P near
// 2^-16 on 65,536 keys, whose dV was off by 7e-4 instead of 3e-4, and dQ by 8e-3 under dO of 0.01).  There they are rounded
// as 2^12 P and 2^k dS, with 2^k from the bound |dS| <= 2 max |dO_i| max |V_j| over the queries and keys of a key head, so that
// nothing overflows either, and the results are multiplied by 2^-12 and 2^-k.  The norms' maxima come with Delta, one for each block
// of that kernel, and every block of the gradient looks through its head's: 3.61 ms against bf16's 3.43 (8192 x 8192, 32 / 8 heads of
// 128), 28.9 against 24.7 us (8 x 256 tokens, 16 heads of 64).
// ----------------------------------------------------------------------------------------------
constexpr int kAttnTile = 128;
constexpr int kFwdThreads = 320;                 // warps 0-7 softmax, 8 copies, 9 products
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnOut { void* p; long long batch, seq, head; };     // element strides
struct AttnRows { const void* p; long long batch, seq, head; };

struct AttnParams {
  int B, Hq, Hkv, Sq, Sk, D;
  int causal;
  int sq_pad;                    // rows of the padded statistics
  int split;                     // blocks of a cluster that share a tile's walk (forward), that may (backward)
  int key_split, query_split;    // backward: how many share a key tile's queries, a query tile's keys: `split` or one
  float scale, scale_log2;       // scale, scale * log2(e)
  const int* kv_lens;            // [B] or null
  float* lse;                    // forward: [B][Hq][Sq]
  const float* lse2;             // backward: lse log2(e) - kAttnShift, +inf where a row has no key or does not exist: [B][Hq][sq_pad]
  const float* delta;            // likewise, 0 there; null: each block makes both for its own queries, from what follows
  const float* peaks;            // fp16, with a workspace: |dO_i|^2 at most, of the queries of each block of the kernel before: [B][Hq][blocks], then |V_j|^2: [B][Hkv][blocks]
  AttnRows dout, o, v;
  const float* lse_in;           // [B][Hq][Sq]
  AttnOut out, dk, dv;           // forward: O; backward: dQ, dK, dV
  uint32_t* flags;
};

// P in an fp16 gradient is 2^kAttnShift P: whole rows of a million keys keep their 11 bits, and a P a little above one still fits.
template <bool BF16> constexpr float kAttnShift = BF16 ? 0.f : 12.f;
template <bool BF16> constexpr float kAttnUnshift = BF16 ? 1.f : 1.f / 4096.f;
template <int D> constexpr int kAttnStatRows = 256 / (D / 8);     // rows of a block of the statistics kernel
constexpr int kAttnPeakRows = 128;                                // of v, of a block that looks for its largest (fp16)

template <int D> struct AttnTile {
  static constexpr uint32_t kBlock = kAttnTile * 128;         // 128 rows x 64 elements
  static constexpr uint32_t kBytes = kBlock * (D / 64);
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if (BF16) return pack_bf16x2_rn(lo, hi);
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool BF16>
__device__ __forceinline__ float2 unpack16(uint32_t u) {
  if (BF16) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}

template <int D>
__device__ __forceinline__ void attn_load_tile(unsigned char* dst, const CUtensorMap* map, uint64_t* bar, int row, int head, int batch) {
#pragma unroll
  for (int h = 0; h < D / 64; ++h) tma_load_4d(dst + h * AttnTile<D>::kBlock, map, bar, h * 64, row, head, batch);
}
// rows [from, to) of a tile become zero; called by one warp, before the tile is an operand
template <int D>
__device__ __forceinline__ void attn_zero_rows(unsigned char* tile, int from, int to) {
  const int lane = threadIdx.x & 31;
  for (int k = lane; k < (to - from) * 8; k += 32)
#pragma unroll
    for (int h = 0; h < D / 64; ++h) *reinterpret_cast<uint4*>(tile + h * AttnTile<D>::kBlock + from * 128 + k * 16) = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  __syncwarp();
}

// The products are issued by one lane, but their descriptors are made by the whole warp, so that they are
// uniform values (made inside the lane's branch they cost more time than the products themselves).  In a cluster a shared
// address has the block's rank in its upper bits, which must not reach the descriptor's other fields.
template <int D> struct AttnDesc {
  static __device__ __forceinline__ uint64_t rows(uint32_t addr) { return desc_kmajor(0) + ((addr & 0x3ffffu) >> 4); }                                  // product over head elements
  static __device__ __forceinline__ uint64_t tokens(uint32_t addr) { return desc_mnmajor(0, AttnTile<D>::kBlock) + ((addr & 0x3ffffu) >> 4); }          // product over tokens
};
// 128 x N product over head elements: rows of `a` with rows of `b`
template <int D, bool BF16, int N>
__device__ __forceinline__ void attn_mma_rows(uint32_t d, uint64_t a, uint64_t b) {
  constexpr uint32_t idesc = mma_idesc(kAttnTile, N, BF16, false, false);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) {
    const uint32_t off = ((k / 4) * AttnTile<D>::kBlock + (k % 4) * 32) >> 4;
    mma_ss(d, a + off, b + off, idesc, k != 0);
  }
}
// 128 x D product over tokens: 16-bit values in tensor memory with the tokens of `b`.  Whoever had columns
// 32 g .. 32 g + 31 of the fp32 scores puts their 16 words of 16-bit values in the first half of that place.
// 32 tokens: k and k + 1 of the groups of 16.
template <int D, bool BF16>
__device__ __forceinline__ void attn_mma_some_tokens(uint32_t d, uint32_t a, uint64_t b, int k, bool accumulate) {
  constexpr uint32_t idesc = mma_idesc(kAttnTile, D, BF16, false, true);
#pragma unroll
  for (int e = 0; e < 2; ++e) mma_ts(d, a + (k / 2) * 32 + e * 8, b + (k + e) * (2048 >> 4), idesc, e != 0 ? 1u : accumulate);
}
template <int D, bool BF16, int TOKENS>
__device__ __forceinline__ void attn_mma_tokens(uint32_t d, uint32_t a, uint64_t b, bool accumulate) {
#pragma unroll
  for (int k = 0; k < TOKENS / 16; k += 2) attn_mma_some_tokens<D, BF16>(d, a, b, k, accumulate || k != 0);
}

// Columns [first, first + 32 BLOCKS) of row `row` of an accumulator (this thread's lane), times `mul`, to global memory.
template <int BLOCKS, bool BF16>
__device__ __forceinline__ void attn_store_row(const AttnParams& p, const AttnOut& o, uint32_t tmem, int first, int batch, int head, int row, bool live, float mul) {
  unsigned short* dst = static_cast<unsigned short*>(o.p) + batch * o.batch + static_cast<long long>(row) * o.seq + head * o.head + first;
#pragma unroll
  for (int c = 0; c < BLOCKS; ++c) {
    uint32_t v[32];
    __syncwarp();
    tmem_ld32(tmem + first + c * 32, v);
    tmem_wait_ld();
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (!live || first + c * 32 + g * 8 >= p.D) continue;       // the head size is a multiple of eight
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = pack16<BF16>(__uint_as_float(v[8 * g + 2 * k]) * mul, __uint_as_float(v[8 * g + 2 * k + 1]) * mul);
      *reinterpret_cast<uint4*>(dst + c * 32 + g * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}
__device__ __forceinline__ void attn_zero_row(const AttnParams& p, const AttnOut& o, int batch, int head, int row) {
  unsigned short* dst = static_cast<unsigned short*>(o.p) + batch * o.batch + static_cast<long long>(row) * o.seq + head * o.head;
  for (int k = 0; k < p.D; k += 8) *reinterpret_cast<uint4*>(dst + k) = make_uint4(0u, 0u, 0u, 0u);
}

__device__ __forceinline__ int attn_kv_len(const AttnParams& p, int batch) {
  if (p.kv_lens == nullptr) return p.Sk;
  const int n = p.kv_lens[batch];
  return n < 0 ? 0 : n > p.Sk ? p.Sk : n;
}

// A share of an accumulator, 128 rows of D fp32 values in shared memory, the 16-byte groups of a row
// exchanged by its lowest three bits: written a row a thread, read a few rows a warp.
template <int D, int BLOCKS>
__device__ __forceinline__ void attn_keep_row(unsigned char* keep, uint32_t tmem, int first, int row) {
#pragma unroll
  for (int c = 0; c < BLOCKS; ++c) {
    uint32_t v[32];
    __syncwarp();
    tmem_ld32(tmem + first + c * 32, v);
    tmem_wait_ld();
#pragma unroll
    for (int g = 0; g < 8; ++g)
      *reinterpret_cast<uint4*>(keep + row * (D * 4) + (((first + c * 32) / 4 + g) ^ (row & 7)) * 16) = make_uint4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
  }
}
// Shares of a query tile, one in each block of the cluster, become the result: every block joins its part of the rows,
//     m = max_c m_c     O = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) sum_c
// in the blocks' order.  `row` stands for the shares' maxima, then their sums.
template <int D, bool BF16>
__device__ __forceinline__ void attn_join(const AttnParams& p, const unsigned char* keep, const float* row_at, int rank, int q0, int head, int batch) {
  const int rows = kAttnTile / p.split;
  for (int n = threadIdx.x; n < rows * (D / 8); n += kFwdThreads) {
    const int lrow = rank * rows + n / (D / 8), e = n % (D / 8) * 8, row = q0 + lrow;
    if (row >= p.Sq) continue;
    float m = -INFINITY;
    for (int c = 0; c < p.split; ++c) m = fmaxf(m, ld_cluster_f32(row_at + lrow, c));
    float sum = 0.f, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < p.split; ++c) {
      const float part = ld_cluster_f32(row_at + kAttnTile + lrow, c);
      if (part == 0.f) continue;                 // no key there that the query sees: nothing was kept
      const float w = exp2_fast(ld_cluster_f32(row_at + lrow, c) - m);      // scores that are all NaN have no maximum, but a sum of NaN
      sum = fmaf(w, part, sum);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 o = ld_cluster_f32x4(keep + lrow * (D * 4) + ((e / 4 + h) ^ (lrow & 7)) * 16, c);
        v[4 * h] = fmaf(w, o.x, v[4 * h]);
        v[4 * h + 1] = fmaf(w, o.y, v[4 * h + 1]);
        v[4 * h + 2] = fmaf(w, o.z, v[4 * h + 2]);
        v[4 * h + 3] = fmaf(w, o.w, v[4 * h + 3]);
      }
    }
    const float by = sum == 0.f ? 0.f : 1.f / sum;
    if (e < p.D)
      *reinterpret_cast<uint4*>(static_cast<unsigned short*>(p.out.p) + batch * p.out.batch + static_cast<long long>(row) * p.out.seq + head * p.out.head + e) =
          make_uint4(pack16<BF16>(v[0] * by, v[1] * by), pack16<BF16>(v[2] * by, v[3] * by), pack16<BF16>(v[4] * by, v[5] * by), pack16<BF16>(v[6] * by, v[7] * by));
    if (e == 0) p.lse[(static_cast<long long>(batch) * p.Hq + head) * p.Sq + row] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
  }
}

// The same for a gradient, whose shares are added as they are: the first `shares` blocks have one.
template <int D, bool BF16, int THREADS>
__device__ __forceinline__ void attn_join_sum(const AttnParams& p, const AttnOut& out, const unsigned char* keep, int rank, int shares, int row0, int len, int head, int batch, float mul) {
  const int rows = kAttnTile / p.split;
  for (int n = threadIdx.x; n < rows * (D / 8); n += THREADS) {
    const int lrow = rank * rows + n / (D / 8), e = n % (D / 8) * 8, row = row0 + lrow;
    if (row >= len || e >= p.D) continue;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < shares; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 o = ld_cluster_f32x4(keep + lrow * (D * 4) + ((e / 4 + h) ^ (lrow & 7)) * 16, c);
        v[4 * h] += o.x;
        v[4 * h + 1] += o.y;
        v[4 * h + 2] += o.z;
        v[4 * h + 3] += o.w;
      }
    *reinterpret_cast<uint4*>(static_cast<unsigned short*>(out.p) + batch * out.batch + static_cast<long long>(row) * out.seq + head * out.head + e) = make_uint4(
        pack16<BF16>(v[0] * mul, v[1] * mul), pack16<BF16>(v[2] * mul, v[3] * mul), pack16<BF16>(v[4] * mul, v[5] * mul), pack16<BF16>(v[6] * mul, v[7] * mul));
  }
}

// ----------------------------------------------------------------------------------------------
// Forward.  A block owns 128 queries of one head and walks over the key tiles: S = Q K^T, softmax, O += P V,
// one after the other; two blocks share an SM, and one's softmax runs while the tensor cores work for the other.
// (One block with two query tiles in turn reads K and V half as often, but is no faster at 8192 tokens, 562 us
// against 573, and slower where blocks are few or short: 2048 causal tokens of 8 heads 42 us against 35.)
// Tensor memory: S (128 columns, later the rounded P in its place) and the accumulator.
// Few query tiles and many keys: the blocks of a cluster share the keys of a query tile and join their shares through one
// another's shared memory, no workspace and no second launch (one query over 4000 keys 57 -> 14 us).
// Two threads share one query's row of scores and exchange their maxima (one thread a row needs none, but with two
// warps per scheduler every instruction's latency shows).  The running maximum is only raised when a row's scores exceed
// it by more than 2^8 in the exponential (the quotient O / sum does not depend on it, and fp32 and bf16 have the
// range): the accumulator is then rescaled in place, which after the first few key tiles hardly happens.
// ----------------------------------------------------------------------------------------------
template <int D> struct AttnFwdSmem {
  static constexpr uint32_t kT = AttnTile<D>::kBytes;
  static constexpr int kSlots = D == 128 ? 2 : 5;              // ring of K and V tiles in turn
  static constexpr uint32_t kKV = kT, kBars = kKV + kSlots * kT, kBytes = kBars + 256 + 1024;
};

// STARVE, here and in the gradient: the self-test's form, whose copies leave the last tile out, so that every wait behind it
// runs out.
template <int D, bool BF16, bool STARVE = false>
__global__ void __launch_bounds__(kFwdThreads, 2)
attn_forward_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const AttnParams p) {
  extern __shared__ unsigned char smem_dyn[];
  using L = AttnFwdSmem<D>;
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  uint64_t* q_full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* kv_full = q_full + 1;                // [kSlots]
  uint64_t* kv_free = kv_full + L::kSlots;       // [kSlots]
  uint64_t* s_full = kv_free + L::kSlots;
  uint64_t* p_full = s_full + 1;                 // [2] the even and the odd 32 keys of either half
  uint64_t* o_full = p_full + 2;
  uint64_t* pair = o_full + 1;                   // [4] the two warps of 32 rows
  uint64_t* drain = pair + 4;
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ float s_row[2][kAttnTile];          // [half][row]
  __shared__ float s_share[2][kAttnTile];        // maxima and sums of this block's share
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int head = blockIdx.y, batch = blockIdx.z;
  const int rank = static_cast<int>(blockIdx.x) % p.split;
  const int q0 = static_cast<int>((gridDim.x - 1 - blockIdx.x) / p.split) * kAttnTile;     // with a causal mask the last queries have the most keys: first

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    for (int s = 0; s < L::kSlots; ++s) { mbar_init(&kv_full[s], 1); mbar_init(&kv_free[s], 1); }
    mbar_init(s_full, 1);
    mbar_init(&p_full[0], 8);
    mbar_init(&p_full[1], 8);
    mbar_init(o_full, 1);
    for (int t = 0; t < 4; ++t) mbar_init(&pair[t], 2);
    mbar_init(drain, 1);
    s_abort = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == 9) tmem_alloc(&s_tmem, 256);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t t_s = s_tmem, t_o = t_s + 128;
  const int kv_len = attn_kv_len(p, batch);
  const int off = p.Sk - p.Sq;
  const int q_last = min(q0 + kAttnTile, p.Sq) - 1;
  const int seen = p.causal ? min(kv_len, max(0, q_last + off + 1)) : kv_len;     // keys that any query of the block sees
  const int all_tiles = (seen + kAttnTile - 1) / kAttnTile, share = (all_tiles + p.split - 1) / p.split;
  const int first = min(rank * share, all_tiles), tiles = min(share, all_tiles - first);        // this block's key tiles

  if (tiles > 0 && warp == 8) {
    if (lane == 0) {
      mbar_expect_tx(q_full, L::kT);
      attn_load_tile<D>(smem, &mq, q_full, q0, head, batch);
      const int kv_head = head / (p.Hq / p.Hkv);
      int slot = 0, issued = 0;
      uint32_t parity = 1;
      for (int n = 0; n < 2 * tiles; ++n) {      // K_0 V_0 K_1 V_1 ..
        if (STARVE && n == 2 * tiles - 1) break;
        if (s_abort || !mbar_wait_bounded(&kv_free[slot], parity)) { s_abort = 1; break; }
        mbar_expect_tx(&kv_full[slot], L::kT);
        attn_load_tile<D>(smem + L::kKV + slot * L::kT, n & 1 ? &mv : &mk, &kv_full[slot], (first + (n >> 1)) * kAttnTile, kv_head, batch);
        ++issued;
        if (++slot == L::kSlots) { slot = 0; parity ^= 1u; }
      }
      if (s_abort) {                             // no copy may land after the block has gone
        mbar_wait_bounded(q_full, 0);
        for (int s = 0; s < L::kSlots && s < issued; ++s) mbar_wait_bounded(&kv_full[s], ((issued - 1 - s) / L::kSlots) & 1);
      }
    }
  } else if (tiles > 0 && warp == 9) {
    const bool issuer = elect_one();
    int slot = 0;
    uint32_t parity = 0;
    bool ok = mbar_wait_bounded(q_full, 0);
    // waits for a slot; V tiles that reach past kv_len get their rows zeroed
    auto take = [&](int valid) -> uint32_t {
      ok = ok && !s_abort && mbar_wait_bounded(&kv_full[slot], parity);
      ok = __all_sync(0xffffffffu, ok);
      if (ok && valid < kAttnTile) attn_zero_rows<D>(smem + L::kKV + slot * L::kT, valid, kAttnTile);
      return smem_addr(smem) + L::kKV + slot * L::kT;
    };
    auto advance = [&]() { if (++slot == L::kSlots) { slot = 0; parity ^= 1u; } };
    const uint64_t q_desc = AttnDesc<D>::rows(smem_addr(smem));
    for (int j = 0; j < tiles; ++j) {
      // S(j) takes the place of P(j - 1), which the product before it has read
      const uint64_t k_desc = AttnDesc<D>::rows(take(kAttnTile));
      tc_fence_after();
      if (ok && issuer) {
        attn_mma_rows<D, BF16, kAttnTile>(t_s, q_desc, k_desc);
        mma_commit(s_full);
        mma_commit(&kv_free[slot]);
      }
      __syncwarp();
      advance();
      const uint64_t v_desc = AttnDesc<D>::tokens(take(min(kv_len - (first + j) * kAttnTile, kAttnTile)));
      // the product over the even 32 keys of either half runs beside the exponentials of the odd ones
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        ok = ok && !s_abort && mbar_wait_bounded(&p_full[c], j & 1);
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        if (ok && issuer) {
          attn_mma_some_tokens<D, BF16>(t_o, t_s, v_desc, 2 * c, j != 0 || c != 0);
          attn_mma_some_tokens<D, BF16>(t_o, t_s, v_desc, 4 + 2 * c, true);
        }
        __syncwarp();
      }
      if (!ok) break;
      if (issuer) {
        mma_commit(&kv_free[slot]);
        if (j == tiles - 1) mma_commit(o_full);
      }
      __syncwarp();
      advance();
    }
    if (!ok) {
      s_abort = 1;
      if (issuer) { mma_commit(drain); mbar_wait_bounded(drain, 0); }
    }
  } else if (warp < 8) {
    const int half = warp >> 2;                  // this warp's 64 keys of each tile
    const int lrow = (warp & 3) * 32 + lane, row = q0 + lrow;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = t_s + half * 64 + lanes, o_at = t_o + lanes;
    const int limit = p.causal ? min(kv_len, row + off + 1) : kv_len;        // this query's keys: [0, limit)
    const int warp_limit = p.causal ? min(kv_len, row - lane + off + 1) : kv_len;   // all of the warp's queries see these
    uint64_t* both = &pair[warp & 3];
    uint32_t turn = 0;
    bool ok = true;
    // The other half's value for this row.  The next exchange comes after the products that both warps' P go
    // into, so a place is never written before it has been read.
    auto exchange = [&](float mine) {
      s_row[half][lrow] = mine;
      __syncwarp();
      if (lane == 0) mbar_arrive_one(both);
      ok = ok && !s_abort && mbar_wait_bounded(both, turn);
      ok = __all_sync(0xffffffffu, ok);
      turn ^= 1u;
      return s_row[half ^ 1][lrow];
    };
    float top = -INFINITY, sum = 0.f;            // running maximum of scale_log2 S, this half's sum under it
    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
    for (int j = 0; ok && j < tiles; ++j) {
      ok = !s_abort && mbar_wait_bounded(s_full, j & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const int k0 = (first + j) * kAttnTile + half * 64;
      const bool masked = k0 + 64 > warp_limit;              // warp-uniform: some score is masked
      // 32 scores at a time, read again for the exponentials: 64 registers more would spill at this block size
      uint32_t s[32];
      auto fetch = [&](int c) {
        tmem_ld32(s_at + c * 32, s);
        tmem_wait_ld();
        if (masked) {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (k0 + c * 32 + e >= limit) s[e] = 0xff800000u;
        }
      };
      float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        fetch(c);
#pragma unroll
        for (int e = 0; e < 32; e += 2) m[(e >> 1) & 1] = max3(m[(e >> 1) & 1], __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
      }
      float tile_top = fmaxf(m[0], m[1]);
      tile_top = fmaxf(tile_top, exchange(tile_top)) * p.scale_log2;
      if (!ok) break;
      const bool raise = tile_top > top + 8.f;   // also the first time a row sees a key
      if (__any_sync(0xffffffffu, raise)) {
        const float next = raise ? tile_top : top;
        const float factor = raise ? exp2_fast(top - next) : 1.f;
        sum *= factor;
        top = next;
        if (j > 0) {                             // half of the accumulator's columns
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            uint32_t o[32];
            tmem_ld32(o_at + half * (D / 2) + c * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
            tmem_st32(o_at + half * (D / 2) + c * 32, o);
          }
        }
      }
      const float base = top == -INFINITY ? 0.f : -top;
      const float2 base2 = make_float2(base, base);
      float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[16];
        fetch(c);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float2 x = fma2(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), scale2, base2);
          x.x = exp2_fast(x.x);
          x.y = exp2_fast(x.y);
          part[e & 1] = add2(part[e & 1], x);
          w[e] = pack16<BF16>(x.x, x.y);
        }
        tmem_st16(s_at + c * 32, w);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_one(&p_full[c]);
        __syncwarp();                            // the reads of tensor memory that follow want the whole warp
      }
      part[0] = add2(part[0], part[1]);
      sum += part[0].x + part[0].y;
    }
    const bool live = row < p.Sq;
    if (ok && tiles > 0) {
      ok = !s_abort && mbar_wait_bounded(o_full, 0);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      sum += exchange(sum);
      if (p.split > 1) attn_keep_row<D, D / 64>(smem + L::kKV, o_at, half * (D / 2), lrow);
      else if (ok) attn_store_row<D / 64, BF16>(p, p.out, o_at, half * (D / 2), batch, head, row, live, sum == 0.f ? 0.f : 1.f / sum);
    } else if (p.split == 1 && tiles == 0 && live && half == 0) {
      attn_zero_row(p, p.out, batch, head, row);
    }
    if (p.split > 1) s_share[half][lrow] = half == 0 ? top : sum;
    else if (ok && live && half == 0) p.lse[(static_cast<long long>(batch) * p.Hq + head) * p.Sq + row] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    if (!ok) s_abort = 1;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (s_abort && threadIdx.x == 0) atomicOr(p.flags, kFlagTimeout);
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(t_s, 256);
  }
  if (p.split > 1) {
    cluster_sync_all();
    attn_join<D, BF16>(p, smem + L::kKV, s_share[0], rank, q0, head, batch);
    cluster_sync_all();                          // the others may still read this block's share
  }
}

// ----------------------------------------------------------------------------------------------
// Before the gradient: Delta_i = sum_d dO_id O_id and the log-sum-exp in base 2, +inf and 0 where a query sees no key.
// D / 8 lanes take a query's row, eight elements each.
//
// With a workspace a kernel of its own writes them there, padded to whole tiles, so that the gradient's blocks copy them a
// tile at a time.  Without one (short queries only) every block of the gradient makes its own, in shared memory: this
// repeats the work in each block of a head and costs up to 2 us of it, but saves a launch.
// ----------------------------------------------------------------------------------------------
// U rows of each group of lanes, `step` places apart from place n on: rows of `heads` heads from `head` on, `pitch` places
// each; `total` places in all.  Whole warps.
template <bool BF16>
__device__ __forceinline__ float attn_dot8(const uint4& x, const uint4& y) {
  const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 a = unpack16<BF16>(xs[k]), b = unpack16<BF16>(ys[k]);
    sum += a.x * b.x + a.y * b.y;
  }
  return sum;
}
template <int D, bool BF16, int U>
__device__ __forceinline__ void attn_row_stats(const AttnParams& p, int batch, int head, int first_row, int pitch, int n, int step, int total, float* lse2, float* delta) {
  constexpr int kLanes = D / 8;
  const int e = 8 * (threadIdx.x % kLanes);
  uint4 x[U], y[U];
  float l[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = n + u * step, h = head + at / pitch, row = first_row + at % pitch;
    x[u] = y[u] = make_uint4(0u, 0u, 0u, 0u);
    l[u] = -INFINITY;
    if (at < total && row < p.Sq) {
      if (e < p.D) {
        x[u] = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p.dout.p) + batch * p.dout.batch + row * p.dout.seq + h * p.dout.head + e);
        y[u] = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p.o.p) + batch * p.o.batch + row * p.o.seq + h * p.o.head + e);
      }
      l[u] = p.lse_in[(static_cast<long long>(batch) * p.Hq + h) * p.Sq + row];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float sum = attn_dot8<BF16>(x[u], y[u]);
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const int at = n + u * step;
    if (e == 0 && at < total) {
      const bool none = l[u] == -INFINITY;
      lse2[at] = none ? INFINITY : fmaf(l[u], kLog2e, -kAttnShift<BF16>);
      delta[at] = none ? 0.f : sum;
    }
  }
}
// All of `total` places by the THREADS elementwise threads of a block, which meet at the end.
template <int D, bool BF16, int THREADS>
__device__ __forceinline__ void attn_block_stats(const AttnParams& p, int batch, int head, int first_row, int pitch, int total, float* lse2, float* delta) {
  constexpr int kStep = THREADS / (D / 8), kU = 4;
  const int n = threadIdx.x / (D / 8);
  for (int base = 0; base < total; base += kU * kStep) attn_row_stats<D, BF16, kU>(p, batch, head, first_row, pitch, base + n, kStep, total, lse2, delta);
  asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
}

// The largest |x|^2 of rows n, n + step, .. below `total`, D / 8 lanes a row.  `row_at`: where place n is, null where it does not count.
template <int D, int STEP, typename RowAt>
__device__ __forceinline__ float attn_peak(const AttnParams& p, int64_t total, RowAt row_at) {
  constexpr int kLanes = D / 8, kU = 4;
  const int e = 8 * (threadIdx.x % kLanes);
  float peak = 0.f;
  for (int64_t base = 0; base < total; base += kU * STEP) {
    uint4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int64_t n = base + u * STEP + threadIdx.x / kLanes;
      const unsigned short* at = n < total && e < p.D ? row_at(n) : nullptr;
      x[u] = at != nullptr ? *reinterpret_cast<const uint4*>(at + e) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      float sum = attn_dot8<false>(x[u], x[u]);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      peak = fmaxf(peak, sum);
    }
  }
  return peak;
}
__device__ __forceinline__ const unsigned short* attn_row(const AttnRows& t, int batch, int64_t row, int head) {
  return static_cast<const unsigned short*>(t.p) + batch * t.batch + row * t.seq + head * t.head;
}
__device__ __forceinline__ bool attn_has_key(const AttnParams& p, int batch, int head, int64_t row) {
  return p.lse_in[(static_cast<long long>(batch) * p.Hq + head) * p.Sq + row] != -INFINITY;
}

// fp16: 2^k for the dS of a key head, by the THREADS elementwise threads of a block, all blocks of the head alike.  The bound's
// slack is a few binades of the forty that fp16 has.
template <int D, int THREADS>
__device__ __forceinline__ float attn_ds_scale(const AttnParams& p, int batch, int kv_head, int kv_len) {
  __shared__ float s_peak[2][THREADS / 32];
  const int group = p.Hq / p.Hkv;
  float peak[2] = {0.f, 0.f};                      // |dO|^2, |V|^2
  if (p.peaks != nullptr) {
    const long long qb = p.sq_pad / kAttnStatRows<D>, kb = (p.Sk + kAttnPeakRows - 1ll) / kAttnPeakRows;
    const float* at[2] = {p.peaks + (static_cast<long long>(batch) * p.Hq + kv_head * group) * qb,
                          p.peaks + static_cast<long long>(p.B) * p.Hq * qb + (static_cast<long long>(batch) * p.Hkv + kv_head) * kb};
    const long long count[2] = {group * qb, kb};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll 4
      for (long long k = threadIdx.x; k < count[t]; k += THREADS) peak[t] = fmaxf(peak[t], at[t][k]);
  } else {
    peak[0] = attn_peak<D, THREADS / (D / 8)>(p, static_cast<int64_t>(group) * p.Sq, [&](int64_t n) {
      const int head = kv_head * group + static_cast<int>(n / p.Sq), row = static_cast<int>(n % p.Sq);
      return attn_has_key(p, batch, head, row) ? attn_row(p.dout, batch, row, head) : nullptr;
    });
    peak[1] = attn_peak<D, THREADS / (D / 8)>(p, kv_len, [&](int64_t n) { return attn_row(p.v, batch, n, kv_head); });
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) peak[t] = fmaxf(peak[t], __shfl_xor_sync(0xffffffffu, peak[t], o));
    if ((threadIdx.x & 31) == 0) s_peak[t][threadIdx.x >> 5] = peak[t];
  }
  asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
#pragma unroll
  for (int t = 0; t < 2; ++t)
    for (int w = 0; w < THREADS / 32; ++w) peak[t] = fmaxf(peak[t], s_peak[t][w]);
  const float square = peak[0] * peak[1];          // 2^-96 .. 2^78
  if (!(square > 0.f && square < INFINITY)) return 1.f;
  const int half = ((__float_as_int(square) >> 23) - 127 >> 1) + 1;      // |dO| |V| < 2^half, so |dS| < 2^(half + 1): 2^k dS < 2^14
  return __int_as_float((13 - half + 127) << 23);
}

template <int D, bool BF16>
__global__ void __launch_bounds__(256) attn_delta_kernel(const AttnParams p, float* lse2, float* delta, float* peaks) {      // grid: rows of a head (fp16: of q, then of v), heads, batch
  pdl_launch_dependents();
  if constexpr (!BF16) {
    __shared__ float s_peak[8];
    constexpr int kRows = kAttnStatRows<D>;
    const int qb = p.sq_pad / kRows, x = static_cast<int>(blockIdx.x), batch = blockIdx.z;
    const bool keys = x >= qb;
    const long long kb = (p.Sk + kAttnPeakRows - 1ll) / kAttnPeakRows;
    // the blocks beyond q's share all key heads' rows of v
    const long long unit = static_cast<long long>(x - qb) * p.Hq + blockIdx.y;
    if (keys && unit >= kb * p.Hkv) return;
    const int head = keys ? static_cast<int>(unit / kb) : static_cast<int>(blockIdx.y);
    const long long block = keys ? unit % kb : x, first = block * (keys ? kAttnPeakRows : kRows);
    const int kv_len = attn_kv_len(p, batch);
    float peak = attn_peak<D, kRows>(p, keys ? kAttnPeakRows : kRows, [&](int64_t n) -> const unsigned short* {
      if (keys) return first + n < kv_len ? attn_row(p.v, batch, first + n, head) : nullptr;
      return first + n < p.Sq && attn_has_key(p, batch, head, first + n) ? attn_row(p.dout, batch, first + n, head) : nullptr;
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) peak = fmaxf(peak, __shfl_xor_sync(0xffffffffu, peak, o));
    if ((threadIdx.x & 31) == 0) s_peak[threadIdx.x >> 5] = peak;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 8; ++w) peak = fmaxf(peak, s_peak[w]);
      peaks[keys ? static_cast<long long>(p.B) * p.Hq * qb + (static_cast<long long>(batch) * p.Hkv + head) * kb + block : (static_cast<long long>(batch) * p.Hq + head) * qb + block] = peak;
    }
    if (keys) return;
  }
  const long long at = (static_cast<long long>(blockIdx.z) * p.Hq + blockIdx.y) * p.sq_pad;
  attn_row_stats<D, BF16, 1>(p, blockIdx.z, blockIdx.y, 0, p.sq_pad, blockIdx.x * (256 / (D / 8)) + threadIdx.x / (D / 8), 0, p.sq_pad, lse2 + at, delta + at);
}

// ----------------------------------------------------------------------------------------------
// dK and dV.  A block owns 128 keys of one key head and walks over the query tiles of all query heads
// that share it: the shared head's gradient is a sum in tensor memory, in a fixed order, without atomics.
// Tensor memory (512 columns at D = 128): S^T, dP^T, dV, dK.  P^T and dS^T, rounded, take the places of S^T
// and dP^T and are the left operands of dV += P^T dO and dK += dS^T Q straight from there.
// The products are issued so that each elementwise phase has two products beside it:
//     P(i) from S(i)       | dK(i-1), dP(i)
//     dS(i) from P, dP(i)  | dV(i), S(i+1)
// Four warps share a block of 32 keys, 32 queries each.
// ----------------------------------------------------------------------------------------------
// The streamed tiles (queries here, keys below) are 128 tokens at D = 128.  At D = 64 they are 64: tensor memory
// then holds two blocks an SM (256 columns each), which overlap where a block is short or waits for its own chain;
// with 128 tokens and one block the encoder shape (512 tokens, 64 elements) took 72 us.
template <int D> struct AttnBwd {
  static constexpr int kTok = D == 128 ? 128 : 64;               // tokens of a streamed tile
  static constexpr int kParts = kTok / 32, kElem = 4 * kParts;   // elementwise warps: 32 rows x 32 columns each
  static constexpr int kCopyWarp = kElem, kMmaWarp = kElem + 1, kThreads = kElem * 32 + 64, kBlocks = D == 128 ? 1 : 2;
  static constexpr uint32_t kTmem = 2 * kTok + 2 * D;
  static constexpr uint32_t kRes = AttnTile<D>::kBytes, kStr = kRes * kTok / 128;      // bytes of a resident, a streamed tile
  // the box of the tensor maps is one streamed tile's rows
  static __device__ __forceinline__ void load_resident(unsigned char* dst, const CUtensorMap* map, uint64_t* bar, int row, int head, int batch) {
#pragma unroll
    for (int h = 0; h < 128 / kTok; ++h) attn_load_tile<D>(dst + h * kStr, map, bar, row + h * kTok, head, batch);
  }
};
template <int D> struct AttnDkvSmem {
  using G = AttnBwd<D>;
  static constexpr int kStages = D == 128 ? 2 : 4;
  static constexpr uint32_t kRing = 2 * G::kRes, kStage = 2 * G::kStr;          // K, V | (Q, dO) per stage
  static constexpr uint32_t kStat = G::kTok * 4;                                // lse2, delta: bytes per stage of each
  static constexpr uint32_t kStats = kRing + kStages * kStage;
  static constexpr uint32_t kTable = kStats + kStages * 2 * kStat;              // short queries' lse2, delta
  static constexpr uint32_t kBars = kTable + 2 * 4 * ADACONS_ATTN_SHORT_ROWS, kBytes = kBars + 256 + 1024;
};

template <int D, bool BF16, bool STARVE>
__device__ __forceinline__ void attn_dkv_block(unsigned char* smem, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mdo,
                                               const AttnParams& p, const int tile, const int kv_head, const int batch, const int rank) {
  using L = AttnDkvSmem<D>;
  using G = AttnBwd<D>;
  uint64_t* kv_full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* full = kv_full + 1;                  // [kStages]
  uint64_t* free_ = full + L::kStages;           // [kStages]
  uint64_t* s_full = free_ + L::kStages;
  uint64_t* p_full = s_full + 1;
  uint64_t* dp_full = p_full + 1;
  uint64_t* ds_full = dp_full + 1;
  uint64_t* done = ds_full + 1;
  uint64_t* drain = done + 1;
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ float s_by_dk;                      // fp16 only
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int k0 = tile * kAttnTile;
  const int group = p.Hq / p.Hkv;

  if (threadIdx.x == 0) {
    mbar_init(kv_full, 1);
    for (int s = 0; s < L::kStages; ++s) { mbar_init(&full[s], 1); mbar_init(&free_[s], 1); }
    mbar_init(s_full, 1);
    mbar_init(p_full, G::kElem);
    mbar_init(dp_full, 1);
    mbar_init(ds_full, G::kElem);
    mbar_init(done, 1);
    mbar_init(drain, 1);
    s_abort = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == G::kMmaWarp) tmem_alloc(&s_tmem, G::kTmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const uint32_t t_s = tmem, t_dp = tmem + G::kTok, t_dv = tmem + 2 * G::kTok, t_dk = t_dv + D;
  const int kv_len = attn_kv_len(p, batch);
  const int off = p.Sk - p.Sq;
  const int q_tiles = (p.Sq + G::kTok - 1) / G::kTok;
  // the first query that sees any of these keys: i >= k0 - off
  const int first = p.causal ? min(q_tiles, max(0, k0 - off) / G::kTok) : 0;
  const int per_head = k0 < kv_len ? q_tiles - first : 0;
  const int all = group * per_head, share = (all + p.key_split - 1) / p.key_split;
  const int skip = min(rank * share, all), items = min(share, all - skip);       // this block's part of the walk
  pdl_wait();                                    // the statistics

  if (items > 0 && warp == G::kCopyWarp) {
    if (lane == 0) {
      mbar_expect_tx(kv_full, 2 * G::kRes);
      G::load_resident(smem, &mk, kv_full, k0, kv_head, batch);
      G::load_resident(smem + G::kRes, &mv, kv_full, k0, kv_head, batch);
      int stage = 0, issued = 0;
      uint32_t parity = 1;
      for (int n = 0; n < items; ++n) {
        if (STARVE && n == items - 1) break;
        const int head = kv_head * group + (skip + n) / per_head, q0 = (first + (skip + n) % per_head) * G::kTok;
        if (s_abort || !mbar_wait_bounded(&free_[stage], parity)) { s_abort = 1; break; }
        unsigned char* at = smem + L::kRing + stage * L::kStage;
        unsigned char* stats = smem + L::kStats + stage * 2 * L::kStat;
        const long long base = (static_cast<long long>(batch) * p.Hq + head) * p.sq_pad + q0;
        mbar_expect_tx(&full[stage], L::kStage + (p.delta != nullptr ? 2 * L::kStat : 0));
        attn_load_tile<D>(at, &mq, &full[stage], q0, head, batch);
        attn_load_tile<D>(at + G::kStr, &mdo, &full[stage], q0, head, batch);
        if (p.delta != nullptr) {
          bulk_load(stats, p.lse2 + base, L::kStat, &full[stage]);
          bulk_load(stats + L::kStat, p.delta + base, L::kStat, &full[stage]);
        }
        ++issued;
        if (++stage == L::kStages) { stage = 0; parity ^= 1u; }
      }
      if (s_abort) {
        mbar_wait_bounded(kv_full, 0);
        for (int s = 0; s < L::kStages && s < issued; ++s) mbar_wait_bounded(&full[s], ((issued - 1 - s) / L::kStages) & 1);
      }
    }
  } else if (items > 0 && warp == G::kMmaWarp) {
    bool ok = __all_sync(0xffffffffu, mbar_wait_bounded(kv_full, 0));
    if (ok && k0 + kAttnTile > kv_len) {
      attn_zero_rows<D>(smem, kv_len - k0, kAttnTile);
      attn_zero_rows<D>(smem + G::kRes, kv_len - k0, kAttnTile);
    }
    const bool issuer = elect_one();
    const uint64_t k_desc = AttnDesc<D>::rows(smem_addr(smem)), v_desc = k_desc + (G::kRes >> 4);
    const uint32_t ring = smem_addr(smem) + L::kRing;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && !s_abort && mbar_wait_bounded(bar, parity);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      return ok;
    };
    // Queries of a head's first tile that see no key at all: what their q and dO hold, Inf and NaN included, must not reach a product.
    const int none = p.causal && k0 == 0 ? -off - first * G::kTok : 0;
    auto blank = [&](int n, int at) {
      if (none <= 0 || (skip + n) % per_head != 0) return;
      attn_zero_rows<D>(smem + L::kRing + at * L::kStage, 0, none);
      attn_zero_rows<D>(smem + L::kRing + at * L::kStage + G::kStr, 0, none);
    };
    if (wait(&full[0], 0)) {
      blank(0, 0);
      const uint64_t q_desc = AttnDesc<D>::rows(ring);
      if (issuer) {
        attn_mma_rows<D, BF16, G::kTok>(t_s, k_desc, q_desc);
        mma_commit(s_full);
        attn_mma_rows<D, BF16, G::kTok>(t_dp, v_desc, q_desc + (G::kStr >> 4));
        mma_commit(dp_full);
      }
      __syncwarp();
    }
    int stage = 0;
    uint32_t next_parity = 0;              // of the next item's stage
    for (int n = 0; ok && n < items; ++n) {
      const bool more = n + 1 < items;
      const int next_stage = stage + 1 == L::kStages ? 0 : stage + 1;
      if (next_stage == 0) next_parity ^= 1u;
      const uint64_t by_tokens = AttnDesc<D>::tokens(ring + stage * L::kStage), next_rows = AttnDesc<D>::rows(ring + next_stage * L::kStage);
      if (!wait(p_full, n & 1)) break;
      if (issuer) attn_mma_tokens<D, BF16, G::kTok>(t_dv, t_s, by_tokens + (G::kStr >> 4), n != 0);
      __syncwarp();
      if (more) {
        if (!wait(&full[next_stage], next_parity)) break;
        blank(n + 1, next_stage);
        if (issuer) {
          attn_mma_rows<D, BF16, G::kTok>(t_s, k_desc, next_rows);
          mma_commit(s_full);
        }
        __syncwarp();
      }
      if (!wait(ds_full, n & 1)) break;
      if (issuer) {
        attn_mma_tokens<D, BF16, G::kTok>(t_dk, t_dp, by_tokens, n != 0);
        mma_commit(&free_[stage]);
        if (more) {
          attn_mma_rows<D, BF16, G::kTok>(t_dp, v_desc, next_rows + (G::kStr >> 4));
          mma_commit(dp_full);
        } else {
          mma_commit(done);
        }
      }
      __syncwarp();
      stage = next_stage;
    }
    if (!ok) {
      s_abort = 1;
      if (issuer) { mma_commit(drain); mbar_wait_bounded(drain, 0); }
    }
  } else if (warp < G::kElem) {
    const int part = warp >> 2;                  // this warp's 32 queries of each tile
    const int key = k0 + (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = t_s + lanes + part * 32, dp_at = t_dp + lanes + part * 32;
    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = !s_abort && mbar_wait_bounded(bar, parity);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      return ok;
    };
    const bool table = p.delta == nullptr;
    if (table && items > 0) {
      float* at = reinterpret_cast<float*>(smem + L::kTable);
      attn_block_stats<D, BF16, G::kElem * 32>(p, batch, kv_head * group, 0, q_tiles * G::kTok, group * q_tiles * G::kTok, at, at + ADACONS_ATTN_SHORT_ROWS);
    }
    float by_ds = 1.f, by_dk = p.scale;            // from 2^shift P (dP - Delta) to what is rounded; from the sum to dK
    if constexpr (!BF16) {
      if (all > 0) {
        const float up = attn_ds_scale<D, G::kElem * 32>(p, batch, kv_head, kv_len);
        by_ds = up * kAttnUnshift<BF16>;
        by_dk = p.scale / up;
        if (threadIdx.x == 0) s_by_dk = by_dk;
      }
    }
    int stage = 0, in_head = items > 0 ? skip % per_head : 0, head_at = items > 0 ? skip / per_head * q_tiles * G::kTok : 0;
    uint32_t stage_parity = 0;
    for (int n = 0; n < items; ++n) {
      const int q0 = (first + in_head) * G::kTok + part * 32;
      const uint32_t place = table ? L::kTable + (head_at + q0) * 4 : L::kStats + stage * 2 * L::kStat + part * 128;
      if (++in_head == per_head) { in_head = 0; head_at += q_tiles * G::kTok; }
      const float4* lse2 = reinterpret_cast<const float4*>(smem + place);
      const float4* delta = reinterpret_cast<const float4*>(smem + place + (table ? 4 * ADACONS_ATTN_SHORT_ROWS : L::kStat));
      // key j is seen by query i when j < kv_len and j - off <= i
      const int from = key >= kv_len ? 0x7fffffff : p.causal ? key - off - q0 : 0;       // first column of this row that is not masked
      const int warp_from = k0 + (warp & 3) * 32 + 31 >= kv_len ? 0x7fffffff : p.causal ? key - lane + 31 - off - q0 : 0;
      if (!wait(&full[stage], stage_parity)) break;                  // the statistics are this thread's to read
      if (++stage == L::kStages) { stage = 0; stage_parity ^= 1u; }
      if (!wait(s_full, n & 1)) break;
      float pr[32];
      {
        uint32_t s[32];
        tmem_ld32(s_at, s);
        tmem_wait_ld();
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const float4 l = lse2[g];
          const float2 a = fma2(make_float2(__uint_as_float(s[4 * g]), __uint_as_float(s[4 * g + 1])), scale2, make_float2(-l.x, -l.y));
          const float2 b = fma2(make_float2(__uint_as_float(s[4 * g + 2]), __uint_as_float(s[4 * g + 3])), scale2, make_float2(-l.z, -l.w));
          pr[4 * g] = exp2_fast(a.x);
          pr[4 * g + 1] = exp2_fast(a.y);
          pr[4 * g + 2] = exp2_fast(b.x);
          pr[4 * g + 3] = exp2_fast(b.y);
        }
      }
      if (warp_from > 0) {
#pragma unroll
        for (int e = 0; e < 32; ++e) pr[e] = e >= from ? pr[e] : 0.f;
      }
      uint32_t w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) w[e] = pack16<BF16>(pr[2 * e], pr[2 * e + 1]);
      tmem_st16(s_at, w);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_one(p_full);
      if (!wait(dp_full, n & 1)) break;
      {
        uint32_t d[32];
        tmem_ld32(dp_at, d);
        tmem_wait_ld();
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const float4 l = delta[g];
          float2 a = add2(make_float2(__uint_as_float(d[4 * g]), __uint_as_float(d[4 * g + 1])), make_float2(-l.x, -l.y));
          float2 b = add2(make_float2(__uint_as_float(d[4 * g + 2]), __uint_as_float(d[4 * g + 3])), make_float2(-l.z, -l.w));
          if constexpr (!BF16) {
            a = mul2(a, make_float2(by_ds, by_ds));
            b = mul2(b, make_float2(by_ds, by_ds));
          }
          a = mul2(a, make_float2(pr[4 * g], pr[4 * g + 1]));
          b = mul2(b, make_float2(pr[4 * g + 2], pr[4 * g + 3]));
          w[2 * g] = pack16<BF16>(a.x, a.y);
          w[2 * g + 1] = pack16<BF16>(b.x, b.y);
        }
      }
      tmem_st16(dp_at, w);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_one(ds_full);
    }
    const bool live = key < p.Sk;
    // half of the warps for each gradient, 64 columns a warp
    constexpr int kShare = G::kParts / 2;
    const bool is_dv = part < kShare;
    const int columns = (part % kShare) * 64;
    const AttnOut& mine = is_dv ? p.dv : p.dk;
    if (items > 0) {
      if (ok) wait(done, 0);
      if (ok && p.key_split > 1) attn_keep_row<D, 2>(smem + (is_dv ? 0 : kAttnTile * D * 4), (is_dv ? t_dv : t_dk) + lanes, columns, (warp & 3) * 32 + lane);
      else if (ok) attn_store_row<2, BF16>(p, mine, (is_dv ? t_dv : t_dk) + lanes, columns, batch, kv_head, key, live, is_dv ? kAttnUnshift<BF16> : by_dk);
      else s_abort = 1;
    } else if (p.key_split == 1 && live && columns == 0) {
      attn_zero_row(p, mine, batch, kv_head, key);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (s_abort && threadIdx.x == 0) atomicOr(p.flags, kFlagTimeout);
  if (warp == G::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, G::kTmem);
  }
  if (p.key_split > 1) {
    const int shares = all == 0 ? 0 : (all + share - 1) / share;
    cluster_sync_all();
    attn_join_sum<D, BF16, G::kThreads>(p, p.dv, smem, rank, shares, k0, p.Sk, kv_head, batch, kAttnUnshift<BF16>);
    attn_join_sum<D, BF16, G::kThreads>(p, p.dk, smem + kAttnTile * D * 4, rank, shares, k0, p.Sk, kv_head, batch, BF16 || all == 0 ? p.scale : s_by_dk);
    cluster_sync_all();                          // the others may still read this block's share
  }
}

// ----------------------------------------------------------------------------------------------
// dQ.  A block owns 128 queries of one head and walks over the key tiles, recomputing S and dP: with
// seven products in all instead of five, but no sum across blocks (adding dQ from the key blocks would
// need fp32 atomics, whose order changes the result, or a pass over fp32 partial sums).
// Where the blocks of both kinds do not fill the device, those of a cluster share a tile's walk, as the forward's do
// (4000 queries on 200 keys 281 -> 47 us, 4000 x 4000 causal of 2 heads 106 -> 62 us).
// Tensor memory: S twice, dP, dQ.  S(j+1) and dP(j+1) run beside the elementwise phase of tile j, and
// dQ += dS(j) K(j), with dS in the place of S(j), beside that of tile j+1.
// ----------------------------------------------------------------------------------------------
template <int D> struct AttnDqSmem {
  using G = AttnBwd<D>;
  static constexpr int kKs = D == 128 ? 3 : 5, kVs = D == 128 ? 2 : 4;
  static constexpr uint32_t kK = 2 * G::kRes, kV = kK + kKs * G::kStr, kTable = kV + kVs * G::kStr, kBars = kTable + 2 * 4 * kAttnTile, kBytes = kBars + 256 + 1024;
};

template <int D, bool BF16, bool STARVE>
__device__ __forceinline__ void attn_dq_block(unsigned char* smem, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mdo,
                                              const AttnParams& p, const int tile, const int head, const int batch, const int rank) {
  using L = AttnDqSmem<D>;
  using G = AttnBwd<D>;
  uint64_t* q_full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* k_full = q_full + 1;                 // [kKs]
  uint64_t* k_free = k_full + L::kKs;            // [kKs]
  uint64_t* v_full = k_free + L::kKs;            // [kVs]
  uint64_t* v_free = v_full + L::kVs;            // [kVs]
  uint64_t* s_full = v_free + L::kVs;            // [2]
  uint64_t* dp_full = s_full + 2;
  uint64_t* dp_read = dp_full + 1;
  // two, by the parity of the tile: S and dP of the next tile do not wait for dS of this one, so the
  // warps could complete a second phase of a single barrier before its first has been looked at
  uint64_t* ds_full = dp_read + 1;
  uint64_t* done = ds_full + 2;
  uint64_t* drain = done + 1;
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  __shared__ float s_by_dq;                      // fp16 only
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int q0 = tile * kAttnTile;

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    for (int s = 0; s < L::kKs; ++s) { mbar_init(&k_full[s], 1); mbar_init(&k_free[s], 1); }
    for (int s = 0; s < L::kVs; ++s) { mbar_init(&v_full[s], 1); mbar_init(&v_free[s], 1); }
    mbar_init(&s_full[0], 1);
    mbar_init(&s_full[1], 1);
    mbar_init(dp_full, 1);
    mbar_init(dp_read, G::kElem);
    mbar_init(&ds_full[0], G::kElem);
    mbar_init(&ds_full[1], G::kElem);
    mbar_init(done, 1);
    mbar_init(drain, 1);
    s_abort = 0;
    mbar_init_fence();
    fence_proxy_async_smem();
  }
  if (warp == G::kMmaWarp) tmem_alloc(&s_tmem, G::kTmem);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const uint32_t t_dp = tmem + 2 * G::kTok, t_dq = t_dp + G::kTok;
  const int kv_len = attn_kv_len(p, batch);
  const int off = p.Sk - p.Sq;
  const int q_last = min(q0 + kAttnTile, p.Sq) - 1;
  const int seen = p.causal ? min(kv_len, max(0, q_last + off + 1)) : kv_len;
  const int all = (seen + G::kTok - 1) / G::kTok, share = (all + p.query_split - 1) / p.query_split;
  const int skip = min(rank * share, all), tiles = min(share, all - skip);       // this block's part of the walk
  pdl_wait();

  if (tiles > 0 && warp == G::kCopyWarp) {
    if (lane == 0) {
      mbar_expect_tx(q_full, 2 * G::kRes);
      G::load_resident(smem, &mq, q_full, q0, head, batch);
      G::load_resident(smem + G::kRes, &mdo, q_full, q0, head, batch);
      const int kv_head = head / (p.Hq / p.Hkv);
      int issued = 0;
      for (int j = 0; j < tiles; ++j) {
        if (STARVE && j == tiles - 1) break;
        const int ks = j % L::kKs, vs = j % L::kVs;
        if (s_abort || !mbar_wait_bounded(&k_free[ks], ((j / L::kKs) & 1) ^ 1)) { s_abort = 1; break; }
        mbar_expect_tx(&k_full[ks], G::kStr);
        attn_load_tile<D>(smem + L::kK + ks * G::kStr, &mk, &k_full[ks], (skip + j) * G::kTok, kv_head, batch);
        issued = 2 * j + 1;
        if (s_abort || !mbar_wait_bounded(&v_free[vs], ((j / L::kVs) & 1) ^ 1)) { s_abort = 1; break; }
        mbar_expect_tx(&v_full[vs], G::kStr);
        attn_load_tile<D>(smem + L::kV + vs * G::kStr, &mv, &v_full[vs], (skip + j) * G::kTok, kv_head, batch);
        issued = 2 * j + 2;
      }
      if (s_abort) {
        mbar_wait_bounded(q_full, 0);
        const int nk = (issued + 1) / 2, nv = issued / 2;
        for (int s = 0; s < L::kKs && s < nk; ++s) mbar_wait_bounded(&k_full[s], ((nk - 1 - s) / L::kKs) & 1);
        for (int s = 0; s < L::kVs && s < nv; ++s) mbar_wait_bounded(&v_full[s], ((nv - 1 - s) / L::kVs) & 1);
      }
    }
  } else if (tiles > 0 && warp == G::kMmaWarp) {
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = ok && !s_abort && mbar_wait_bounded(bar, parity);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      return ok;
    };
    const bool issuer = elect_one();
    const uint64_t q_desc = AttnDesc<D>::rows(smem_addr(smem)), do_desc = q_desc + (G::kRes >> 4);
    auto scores = [&](int j) {                   // S(j)
      const int ks = j % L::kKs;
      if (!wait(&k_full[ks], (j / L::kKs) & 1)) return;
      unsigned char* at = smem + L::kK + ks * G::kStr;
      if ((skip + j + 1) * G::kTok > kv_len) attn_zero_rows<D>(at, kv_len - (skip + j) * G::kTok, G::kTok);
      const uint64_t k_desc = AttnDesc<D>::rows(smem_addr(at));
      if (issuer) {
        attn_mma_rows<D, BF16, G::kTok>(tmem + (j & 1) * G::kTok, q_desc, k_desc);
        mma_commit(&s_full[j & 1]);
      }
      __syncwarp();
    };
    auto dprobs = [&](int j) {                   // dP(j)
      const int vs = j % L::kVs;
      if (!wait(&v_full[vs], (j / L::kVs) & 1)) return;
      unsigned char* at = smem + L::kV + vs * G::kStr;
      if ((skip + j + 1) * G::kTok > kv_len) attn_zero_rows<D>(at, kv_len - (skip + j) * G::kTok, G::kTok);
      const uint64_t v_desc = AttnDesc<D>::rows(smem_addr(at));
      if (issuer) {
        attn_mma_rows<D, BF16, G::kTok>(t_dp, do_desc, v_desc);
        mma_commit(dp_full);
        mma_commit(&v_free[vs]);
      }
      __syncwarp();
    };
    if (wait(q_full, 0)) {
      if (p.causal && q0 + off < 0) {            // queries that see no key, as on the key side
        attn_zero_rows<D>(smem, 0, -off - q0);
        attn_zero_rows<D>(smem + G::kRes, 0, -off - q0);
      }
      scores(0);
      if (ok) dprobs(0);
    }
    for (int j = 0; ok && j < tiles; ++j) {
      if (j + 1 < tiles) {
        scores(j + 1);
        if (!ok || !wait(dp_read, j & 1)) break;
        dprobs(j + 1);
        if (!ok) break;
      }
      if (!wait(&ds_full[j & 1], (j >> 1) & 1)) break;
      const uint64_t k_desc = AttnDesc<D>::tokens(smem_addr(smem) + L::kK + (j % L::kKs) * G::kStr);
      if (issuer) {
        attn_mma_tokens<D, BF16, G::kTok>(t_dq, tmem + (j & 1) * G::kTok, k_desc, j != 0);
        mma_commit(&k_free[j % L::kKs]);
        if (j == tiles - 1) mma_commit(done);
      }
      __syncwarp();
    }
    if (!ok) {
      s_abort = 1;
      if (issuer) { mma_commit(drain); mbar_wait_bounded(drain, 0); }
    }
  } else if (warp < G::kElem) {
    const int part = warp >> 2;                  // this warp's 32 keys of each tile
    const int row = q0 + (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    float lse2 = INFINITY, delta = 0.f;
    if (p.delta != nullptr) {
      const long long stat = (static_cast<long long>(batch) * p.Hq + head) * p.sq_pad + row;    // rows are padded: always there
      lse2 = p.lse2[stat];
      delta = p.delta[stat];
    } else if (tiles > 0) {
      float* at = reinterpret_cast<float*>(smem + L::kTable);
      attn_block_stats<D, BF16, G::kElem * 32>(p, batch, head, q0, kAttnTile, kAttnTile, at, at + kAttnTile);
      lse2 = at[row - q0];
      delta = at[kAttnTile + row - q0];
    }
    float by_ds = 1.f, by_dq = p.scale;
    if constexpr (!BF16) {
      if (all > 0) {
        const float up = attn_ds_scale<D, G::kElem * 32>(p, batch, head / (p.Hq / p.Hkv), kv_len);
        by_ds = up * kAttnUnshift<BF16>;
        by_dq = p.scale / up;
        if (threadIdx.x == 0) s_by_dq = by_dq;
      }
    }
    const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), lse22 = make_float2(-lse2, -lse2), delta2 = make_float2(-delta * by_ds, -delta * by_ds);
    const int limit = p.causal ? min(kv_len, row + off + 1) : kv_len;
    const int warp_limit = p.causal ? min(kv_len, row - lane + off + 1) : kv_len;
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      ok = !s_abort && mbar_wait_bounded(bar, parity);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      return ok;
    };
    for (int j = 0; j < tiles; ++j) {
      const uint32_t s_at = tmem + (j & 1) * G::kTok + lanes + part * 32, dp_at = t_dp + lanes + part * 32;
      const int k0 = (skip + j) * G::kTok + part * 32;
      if (!wait(&s_full[j & 1], (j >> 1) & 1)) break;
      float pr[32];
      {
        uint32_t s[32];
        tmem_ld32(s_at, s);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 a = fma2(make_float2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), scale2, lse22);
          pr[e] = exp2_fast(a.x);
          pr[e + 1] = exp2_fast(a.y);
        }
      }
      if (k0 + 32 > warp_limit) {
#pragma unroll
        for (int e = 0; e < 32; ++e) pr[e] = k0 + e < limit ? pr[e] : 0.f;
      }
      if (!wait(dp_full, j & 1)) break;
      uint32_t w[16];
      {
        uint32_t d[32];
        tmem_ld32(dp_at, d);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_one(dp_read);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float2 dp = make_float2(__uint_as_float(d[2 * e]), __uint_as_float(d[2 * e + 1]));
          const float2 a = mul2(BF16 ? add2(dp, delta2) : fma2(dp, make_float2(by_ds, by_ds), delta2), make_float2(pr[2 * e], pr[2 * e + 1]));
          w[e] = pack16<BF16>(a.x, a.y);
        }
      }
      tmem_st16(s_at, w);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_one(&ds_full[j & 1]);
    }
    const bool live = row < p.Sq;
    if (tiles > 0) {
      if (ok) wait(done, 0);
      if (p.query_split > 1) {
        if (ok && part < D / 64) attn_keep_row<D, 2>(smem, t_dq + lanes, part * 64, row - q0);
      } else if (ok && part < D / 64) attn_store_row<2, BF16>(p, p.out, t_dq + lanes, part * 64, batch, head, row, live, by_dq);
      if (!ok) s_abort = 1;
    } else if (p.query_split == 1 && live && part == 0) {
      attn_zero_row(p, p.out, batch, head, row);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (s_abort && threadIdx.x == 0) atomicOr(p.flags, kFlagTimeout);
  if (warp == G::kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, G::kTmem);
  }
  if (p.query_split > 1) {
    cluster_sync_all();
    attn_join_sum<D, BF16, G::kThreads>(p, p.out, smem, rank, all == 0 ? 0 : (all + share - 1) / share, q0, p.Sq, head, batch, BF16 || all == 0 ? p.scale : s_by_dq);
    cluster_sync_all();
  }
}

// Both in one launch: the key blocks first (four products a tile and, with shared heads, several query
// heads), the query blocks fill the device as those run out.  With a causal mask the first keys have the
// most queries and the last queries the most keys: long blocks first in either part, all heads of one tile together.
template <int D> constexpr uint32_t attn_backward_smem() { return AttnDkvSmem<D>::kBytes > AttnDqSmem<D>::kBytes ? AttnDkvSmem<D>::kBytes : AttnDqSmem<D>::kBytes; }

template <int D, bool BF16, bool STARVE = false>
__global__ void __launch_bounds__(AttnBwd<D>::kThreads, AttnBwd<D>::kBlocks)
attn_backward_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                     const __grid_constant__ CUtensorMap mdo, const AttnParams p, const int key_blocks, const int q_tiles) {
  extern __shared__ unsigned char smem_dyn[];
  unsigned char* smem = smem_dyn + ((1024u - (smem_addr(smem_dyn) & 1023u)) & 1023u);
  int n = blockIdx.x;
  if (n < key_blocks) {
    const int heads = p.Hkv * p.B, unit = n / p.key_split, tile = unit / heads, rank = n % p.key_split;
    if (tile * kAttnTile >= p.Sk) return;        // rounds the key blocks up to whole clusters
    n = unit - tile * heads;
    attn_dkv_block<D, BF16, STARVE>(smem, mq, mk, mv, mdo, p, tile, n % p.Hkv, n / p.Hkv, rank);
  } else {
    n -= key_blocks;
    const int heads = p.Hq * p.B, unit = n / p.query_split, tile = unit / heads, rank = n % p.query_split;
    if (tile >= q_tiles) return;
    n = unit - tile * heads;
    attn_dq_block<D, BF16, STARVE>(smem, mq, mk, mv, mdo, p, q_tiles - 1 - tile, n % p.Hq, n / p.Hq, rank);
  }
}

}  // namespace adacons
