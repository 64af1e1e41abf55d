// Norms before and after a block with its gate and the residual addition: kernels (sm_100a).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "adacons_common.cuh"

namespace adacons {

// ----------------------------------------------------------------------------------------------
// Rows of D elements: the residual stream x, a block's output f, the block's gate a, gains `post` and `pre`.
//     n = f r_f,   r_f = (mean f^2 + eps)^-1/2          (without `post`: n = f and no factor)
//     x' = x + scale act(a) n post
//     h = x' r_x pre,   r_x = (mean x'^2 + eps)^-1/2
// and back, with xh = x' r_x, c = scale act(a):
//     t = dx' + r_x (dh pre - xh mean(dh pre xh))        = dx
//     df = r_f (c t post - n mean(c t post n)),   da = scale act'(a) t n post
//     dpost = sum c t n,   dpre = sum dh xh
// A gate is one row for all tokens (channel), one for each sequence, or one for each token.  The first two
// leave sums over tokens: with s = sum t n over the tokens that share a gate row, dpost and da are
// both s times something that does not depend on the token, so one running sum per column serves both.
//
// Bound by memory: every element is read and written once.  A row belongs to `tpr` threads (a warp up to 256 elements, 512 threads
// from 2049 on), each with kNormN elements of every kNormN * tpr; a block keeps its gains in registers, walks over
// its rows and has the next row's loads under way while it adds up this one's (D up to 4096; beyond, there are no registers
// for it).  Means are sums in fp32 by shuffles and one shared-memory exchange, in a fixed order.
// The sums over tokens are kept in registers by every thread for its columns, leave as one record per block, and a second
// launch adds the records in order: no atomics.
// ----------------------------------------------------------------------------------------------
constexpr int kNormN = 8;                       // elements of a thread's group: 16 bytes of 16-bit values
constexpr int kNormMaxDim = 16384;
constexpr int kNormSumThreads = 1024;           // of the second launch: 32 columns, 32 shares of the records

enum NormGate { kGateNone = 0, kGateChannel = 1, kGateSequence = 2, kGateToken = 3 };
enum NormBy { kByItself = 0, kBySigmoid = 1, kByTanh = 2 };

template <typename T> struct NormPair;
template <> struct NormPair<__nv_bfloat16> {
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2_rn(a, b); }
};
template <> struct NormPair<__half> {
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <typename T> __device__ __forceinline__ float norm_float(T v) { return static_cast<float>(v); }
template <typename T> __device__ __forceinline__ T norm_round(float v);
template <> __device__ __forceinline__ float norm_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 norm_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half norm_round<__half>(float v) { return __float2half_rn(v); }

// A thread's share of a row, as it lies in memory: vectors of 16 bytes, or (VEC false) single elements.
template <typename T, bool VEC> struct NormRaw {
  static constexpr int kVectors = sizeof(T) / 2;               // fp32: two of them
  uint4 v[kVectors];
  __device__ __forceinline__ void load(const T* row, int col) {
#pragma unroll
    for (int k = 0; k < kVectors; ++k) v[k] = *reinterpret_cast<const uint4*>(row + col + k * (16 / static_cast<int>(sizeof(T))));
  }
  __device__ __forceinline__ void get(float (&f)[kNormN]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        f[4 * k] = __uint_as_float(v[k].x); f[4 * k + 1] = __uint_as_float(v[k].y);
        f[4 * k + 2] = __uint_as_float(v[k].z); f[4 * k + 3] = __uint_as_float(v[k].w);
      }
    } else {
      const uint32_t u[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 p = NormPair<T>::unpack(u[k]);
        f[2 * k] = p.x;
        f[2 * k + 1] = p.y;
      }
    }
  }
};
template <typename T> struct NormRaw<T, false> {
  T v[kNormN];
};

// Where a thread's elements are: group c is kNormN neighbours (VEC), or kNormN elements tpr apart.
template <bool VEC>
struct NormColumns {
  int tpr, t, dim;
  __device__ __forceinline__ int at(int c, int e) const { return VEC ? (c * tpr + t) * kNormN + e : (c * kNormN + e) * tpr + t; }
  __device__ __forceinline__ bool has(int c) const { return !VEC || (c * tpr + t) * kNormN < dim; }
};

template <typename T, bool VEC>
__device__ __forceinline__ void norm_fetch(NormRaw<T, VEC>& raw, const T* row, const NormColumns<VEC>& cols, int c) {
  if constexpr (VEC) {
    if (cols.has(c)) raw.load(row, cols.at(c, 0));
    else
#pragma unroll
      for (int k = 0; k < NormRaw<T, true>::kVectors; ++k) raw.v[k] = make_uint4(0u, 0u, 0u, 0u);
  } else {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) {
      const int col = cols.at(c, e);
      raw.v[e] = col < cols.dim ? row[col] : norm_round<T>(0.f);
    }
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void norm_get(const NormRaw<T, VEC>& raw, float (&f)[kNormN]) {
  if constexpr (VEC) raw.get(f);
  else
#pragma unroll
    for (int e = 0; e < kNormN; ++e) f[e] = norm_float(raw.v[e]);
}
template <typename T, bool VEC>
__device__ __forceinline__ void norm_load(float (&f)[kNormN], const T* row, const NormColumns<VEC>& cols, int c) {
  NormRaw<T, VEC> raw;
  norm_fetch(raw, row, cols, c);
  norm_get(raw, f);
}
template <typename T, bool VEC>
__device__ __forceinline__ void norm_store(T* row, const NormColumns<VEC>& cols, int c, const float (&f)[kNormN]) {
  if constexpr (VEC) {
    if (!cols.has(c)) return;
    T* to = row + cols.at(c, 0);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) *reinterpret_cast<float4*>(to + 4 * k) = make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]);
    } else {
      *reinterpret_cast<uint4*>(to) = make_uint4(NormPair<T>::pack(f[0], f[1]), NormPair<T>::pack(f[2], f[3]), NormPair<T>::pack(f[4], f[5]), NormPair<T>::pack(f[6], f[7]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) {
      const int col = cols.at(c, e);
      if (col < cols.dim) row[col] = norm_round<T>(f[e]);
    }
  }
}

// Gains and gates are fp32 or of the block's type, whichever the caller keeps them in.
struct NormGain {
  const void* data;
  int wide;                                     // fp32
};
template <typename T, bool VEC>
__device__ __forceinline__ void norm_gain(float (&f)[kNormN], const NormGain& g, long long at, const NormColumns<VEC>& cols, int c) {
  if (g.wide) norm_load<float, VEC>(f, static_cast<const float*>(g.data) + at, cols, c);
  else norm_load<T, VEC>(f, static_cast<const T*>(g.data) + at, cols, c);
}
template <typename T> __device__ __forceinline__ float norm_gain_one(const NormGain& g, long long at) {
  return g.wide ? static_cast<const float*>(g.data)[at] : norm_float(static_cast<const T*>(g.data)[at]);
}

__device__ __forceinline__ float norm_act(int by, float a) {
  if (by == kBySigmoid) return 1.f / (1.f + expf(-a));
  if (by == kByTanh) return tanhf(a);
  return a;
}
// the derivative, without the cancellation of 1 - tanh^2 far out
__device__ __forceinline__ float norm_slope(int by, float a) {
  if (by == kBySigmoid) {
    const float e = expf(-fabsf(a)), d = 1.f / (1.f + e);
    return e * d * d;
  }
  if (by == kByTanh) {
    const float e = expf(-2.f * fabsf(a)), d = 1.f / (1.f + e);
    return 4.f * e * d * d;
  }
  return 1.f;
}

struct NormRows {                               // a tensor of (batch, token) rows: strides in elements
  void* data;
  long long batch, row;
};
struct NormDivisor {                            // n / d for 0 <= n < 2^31, as in the rotary kernel
  unsigned m;
  int s;
  __device__ __forceinline__ int divide(int n) const { return static_cast<int>((static_cast<unsigned long long>(static_cast<unsigned>(n)) * m) >> (31 + s)); }
};

struct NormParams {
  NormRows x, f, gate, out, normed;             // forward: out is x'
  NormRows dout, dnormed, dx, df, dgate;        // backward: `out` is read
  NormGain gate_as, post, pre;                  // gate_as: type of the gate; its rows are in `gate`
  float* rows;                                  // [2][tokens]: r_f, r_x
  void *dpost, *dpre;                           // of the gains' types
  float *sums, *pre_sums;                       // records: [items][dim], [blocks][dim]
  long long tokens;
  int len, dim, tpr;
  int gate_kind, by;
  int groups, parts;                            // backward: sequences that have a gate row of their own (or 1), and blocks' shares of each
  int blocks;
  float scale, eps;
  NormDivisor by_len;
};

template <typename T>
__device__ __forceinline__ T* norm_row(const NormRows& r, int b, int s) { return static_cast<T*>(r.data) + b * r.batch + s * r.row; }

// Sum over the threads of a row.  `slot` alternates, so that one barrier a sum is enough.
struct NormSum {
  float* shared;                                // [2][warps of the block]
  int tpr, group, slot;
  __device__ __forceinline__ float operator()(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (tpr == 32) return v;
    float* at = shared + slot * 32;
    slot ^= 1;
    if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(tpr) : "memory");
    const int first = group * (tpr >> 5);
    v = 0.f;
    for (int w = 0; w < (tpr >> 5); ++w) v += at[first + w];
    return v;
  }
};

// C: groups of a thread.  Blocks of 256 threads, or of 512 where a row takes as many.
template <typename X, typename F, int C, bool VEC>
__global__ void __launch_bounds__(512, C == 1 ? 2 : 1) norm_forward_kernel(const NormParams p) {
  __shared__ float s_sum[64];
  const int group = threadIdx.x / p.tpr, per_block = blockDim.x / p.tpr;
  const NormColumns<VEC> cols = {p.tpr, static_cast<int>(threadIdx.x) - group * p.tpr, p.dim};
  NormSum sum = {s_sum, p.tpr, group, 0};
  const bool has_f = p.f.data != nullptr, has_post = p.post.data != nullptr, has_pre = p.pre.data != nullptr;
  const bool gate_rows = p.gate_kind >= kGateSequence;
  constexpr bool kHold = C <= 2;                // gains in registers
  float factor[kHold ? C : 1][kNormN], gain[kHold ? C : 1][kNormN];
  // scale act(channel gate) post: what n is multiplied by, but for a gate's rows
  auto factors = [&](int c, float (&to)[kNormN]) {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) to[e] = p.scale;
    if (p.gate_kind == kGateChannel) {
      float a[kNormN];
      norm_gain<F, VEC>(a, {p.gate.data, p.gate_as.wide}, 0, cols, c);
#pragma unroll
      for (int e = 0; e < kNormN; ++e) to[e] *= norm_act(p.by, a[e]);
    }
    if (has_post) {
      float w[kNormN];
      norm_gain<F, VEC>(w, p.post, 0, cols, c);
#pragma unroll
      for (int e = 0; e < kNormN; ++e) to[e] *= w[e];
    }
  };
  if (kHold) {
#pragma unroll
    for (int c = 0; c < (kHold ? C : 0); ++c) {
      if (has_f) factors(c, factor[c]);
      if (has_pre) norm_gain<F, VEC>(gain[c], p.pre, 0, cols, c);
    }
  }
  const long long step = static_cast<long long>(gridDim.x) * per_block;
  long long at = static_cast<long long>(blockIdx.x) * per_block + group;
  NormRaw<X, VEC> next_x[C];
  NormRaw<F, VEC> next_f[C];
  auto fetch = [&](long long r) {
    const int b = p.by_len.divide(static_cast<int>(r)), s = static_cast<int>(r) - b * p.len;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      norm_fetch(next_x[c], static_cast<const X*>(norm_row<X>(p.x, b, s)), cols, c);
      if (has_f) norm_fetch(next_f[c], static_cast<const F*>(norm_row<F>(p.f, b, s)), cols, c);
    }
  };
  if (C == 1 && at < p.tokens) fetch(at);
  for (; at < p.tokens; at += step) {
    const int row = static_cast<int>(at), b = p.by_len.divide(row), s = row - b * p.len;
    if (C > 1) fetch(at);
    float x[C][kNormN], f[C][kNormN];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      norm_get(next_x[c], x[c]);
      if (has_f) norm_get(next_f[c], f[c]);
    }
    if (C == 1 && at + step < p.tokens) fetch(at + step);
    if (has_f) {
      float r = 1.f;
      if (has_post) {
        float square = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < kNormN; ++e) square = fmaf(f[c][e], f[c][e], square);
        r = rsqrtf(sum(square) / p.dim + p.eps);
      }
      if (cols.t == 0) p.rows[row] = has_post ? r : 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float by[kNormN];
        if (kHold) {
#pragma unroll
          for (int e = 0; e < kNormN; ++e) by[e] = factor[kHold ? c : 0][e];
        } else {
          factors(c, by);
        }
        if (gate_rows) {
          float a[kNormN];
          norm_gain<F, VEC>(a, {p.gate.data, p.gate_as.wide}, b * p.gate.batch + s * p.gate.row, cols, c);
#pragma unroll
          for (int e = 0; e < kNormN; ++e) by[e] *= norm_act(p.by, a[e]);
        }
#pragma unroll
        for (int e = 0; e < kNormN; ++e) x[c][e] = fmaf(f[c][e] * r, by[e], x[c][e]);
        norm_store(norm_row<X>(p.out, b, s), cols, c, x[c]);
      }
    }
    if (cols.t == 0 && !has_f) p.rows[row] = 0.f;
    if (cols.t == 0 && !has_pre) p.rows[p.tokens + row] = 0.f;
    if (has_pre) {
      float square = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < kNormN; ++e) square = fmaf(x[c][e], x[c][e], square);
      const float r = rsqrtf(sum(square) / p.dim + p.eps);
      if (cols.t == 0) p.rows[p.tokens + row] = r;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float w[kNormN];
        if (kHold) {
#pragma unroll
          for (int e = 0; e < kNormN; ++e) w[e] = gain[kHold ? c : 0][e];
        } else {
          norm_gain<F, VEC>(w, p.pre, 0, cols, c);
        }
#pragma unroll
        for (int e = 0; e < kNormN; ++e) w[e] *= x[c][e] * r;
        norm_store(norm_row<F>(p.normed, b, s), cols, c, w);
      }
    }
  }
}

// A block's item is a run of tokens of one group (of all tokens where no sequence has a gate of its own): its sums of t n leave as
// record `item`; the sums for `pre` leave once, as record `block`.
template <typename X, typename F, int C, bool VEC>
__global__ void __launch_bounds__(512, 1) norm_backward_kernel(const NormParams p) {
  extern __shared__ float s_fold[];             // [threads][kNormN] where rows are shorter than a block
  __shared__ float s_sum[64];
  pdl_launch_dependents();
  const int group = threadIdx.x / p.tpr, per_block = blockDim.x / p.tpr;
  const NormColumns<VEC> cols = {p.tpr, static_cast<int>(threadIdx.x) - group * p.tpr, p.dim};
  NormSum sum = {s_sum, p.tpr, group, 0};
  const bool has_f = p.f.data != nullptr, has_post = p.post.data != nullptr, has_pre = p.pre.data != nullptr && p.dnormed.data != nullptr;
  const bool gate_rows = p.gate_kind >= kGateSequence, wants_sum = p.sums != nullptr;
  constexpr bool kHold = C == 1;                // gains in registers
  float held_pre[kNormN], held_post[kNormN], held_by[kNormN];
  auto pre_of = [&](int c, float (&to)[kNormN]) {
    if (!kHold) norm_gain<F, VEC>(to, p.pre, 0, cols, c);
    else
#pragma unroll
      for (int e = 0; e < kNormN; ++e) to[e] = held_pre[e];
  };
  auto make_by = [&](int c, float (&to)[kNormN]) {       // scale act(channel gate)
#pragma unroll
    for (int e = 0; e < kNormN; ++e) to[e] = p.scale;
    if (p.gate_kind != kGateChannel) return;
    float a[kNormN];
    norm_gain<F, VEC>(a, {p.gate.data, p.gate_as.wide}, 0, cols, c);
#pragma unroll
    for (int e = 0; e < kNormN; ++e) to[e] *= norm_act(p.by, a[e]);
  };
  auto post_of = [&](int c, float (&to)[kNormN]) {
    if (kHold) {
#pragma unroll
      for (int e = 0; e < kNormN; ++e) to[e] = held_post[e];
    } else if (has_post) {
      norm_gain<F, VEC>(to, p.post, 0, cols, c);
    } else {
#pragma unroll
      for (int e = 0; e < kNormN; ++e) to[e] = 1.f;
    }
  };
  if (kHold) {
    if (has_pre) norm_gain<F, VEC>(held_pre, p.pre, 0, cols, 0);
#pragma unroll
    for (int e = 0; e < kNormN; ++e) held_post[e] = 1.f;
    if (has_post) norm_gain<F, VEC>(held_post, p.post, 0, cols, 0);
    if (has_f) make_by(0, held_by);
  }
  float acc[C][kNormN], acc_pre[C][kNormN];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int e = 0; e < kNormN; ++e) acc[c][e] = acc_pre[c][e] = 0.f;

  NormRaw<X, VEC> next_dout[C], next_out[C];
  NormRaw<F, VEC> next_dh[C], next_f[C];
  float next_rf = 1.f, next_rx = 1.f;
  auto fetch = [&](int r) {
    const int b = p.by_len.divide(r), s = r - b * p.len;
    if (has_post) next_rf = p.rows[r];
    if (has_pre) next_rx = p.rows[p.tokens + r];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (p.dout.data != nullptr) norm_fetch(next_dout[c], static_cast<const X*>(norm_row<X>(p.dout, b, s)), cols, c);
      if (has_pre) {
        norm_fetch(next_out[c], static_cast<const X*>(norm_row<X>(p.out, b, s)), cols, c);
        norm_fetch(next_dh[c], static_cast<const F*>(norm_row<F>(p.dnormed, b, s)), cols, c);
      }
      if (has_f) norm_fetch(next_f[c], static_cast<const F*>(norm_row<F>(p.f, b, s)), cols, c);
    }
  };
  // the threads that have the same columns in a block's other rows add up, in the rows' order
  auto leave = [&](float (&a)[C][kNormN], float* record) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (per_block > 1) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kNormN; ++e) s_fold[e * blockDim.x + threadIdx.x] = a[c][e];
        __syncthreads();
      }
      if (group == 0) {
#pragma unroll
        for (int e = 0; e < kNormN; ++e) {
          float v = a[c][e];
          for (int g = 1; g < per_block; ++g) v += s_fold[e * blockDim.x + g * p.tpr + threadIdx.x];
          const int col = cols.at(c, e);
          if (col < p.dim) record[col] = v;
        }
      }
#pragma unroll
      for (int e = 0; e < kNormN; ++e) a[c][e] = 0.f;
    }
  };

  const int items = p.groups * p.parts;
  const long long of_group = p.tokens / p.groups;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int g = item / p.parts, part = item - g * p.parts;
    const long long share = (of_group + p.parts - 1) / p.parts;
    const long long begin = g * of_group + min(of_group, part * share), end = g * of_group + min(of_group, (part + 1) * share);
    long long at = begin + group;
    if (C == 1 && at < end) fetch(static_cast<int>(at));
    for (; at < end; at += per_block) {
      const int row = static_cast<int>(at), b = p.by_len.divide(row), s = row - b * p.len;
      if (C > 1) fetch(row);
      float t[C][kNormN];
      const float rf = next_rf, rx = next_rx;
      NormRaw<F, VEC> f_raw[C];
      float hat[C][kNormN], a[C][kNormN];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (p.dout.data != nullptr) norm_get(next_dout[c], t[c]);
        else
#pragma unroll
          for (int e = 0; e < kNormN; ++e) t[c][e] = 0.f;
        if (has_pre) {
          norm_get(next_out[c], hat[c]);
          norm_get(next_dh[c], a[c]);
        }
        f_raw[c] = next_f[c];
      }
      if (C == 1 && at + per_block < end) fetch(static_cast<int>(at + per_block));
      if (has_pre) {
        float inner = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          float w[kNormN];
          pre_of(c, w);
#pragma unroll
          for (int e = 0; e < kNormN; ++e) {
            hat[c][e] *= rx;
            acc_pre[c][e] = fmaf(a[c][e], hat[c][e], acc_pre[c][e]);
            a[c][e] *= w[e];
            inner = fmaf(a[c][e], hat[c][e], inner);
          }
        }
        inner = sum(inner) / p.dim;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < kNormN; ++e) t[c][e] = fmaf(rx, fmaf(-hat[c][e], inner, a[c][e]), t[c][e]);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) norm_store(norm_row<X>(p.dx, b, s), cols, c, t[c]);
      if (!has_f) continue;
      // t becomes c t post, `hat` n
      float inner = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float n[kNormN], by[kNormN], w[kNormN];
        norm_get(f_raw[c], n);
        post_of(c, w);
        if (kHold)
#pragma unroll
          for (int e = 0; e < kNormN; ++e) by[e] = held_by[e];
        else make_by(c, by);
        if (has_post)
#pragma unroll
          for (int e = 0; e < kNormN; ++e) n[e] *= rf;
        if (gate_rows) {
          float g_in[kNormN], dg[kNormN];
          norm_gain<F, VEC>(g_in, {p.gate.data, p.gate_as.wide}, b * p.gate.batch + s * p.gate.row, cols, c);
#pragma unroll
          for (int e = 0; e < kNormN; ++e) {
            by[e] *= norm_act(p.by, g_in[e]);
            dg[e] = p.scale * norm_slope(p.by, g_in[e]) * t[c][e] * n[e] * w[e];
          }
          if (p.gate_kind == kGateToken) {
            if (p.gate_as.wide) norm_store(norm_row<float>(p.dgate, b, s), cols, c, dg);
            else norm_store(norm_row<F>(p.dgate, b, s), cols, c, dg);
          }
        }
        const bool by_token = p.gate_kind == kGateToken;         // its factor differs from token to token: it goes into the sum
#pragma unroll
        for (int e = 0; e < kNormN; ++e) {
          const float tn = t[c][e] * n[e];
          acc[c][e] = fmaf(by_token ? by[e] : 1.f, tn, acc[c][e]);
          t[c][e] *= by[e] * w[e];
          inner = fmaf(t[c][e], n[e], inner);
          hat[c][e] = n[e];
        }
      }
      if (has_post) {
        inner = sum(inner) / p.dim;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < kNormN; ++e) t[c][e] = rf * fmaf(-hat[c][e], inner, t[c][e]);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) norm_store(norm_row<F>(p.df, b, s), cols, c, t[c]);
    }
    if (wants_sum) leave(acc, p.sums + static_cast<long long>(item) * p.dim);
  }
  if (p.pre_sums != nullptr) leave(acc_pre, p.pre_sums + static_cast<long long>(blockIdx.x) * p.dim);
}

// dpost, dpre and the gate's gradient (channel, sequence) from the records: 32 columns a block, whose 32 warps take
// the records in turn and add their shares in order.  A sequence's records are one warp's.
template <typename F>
__global__ void __launch_bounds__(kNormSumThreads) norm_sum_kernel(const NormParams p) {
  __shared__ float s_part[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const bool in = col < p.dim;
  auto total = [&](float v) {                   // over the warps; valid in warp 0
    __syncthreads();
    s_part[warp][lane] = v;
    __syncthreads();
    v = 0.f;
    if (warp == 0)
#pragma unroll
      for (int w = 0; w < 32; ++w) v += s_part[w][lane];
    return v;
  };
  auto put = [&](void* to, bool wide, long long at, float v) {
    if (wide) static_cast<float*>(to)[at] = v;
    else static_cast<F*>(to)[at] = norm_round<F>(v);
  };
  const float post = in && p.post.data != nullptr ? norm_gain_one<F>(p.post, col) : 1.f;
  if (p.sums != nullptr) {
    float v = 0.f;
    if (p.gate_kind == kGateSequence) {
      for (int g = warp; in && g < p.groups; g += 32) {
        float s = 0.f;
#pragma unroll 4
        for (int k = 0; k < p.parts; ++k) s += p.sums[(static_cast<long long>(g) * p.parts + k) * p.dim + col];
        const float a = norm_gain_one<F>({p.gate.data, p.gate_as.wide}, g * p.gate.batch + col);
        v = fmaf(p.scale * norm_act(p.by, a), s, v);
        put(p.dgate.data, p.gate_as.wide, g * p.dgate.batch + col, p.scale * norm_slope(p.by, a) * post * s);
      }
      v = total(v);
    } else {
#pragma unroll 8
      for (int k = warp; k < p.parts; k += 32)
        if (in) v += p.sums[static_cast<long long>(k) * p.dim + col];
      v = total(v);
      if (p.gate_kind == kGateChannel && in && warp == 0) {
        const float a = norm_gain_one<F>({p.gate.data, p.gate_as.wide}, col);
        put(p.dgate.data, p.gate_as.wide, col, p.scale * norm_slope(p.by, a) * post * v);
        v *= p.scale * norm_act(p.by, a);
      } else if (p.gate_kind == kGateNone) {
        v *= p.scale;
      }
    }
    if (p.dpost != nullptr && in && warp == 0) put(p.dpost, p.post.wide, col, v);
  }
  if (p.dpre != nullptr) {
    float v = 0.f;
    if (p.pre_sums != nullptr)
#pragma unroll 8
      for (int k = warp; k < p.blocks; k += 32)
        if (in) v += p.pre_sums[static_cast<long long>(k) * p.dim + col];
    v = total(v);
    if (in && warp == 0) put(p.dpre, p.pre.wide, col, v);
  }
}

}  // namespace adacons
