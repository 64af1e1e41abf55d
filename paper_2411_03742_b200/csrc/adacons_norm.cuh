// Norms before and after a block with its gate and the residual addition: kernels (sm_100a).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "adacons_tc.cuh"

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
// Bound by memory: every element is read and written once.  A block of 512 threads, one an SM, holds one row or several: a row belongs to `tpr` of them, each with one or
// two groups of kNormN neighbours (a warp up to 512 elements, 256 threads for 4096).  The gradient at 4096 elements, fp32 stream, 32,768 tokens: 0.51 ms, 4.7 TB/s; when every fp32 sector was asked for
// twice (see norm_ask) 0.56, and then with one group and 1024 threads 0.91 (the instructions around 8 elements are more than for them), with four groups and 256 threads 0.57;
// forward, bf16, 0.27 ms, 0.31 and 0.34.  What holds it below the copy rate, 6.6 TB/s, is that a row's loads go out in one burst, 4300 to 5000 of its 10,000 cycles: asked for
// piece by piece between the sums they come too late (0.62), rows brought into L2 before do not help (0.60), nor does one exchange for both sums (0.51).  The gains lie in shared memory as fp32, multiplied with
// what else does not change.  The next rows are on their way meanwhile, by asynchronous copies of 16 bytes into places of shared memory that only threads
// of the same warp read, so that nothing waits for another warp (D up to 8192; beyond, a row fills shared memory, and
// rows of odd sizes or strides are loaded element by element).  Means are sums in fp32 by shuffles and one shared-memory exchange, in a fixed order.
// The sums over tokens are kept in registers by every thread for its columns, leave as one record per block, and a second
// launch adds the records in order: no atomics.
// ----------------------------------------------------------------------------------------------
constexpr int kNormThreads = 512;
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

// A group of a thread's elements as pairs: B200 has additions, multiplications and multiply-adds of two fp32 values.
struct Norm8 {
  float2 p[kNormN / 2];
  __device__ __forceinline__ float& operator[](int e) { return e & 1 ? p[e / 2].y : p[e / 2].x; }
  __device__ __forceinline__ float operator[](int e) const { return e & 1 ? p[e / 2].y : p[e / 2].x; }
};
__device__ __forceinline__ Norm8 norm_all(float v) {
  Norm8 r;
#pragma unroll
  for (int k = 0; k < kNormN / 2; ++k) r.p[k] = make_float2(v, v);
  return r;
}
__device__ __forceinline__ Norm8 operator*(const Norm8& a, const Norm8& b) {
  Norm8 r;
#pragma unroll
  for (int k = 0; k < kNormN / 2; ++k) r.p[k] = mul2(a.p[k], b.p[k]);
  return r;
}
__device__ __forceinline__ Norm8 operator*(const Norm8& a, float b) { return a * norm_all(b); }
__device__ __forceinline__ Norm8 operator+(const Norm8& a, const Norm8& b) {
  Norm8 r;
#pragma unroll
  for (int k = 0; k < kNormN / 2; ++k) r.p[k] = add2(a.p[k], b.p[k]);
  return r;
}
__device__ __forceinline__ Norm8 norm_fma(const Norm8& a, const Norm8& b, const Norm8& c) {
  Norm8 r;
#pragma unroll
  for (int k = 0; k < kNormN / 2; ++k) r.p[k] = fma2(a.p[k], b.p[k], c.p[k]);
  return r;
}
__device__ __forceinline__ Norm8 norm_fma(const Norm8& a, float b, const Norm8& c) { return norm_fma(a, norm_all(b), c); }
__device__ __forceinline__ float norm_fold(const Norm8& a) {
  const float2 s = add2(add2(a.p[0], a.p[1]), add2(a.p[2], a.p[3]));
  return s.x + s.y;
}

// A thread's share of a row, as it lies in memory: vectors of 16 bytes, or (VEC false) single elements.
template <typename T, bool VEC> struct NormRaw {
  static constexpr int kVectors = sizeof(T) / 2;               // fp32: two of them
  uint4 v[kVectors];
  __device__ __forceinline__ void load(const T* row, int col) {
#pragma unroll
    for (int k = 0; k < kVectors; ++k) v[k] = *reinterpret_cast<const uint4*>(row + col + k * (16 / static_cast<int>(sizeof(T))));
  }
  __device__ __forceinline__ void get(Norm8& f) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        f.p[2 * k] = make_float2(__uint_as_float(v[k].x), __uint_as_float(v[k].y));
        f.p[2 * k + 1] = make_float2(__uint_as_float(v[k].z), __uint_as_float(v[k].w));
      }
    } else {
      f.p[0] = NormPair<T>::unpack(v[0].x);
      f.p[1] = NormPair<T>::unpack(v[0].y);
      f.p[2] = NormPair<T>::unpack(v[0].z);
      f.p[3] = NormPair<T>::unpack(v[0].w);
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
__device__ __forceinline__ void norm_get(const NormRaw<T, VEC>& raw, Norm8& f) {
  if constexpr (VEC) raw.get(f);
  else
#pragma unroll
    for (int e = 0; e < kNormN; ++e) f[e] = norm_float(raw.v[e]);
}
template <typename T, bool VEC>
__device__ __forceinline__ void norm_load(Norm8& f, const T* row, const NormColumns<VEC>& cols, int c) {
  NormRaw<T, VEC> raw;
  norm_fetch(raw, row, cols, c);
  norm_get(raw, f);
}
template <typename T, bool VEC>
__device__ __forceinline__ void norm_store(T* row, const NormColumns<VEC>& cols, int c, const Norm8& f) {
  if constexpr (VEC) {
    if (!cols.has(c)) return;
    T* to = row + cols.at(c, 0);
    if constexpr (sizeof(T) == 4) {
      uint4 v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) v[k] = make_uint4(__float_as_uint(f[4 * k]), __float_as_uint(f[4 * k + 1]), __float_as_uint(f[4 * k + 2]), __float_as_uint(f[4 * k + 3]));
      if ((reinterpret_cast<uintptr_t>(to) & 31) == 0) {       // whole sectors
        st_global_v8(to, v[0], v[1], 0ull);
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4*>(to + 4 * k) = v[k];
      }
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

// 16 bytes global -> shared, asynchronously; the copies of a thread form groups
__device__ __forceinline__ void norm_copy(unsigned char* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void norm_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void norm_await(int pending) {      // until all but the last `pending` groups are there
  if (pending == 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
  else if (pending == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else if (pending == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else asm volatile("cp.async.wait_group 3;" ::: "memory");
}
// A thread's places for one row: vector v is kNormThreads * 16 bytes behind vector 0.  Of fp32 rows a warp's copies follow one another, 512 bytes an instruction, each into the
// place of the thread that wants it: two halves of a thread's own 32 bytes would ask for every sector twice (the gradient of a 4096-element fp32 stream 560 us, 511 like this).  So a row is
// complete for a thread when its warp has waited and met.
template <typename T>
__device__ __forceinline__ void norm_ask(unsigned char* to, const T* row, const NormColumns<true>& cols, int c) {
  if constexpr (sizeof(T) == 2) {
    if (cols.has(c)) norm_copy(to, row + cols.at(c, 0));
  } else {
    const int lane = threadIdx.x & 31, first = cols.at(c, 0) - lane * kNormN;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int vector = k * 32 + lane, owner = vector >> 1;
      if (first + owner * kNormN < cols.dim) norm_copy(to + (owner - lane) * 16 + (vector & 1) * kNormThreads * 16, row + first + vector * 4);
    }
  }
}
// Places of groups outside the row hold zeros from the start (norm_clear) and are never written.
template <typename T>
__device__ __forceinline__ void norm_take(const unsigned char* from, Norm8& f) {
  NormRaw<T, true> raw;
#pragma unroll
  for (int k = 0; k < NormRaw<T, true>::kVectors; ++k) raw.v[k] = *reinterpret_cast<const uint4*>(from + k * kNormThreads * 16);
  raw.get(f);
}
// Zeros in `count` vectors of every row of a thread's ring, from vector `first` on.
__device__ __forceinline__ void norm_clear(unsigned char* ring, const int depth, const int vectors, int first, int count) {
  for (int d = 0; d < depth; ++d)
    for (int k = 0; k < count; ++k) *reinterpret_cast<uint4*>(ring + (d * vectors + first + k) * kNormThreads * 16) = make_uint4(0u, 0u, 0u, 0u);
}

// Gains and gates are fp32 or of the block's type, whichever the caller keeps them in.
struct NormGain {
  const void* data;
  int wide;                                     // fp32
};
template <typename T, bool VEC>
__device__ __forceinline__ void norm_gain(Norm8& f, const NormGain& g, long long at, const NormColumns<VEC>& cols, int c) {
  if (g.wide) norm_load<float, VEC>(f, static_cast<const float*>(g.data) + at, cols, c);
  else norm_load<T, VEC>(f, static_cast<const T*>(g.data) + at, cols, c);
}
template <typename T> __device__ __forceinline__ float norm_gain_one(const NormGain& g, long long at) {
  return g.wide ? static_cast<const float*>(g.data)[at] : norm_float(static_cast<const T*>(g.data)[at]);
}

// tanh: (1 - e) / (1 + e) with e = exp(-2 |a|), and below 1/4, where that cancels, the first five terms of its series (error 2e-8 of it)
__device__ __forceinline__ float norm_act(int by, float a) {
  if (by == kBySigmoid) return __fdividef(1.f, 1.f + __expf(-a));
  if (by == kByTanh) {
    const float e = __expf(-2.f * fabsf(a)), q = a * a;
    const float near = a * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return q < 0.0625f ? near : copysignf(__fdividef(1.f - e, 1.f + e), a);
  }
  return a;
}
// the derivative, without the cancellation of 1 - tanh^2 far out
__device__ __forceinline__ float norm_slope(int by, float a) {
  if (by == kBySigmoid) {
    const float e = __expf(-fabsf(a)), d = __fdividef(1.f, 1.f + e);
    return e * d * d;
  }
  if (by == kByTanh) {
    const float e = __expf(-2.f * fabsf(a)), d = __fdividef(1.f, 1.f + e);
    return 4.f * e * d * d;
  }
  return 1.f;
}

// either for a group, with the choice made once
__device__ __forceinline__ void norm_act_all(int by, Norm8& a) {
  if (by == kByItself) return;
  if (by == kBySigmoid) {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) a[e] = norm_act(kBySigmoid, a[e]);
  } else {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) a[e] = norm_act(kByTanh, a[e]);
  }
}
__device__ __forceinline__ void norm_slope_all(int by, Norm8& a) {
  if (by == kBySigmoid) {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) a[e] = norm_slope(kBySigmoid, a[e]);
  } else {
#pragma unroll
    for (int e = 0; e < kNormN; ++e) a[e] = by == kByItself ? 1.f : norm_slope(kByTanh, a[e]);
  }
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
  int vectors, depth;                           // of the ring: 16-byte vectors of a thread and row, rows
  int ring;                                     // where it starts in shared memory, behind the gains
  float scale, eps, share;                      // share: 1 / dim
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
    // every lane takes one warp's sum, several the same
    const int warps = tpr >> 5;
    v = at[group * warps + (threadIdx.x & (warps - 1))];
    for (int o = warps >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
};

// The gains of all columns in shared memory, each half of a group of kNormN apart so that a warp's reads of 16 bytes meet all banks.
// `make` gives a column's value.
template <bool VEC>
struct NormTable {
  float* at;
  NormColumns<VEC> cols;
  int width;                                    // columns, padded
  __device__ __forceinline__ int place(int col) const { return VEC ? ((col >> 2) & 1) * (width / 2) + (col >> 3) * 4 + (col & 3) : col; }
  template <typename Make>
  __device__ __forceinline__ void fill(Make make) {
    for (int col = threadIdx.x; col < width; col += kNormThreads) at[place(col)] = col < cols.dim ? make(col) : 0.f;
  }
  __device__ __forceinline__ void get(int c, Norm8& f) const {
    if constexpr (VEC) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 v = *reinterpret_cast<const float4*>(at + h * (width / 2) + (c * cols.tpr + cols.t) * 4);
        f[4 * h] = v.x; f[4 * h + 1] = v.y; f[4 * h + 2] = v.z; f[4 * h + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kNormN; ++e) f[e] = at[cols.at(c, e)];
    }
  }
};
// pre, and scale act(channel gate) post
template <typename F>
__device__ __forceinline__ float norm_factor(const NormParams& p, int col) {
  float v = p.scale;
  if (p.gate_kind == kGateChannel) v *= norm_act(p.by, norm_gain_one<F>({p.gate.data, p.gate_as.wide}, col));
  if (p.post.data != nullptr) v *= norm_gain_one<F>(p.post, col);
  return v;
}

// C: groups of a thread
template <typename X, typename F, int C, bool VEC>
__global__ void __launch_bounds__(kNormThreads, 1) norm_forward_kernel(const NormParams p) {
  extern __shared__ __align__(16) unsigned char s_dyn[];
  __shared__ float s_sum[64];
  constexpr bool kRing = VEC && C <= 2;
  constexpr int kX = static_cast<int>(sizeof(X)) / 2, kF = static_cast<int>(sizeof(F)) / 2;        // vectors of a group
  constexpr int kAtF = C * kX, kAtGate = kAtF + C * kF;
  const int group = threadIdx.x / p.tpr, per_block = kNormThreads / p.tpr;
  const NormColumns<VEC> cols = {p.tpr, static_cast<int>(threadIdx.x) - group * p.tpr, p.dim};
  NormSum sum = {s_sum, p.tpr, group, 0};
  const bool has_f = p.f.data != nullptr, has_post = p.post.data != nullptr, has_pre = p.pre.data != nullptr;
  const bool by_token = p.gate_kind == kGateToken, by_sequence = p.gate_kind == kGateSequence;
  const long long step = static_cast<long long>(gridDim.x) * per_block;
  long long at = static_cast<long long>(blockIdx.x) * per_block + group;
  unsigned char* const ring = s_dyn + p.ring + threadIdx.x * 16;
  const int row_bytes = p.vectors * kNormThreads * 16;
  auto ask = [&](long long r, int slot) {
    if constexpr (kRing) {
      __syncwarp();                              // the slot's last row is read
      if (r < p.tokens) {
        const int b = p.by_len.divide(static_cast<int>(r)), s = static_cast<int>(r) - b * p.len;
        unsigned char* to = ring + slot * row_bytes;
        auto all = [&](const auto* from, int first, int each) {
#pragma unroll
          for (int c = 0; c < C; ++c) norm_ask(to + (first + c * each) * kNormThreads * 16, from, cols, c);
        };
        all(norm_row<X>(p.x, b, s), 0, kX);
        if (has_f) all(norm_row<F>(p.f, b, s), kAtF, kF);
        if (by_token) {
          if (p.gate_as.wide) all(norm_row<float>(p.gate, b, s), kAtGate, 2);
          else all(norm_row<F>(p.gate, b, s), kAtGate, kF);
        }
      }
      norm_close();
    }
  };
  for (int c = 0; kRing && c < C; ++c) {
    if (cols.has(c)) continue;
    norm_clear(ring, p.depth, p.vectors, c * kX, kX);
    if (has_f) norm_clear(ring, p.depth, p.vectors, kAtF + c * kF, kF);
    if (by_token) norm_clear(ring, p.depth, p.vectors, kAtGate + c * (p.gate_as.wide ? 2 : kF), p.gate_as.wide ? 2 : kF);
  }
  for (int k = 0; k < p.depth - 1; ++k) ask(at + k * step, k);
  const int width = C * p.tpr * kNormN;
  NormTable<VEC> pre = {reinterpret_cast<float*>(s_dyn), cols, width}, factor = {reinterpret_cast<float*>(s_dyn) + width, cols, width};
  if (has_pre) pre.fill([&](int col) { return norm_gain_one<F>(p.pre, col); });
  if (has_f) factor.fill([&](int col) { return norm_factor<F>(p, col); });
  __syncthreads();
  for (int slot = 0; at < p.tokens; at += step) {
    const int row = static_cast<int>(at), b = p.by_len.divide(row), s = row - b * p.len;
    const unsigned char* from = ring + slot * row_bytes;
    Norm8 x[C], f[C];
    if constexpr (kRing) {
      ask(at + (p.depth - 1) * step, slot == 0 ? p.depth - 1 : slot - 1);
      norm_await(p.depth - 1);
      __syncwarp();
      if (++slot == p.depth) slot = 0;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (kRing) {
        norm_take<X>(from + c * kX * kNormThreads * 16, x[c]);
        if (has_f) norm_take<F>(from + (kAtF + c * kF) * kNormThreads * 16, f[c]);
      } else {
        norm_load<X, VEC>(x[c], norm_row<X>(p.x, b, s), cols, c);
        if (has_f) norm_load<F, VEC>(f[c], norm_row<F>(p.f, b, s), cols, c);
      }
    }
    if (has_f) {
      float r = 1.f;
      if (has_post) {
        Norm8 square = f[0] * f[0];
#pragma unroll
        for (int c = 1; c < C; ++c) square = norm_fma(f[c], f[c], square);
        r = rsqrtf(fmaf(sum(norm_fold(square)), p.share, p.eps));
      }
      if (cols.t == 0) p.rows[row] = has_post ? r : 0.f;
      X* out = norm_row<X>(p.out, b, s);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        Norm8 by;
        factor.get(c, by);
        if (by_token || by_sequence) {
          Norm8 a;
          if (by_sequence || !kRing) norm_gain<F, VEC>(a, {p.gate.data, p.gate_as.wide}, b * p.gate.batch + s * p.gate.row, cols, c);
          else if (p.gate_as.wide) norm_take<float>(from + (kAtGate + c * 2) * kNormThreads * 16, a);
          else norm_take<F>(from + (kAtGate + c * kF) * kNormThreads * 16, a);
          norm_act_all(p.by, a);
          by = by * a;
        }
        x[c] = norm_fma(f[c] * r, by, x[c]);
        norm_store(out, cols, c, x[c]);
      }
    }
    if (cols.t == 0 && !has_f) p.rows[row] = 0.f;
    if (cols.t == 0 && !has_pre) p.rows[p.tokens + row] = 0.f;
    if (has_pre) {
      Norm8 square = x[0] * x[0];
#pragma unroll
      for (int c = 1; c < C; ++c) square = norm_fma(x[c], x[c], square);
      const float r = rsqrtf(fmaf(sum(norm_fold(square)), p.share, p.eps));
      if (cols.t == 0) p.rows[p.tokens + row] = r;
      F* normed = norm_row<F>(p.normed, b, s);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        Norm8 w;
        pre.get(c, w);
        norm_store(normed, cols, c, x[c] * r * w);
      }
    }
  }
}

// A block's item is a run of tokens of one group (of all tokens where no sequence has a gate of its own): its sums of t n leave as
// record `item`; the sums for `pre` leave once, as record `block`.
template <typename X, typename F, int C, bool VEC>
__global__ void __launch_bounds__(kNormThreads, 1) norm_backward_kernel(const NormParams p) {
  extern __shared__ __align__(16) unsigned char s_dyn[];
  __shared__ float s_sum[64];
  constexpr bool kRing = VEC && C <= 2;
  constexpr int kX = static_cast<int>(sizeof(X)) / 2, kF = static_cast<int>(sizeof(F)) / 2;        // vectors of a group
  constexpr int kAtOut = C * kX, kAtDh = kAtOut + C * kX, kAtF = kAtDh + C * kF, kAtGate = kAtF + C * kF;
  pdl_launch_dependents();
  const int group = threadIdx.x / p.tpr, per_block = kNormThreads / p.tpr;
  const NormColumns<VEC> cols = {p.tpr, static_cast<int>(threadIdx.x) - group * p.tpr, p.dim};
  NormSum sum = {s_sum, p.tpr, group, 0};
  const bool has_f = p.f.data != nullptr, has_post = p.post.data != nullptr, has_pre = p.pre.data != nullptr && p.dnormed.data != nullptr;
  const bool has_dout = p.dout.data != nullptr, wants_sum = p.sums != nullptr;
  const bool by_token = p.gate_kind == kGateToken, by_sequence = p.gate_kind == kGateSequence;
  unsigned char* const ring = s_dyn + p.ring + threadIdx.x * 16;
  float* s_fold = reinterpret_cast<float*>(s_dyn + p.ring);       // [C kNormN][threads] where rows are shorter than a block: once a run's rows are through
  const int row_bytes = p.vectors * kNormThreads * 16;
  auto ask = [&](long long r, long long end, int slot) {
    if constexpr (kRing) {
      __syncwarp();                              // the slot's last row is read
      if (r < end) {
        const int b = p.by_len.divide(static_cast<int>(r)), s = static_cast<int>(r) - b * p.len;
        unsigned char* to = ring + slot * row_bytes;
        auto all = [&](const auto* from, int first, int each) {
#pragma unroll
          for (int c = 0; c < C; ++c) norm_ask(to + (first + c * each) * kNormThreads * 16, from, cols, c);
        };
        if (has_dout) all(norm_row<X>(p.dout, b, s), 0, kX);
        if (has_pre) {
          all(norm_row<X>(p.out, b, s), kAtOut, kX);
          all(norm_row<F>(p.dnormed, b, s), kAtDh, kF);
        }
        if (has_f) all(norm_row<F>(p.f, b, s), kAtF, kF);
        if (by_token) {
          if (p.gate_as.wide) all(norm_row<float>(p.gate, b, s), kAtGate, 2);
          else all(norm_row<F>(p.gate, b, s), kAtGate, kF);
        }
      }
      norm_close();
    }
  };
  const int items = p.groups * p.parts;
  const long long of_group = p.tokens / p.groups;
  // even shares, the first ones a token longer
  const long long share = of_group / p.parts, longer = of_group - share * p.parts;
  auto run_of = [&](int item, long long& begin, long long& end) {
    const int g = item / p.parts, part = item - g * p.parts;
    begin = g * of_group + part * share + min(static_cast<long long>(part), longer);
    end = begin + share + (part < longer ? 1 : 0);
  };
  long long begin, end;
  run_of(blockIdx.x, begin, end);
  auto clear = [&]() {
    for (int c = 0; kRing && c < C; ++c) {
      if (cols.has(c)) continue;
      norm_clear(ring, p.depth, p.vectors, c * kX, kX);
      norm_clear(ring, p.depth, p.vectors, kAtOut + c * kX, kX);
      norm_clear(ring, p.depth, p.vectors, kAtDh + c * kF, kF);
      norm_clear(ring, p.depth, p.vectors, kAtF + c * kF, kF);
      if (by_token) norm_clear(ring, p.depth, p.vectors, kAtGate + c * (p.gate_as.wide ? 2 : kF), p.gate_as.wide ? 2 : kF);
    }
  };
  clear();
  if (kRing)
    for (int k = 0; k < p.depth - 1; ++k) ask(begin + group + k * per_block, end, k);
  const int width = C * p.tpr * kNormN;
  NormTable<VEC> pre = {reinterpret_cast<float*>(s_dyn), cols, width}, factor = {reinterpret_cast<float*>(s_dyn) + width, cols, width};
  if (has_pre) pre.fill([&](int col) { return norm_gain_one<F>(p.pre, col); });
  if (has_f) factor.fill([&](int col) { return norm_factor<F>(p, col); });
  __syncthreads();
  Norm8 acc[C], acc_pre[C];
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = acc_pre[c] = norm_all(0.f);
  // what the threads of a block's rows have for the same columns, added in the rows' order
  auto leave = [&](Norm8 (&a)[C], float* record) {
    if (per_block > 1) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < kNormN; ++e) s_fold[(c * kNormN + e) * kNormThreads + threadIdx.x] = a[c][e];
      __syncthreads();
      const int shift = 31 - __clz(p.tpr);
      for (int k = threadIdx.x; k < C * kNormN * p.tpr; k += kNormThreads) {
        const int t = k & (p.tpr - 1), ce = k >> shift, c = ce / kNormN, e = ce % kNormN;
        float v = 0.f;
        for (int g = 0; g < per_block; ++g) v += s_fold[ce * kNormThreads + g * p.tpr + t];
        const int col = VEC ? (c * p.tpr + t) * kNormN + e : (c * kNormN + e) * p.tpr + t;
        if (col < p.dim) record[col] = v;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < kNormN; ++e) {
          const int col = cols.at(c, e);
          if (col < p.dim) record[col] = a[c][e];
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c) a[c] = norm_all(0.f);
  };
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    if (item != static_cast<int>(blockIdx.x)) {
      run_of(item, begin, end);
      clear();                                   // sums have been there
      if (kRing)
        for (int k = 0; k < p.depth - 1; ++k) ask(begin + group + k * per_block, end, k);
    }
    long long at = begin + group;
    float next_rf = 1.f, next_rx = 1.f;
    auto factors_of = [&](long long r) {
      if (r >= end) return;
      if (has_post) next_rf = p.rows[r];
      if (has_pre) next_rx = p.rows[p.tokens + r];
    };
    factors_of(at);
    for (int slot = 0; at < end; at += per_block) {
      const int row = static_cast<int>(at), b = p.by_len.divide(row), s = row - b * p.len;
      const float rf = next_rf, rx = next_rx;
      const unsigned char* from = ring + slot * row_bytes;
      factors_of(at + per_block);
      if constexpr (kRing) {
        ask(at + static_cast<long long>(p.depth - 1) * per_block, end, slot == 0 ? p.depth - 1 : slot - 1);
        norm_await(p.depth - 1);
        __syncwarp();
        if (++slot == p.depth) slot = 0;
      }
      // group c of a tensor's row, from the ring or from memory; with one group a thread (rows up to 4096 elements) all that comes from memory is asked for at once
      constexpr bool kAtOnce = !kRing && C == 1;
      NormRaw<X, VEC> raw_out, raw_dout;
      NormRaw<F, VEC> raw_dh, raw_f;
      if constexpr (kAtOnce) {
        if (has_pre) {
          norm_fetch(raw_out, static_cast<const X*>(norm_row<X>(p.out, b, s)), cols, 0);
          norm_fetch(raw_dh, static_cast<const F*>(norm_row<F>(p.dnormed, b, s)), cols, 0);
        }
        if (has_dout) norm_fetch(raw_dout, static_cast<const X*>(norm_row<X>(p.dout, b, s)), cols, 0);
        if (has_f) norm_fetch(raw_f, static_cast<const F*>(norm_row<F>(p.f, b, s)), cols, 0);
      }
      auto x_row = [&](const NormRows& r, int first, int c, Norm8& to) {
        if constexpr (kAtOnce) norm_get(first == kAtOut ? raw_out : raw_dout, to);
        else if constexpr (kRing) norm_take<X>(from + (first + c * kX) * kNormThreads * 16, to);
        else norm_load<X, VEC>(to, norm_row<X>(r, b, s), cols, c);
      };
      auto f_row = [&](const NormRows& r, int first, int c, Norm8& to) {
        if constexpr (kAtOnce) norm_get(first == kAtDh ? raw_dh : raw_f, to);
        else if constexpr (kRing) norm_take<F>(from + (first + c * kF) * kNormThreads * 16, to);
        else norm_load<F, VEC>(to, norm_row<F>(r, b, s), cols, c);
      };
      Norm8 t[C];
      if (has_pre) {
        Norm8 hat[C], mean = norm_all(0.f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          Norm8 w;
          pre.get(c, w);
          x_row(p.out, kAtOut, c, hat[c]);
          f_row(p.dnormed, kAtDh, c, t[c]);
          hat[c] = hat[c] * rx;
          const Norm8 product = t[c] * hat[c];
          acc_pre[c] = acc_pre[c] + product;
          mean = norm_fma(product, w, mean);
          t[c] = t[c] * w;
        }
        const float minus = -sum(norm_fold(mean)) * p.share;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          Norm8 d = norm_all(0.f);
          if (has_dout) x_row(p.dout, 0, c, d);
          t[c] = norm_fma(norm_fma(hat[c], minus, t[c]), rx, d);
        }
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
          t[c] = norm_all(0.f);
          if (has_dout) x_row(p.dout, 0, c, t[c]);
        }
      }
      X* dx = norm_row<X>(p.dx, b, s);
#pragma unroll
      for (int c = 0; c < C; ++c) norm_store(dx, cols, c, t[c]);
      if (!has_f) continue;
      // t becomes c t post
      Norm8 inner = norm_all(0.f);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        Norm8 n, by;
        f_row(p.f, kAtF, c, n);
        factor.get(c, by);
        const Norm8 tn = t[c] * n * rf;
        if (by_token || by_sequence) {
          Norm8 gate;
          if (by_sequence || !kRing) norm_gain<F, VEC>(gate, {p.gate.data, p.gate_as.wide}, b * p.gate.batch + s * p.gate.row, cols, c);
          else if (p.gate_as.wide) norm_take<float>(from + (kAtGate + c * 2) * kNormThreads * 16, gate);
          else norm_take<F>(from + (kAtGate + c * kF) * kNormThreads * 16, gate);
          if (by_token) {
            Norm8 slope = gate;
            norm_slope_all(p.by, slope);
            const Norm8 dg = slope * by * tn;
            if (p.gate_as.wide) norm_store(norm_row<float>(p.dgate, b, s), cols, c, dg);
            else norm_store(norm_row<F>(p.dgate, b, s), cols, c, dg);
          }
          norm_act_all(p.by, gate);
          acc[c] = by_token ? norm_fma(gate * p.scale, tn, acc[c]) : acc[c] + tn;        // a token's gate differs from its neighbours': it goes into the sum
          by = by * gate;
        } else {
          acc[c] = acc[c] + tn;
        }
        t[c] = t[c] * by;
        inner = norm_fma(t[c], n, inner);
      }
      F* df = norm_row<F>(p.df, b, s);
      if (has_post) {
        const float minus = -sum(norm_fold(inner)) * p.share * rf * rf * rf;       // of c t post and n: two factors r_f, and one on the result
#pragma unroll
        for (int c = 0; c < C; ++c) {
          Norm8 n;
          f_row(p.f, kAtF, c, n);
          norm_store(df, cols, c, norm_fma(n, minus, t[c] * rf));
        }
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) norm_store(df, cols, c, t[c]);
      }
    }
    if (kRing) norm_await(0);                    // what follows may take the ring's place
    if (wants_sum) leave(acc, p.sums + static_cast<long long>(item) * p.dim);
  }
  if (p.pre_sums != nullptr) leave(acc_pre, p.pre_sums + static_cast<long long>(blockIdx.x) * p.dim);
}

// dpost, dpre and the gate's gradient (channel, sequence) from the records: 32 columns a block, whose 32 warps divide into as many for each
// group of records (a sequence's, or all); they take its records in turn and their sums are added in order.
template <typename F>
__global__ void __launch_bounds__(kNormSumThreads) norm_sum_kernel(const NormParams p) {
  __shared__ float s_part[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const bool in = col < p.dim;
  // over `count` warps from the first of them on, which has the result
  auto total = [&](float v, int first, int count) {
    __syncthreads();
    s_part[warp][lane] = v;
    __syncthreads();
    v = 0.f;
    if (warp == first)
      for (int w = 0; w < count; ++w) v += s_part[first + w][lane];
    return v;
  };
  auto put = [&](void* to, bool wide, long long at, float v) {
    if (wide) static_cast<float*>(to)[at] = v;
    else static_cast<F*>(to)[at] = norm_round<F>(v);
  };
  const float post = in && p.post.data != nullptr ? norm_gain_one<F>(p.post, col) : 1.f;
  float by_pre = 0.f;
  if (p.pre_sums != nullptr && in)
#pragma unroll 8
    for (int k = warp; k < p.blocks; k += 32) by_pre += p.pre_sums[static_cast<long long>(k) * p.dim + col];
  if (p.sums != nullptr) {
    int at_once = 1;                             // groups
    while (at_once < 32 && at_once < p.groups) at_once *= 2;
    const int each = 32 / at_once, first = warp / each * each;
    float v = 0.f;
    for (int g0 = 0; g0 < p.groups; g0 += at_once) {
      const int g = g0 + warp / each;
      float s = 0.f;
      if (in && g < p.groups)
#pragma unroll 8
        for (int k = warp - first; k < p.parts; k += each) s += p.sums[(static_cast<long long>(g) * p.parts + k) * p.dim + col];
      if (each > 1) s = total(s, first, each);
      if (!in || g >= p.groups || warp != first) continue;
      if (p.gate_kind == kGateSequence || p.gate_kind == kGateChannel) {
        const bool sequence = p.gate_kind == kGateSequence;
        const float a = norm_gain_one<F>({p.gate.data, p.gate_as.wide}, (sequence ? g * p.gate.batch : 0) + col);
        v = fmaf(p.scale * norm_act(p.by, a), s, v);
        put(p.dgate.data, p.gate_as.wide, (sequence ? g * p.dgate.batch : 0) + col, p.scale * norm_slope(p.by, a) * post * s);
      } else {
        v += p.gate_kind == kGateNone ? p.scale * s : s;
      }
    }
    if (p.groups > 1) v = total(v, 0, 32);
    if (p.dpost != nullptr && in && warp == 0) put(p.dpost, p.post.wide, col, v);
  }
  if (p.dpre != nullptr) {
    const float v = total(by_pre, 0, 32);
    if (in && warp == 0) put(p.dpre, p.pre.wide, col, v);
  }
}

}  // namespace adacons
