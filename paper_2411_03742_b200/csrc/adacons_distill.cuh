// Distillation from a teacher's top logits: kernels (sm_100a).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "adacons_common.cuh"
#include "adacons_tc.cuh"

namespace adacons {

// ----------------------------------------------------------------------------------------------
// For every token: the student's logits z (V of them), the teacher's logits t_j at K entries i_j, a label y or none.
//     p = softmax(t / tau) over the entries that are there,   L = ln sum_v exp(z_v / tau),   L1 = ln sum_v exp(z_v)
//     loss = mix tau^2 sum_j p_j (ln p_j - z_{i_j} / tau + L)  +  (1 - mix) (L1 - z_y)
//     dz_v = dloss (mix tau (exp(z_v / tau - L) - sum_{j: i_j = v} p_j) + (1 - mix) (exp(z_v - L1) - [v = y]))
// An entry is there when its index lies in 0 .. V-1 and its logit is not -inf; a token without entries has no first term, one
// without a label no second, one without either is not read at all.
//
// Bound by memory: z is read once forward, read and written once back.  A block goes through a token's logits (or a share of
// them, when there are few tokens: the blocks of a cluster join their maxima and sums in a fixed order through one another's shared memory)
// with one running maximum and sum a thread, 32 elements between two looks at the maximum.  Both sums need an exponential
// of every logit where tau is not one, and the exponential unit would then be the limit (16 a cycle and SM against 12 bf16 logits
// that memory brings): for tau = 2, 3 and 4 the second is a power of the first, exp(z) = exp(z / tau)^tau (backward: of exp((z - L1) / tau), so that small probabilities are not lost
// on the way).
// ----------------------------------------------------------------------------------------------
constexpr int kDistillMaxK = 1024;
constexpr float kDistillLow = -3.402823466e38f;
constexpr float kDistillLog2e = 1.4426950408889634f;

template <typename T> struct DistillVec;
template <> struct DistillVec<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) { f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w); }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
  static __device__ __forceinline__ float round(float v) { return v; }
};
template <> struct DistillVec<__nv_bfloat16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) { const float2 p = unpack_pair<1>(v, k); f[2 * k] = p.x; f[2 * k + 1] = p.y; }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack_bf16x2_rn(f[0], f[1]), pack_bf16x2_rn(f[2], f[3]), pack_bf16x2_rn(f[4], f[5]), pack_bf16x2_rn(f[6], f[7]));
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ __nv_bfloat16 round(float v) { return __float2bfloat16_rn(v); }
};
template <> struct DistillVec<__half> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&u[k])); f[2 * k] = p.x; f[2 * k + 1] = p.y; }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) { const __half2 h = __floats2half2_rn(f[2 * k], f[2 * k + 1]); u[k] = *reinterpret_cast<const uint32_t*>(&h); }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
  static __device__ __forceinline__ float one(const __half* p) { return __half2float(*p); }
  static __device__ __forceinline__ __half round(float v) { return __float2half_rn(v); }
};

struct DistillParams {
  const void *z, *ids, *teacher, *labels;        // labels may be null
  long long z_row, ids_row, teacher_row;         // strides in elements
  int vocab, top;
  int ids_wide, labels_wide;                     // 64-bit indices
  int teacher_type;                              // adacons_dtype
  float tau, mix;
  float* loss;                                   // forward
  float* rows;                                   // [2][tokens]: L, L1
  long long tokens;
  const float* dloss;                            // backward
  long long dloss_step;
  void* dz;
  long long dz_row;
  int shares;                                    // blocks of a token
  int vectors;                                   // z and dz lie alike relative to 16 bytes
};

__device__ __forceinline__ float distill_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <int POWER>
__device__ __forceinline__ float distill_power(float e) {
  const float e2 = e * e;
  return POWER == 2 ? e2 : POWER == 3 ? e2 * e : e2 * e2;
}
// the larger of two in each half of a vector's words, and of all of them; NaN where nothing else is left
__device__ __forceinline__ uint32_t distill_max2(uint32_t a, uint32_t b, __nv_bfloat16) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ uint32_t distill_max2(uint32_t a, uint32_t b, __half) {
  const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ long long distill_index(const void* p, int wide, long long at) {
  return wide ? static_cast<const long long*>(p)[at] : static_cast<const int*>(p)[at];
}
__device__ __forceinline__ float distill_teacher(const DistillParams& p, long long at) {
  if (p.teacher_type == 0) return static_cast<const float*>(p.teacher)[at];
  return p.teacher_type == 1 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p.teacher)[at]) : __half2float(static_cast<const __half*>(p.teacher)[at]);
}
// the entry's index, or -1 where there is none
__device__ __forceinline__ int distill_entry(const DistillParams& p, long long row, int j, float& t) {
  const long long id = distill_index(p.ids, p.ids_wide, row * p.ids_row + j);
  t = distill_teacher(p, row * p.teacher_row + j);
  return id >= 0 && id < p.vocab && !(t == -INFINITY) ? static_cast<int>(id) : -1;
}
__device__ __forceinline__ int distill_label(const DistillParams& p, long long row) {
  if (p.labels == nullptr) return -1;
  const long long y = distill_index(p.labels, p.labels_wide, row);
  return y >= 0 && y < p.vocab ? static_cast<int>(y) : -1;
}

// Maximum and sum over a block; `shared` has 32 places, and a barrier lies between two uses.
__device__ __forceinline__ float distill_block_max(float v, float* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (blockDim.x == 32) return v;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  v = kDistillLow;
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v = fmaxf(v, shared[w]);
  return v;
}
__device__ __forceinline__ float distill_block_sum(float v, float* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (blockDim.x == 32) return v;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v += shared[w];
  return v;
}

// Elements [begin, end) of a row as a thread meets them: some before the first 16-byte boundary, vectors, the rest.
template <typename T>
struct DistillSpan {
  const T* from;
  int head, vectors, tail;
  __device__ __forceinline__ DistillSpan(const T* row, int begin, int end) : from(row + begin) {
    const int n = end - begin, off = static_cast<int>(reinterpret_cast<uintptr_t>(from) & 15) / static_cast<int>(sizeof(T));
    head = min(n, off == 0 ? 0 : DistillVec<T>::kN - off);
    vectors = (n - head) / DistillVec<T>::kN;
    tail = n - head - vectors * DistillVec<T>::kN;
  }
};

// A share of a token's logits: whole multiples of 64 elements, the last one what is left.
__device__ __forceinline__ void distill_share(int vocab, int shares, int share, int& begin, int& end) {
  const int size = (static_cast<int>((static_cast<long long>(vocab) + shares - 1) / shares) + 63) / 64 * 64;
  begin = static_cast<int>(min(static_cast<long long>(vocab), static_cast<long long>(share) * size));
  end = static_cast<int>(min(static_cast<long long>(vocab), static_cast<long long>(begin) + size));
}

// MODE 0: L alone; 1: L1 by exponentials of its own; 2, 3, 4: L1 from powers of L's.
template <int MODE>
struct DistillState {
  float m, s, s1;
  float k;                                       // log2(e) / tau
  __device__ __forceinline__ DistillState(const DistillParams& p) : m(kDistillLow), s(0.f), s1(0.f), k(kDistillLog2e / p.tau) {}
  // the factor on s1 that goes with the factor e = 2^(d k) on s
  __device__ __forceinline__ float second(float d, float e) const { return MODE == 1 ? distill_ex2(d * kDistillLog2e) : distill_power<MODE>(e); }
  __device__ __forceinline__ void rescale(float top) {         // to a larger maximum
    const float e = distill_ex2((m - top) * k);
    s *= e;
    if (MODE != 0) s1 *= second(m - top, e);
    m = top;
  }
  __device__ __forceinline__ void add(float z) {
    if (z > m) rescale(z);
    const float d = z - m, e = distill_ex2(d * k);
    s += e;
    if (MODE != 0) s1 += second(d, e);
  }
  template <int N> __device__ __forceinline__ void add_all(const float (&z)[N], float2& a, float2& b) const {      // none above m
    const float2 minus = make_float2(-m, -m), by = make_float2(k, k), by1 = make_float2(kDistillLog2e, kDistillLog2e);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 d = add2(make_float2(z[i], z[i + 1]), minus), x = mul2(d, by);
      const float2 e = make_float2(distill_ex2(x.x), distill_ex2(x.y));
      a = add2(a, e);
      if (MODE == 1) {
        const float2 y = mul2(d, by1);
        b = add2(b, make_float2(distill_ex2(y.x), distill_ex2(y.y)));
      } else if (MODE != 0) {
        const float2 e2 = mul2(e, e);
        b = MODE == 2 ? fma2(e, e, b) : fma2(e2, MODE == 3 ? e : e2, b);
      }
    }
  }
  __device__ __forceinline__ void join(float m2, float s2, float t2) {
    const float top = fmaxf(m, m2);
    if (top > m) rescale(top);
    const float e = distill_ex2((m2 - top) * k);
    s = fmaf(s2, e, s);
    if (MODE != 0) s1 = fmaf(t2, second(m2 - top, e), s1);
  }
};
template <typename T, int N>
__device__ __forceinline__ float distill_top(const uint4 (&raw)[N]) {
  if constexpr (sizeof(T) == 4) {
    float m = kDistillLow;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(raw[i].x), __uint_as_float(raw[i].y)), fmaxf(__uint_as_float(raw[i].z), __uint_as_float(raw[i].w))));
    return m;
  } else {
    uint32_t m = raw[0].x;
#pragma unroll
    for (int i = 0; i < N; ++i) m = distill_max2(distill_max2(m, raw[i].x, T()), distill_max2(distill_max2(raw[i].y, raw[i].z, T()), raw[i].w, T()), T());
    const uint4 all = make_uint4(m, m, m, m);
    float f[DistillVec<T>::kN];
    DistillVec<T>::unpack(all, f);
    return fmaxf(f[0], f[1]);
  }
}

template <typename T, int MODE>
__global__ void __launch_bounds__(512, 2) distill_forward_kernel(const DistillParams p) {
  __shared__ float s_part[3][32];
  __shared__ float s_join[3];
  using V = DistillVec<T>;
  const int shares = p.shares, share = shares > 1 ? static_cast<int>(cluster_rank()) : 0;
  const long long row = blockIdx.x / shares;
  const int tid = threadIdx.x, threads = blockDim.x;
  const T* z = static_cast<const T*>(p.z) + row * p.z_row;
  const int label = distill_label(p, row);
  // this thread's entries: the loads are under way while the row is
  constexpr int kMine = 2;                       // of 512 threads; smaller blocks go round again below
  int id[kMine];
  float t[kMine], at[kMine];
  bool some = false;
  for (int j = tid; j < p.top; j += threads) {
    float v;
    some = some || distill_entry(p, row, j, v) >= 0;
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int j = tid + i * threads;
    id[i] = -1;
    t[i] = kDistillLow;
    at[i] = 0.f;
    if (share == 0 && j < p.top) {
      id[i] = distill_entry(p, row, j, t[i]);
      if (id[i] >= 0) at[i] = V::one(z + id[i]);
    }
  }
  const bool taught = __syncthreads_or(some);
  if (!taught && label < 0) {                    // the same in all blocks of the token
    if (share == 0 && tid == 0) {
      p.loss[row] = 0.f;
      p.rows[row] = p.rows[p.tokens + row] = 0.f;
    }
    return;
  }
  DistillState<MODE> st(p);
  {
    int begin, end;
    distill_share(p.vocab, shares, share, begin, end);
    const DistillSpan<T> span(z, begin, end);
    if (tid < span.head) st.add(V::one(span.from + tid));
    const uint4* body = reinterpret_cast<const uint4*>(span.from + span.head);
    constexpr int kDeep = 4;                     // vectors between two looks; the next ones are on their way meanwhile
    auto take = [&](const auto& raw) {
      const float top = distill_top<T>(raw);
      if (top > st.m) st.rescale(top);
      float2 a = make_float2(0.f, 0.f), b = make_float2(0.f, 0.f);
#pragma unroll
      for (const uint4& v : raw) {
        float g[V::kN];
        V::unpack(v, g);
        st.add_all(g, a, b);
      }
      st.s += a.x + a.y;
      if (MODE != 0) st.s1 += b.x + b.y;
    };
    int at_vector = tid;
    const int last = span.vectors - (kDeep - 1) * threads;       // where a thread's kDeep vectors may start at most
    uint4 raw[kDeep];
    if (at_vector < last) {
#pragma unroll
      for (int i = 0; i < kDeep; ++i) raw[i] = ld_stream_v4(body + at_vector + i * threads);
    }
    while (at_vector < last) {
      uint4 next[kDeep];
      const int ahead = at_vector + kDeep * threads;
      if (ahead < last) {
#pragma unroll
        for (int i = 0; i < kDeep; ++i) next[i] = ld_stream_v4(body + ahead + i * threads);
      }
      take(raw);
#pragma unroll
      for (int i = 0; i < kDeep; ++i) raw[i] = next[i];
      at_vector = ahead;
    }
    for (; at_vector < span.vectors; at_vector += threads) {
      const uint4 one[1] = {ld_stream_v4(body + at_vector)};
      take(one);
    }
    if (tid < span.tail) st.add(V::one(span.from + span.head + span.vectors * V::kN + tid));
  }
  // lanes, warps, blocks
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2 = __shfl_down_sync(0xffffffffu, st.m, o), s2 = __shfl_down_sync(0xffffffffu, st.s, o);
    st.join(m2, s2, MODE == 0 ? 0.f : __shfl_down_sync(0xffffffffu, st.s1, o));
  }
  if ((tid & 31) == 0) { s_part[0][tid >> 5] = st.m; s_part[1][tid >> 5] = st.s; s_part[2][tid >> 5] = st.s1; }
  __syncthreads();
  DistillState<MODE> all(p);
  for (int w = 0; w < (threads >> 5); ++w) all.join(s_part[0][w], s_part[1][w], s_part[2][w]);
  if (shares > 1) {
    if (tid == 0) { s_join[0] = all.m; s_join[1] = all.s; s_join[2] = all.s1; }
    cluster_sync_all();
    if (share == 0) {
      DistillState<MODE> joined(p);
      for (int r = 0; r < shares; ++r) joined.join(ld_cluster_f32(&s_join[0], r), ld_cluster_f32(&s_join[1], r), ld_cluster_f32(&s_join[2], r));
      all = joined;
    }
    cluster_sync_all();                          // nobody leaves while its sums are read
    if (share != 0) return;
  }
  const float inv_tau = 1.f / p.tau, log_s = logf(all.s), log_s1 = MODE == 0 ? log_s : logf(all.s1);
  float loss = 0.f;
  if (taught) {
    float top = kDistillLow;
    for (int j = tid; j < p.top; j += threads) {
      float v;
      if (distill_entry(p, row, j, v) >= 0) top = fmaxf(top, v);
    }
    top = distill_block_max(top, s_part[0]);
    // sum of e_j and of e_j ((t_j - top) - (z_j - m)) / tau
    float sum = 0.f, inner = 0.f;
    auto take = [&](float tj, float zj) {
      const float d = (tj - top) * inv_tau, e = expf(d);
      sum += e;
      if (e != 0.f) inner = fmaf(e, d - (zj - all.m) * inv_tau, inner);
    };
#pragma unroll
    for (int i = 0; i < kMine; ++i)
      if (id[i] >= 0) take(t[i], at[i]);
    for (int j = tid + kMine * threads; j < p.top; j += threads) {
      float v;
      const int e = distill_entry(p, row, j, v);
      if (e >= 0) take(v, V::one(z + e));
    }
    sum = distill_block_sum(sum, s_part[0]);
    inner = distill_block_sum(inner, s_part[1]);
    loss = p.mix * p.tau * p.tau * (inner / sum - logf(sum) + log_s);
  }
  if (tid == 0) {
    if (label >= 0) loss += (1.f - p.mix) * (log_s1 - (V::one(z + label) - all.m));
    p.loss[row] = loss;
    p.rows[row] = all.m * inv_tau + log_s;
    p.rows[p.tokens + row] = p.labels == nullptr ? 0.f : all.m + log_s1;
  }
}

// A block writes a token's gradient, or a share of it: first exp alone everywhere, then, after a barrier, once more where
// entries or the label are, with everything that falls on one index summed up before it is rounded.  The logits there are fetched before
// the first writes: dz may be z.
template <typename T, int MODE>
__global__ void __launch_bounds__(512, 2) distill_backward_kernel(const DistillParams p) {
  __shared__ int s_id[kDistillMaxK + 1];
  __shared__ float s_weight[kDistillMaxK + 1], s_z[kDistillMaxK + 1];
  __shared__ float s_part[32];
  using V = DistillVec<T>;
  const long long row = blockIdx.x / p.shares;
  const int share = static_cast<int>(blockIdx.x - row * p.shares);
  const int tid = threadIdx.x, threads = blockDim.x;
  const T* z = static_cast<const T*>(p.z) + row * p.z_row;
  T* dz = static_cast<T*>(p.dz) + row * p.dz_row;
  int begin, end;
  distill_share(p.vocab, p.shares, share, begin, end);
  const int label = distill_label(p, row);
  const float inv_tau = 1.f / p.tau, dloss = p.dloss[row * p.dloss_step];
  float top = kDistillLow;
  bool some = false;
  for (int j = tid; j < p.top; j += threads) {
    float t;
    const int id = distill_entry(p, row, j, t);
    s_id[j] = id;
    s_weight[j] = t;
    if (id >= begin && id < end) s_z[j] = V::one(z + id);
    if (id >= 0) { some = true; top = fmaxf(top, t); }
  }
  const bool taught = __syncthreads_or(some);
  if (!taught && label < 0) {                    // nothing falls on this token
    for (int i = begin + tid; i < end; i += threads) dz[i] = V::round(0.f);
    return;
  }
  top = distill_block_max(top, s_part);
  float sum = 0.f;
  for (int j = tid; j < p.top; j += threads)
    if (s_id[j] >= 0) sum += s_weight[j] = expf((s_weight[j] - top) * inv_tau);
  sum = distill_block_sum(sum, s_part);
  const float soft = taught ? dloss * p.mix * p.tau : 0.f, hard = label >= 0 ? dloss * (1.f - p.mix) : 0.f;
  const float each = taught ? soft / sum : 0.f;
  for (int j = tid; j < p.top; j += threads)
    if (s_id[j] >= 0) s_weight[j] *= each;
  if (tid == 0) {
    s_id[p.top] = label;
    s_weight[p.top] = hard;
    if (label >= begin && label < end) s_z[p.top] = V::one(z + label);
  }
  __syncthreads();
  // Powers: exp(z - L1) = exp(z / tau - L1 / tau)^tau, which leaves fp32 no sooner than it does itself, and exp(z / tau - L) = exp(z / tau - L1 / tau) exp(L1 / tau - L), whose last
  // factor lies between V^(1 / tau - 1) and 1.
  const float L = p.rows[row], L1 = p.rows[p.tokens + row];
  const bool powers = MODE > 1 && label >= 0;
  const float from = powers ? L1 * inv_tau : L;
  const float with = MODE == 0 ? soft + hard : powers ? soft * expf(from - L) : soft;
  auto gradient = [&](float v) {
    const float e = distill_ex2(fmaf(v, inv_tau, -from) * kDistillLog2e);
    if (MODE == 0) return with * e;
    if (MODE == 1) return fmaf(hard, distill_ex2((v - L1) * kDistillLog2e), with * e);
    return fmaf(hard, distill_power<MODE>(e), with * e);
  };
  if (p.vectors) {
    const DistillSpan<T> span(z, begin, end);
    T* to = dz + begin;
    if (tid < span.head) to[tid] = V::round(gradient(V::one(span.from + tid)));
    const uint4* body = reinterpret_cast<const uint4*>(span.from + span.head);
    uint4* out = reinterpret_cast<uint4*>(to + span.head);
    constexpr int kDeep = 4;
    for (int at = tid; at < span.vectors; at += kDeep * threads) {
      uint4 raw[kDeep];
#pragma unroll
      for (int i = 0; i < kDeep; ++i)
        if (at + i * threads < span.vectors) raw[i] = *(body + at + i * threads);
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        if (at + i * threads >= span.vectors) continue;
        float g[V::kN];
        V::unpack(raw[i], g);
#pragma unroll
        for (int e = 0; e < V::kN; ++e) g[e] = gradient(g[e]);
        out[at + i * threads] = V::pack(g);
      }
    }
    const int last = span.head + span.vectors * V::kN + tid;
    if (tid < span.tail) to[last] = V::round(gradient(V::one(span.from + last)));
  } else {
#pragma unroll 4
    for (int i = begin + tid; i < end; i += threads) dz[i] = V::round(gradient(V::one(z + i)));
  }
  __syncthreads();
  for (int j = tid; j <= p.top; j += threads) {
    const int id = s_id[j];
    if (id < begin || id >= end) continue;
    bool first = true;
    float weight = 0.f;
    for (int i = 0; i <= p.top; ++i) {
      if (s_id[i] != id) continue;
      if (i < j) { first = false; break; }
      weight += s_weight[i];
    }
    if (first) dz[id] = V::round(gradient(s_z[j]) - weight);
  }
}

}  // namespace adacons
