// Rotary positions: kernel (sm_100a).
#pragma once

#include "adacons_common.cuh"

namespace adacons {

// ----------------------------------------------------------------------------------------------
// Pair i of a head, at position t, is turned by the angle t f_i and multiplied by `gain`:
//     (a, b) -> gain (a cos - b sin, a sin + b cos)        gradient: the turn by -t f_i, same gain
// with (a, b) = (x_i, x_{i + rot/2}) or, interleaved, (x_2i, x_2i+1).  Elements from `rot` on pass through.
//
// The angle of a late position is thousands of turns: t f_i is formed in fp64, whole turns are taken off
// there, and only the remainder (|phi| <= 1/2 turn, exact to 2^-36 even at t = 2^20) goes to fp32 sine and
// cosine.  That is rot/2 sines per token, shared by all of its heads: a block takes a few tokens, its threads first make
// the table in shared memory and then walk over the tokens' heads, 16 bytes of each half (or 32 adjacent bytes) a thread.
// Bound by memory: every element is read and written once.
// ----------------------------------------------------------------------------------------------
constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTable = 2048;            // (cos, sin) pairs in a block's table
constexpr int kRopeMaxTokens = 64;             // of a block

// n / d for 0 <= n < 2^31 by a multiplication: m = ceil(2^(31 + s) / d) with s = ceil(log2 d)
struct RopeDivisor {
  unsigned m;
  int s;
  __device__ __forceinline__ int divide(int n) const { return static_cast<int>((static_cast<unsigned long long>(static_cast<unsigned>(n)) * m) >> (31 + s)); }
};

struct RopeParams {
  const void* x;
  void* y;
  const int* positions;        // [tokens] contiguous, or null: token index within its sequence plus `first`
  const double* turns;         // f_i / (2 pi)
  long long first;
  long long tokens;            // batch * seq
  int seq, heads, dim, rot;
  long long xb, xs, xh, yb, ys, yh;      // element strides
  float gain;
  int inverse;
  int tokens_per_block;
  RopeDivisor per_token, per_head;       // work items
};

template <int DT> struct RopeVec;
template <> struct RopeVec<0> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) { f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w); }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); }
};
template <> struct RopeVec<1> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) { const float2 p = unpack_pair<1>(v, k); f[2 * k] = p.x; f[2 * k + 1] = p.y; }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack_bf16x2_rn(f[0], f[1]), pack_bf16x2_rn(f[2], f[3]), pack_bf16x2_rn(f[4], f[5]), pack_bf16x2_rn(f[6], f[7]));
  }
};
template <int DT> __device__ __forceinline__ float rope_get(const void* p, long long i) {
  return DT == 0 ? static_cast<const float*>(p)[i] : __uint_as_float(static_cast<uint32_t>(static_cast<const unsigned short*>(p)[i]) << 16);
}
template <int DT> __device__ __forceinline__ void rope_put(void* p, long long i, float v) {
  if (DT == 0) static_cast<float*>(p)[i] = v;
  else static_cast<unsigned short*>(p)[i] = static_cast<unsigned short>(pack_bf16x2_rn(v, 0.f) & 0xffffu);
}

// Work items of one (token, head).  VEC: rotated pairs in groups of kN (two 16-byte vectors), then the rest two
// vectors at a time; otherwise one pair, then one element.
template <int DT, bool INTERLEAVED, bool VEC>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p) {
  __shared__ float2 table[kRopeMaxTable];
  __shared__ long long s_x[kRopeMaxTokens], s_y[kRopeMaxTokens];       // where the tokens start, in elements
  using V = RopeVec<DT>;
  constexpr int N = VEC ? V::kN : 1;
  const int pairs = p.rot / 2;
  const long long t0 = static_cast<long long>(blockIdx.x) * p.tokens_per_block;
  const int count = static_cast<int>(min(static_cast<long long>(p.tokens_per_block), p.tokens - t0));
  for (int k = threadIdx.x; k < count * pairs; k += kRopeThreads) {
    const int tok = k / pairs, i = k - tok * pairs;
    const long long t = t0 + tok;
    const long long pos = p.positions != nullptr ? p.positions[t] : p.first + t % p.seq;
    double turn = static_cast<double>(pos) * p.turns[i];
    turn -= rint(turn);
    float s, c;
    sincospif(static_cast<float>(2.0 * turn), &s, &c);
    table[k] = make_float2(c * p.gain, (p.inverse ? -s : s) * p.gain);
  }
  if (threadIdx.x < count) {
    const long long t = t0 + threadIdx.x, b = t / p.seq, sq = t - b * p.seq;
    s_x[threadIdx.x] = b * p.xb + sq * p.xs;
    s_y[threadIdx.x] = b * p.yb + sq * p.ys;
  }
  __syncthreads();
  // in place, what is not turned is where it belongs
  const int rest = p.x == p.y ? 0 : (p.dim - p.rot) / N, turned = pairs / N, per_head = turned + (VEC ? (rest + 1) / 2 : rest), per_token = per_head * p.heads;
  const int work = count * per_token;
  constexpr int kElem = DT == 0 ? 4 : 2;
#pragma unroll 4
  for (int k = threadIdx.x; k < work; k += kRopeThreads) {
    const int tok = p.per_token.divide(k), in_token = k - tok * per_token;
    const int head = p.per_head.divide(in_token), item = in_token - head * per_head;
    const char* x = static_cast<const char*>(p.x) + (s_x[tok] + head * p.xh) * kElem;
    char* y = static_cast<char*>(p.y) + (s_y[tok] + head * p.yh) * kElem;
    const float2* cs = table + tok * pairs + item * N;
    const bool turn = item < turned;
    if (!VEC) {
      if (!turn) {
        const int e = p.rot + item - turned;
        rope_put<DT>(y, e, rope_get<DT>(x, e));
        continue;
      }
      const int ia = INTERLEAVED ? 2 * item : item, ib = INTERLEAVED ? 2 * item + 1 : item + pairs;
      const float a = rope_get<DT>(x, ia), q = rope_get<DT>(x, ib);
      rope_put<DT>(y, ia, a * cs[0].x - q * cs[0].y);
      rope_put<DT>(y, ib, a * cs[0].y + q * cs[0].x);
      continue;
    }
    // two vectors either way, so that turned and untouched items of a warp load and store together
    const int ea = turn ? (INTERLEAVED ? 2 * item * N : item * N) : p.rot + 2 * (item - turned) * N;
    const int eb = turn && !INTERLEAVED ? ea + pairs : ea + N;
    const bool two = turn || 2 * (item - turned) + 1 < rest;
    uint4 va = *reinterpret_cast<const uint4*>(x + ea * kElem), vb = make_uint4(0u, 0u, 0u, 0u);
    if (two) vb = *reinterpret_cast<const uint4*>(x + eb * kElem);
    if (turn) {
      float u[V::kN], w[V::kN], ou[V::kN], ow[V::kN];
      V::unpack(va, u);
      V::unpack(vb, w);
      if (INTERLEAVED) {
#pragma unroll
        for (int e = 0; e < V::kN; e += 2) {
          const float2 c0 = cs[e / 2], c1 = cs[V::kN / 2 + e / 2];
          ou[e] = u[e] * c0.x - u[e + 1] * c0.y;
          ou[e + 1] = u[e] * c0.y + u[e + 1] * c0.x;
          ow[e] = w[e] * c1.x - w[e + 1] * c1.y;
          ow[e + 1] = w[e] * c1.y + w[e + 1] * c1.x;
        }
      } else {
#pragma unroll
        for (int e = 0; e < V::kN; ++e) {
          const float2 c0 = cs[e];
          ou[e] = u[e] * c0.x - w[e] * c0.y;
          ow[e] = u[e] * c0.y + w[e] * c0.x;
        }
      }
      va = V::pack(ou);
      vb = V::pack(ow);
    }
    *reinterpret_cast<uint4*>(y + ea * kElem) = va;
    if (two) *reinterpret_cast<uint4*>(y + eb * kElem) = vb;
  }
}

}  // namespace adacons
