// Rows of logits, 16 bytes a lane at a time, and their exponentials.
#pragma once

#include "ssm_common.h"

namespace logits {

using namespace ssm;

typedef uint32_t Four __attribute__((ext_vector_type(4)));
typedef Four Loose __attribute__((aligned(2)));

// Eight 16-bit or four 32-bit logits as they were loaded, and the value of one.  (Of one vector: an array that is loaded in a branch is taken apart
// there, which waits for the load.)
template <typename E>
struct Chunk {
  static constexpr int N = 16 / sizeof(E);
  Four w;
  // the first n become minus infinity
  __device__ __forceinline__ void leave_out(int n) {
    constexpr uint32_t none = sizeof(E) == 4 ? 0xFF800000u : std::is_same_v<E, bf16_t> ? 0xFF80u : 0xFC00u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(E) == 4) {
        if (i < n) w[i] = none;
      } else {
        if (2 * i < n) w[i] = (w[i] & 0xFFFF0000u) | none;
        if (2 * i + 1 < n) w[i] = (w[i] & 0xFFFFu) | none << 16;
      }
    }
  }
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[k]);
    else if constexpr (std::is_same_v<E, bf16_t>) return __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
    else return static_cast<float>(__builtin_bit_cast(E, (uint16_t)(k & 1 ? w[k / 2] >> 16 : w[k / 2])));
  }
};
// A whole chunk at a place that is the same for all threads and a thread's offset of 32 bits: one address of scalar registers for
// each, where sixteen of vector registers would push the row out.
template <typename E>
__device__ __forceinline__ Chunk<E> load_whole(const E* place, uint32_t byte) {
  uint64_t at = (uint64_t)place;
  asm("" : "+s"(at), "+v"(byte));
  return Chunk<E>{*(const __attribute__((address_space(1))) Loose*)(at + byte)};
}
template <typename E>
__device__ __forceinline__ void store_whole(E* place, uint32_t byte, const float (&v)[Chunk<E>::N]) {
  uint64_t at = (uint64_t)place;
  asm("" : "+s"(at), "+v"(byte));
  Some<E, Chunk<E>::N> s;
#pragma unroll
  for (int k = 0; k < Chunk<E>::N; ++k) s.v[k] = static_cast<E>(v[k]);
  *(__attribute__((address_space(1))) Loose*)(at + byte) = __builtin_bit_cast(Four, s);
}
// What lies behind the row's end counts as minus infinity, which has no share.
template <typename E>
__device__ __forceinline__ Chunk<E> load_chunk(const E* x, int at, int V) {
  constexpr int N = Chunk<E>::N;
  if (at + N <= V) return __builtin_bit_cast(Chunk<E>, load_some<E, N>(x + at));
  Some<E, N> s;
#pragma unroll
  for (int k = 0; k < N; ++k) s.v[k] = at + k < V ? x[at + k] : static_cast<E>(-INFINITY);
  return __builtin_bit_cast(Chunk<E>, s);
}
template <typename E>
__device__ __forceinline__ void store_chunk(E* x, int at, int V, const float (&v)[Chunk<E>::N]) {
  constexpr int N = Chunk<E>::N;
  if (at + N <= V) return store_some<E, N>(x + at, v);
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (at + k < V) store(x + at + k, v[k]);
}

// exp((x - m) scale) for logits of which m is the largest.  float32 logits take the corrected exponential.  For 16-bit ones it is one
// multiply-add in front of the exponential, 2^(k x - k m) with k = scale log2(e): what the rounding of k m leaves is the same factor
// 2^off in all of a row's, and is taken from the logarithm of their sum.  Where k m passes 2^20 the next smaller logit of 16
// bits has no share left, with a k of 2^20 / m either: so nothing overflows.
template <typename E>
struct Exponential {
  float m, scale, k, km, off;
  __device__ __forceinline__ Exponential(float largest, float scale)
      : m(largest), scale(scale), k(fminf(scale * kLog2e, 0x1p20f / fabsf(largest))), km(largest * k), off(fmaf(largest, k, -km)) {}
  __device__ __forceinline__ float operator()(float x) const {
    if constexpr (kExact<E>) return exp_of<true>((x - m) * scale);
    else return exp2_fast(fmaf(x, k, -km));
  }
  // what comes off the logarithm of a sum of such
  __device__ __forceinline__ double log_off() const { return kExact<E> ? 0.0 : 0.69314718055994531 * (double)off; }
};

// log(v), within 2^-23: the exponent's part is exact, and the instruction sees values from 0.7 to 1.4 alone, whose logarithms are small.
__device__ __forceinline__ double log_of(float v) {
  int e = __builtin_amdgcn_frexp_expf(v);
  float f = __builtin_amdgcn_frexp_mantf(v);
  if (f < 0.70710678f) f += f, --e;
  return ((double)e + (double)__builtin_amdgcn_logf(f)) * 0.69314718055994531;
}

}  // namespace logits
