// Rows of logits, 16 bytes a lane at a time.
#pragma once

#include "ssm_common.h"

namespace chunks {

using namespace ssm;

// Eight 16-bit or four 32-bit logits as they were loaded, and the value of one.
template <typename E>
struct Chunk {
  static constexpr int N = 16 / sizeof(E);
  uint32_t w[4];
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
typedef uint32_t Four __attribute__((ext_vector_type(4)));
typedef Four Loose __attribute__((aligned(2)));
// A whole chunk at a place that is the same for all threads and a thread's offset of 32 bits: one address of scalar registers for
// each, where sixteen of vector registers would push the row out.
template <typename E>
__device__ __forceinline__ Chunk<E> load_whole(const E* place, uint32_t byte) {
  uint64_t at = (uint64_t)place;
  asm("" : "+s"(at));
  const Four w = *(const __attribute__((address_space(1))) Loose*)(at + byte);
  return Chunk<E>{{w.x, w.y, w.z, w.w}};
}
template <typename E>
__device__ __forceinline__ void store_whole(E* place, uint32_t byte, const float (&v)[Chunk<E>::N]) {
  uint64_t at = (uint64_t)place;
  asm("" : "+s"(at));
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

}  // namespace chunks
