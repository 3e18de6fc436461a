// Sums, largest values and the like over the 64 lanes of a wave, in every lane: halves and rows of lanes exchange registers, then
// rows of sixteen are turned by eight, four, two and one.  Every level joins the same two groups in all lanes, so all lanes have
// the same bits.  None of it goes through LDS, as a general shuffle does.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lanes {

template <typename T>
struct Pair {
  T a, b;
};
template <int ROW>                 // 32 or 16: each lane has the values of itself and of the lane so many away
__device__ __forceinline__ Pair<uint32_t> exchange(uint32_t v) {
  if constexpr (ROW == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return Pair<uint32_t>{r[0], r[1]};
  } else {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return Pair<uint32_t>{r[0], r[1]};
  }
}
template <int BY>
__device__ __forceinline__ uint32_t turn(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + BY, 0xf, 0xf, true);
}

template <int ROW, typename T>
__device__ __forceinline__ Pair<T> exchanged(T v) {
  if constexpr (sizeof(T) == 4) {
    const Pair<uint32_t> r = exchange<ROW>(__builtin_bit_cast(uint32_t, v));
    return Pair<T>{__builtin_bit_cast(T, r.a), __builtin_bit_cast(T, r.b)};
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const Pair<uint32_t> lo = exchange<ROW>((uint32_t)u), hi = exchange<ROW>((uint32_t)(u >> 32));
    return Pair<T>{__builtin_bit_cast(T, (uint64_t)hi.a << 32 | lo.a), __builtin_bit_cast(T, (uint64_t)hi.b << 32 | lo.b)};
  }
}
template <int BY, typename T>
__device__ __forceinline__ T turned(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, turn<BY>(__builtin_bit_cast(uint32_t, v)));
  } else {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(T, (uint64_t)turn<BY>((uint32_t)(u >> 32)) << 32 | turn<BY>((uint32_t)u));
  }
}

// f has to be symmetric.
template <typename T, typename F>
__device__ __forceinline__ T all(T v, F&& f) {
  const Pair<T> halves = exchanged<32>(v);
  v = f(halves.a, halves.b);
  const Pair<T> rows = exchanged<16>(v);
  v = f(rows.a, rows.b);
  v = f(v, turned<8>(v)), v = f(v, turned<4>(v)), v = f(v, turned<2>(v));
  return f(v, turned<1>(v));
}
template <typename T>
__device__ __forceinline__ T sum(T v) {
  return all(v, [](T a, T b) { return a + b; });
}
template <typename T>
__device__ __forceinline__ T largest(T v) {
  if constexpr (sizeof(T) == 4 && __is_floating_point(T)) return all(v, [](T a, T b) { return fmaxf(a, b); });
  else return all(v, [](T a, T b) { return a > b ? a : b; });
}

}  // namespace lanes
