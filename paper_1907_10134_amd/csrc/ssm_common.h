// Shared by the state space kernels: the types of activations, strided rows, the step's softplus and the gate.
#pragma once

#include <type_traits>

#include "bppsa_internal.h"

namespace ssm {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Base of row (t, b) of a strided array; offsets in 64 bits, a long prompt's array passes 2^31 elements.
template <typename E>
struct Rows {
  E* data;
  int64_t st, sb;
  __device__ __forceinline__ E* at(int t, int b) const { return data + (int64_t)t * st + (int64_t)b * sb; }
};
template <typename E>
Rows<E> rows_of(const bppsa_rows& r) {
  return Rows<E>{static_cast<E*>(r.data), r.stride_t, r.stride_b};
}

// Activations are computed in fp32 and rounded once, to the nearest even, when they are stored.
template <typename E>
__device__ __forceinline__ void store(E* p, float v) { *p = static_cast<E>(v); }

// An element as it was loaded, in a register of its own, and its value.
template <typename E>
__device__ __forceinline__ uint32_t bits_at(uint64_t address) {
  typedef std::conditional_t<sizeof(E) == 4, uint32_t, uint16_t> U;
  return *(const __attribute__((address_space(1))) U*)address;
}
template <typename E>
__device__ __forceinline__ float value(uint32_t bits) {
  if constexpr (sizeof(E) == 4) return __uint_as_float(bits);
  else return static_cast<float>(__builtin_bit_cast(E, (uint16_t)bits));
}

// The rows of an array that a wave walks through: a lane's address in vector registers, moved on by a stride in scalar ones.
// (Both in scalar registers, with the lane's offset added by the access, left too few of them while Bm and Cm were scalars too; not
// tried since those are in LDS.)
template <typename E>
struct Walk {
  uint64_t lane;
  int64_t step, move_by;           // bytes of a row and of a pass
  __device__ __forceinline__ Walk(const Rows<E>& r, int t, int b, uint32_t byte, int rows_of_pass)
      : lane((uint64_t)r.at(t, b) + byte), step(r.st * (int64_t)sizeof(E)), move_by(rows_of_pass * step) {
    asm("" : "+s"(move_by));       // or a pass back is taken off by two instructions instead of added by one
  }
  __device__ __forceinline__ uint32_t bits(int rows_on) const { return bits_at<E>(lane + rows_on * step); }
  __device__ __forceinline__ void put(int rows_on, float v) const {
    *(__attribute__((address_space(1))) E*)(lane + rows_on * step) = static_cast<E>(v);
  }
  __device__ __forceinline__ void move() { lane += move_by; }
};

// V neighbouring elements by one access of any alignment: the memory path takes 16 bytes from an odd element as well, and a
// line that is crossed costs less than eight accesses do.
template <typename E, int V>
struct __attribute__((packed, aligned(sizeof(E)))) Some {
  E v[V];
};
template <typename E, int V>
__device__ __forceinline__ Some<E, V> load_some(const E* p) { return *reinterpret_cast<const Some<E, V>*>(p); }
template <typename E, int V>
__device__ __forceinline__ void store_some(E* p, const float (&x)[V]) {
  Some<E, V> s;
#pragma unroll
  for (int i = 0; i < V; ++i) s.v[i] = static_cast<E>(x[i]);
  *reinterpret_cast<Some<E, V>*>(p) = s;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp, 2^x
constexpr float kLog2e = 1.44269504088896340736f;

// exp(a).  EXACT, for a of at most 87: the product with log2(e) loses |x| 2^-24 of the
// result; its rounding and the constant's own come back as a first-order term, which leaves v_exp_f32's error.  Without, for
// activations of 16 bits, whose own rounding is 2^8 times as much.
template <bool EXACT>
__device__ __forceinline__ float exp_of(float a) {
  const float p = a * kLog2e;
  const float e = exp2_fast(p);
  if (!EXACT) return e;
  const float lost = fmaf(a, 1.92596299112661746887e-8f, fmaf(a, kLog2e, -p));
  return a < -87.0f ? e : fmaf(e, lost * 0.69314718055994530942f, e);          // a = -infinity: p - p is none
}

// 1 / (c + e), c a whole number.  EXACT: v_rcp_f32 (1 ulp) corrected once, with what the sum's rounding lost.
template <bool EXACT>
__device__ __forceinline__ float reciprocal_sum(float c, float e) {
  const float y = c + e, r = __builtin_amdgcn_rcpf(y);
  if (!EXACT) return r;
  const float lost = c > e ? e - (y - c) : c - (y - e);
  return fmaf(fmaf(-y, r, 1.0f) - lost * r, r, r);
}

template <typename E>
constexpr bool kExact = sizeof(E) == 4;

// 1 / (1 + exp(-x)); nothing is left of it for very negative x, down to the lowest value of a type, of which x times this and
// its derivative have to be zero.  EXACT: from exp(-|x|), so that no exponential is infinite and needs a correction; without, an
// infinite one gives zero by itself.
template <typename E>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (kExact<E>) {
    const float e = exp_of<true>(-fabsf(x)), r = reciprocal_sum<true>(1.0f, e);
    return x >= 0.0f ? r : e * r;
  } else {
    return reciprocal_sum<false>(1.0f, exp_of<false>(-x));
  }
}

// max(x, 0) + log1p(exp(-|x|)).  log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3, as an odd polynomial in s: log(1 + e)
// by the logarithm instruction would lose the small steps (e = 1e-3 keeps 2^-14 of its value in 1 + e).
// (atanh(s) / s - 1) / s^2 interpolated at the four Chebyshev nodes of s^2 in [0, 1/9]: within 2^-25 of 2 atanh(s).
template <typename E>
__device__ __forceinline__ float softplus(float x) {
  const float e = exp_of<kExact<E>>(-fabsf(x));
  const float s = e * reciprocal_sum<kExact<E>>(2.0f, e);
  const float w = s * s;
  const float p = w * fmaf(fmaf(fmaf(0.13426013f, w, 0.14118274f), w, 0.20003782f), w, 0.3333332f);
  return fmaf(2.0f, fmaf(s, p, s), fmaxf(x, 0.0f));
}

__device__ __forceinline__ int clamp_length(const int32_t* lengths, int b, int T) {
  if (!lengths) return T;
  const int n = lengths[b];
  return n < 0 ? 0 : (n > T ? T : n);
}

// Whether no two rows of an output share a place: a stride of zero repeats a row, which is an input's privilege.
static inline bool writable(const bppsa_rows& r, int T, int B) {
  return r.data && (T == 1 || r.stride_t != 0) && (B == 1 || r.stride_b != 0);
}

template <typename F>
bppsa_status by_type(int type, F&& f) {
  switch (type) {
    case BPPSA_F32: return f(float{});
    case BPPSA_BF16: return f(bf16_t{});
    case BPPSA_F16: return f(f16_t{});
    default: return BPPSA_EUNSUPPORTED;
  }
}

}  // namespace ssm
