// Shared by the state space kernels: the types of activations, strided rows, the step's softplus and the gate.
#pragma once

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
__device__ __forceinline__ float load(const E* p) { return static_cast<float>(*p); }
template <typename E>
__device__ __forceinline__ void store(E* p, float v) { *p = static_cast<E>(v); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp, 2^x
constexpr float kLog2e = 1.44269504088896340736f;

// exp(-|x|).  The product with log2(e) loses |x| 2^-24 of the result; its rounding and the constant's own come back as a
// first-order term, which leaves v_exp_f32's error.
__device__ __forceinline__ float exp_of_minus(float x) {
  const float a = -fabsf(x), p = a * kLog2e;
  float lost = fmaf(a, kLog2e, -p);
  lost = fmaf(a, 1.92596299112661746887e-8f, lost);
  const float e = exp2_fast(p);
  return p < -150.0f ? 0.0f : fmaf(e, lost * 0.69314718055994530942f, e);      // an infinite x: infinity minus itself above
}

// 1 / y, v_rcp_f32 and a correction: to half a step.
__device__ __forceinline__ float reciprocal(float y) {
  const float r = __builtin_amdgcn_rcpf(y);
  return fmaf(fmaf(-y, r, 1.0f), r, r);
}

// 1 / (1 + exp(-x)): exp of the negative magnitude only, so nothing overflows.
__device__ __forceinline__ float sigmoid(float x) {
  const float e = exp_of_minus(x), r = reciprocal(1.0f + e);
  return x >= 0.0f ? r : e * r;
}

// max(x, 0) + log1p(exp(-|x|)).  log1p(e) = 2 atanh(s), s = e / (2 + e) <= 1/3, as an odd polynomial in s: log(1 + e)
// by the logarithm instruction would lose the small steps (e = 1e-3 keeps 2^-14 of its value in 1 + e).
// Series terms to s^15; the next is 2^-29 of the first at s = 1/3.
__device__ __forceinline__ float softplus(float x) {
  const float e = exp_of_minus(x);
  const float s = e * reciprocal(2.0f + e);
  const float w = s * s;
  float p = 1.0f / 15;
  p = fmaf(p, w, 1.0f / 13);
  p = fmaf(p, w, 1.0f / 11);
  p = fmaf(p, w, 1.0f / 9);
  p = fmaf(p, w, 1.0f / 7);
  p = fmaf(p, w, 1.0f / 5);
  p = fmaf(p, w, 1.0f / 3);
  p *= w;
  return fmaxf(x, 0.0f) + 2.0f * fmaf(s, p, s);
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
