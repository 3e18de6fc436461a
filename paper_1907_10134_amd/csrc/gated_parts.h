// What the gated recurrence's kernels share: the layer, how the work is cut, and the gates of a step.
#pragma once

#include <algorithm>

#include "ssm_common.h"

namespace gated {

using namespace ssm;

constexpr int kWaves = 8;        // of a workgroup, each with a run of neighbouring steps of a tile
constexpr int kKept = 64;        // steps between two states kept for the backward pass, whose tiles are as long

// A lane has V neighbouring channels, a workgroup 64 V.  The last lane of a row starts early enough to have V too and repeats
// some of its neighbour's, with the same results.
template <typename E>
struct Layer {
  Rows<const E> x, r, i, z;
  const float *decay, *r_bias, *i_bias, *h0;
  const int32_t* lengths;
  int T, B, D, columns;
};
template <typename E>
Layer<E> layer_of(const bppsa_gated& l, int wide) {
  return Layer<E>{rows_of<const E>(l.x), rows_of<const E>(l.r), rows_of<const E>(l.i), rows_of<const E>(l.z), l.decay, l.r_bias,
                  l.i_bias, l.h0, l.lengths, l.T, l.B, l.D, bppsa_ceil_div(l.D, wide)};
}

template <int V>
struct Own {                     // a lane's channels, of which the first `repeated` are its neighbour's
  int d, repeated;
  bool on;
  __device__ __forceinline__ Own(int column, int lane, int D) {
    d = (column * 64 + lane) * V;
    on = d < D;
    repeated = on && d > D - V ? d - (D - V) : 0;
    if (d > D - V) d = D - V;
  }
};
template <int V>
__device__ __forceinline__ void parameter(const float* p, int d, float (&v)[V]) {
#pragma unroll
  for (int c = 0; c < V; ++c) v[c] = p ? p[d + c] : 0.0f;
}

// 1 - exp(-x) for x >= 0, given e = exp(-x): below 1/4, where the difference would lose bits, x times the series of
// (1 - exp(-x)) / x up to x^6 / 7!, within 2^-26 of it.
__device__ __forceinline__ float one_minus(float e, float x) {
  float p = fmaf(x, 1.0f / 5040.0f, -1.0f / 720.0f);
  p = fmaf(p, x, 1.0f / 120.0f), p = fmaf(p, x, -1.0f / 24.0f), p = fmaf(p, x, 1.0f / 6.0f), p = fmaf(p, x, -0.5f);
  p = fmaf(p, x, 1.0f);
  return x < 0.25f ? x * p : 1.0f - e;
}

// A step's gates: rho and iota, the decay a = exp(-decay rho) and m2 = 1 - a^2, of which what enters is the root.
struct Gates {
  float rho, iota, a, m2;
};
template <typename E>
__device__ __forceinline__ Gates gates_of(float r, float i, float decay) {
  Gates g;
  g.rho = sigmoid<E>(r), g.iota = sigmoid<E>(i);
  const float size = decay * g.rho;
  g.a = exp_of<kExact<E>>(-size);
  g.m2 = one_minus(g.a * g.a, size + size);
  return g;
}

// One grid axis counts tiles, samples and columns; a launch has fewer than 2^32 threads.
static inline int64_t workgroups(int T, int B, int D) {
  return (int64_t)bppsa_ceil_div(T, kKept) * B * bppsa_ceil_div(D, 64);
}
static inline bool too_large(int T, int B, int D) {
  return bppsa_mul_overflows(T, B, D, 4) || T > 0x7FFFFFFF - 1024 || D > 1 << 24 || workgroups(T, B, D) >= 1 << 23;
}
static inline bool sizes_ok(int T, int B, int D) { return T > 0 && B > 0 && D > 0 && !too_large(T, B, D); }

static inline bppsa_status check_layer(const bppsa_gated* l) {
  if (!l || l->T < 1 || l->B < 1 || l->D < 1) return BPPSA_EINVAL;
  if (!l->x.data || !l->r.data || !l->i.data || !l->decay) return BPPSA_EINVAL;
  if (l->type < BPPSA_F32 || l->type > BPPSA_F16) return BPPSA_EUNSUPPORTED;
  return too_large(l->T, l->B, l->D) ? BPPSA_EOVERFLOW : BPPSA_OK;
}

static inline bppsa_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need && (!workspace || have < need)) return BPPSA_EWORKSPACE;
  return need && ((uintptr_t)workspace & 255) ? BPPSA_EINVAL : BPPSA_OK;
}

// Two channels a lane, or one where there is only one.
template <typename F>
bppsa_status by_width(int D, F&& f) {
  if (D >= 2) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 1>{});
}

}  // namespace gated
