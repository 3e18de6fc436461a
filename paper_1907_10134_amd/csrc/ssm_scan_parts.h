// What the selective scan's kernels share: how the work is cut, and the arrays between launches.
//
// A workgroup takes 64 channels of one group, one a lane, of one sample.  Its waves split the states: wave w holds states
// 4 w .. 4 w + 3 of all 64 channels.  What the waves share goes through LDS: a step's size, made once for a channel, the
// sums over the states, and Bm and Cm, which are the same number for a whole wave.  (Those were scalar operands first, of
// no cost to the vector unit; but a scalar load can only be waited for with all others that are out, at every second step,
// and 32 of them at a time left so few scalar registers that a tenth of the vector instructions moved others out of the
// way.)  States along the lanes instead would need two vector additions a step for the sum over them.
#pragma once

#include "ssm_common.h"

namespace ssm {

constexpr int kTile = 64;        // channels of a workgroup, one a lane
constexpr int kHeld = 4;         // states of a channel that a wave holds
constexpr int kKept = 8;         // steps between two states kept for the backward pass

template <typename E>
struct Layer {
  Rows<const E> u, dt, z, Bm, Cm;
  const float *A, *skip, *dt_bias, *h0;
  const int32_t* lengths;
  int T, B, D, N, G, wide, tiles;      // wide = D / G channels a group, tiles = ceil(wide / 64) tiles a group
};

template <typename E>
Layer<E> layer_of(const bppsa_ssm& l) {
  const int wide = l.D / l.G;
  return Layer<E>{rows_of<const E>(l.u), rows_of<const E>(l.dt), rows_of<const E>(l.z), rows_of<const E>(l.Bm),
                  rows_of<const E>(l.Cm), l.A, l.skip, l.dt_bias, l.h0, l.lengths, l.T, l.B, l.D, l.N, l.G, wide,
                  bppsa_ceil_div(wide, kTile)};
}

// Waves of a workgroup for N states: the next of 1, 2, 4, 6, 8, 12, 16.
static inline int waves_of(int N) {
  const int need = (N + kHeld - 1) / kHeld;
  for (int w : {1, 2, 4, 6, 8, 12})
    if (need <= w) return w;
  return 16;
}
template <typename F>
bppsa_status by_waves(int waves, F&& f) {
  switch (waves) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 6: return f(std::integral_constant<int, 6>{});
    case 8: return f(std::integral_constant<int, 8>{});
    case 12: return f(std::integral_constant<int, 12>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

// Offsets of an array of states, float4 a channel and wave: [first][b][wave][d][4].
__host__ __device__ __forceinline__ int64_t state_at(int64_t first, int B, int b, int waves, int w, int D, int d) {
  return (((first * B + b) * waves + w) * D + d) * kHeld;
}

// Bm and Cm of a pass of kKept steps, for all waves of a workgroup: [step][wave][four Bm, four Cm], one value a thread.
// A thread fetches its value of a pass ahead, as an element, and leaves it in LDS as a float; a wave reads its eight of a
// step from one place, 16 bytes an access.  Zero beyond the states there are and behind a sample's end.
template <typename E>
struct Coef {
  uint64_t at;
  int64_t step;                    // of a pass
  int row;                         // of the pass
  bool real;
  __device__ __forceinline__ Coef(const Layer<E>& l, int waves, int thread, int first, int b, int g) {
    const int k = thread % (2 * kHeld), n = thread / (2 * kHeld) % waves * kHeld + k % kHeld;
    row = thread / (2 * kHeld) / waves, real = n < l.N;
    const Rows<const E> r{k < kHeld ? l.Bm.data : l.Cm.data, k < kHeld ? l.Bm.st : l.Cm.st, k < kHeld ? l.Bm.sb : l.Cm.sb};
    at = (uint64_t)(r.at(first + row, b) + g * l.N + (real ? n : 0));
    step = r.st * (int64_t)sizeof(E) * kKept;
  }
  __device__ __forceinline__ uint32_t fetch(int left) const { return real && row < left ? bits_at<E>(at) : 0; }   // left: steps of the pass that there are
  __device__ __forceinline__ void move(int passes) { at += passes * step; }
};
template <int SECOND, typename X>
__device__ __forceinline__ X& pick(X& a, X& b) {
  if constexpr (SECOND) return b;
  else return a;
}

// Two steps' instructions stay together: without a limit the compiler starts a whole pass's products and exponentials, twice
// the registers.
__device__ __forceinline__ void two_by_two(int i) {
  if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);
}
// The states are computed here and not later: nothing but the next pass needs them, and the compiler keeps the operands of
// several passes instead.
__device__ __forceinline__ void now(float (&h)[kHeld]) { asm volatile("" : "+v"(h[0]), "+v"(h[1]), "+v"(h[2]), "+v"(h[3])); }
__device__ __forceinline__ void four(const float* from, float (&v)[kHeld]) {
  const float4 x = *reinterpret_cast<const float4*>(from);
  v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
}

// A long sequence with few channels is cut into spans, each scanned by workgroups of its own.  A first launch scans each
// span from a state of zero and keeps only where that ends and the sum of its steps; a channel's decay over a span is
// exp(A sum), so that the second launch can join the spans between its own and the start in a multiply-add each, and scan
// its own from its true start.
struct Spans {
  int count, steps;
};
struct Summary {
  float *ends, *sums;              // [span][b][wave][d][4], [span][b][d]
};

// Carries h over `count` spans, from `first` on, one after the other by `step`.  Eight of them are asked for together: one at
// a time, the 47 of T = 30000 took some 20 us.
__device__ __forceinline__ void join_spans(const Summary& sum, int first, int step, int count, int B, int b, int waves, int w,
                                           int D, int d, const float (&A2)[kHeld], float (&h)[kHeld]) {
  constexpr int AHEAD = 8;
  for (int k = 0; k < count; k += AHEAD) {
    float4 end[AHEAD];
    float s[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int at = first + step * (k + j < count ? k + j : count - 1);
      end[j] = *reinterpret_cast<const float4*>(sum.ends + state_at(at, B, b, waves, w, D, d));
      s[j] = sum.sums[((int64_t)at * B + b) * D + d];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (k + j >= count) break;
      h[0] = fmaf(exp2_fast(A2[0] * s[j]), h[0], end[j].x), h[1] = fmaf(exp2_fast(A2[1] * s[j]), h[1], end[j].y);
      h[2] = fmaf(exp2_fast(A2[2] * s[j]), h[2], end[j].z), h[3] = fmaf(exp2_fast(A2[3] * s[j]), h[3], end[j].w);
    }
  }
}

// As many spans as give every SIMD `waves` waves, none shorter than 32 steps (a multiple of kKept), 64 at most.
static inline Spans spans_of(int T, int B, int D, int N, int G, int waves) {
  const int64_t have = (int64_t)G * bppsa_ceil_div(D / G, kTile) * B * waves_of(N);
  int64_t count = (int64_t)bppsa_compute_units() * 4 * waves / have;
  if (count > T / 32) count = T / 32;
  if (count > 64) count = 64;
  if (count < 2) return Spans{1, T};
  const int steps = bppsa_ceil_div(bppsa_ceil_div(T, (int)count), kKept) * kKept;
  return Spans{bppsa_ceil_div(T, steps), steps};
}

// Offsets of a workspace's arrays.
struct Arena {
  size_t at = 0;
  size_t operator()(int64_t floats) {
    const size_t o = at;
    at += bppsa_align_up((size_t)floats * sizeof(float), 256);
    return o;
  }
};

static inline bool sizes_ok(int T, int B, int D, int N, int G) {
  return T > 0 && B > 0 && D > 0 && N > 0 && G > 0 && N <= BPPSA_SSM_MAX_N && D % G == 0;
}

static inline bppsa_status check_layer(const bppsa_ssm* l) {
  if (!l || l->T < 1 || l->B < 1 || l->D < 1 || l->N < 1 || l->G < 1) return BPPSA_EINVAL;
  if (!l->u.data || !l->dt.data || !l->Bm.data || !l->Cm.data || !l->A) return BPPSA_EINVAL;
  if (l->D % l->G) return BPPSA_ESHAPE;
  if (l->N > BPPSA_SSM_MAX_N || l->type < BPPSA_F32 || l->type > BPPSA_F16) return BPPSA_EUNSUPPORTED;
  // one grid axis counts the samples; rows are addressed by 32 bits of bytes
  if (bppsa_mul_overflows(l->T, l->B, l->D, 2) || bppsa_mul_overflows(l->B, l->D, l->N, 1) || l->B > 65535 || l->D > 1 << 28 ||
      l->T > 0x7FFFFFFF - 64)
    return BPPSA_EOVERFLOW;
  return BPPSA_OK;
}

static inline bppsa_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need && (!workspace || have < need)) return BPPSA_EWORKSPACE;
  return need && ((uintptr_t)workspace & 255) ? BPPSA_EINVAL : BPPSA_OK;
}

}  // namespace ssm
