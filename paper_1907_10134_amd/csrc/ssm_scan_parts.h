// What the selective scan's kernels share: how the work is cut, and the arrays between launches.
//
// A workgroup takes 64 channels of one group, one a lane, of one sample.  Its waves split the states: wave w holds H states of all
// 64 channels, from H w on.  What the waves share goes through LDS: a step's size, made once for a channel, the
// sums over the states, and Bm and Cm, which are the same number for a whole wave.  (Those were scalar operands first, of
// no cost to the vector unit; but a scalar load can only be waited for with all others that are out, at every second step,
// and 32 of them at a time left so few scalar registers that a tenth of the vector instructions moved others out of the
// way.)  States along the lanes instead would need two vector additions a step for the sum over them.
#pragma once

#include <algorithm>

#include "ssm_common.h"

namespace ssm {

constexpr int kTile = 64;        // channels of a workgroup, one a lane
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

// The waves of a workgroup for N states and how many of them each holds: four, but two where there are few, or as many rows as
// eight would be a wave's to prepare (at N = 8 two waves of four states took longer than N = 16 does).
static inline int held_of(int N) { return N <= 8 ? 2 : 4; }
static inline int waves_of(int N) {
  return N <= 4 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : N <= 48 ? 12 : 16;
}
static inline int padded_of(int N) { return waves_of(N) * held_of(N); }
template <typename F>
bppsa_status by_states(int N, F&& f) {
  typedef std::integral_constant<int, 2> Two;
  typedef std::integral_constant<int, 4> Four;
  if (N <= 4) return f(std::integral_constant<int, 2>{}, Two{});
  if (N <= 8) return f(std::integral_constant<int, 4>{}, Two{});
  if (N <= 16) return f(std::integral_constant<int, 4>{}, Four{});
  if (N <= 32) return f(std::integral_constant<int, 8>{}, Four{});
  if (N <= 48) return f(std::integral_constant<int, 12>{}, Four{});
  return f(std::integral_constant<int, 16>{}, Four{});
}

// Offsets of an array of states, `held` floats a channel and wave: [first][b][wave][d][held].
__host__ __device__ __forceinline__ int64_t state_at(int held, int64_t first, int B, int b, int waves, int w, int D, int d) {
  return (((first * B + b) * waves + w) * D + d) * held;
}
template <int H>
struct alignas(4 * H) States {
  float v[H];
};
template <int H>
__device__ __forceinline__ void get(const float* from, float (&v)[H]) {
  const States<H> x = *reinterpret_cast<const States<H>*>(from);
#pragma unroll
  for (int i = 0; i < H; ++i) v[i] = x.v[i];
}
template <int H>
__device__ __forceinline__ void put(float* to, const float (&v)[H]) {
  States<H> x;
#pragma unroll
  for (int i = 0; i < H; ++i) x.v[i] = v[i];
  *reinterpret_cast<States<H>*>(to) = x;
}

// Bm and Cm of a pass of kKept steps, for all waves of a workgroup: [step][wave][H of Bm, H of Cm], one value a thread.
// A thread fetches its value of a pass ahead, as an element, and leaves it in LDS as a float; a wave reads those of its
// states of a step from one place, all at once.  Zero beyond the states there are and behind a sample's end.
template <typename E, int H>
struct Coef {
  uint64_t at;
  int64_t step;                    // of a pass
  int row;                         // of the pass
  bool real;
  __device__ __forceinline__ Coef(const Layer<E>& l, int waves, int thread, int first, int b, int g) {
    const int k = thread % (2 * H), n = thread / (2 * H) % waves * H + k % H;
    row = thread / (2 * H) / waves, real = n < l.N && row < kKept;
    const Rows<const E> r{k < H ? l.Bm.data : l.Cm.data, k < H ? l.Bm.st : l.Cm.st, k < H ? l.Bm.sb : l.Cm.sb};
    at = (uint64_t)(r.at(first + (row < kKept ? row : 0), b) + g * l.N + (real ? n : 0));
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
template <int H>
__device__ __forceinline__ void now(float (&h)[H]) {
#pragma unroll
  for (int i = 0; i < H; ++i) asm volatile("" : "+v"(h[i]));
}

// A long sequence with few channels is cut into spans, each scanned by workgroups of its own.  A first launch scans each
// span from a state of zero and keeps only where that ends and the sum of its steps; a channel's decay over a span is
// exp(A sum), so that the second launch can join the spans between its own and the start in a multiply-add each, and scan
// its own from its true start.
struct Spans {
  int count, steps;
};
struct Summary {
  float *ends, *sums;              // [span][b][wave][d][held], [span][b][d]
};

// Carries h over `count` spans, from `first` on, one after the other by `step`.  Eight of them are asked for together: one at
// a time, the 47 of T = 30000 took some 20 us.
// Where a state grows (a positive A), a span's factor may pass the largest float though its product with a small state does
// not: three factors of a third of the exponent, one after the other, are as large as a product of floats can be made.
// Such states go one span at a time, by a loop that is short: both ways eight at a time cost a kernel that joins one span
// 15.6 us instead of 14.5 (T = 64, B = 24, D = 254, N = 64).
template <int H>
__device__ __forceinline__ void join_spans(const Summary& sum, int first, int step, int count, int B, int b, int waves, int w,
                                           int D, int d, const float (&A2)[H], float (&h)[H]) {
  constexpr int AHEAD = 8;
  bool grows = false;
#pragma unroll
  for (int i = 0; i < H; ++i) grows |= A2[i] > 0.0f;
  if (__any(grows)) {
#pragma unroll 1
    for (int k = 0; k < count; ++k) {
      const int at = first + step * k;
      float end[H];
      get(sum.ends + state_at(H, at, B, b, waves, w, D, d), end);
      const float third = sum.sums[((int64_t)at * B + b) * D + d] * (1.0f / 3.0f);
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const float factor = exp2_fast(A2[i] * third);
        h[i] = h[i] == 0.0f ? end[i] : fmaf(h[i] * factor * factor, factor, end[i]);      // zero stays zero
      }
    }
    return;
  }
  for (int k = 0; k < count; k += AHEAD) {
    float end[AHEAD][H], s[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int at = first + step * (k + j < count ? k + j : count - 1);
      get(sum.ends + state_at(H, at, B, b, waves, w, D, d), end[j]);
      s[j] = sum.sums[((int64_t)at * B + b) * D + d];
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (k + j >= count) break;
#pragma unroll
      for (int i = 0; i < H; ++i) h[i] = fmaf(exp2_fast(A2[i] * s[j]), h[i], end[j][i]);
    }
  }
}

// As many spans as give every SIMD `waves` waves, none shorter than 32 steps (a multiple of kKept), 64 at most.  Where samples
// have lengths of their own, three quarters more: spans behind an end leave units free for others (T = 1000, B =
// 16, D = 640: 76 us with twice the spans, 87 with as many as below; without lengths twice as many cost T = 2048, B =
// 64, D = 32 a sixth).
static inline Spans spans_of(int T, int B, int D, int N, int G, int waves, bool ragged) {
  const int64_t have = (int64_t)G * bppsa_ceil_div(D / G, kTile) * B * waves_of(N);
  int64_t count = (int64_t)bppsa_compute_units() * 4 * (ragged ? waves * 7 / 4 : waves) / have;
  if (count > T / 32) count = T / 32;
  if (count > 64) count = 64;
  if (count < 2) return Spans{1, T};
  const int steps = bppsa_ceil_div(bppsa_ceil_div(T, (int)count), kKept) * kKept;
  return Spans{bppsa_ceil_div(T, steps), steps};
}
// What a workspace, whose size is asked for without lengths, has to hold.
static inline int most_spans(int T, int B, int D, int N, int G, int waves) {
  return std::max(spans_of(T, B, D, N, G, waves, false).count, spans_of(T, B, D, N, G, waves, true).count);
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

// One grid axis counts the samples, rows are addressed by 32 bits of bytes, and a launch has fewer than 2^32 threads.
static inline bool too_large(int T, int B, int D, int N, int G) {
  return bppsa_mul_overflows(T, B, D, 2) || bppsa_mul_overflows(B, D, N, 1) || B > 65535 || D > 1 << 24 || T > 0x7FFFFFFF - 64 ||
         (int64_t)G * bppsa_ceil_div(D / G, kTile) >= 1 << 22;
}

static inline bool sizes_ok(int T, int B, int D, int N, int G) {
  return T > 0 && B > 0 && D > 0 && N > 0 && G > 0 && N <= BPPSA_SSM_MAX_N && D % G == 0 && !too_large(T, B, D, N, G);
}

static inline bppsa_status check_layer(const bppsa_ssm* l) {
  if (!l || l->T < 1 || l->B < 1 || l->D < 1 || l->N < 1 || l->G < 1) return BPPSA_EINVAL;
  if (!l->u.data || !l->dt.data || !l->Bm.data || !l->Cm.data || !l->A) return BPPSA_EINVAL;
  if (l->D % l->G) return BPPSA_ESHAPE;
  if (l->N > BPPSA_SSM_MAX_N || l->type < BPPSA_F32 || l->type > BPPSA_F16) return BPPSA_EUNSUPPORTED;
  return too_large(l->T, l->B, l->D, l->N, l->G) ? BPPSA_EOVERFLOW : BPPSA_OK;
}

// The kept states are read and written by 8 and 16 bytes.
static inline bool states_ok(const void* states) { return ((uintptr_t)states & 15) == 0; }

static inline bppsa_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need && (!workspace || have < need)) return BPPSA_EWORKSPACE;
  return need && ((uintptr_t)workspace & 255) ? BPPSA_EINVAL : BPPSA_OK;
}

}  // namespace ssm
