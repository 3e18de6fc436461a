// What the selective scan's kernels share: how the work is cut, and the arrays between launches.
//
// A workgroup takes 64 channels of one group, one a lane, of one sample.  Its waves split the states: wave w holds states
// 4 w .. 4 w + 3 of all 64 channels, so that Bm and Cm of a step are the same number for a whole wave.  They come through
// the scalar cache into scalar registers from a float array that a first small launch writes (`coef`), and cost the vector
// unit nothing; what the waves share, the step's size and the sums over the states, goes through LDS once a channel.
// The other layout that was thought through, states along the lanes, needs two vector additions a step and four states
// for the sum over them and 16 bytes of LDS reads a state for Bm and Cm, which by itself would bind the kernel.
#pragma once

#include "ssm_common.h"

namespace ssm {

constexpr int kTile = 64;        // channels of a workgroup, one a lane
constexpr int kHeld = 4;         // states of a channel that a wave holds
constexpr int kKept = 8;         // steps between two states kept for the backward pass
constexpr int kPad = kKept;      // `coef` reaches to the next multiple of so many steps: a span's last steps are not tested for

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

// coef [b][g][w][t][8]: four Bm, then four Cm, zero beyond the states there are and behind a sample's end.
static inline int64_t coef_floats(int64_t T, int64_t B, int64_t N, int64_t G) {
  return B * G * ((T + kPad - 1) / kPad * kPad) * waves_of((int)N) * 2 * kHeld;
}

// A forward call that keeps states for the backward pass keeps coef in front of them, up to this many groups (the size of
// the states is asked for without G): one launch less there.
constexpr int kGroupsKept = 4;
static inline size_t kept_coef_floats(int64_t T, int64_t B, int64_t N) {
  return bppsa_align_up((size_t)coef_floats(T, B, N, kGroupsKept), 64);
}

template <typename E>
static __global__ void __launch_bounds__(256)
coef_kernel(const Layer<E> l, int waves, int64_t all, float* __restrict__ coef) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= all) return;
  const int of = (int)(i % 8), padded = (l.T + kPad - 1) / kPad * kPad;
  const int64_t row = i / 8;
  const int t = (int)(row % padded), w = (int)(row / padded % waves);
  const int64_t bg = row / padded / waves;
  const int g = (int)(bg % l.G), b = (int)(bg / l.G), n = w * kHeld + of % kHeld;
  const bool in = n < l.N && t < clamp_length(l.lengths, b, l.T);
  coef[i] = in ? load((of < kHeld ? l.Bm : l.Cm).at(t, b) + g * l.N + n) : 0.0f;
}

// Bm and Cm of STEPS steps in scalar registers.  Scalar loads come back in any order, so the only wait for one is the wait
// for all that are out, LDS reads among them: a batch's loads go out together, right behind the wait for the batch
// before, and have the time of that one's steps.  (Left to the compiler, which asks for one step's at a time, a wave
// waited for every one: 492 us instead of 344 at T = 30000, D = 2048.)  Batches of four steps, 64 registers for two of them,
// suit the summaries; in the main kernels they left so few that a quarter of the backward pass's vector instructions moved
// scalars to and from vector lanes: batches of two there.
typedef float TwoSteps __attribute__((ext_vector_type(4 * kHeld)));
typedef const __attribute__((address_space(4))) TwoSteps* ScalarCoef;       // read through the scalar cache
template <int STEPS>
struct Coef {
  TwoSteps at[STEPS / 2];
  __device__ __forceinline__ void ask(const float* from) {
#pragma unroll
    for (int k = 0; k < STEPS / 2; ++k) at[k] = ((ScalarCoef)from)[k];
  }
  __device__ __forceinline__ float B(int i, int k) const { return at[i / 2][i % 2 * 2 * kHeld + k]; }
  __device__ __forceinline__ float C(int i, int k) const { return at[i / 2][i % 2 * 2 * kHeld + kHeld + k]; }
};
// All scalar loads and LDS accesses of this wave are done; none of what follows is moved in front of it.
__device__ __forceinline__ void wait_for_scalars() {
  __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0), nothing else
  __builtin_amdgcn_sched_barrier(0);
}

template <typename E>
static void launch_coef(const Layer<E>& l, float* coef, hipStream_t s) {
  const int64_t all = coef_floats(l.T, l.B, l.N, l.G);
  coef_kernel<E><<<(unsigned)((all + 255) / 256), 256, 0, s>>>(l, waves_of(l.N), all, coef);
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

// As many spans as give every SIMD `waves` waves, none shorter than 32 steps (a multiple of kPad), 64 at most.
static inline Spans spans_of(int T, int B, int D, int N, int G, int waves) {
  const int64_t have = (int64_t)G * bppsa_ceil_div(D / G, kTile) * B * waves_of(N);
  int64_t count = (int64_t)bppsa_compute_units() * 4 * waves / have;
  if (count > T / 32) count = T / 32;
  if (count > 64) count = 64;
  if (count < 2) return Spans{1, T};
  const int steps = bppsa_ceil_div(bppsa_ceil_div(T, (int)count), kPad) * kPad;
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
