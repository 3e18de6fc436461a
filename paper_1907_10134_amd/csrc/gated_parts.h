// What the gated recurrence's kernels share: the layer, how the work is cut, and the gates of a step.
#pragma once

#include <algorithm>

#include "barriers.h"
#include "ssm_common.h"

namespace gated {

using namespace ssm;

constexpr int kWaves = 8;        // of a workgroup, each with a run of neighbouring steps of a tile
constexpr int kRun = 16, kRunBack = 8;         // steps of a run, forward and backward
constexpr int kTile = kWaves * kRun, kKept = kWaves * kRunBack;      // steps of a tile; a state is kept before each of the backward pass

// A lane has V neighbouring channels, 4 bytes of them, a workgroup 64 V.  The last lane of a row starts early enough to have V too and repeats
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
// Values stay as they were loaded up to here: the compiler would widen them as soon as it can and hold twice the registers.
template <typename E, int V>
__device__ __forceinline__ void as_loaded(Some<E, V>& x) {
  static_assert(sizeof(x) <= 4);
  typedef std::conditional_t<sizeof(x) == 4, uint32_t, uint16_t> U;
  uint32_t bits = __builtin_bit_cast(U, x);
  asm volatile("" : "+v"(bits));
  x = __builtin_bit_cast(Some<E, V>, (U)bits);
}

// The channel of place `at` of a workgroup's 64 V.
template <int V>
__device__ __forceinline__ int channel_of(int column, int at, int D) { return Own<V>(column, at / V, D).d + at % V; }
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

// One grid axis counts tiles, samples and columns; a launch has fewer than 2^32 threads, 512 a tile.
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

// Two channels of 16 bits a lane, or one where there is only one.
template <typename E, typename F>
bppsa_status by_width(int D, F&& f) {
  if (sizeof(E) == 2 && D >= 2) return f(std::integral_constant<int, 4 / sizeof(E)>{});
  return f(std::integral_constant<int, 1>{});
}

// How the tiles of a sequence are joined in one launch.  A tile reads its inputs once, into registers; what it does to a state that
// comes in is the product of its decays and where it arrives from zero.  It leaves these two in a word and looks back over
// the words of the tiles before it to the nearest one that already knows the state behind it, then leaves its own:
// whichever that is, the state that comes in is the same chain of multiply-adds from the first tile on, so the bits do not
// depend on who was first.  Workgroups take tiles by a ticket, in the order in which they wait for each other: a tile that another
// waits for has been taken before and is running or done, so every wait ends.
// A word: the product's bits above, the end's below.  The sign of the product, which is never negative, says that the end
// is the state itself; all ones: nothing yet.  A word is one 64-bit access, so its halves belong together.
constexpr uint64_t kEmpty = ~(uint64_t)0;
constexpr uint32_t kSettled = 0x80000000u;
__device__ __forceinline__ uint64_t word_of(float product, float end) {
  uint32_t p = __float_as_uint(product) & 0x7FFFFFFFu;
  if (p > 0x7F800000u) p = 0x7FC00000u;
  return (uint64_t)p << 32 | __float_as_uint(end);
}
__device__ __forceinline__ uint64_t settled(float state) { return (uint64_t)kSettled << 32 | __float_as_uint(state); }
__device__ __forceinline__ bool is_settled(uint64_t w) { return (uint32_t)(w >> 32) == kSettled; }
__device__ __forceinline__ float through(uint64_t w, float h) {
  const float end = __uint_as_float((uint32_t)w);
  return is_settled(w) ? end : fmaf(__uint_as_float((uint32_t)(w >> 32)), h, end);
}
__device__ __forceinline__ uint64_t peek(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void leave(uint64_t* p, uint64_t w) { __hip_atomic_store(p, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The state that comes into a tile: `mine` is this tile's word of a channel, `step` the words to the next tile, `tiles` how many
// lie in front of it (the farthest one's word becomes settled without waiting for any other).
__device__ __forceinline__ float look_back(const uint64_t* mine, int64_t step, int tiles) {
  constexpr int WINDOW = 8;
  int far = 0;                                 // windows behind this one that hold no settled word
  uint64_t w[WINDOW];
  auto window = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < WINDOW; ++j) {
      const int back = k * WINDOW + j + 1;
      w[j] = peek(mine - step * (back <= tiles ? back : tiles));
    }
  };
  for (;;) {
    window(far);
    bool wait = false, found = false;
#pragma unroll
    for (int j = 0; j < WINDOW; ++j) {
      wait |= !found && w[j] == kEmpty;
      found |= is_settled(w[j]);
    }
    if (__any(wait)) {
      __builtin_amdgcn_s_sleep(1);
      continue;
    }
    if (__all(found)) break;
    ++far;
  }
  float h = 0.0f;
  for (;;) {
#pragma unroll
    for (int j = WINDOW - 1; j >= 0; --j) h = through(w[j], h);
    if (far == 0) return h;
    window(--far);
  }
}

// Empties the words of a call and its ticket, which lies in front of them.
constexpr int kTicketBytes = 256;
static __global__ void __launch_bounds__(256) empty_words_kernel(char* workspace, int64_t sixteens) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= sixteens) return;
  const uint32_t v = i < kTicketBytes / 16 ? 0u : ~0u;
  reinterpret_cast<uint4*>(workspace)[i] = make_uint4(v, v, v, v);
}
static inline size_t words_bytes(int tiles, int B, int columns, int V) {
  return tiles > 1 ? kTicketBytes + bppsa_align_up((size_t)tiles * B * columns * 64 * V * sizeof(uint64_t), 256) : 0;
}
static inline void empty_words(void* workspace, size_t bytes, hipStream_t s) {
  empty_words_kernel<<<(unsigned)((bytes / 16 + 255) / 256), 256, 0, s>>>(static_cast<char*>(workspace), (int64_t)(bytes / 16));
}

}  // namespace gated
