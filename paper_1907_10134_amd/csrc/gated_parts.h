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
  const float *decay, *r_bias, *i_bias, *h0;   // a bias that there is not: the decays, with a mask that leaves nothing of them
  const int32_t* lengths;
  int T, B, D, columns;
  uint32_t r_mask, i_mask;
};
template <typename E>
Layer<E> layer_of(const bppsa_gated& l, int wide) {
  return Layer<E>{rows_of<const E>(l.x), rows_of<const E>(l.r), rows_of<const E>(l.i), rows_of<const E>(l.z), l.decay,
                  l.r_bias ? l.r_bias : l.decay, l.i_bias ? l.i_bias : l.decay, l.h0, l.lengths, l.T, l.B, l.D,
                  bppsa_ceil_div(l.D, wide), l.r_bias ? ~0u : 0u, l.i_bias ? ~0u : 0u};
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
// A lane's V channels of a row as they were loaded, in one register, and the value of one of them.  (As an array of V the compiler
// takes them apart where they are loaded, for twice the registers.)
template <typename E>
__device__ __forceinline__ float part(uint32_t bits, int c) {
  if constexpr (sizeof(E) == 4) return __uint_as_float(bits);
  else if constexpr (std::is_same_v<E, bf16_t>) return __uint_as_float(c ? bits & 0xFFFF0000u : bits << 16);
  else return static_cast<float>(__builtin_bit_cast(E, (uint16_t)(c ? bits >> 16 : bits)));
}
// Such values stay as they are up to here: widened as soon as they can be they would take twice the registers again.
__device__ __forceinline__ void as_loaded(uint32_t& bits) { asm volatile("" : "+v"(bits)); }

// The rows of a wave's run in an array: the first one's address and the bytes to the next, both the same for the whole wave, so that
// an access is a scalar address and a lane's offset of 32 bits, and a row costs one scalar addition.
template <typename E>
struct Run {
  typedef std::remove_const_t<E> T;
  uint64_t at;
  int64_t step;
  __device__ __forceinline__ Run(const Rows<E>& r, int t, int b) : at((uint64_t)r.at(t, b)), step(r.st * (int64_t)sizeof(E)) {}
  template <int V>
  using Bits = std::conditional_t<sizeof(Some<T, V>) == 4, uint32_t, uint16_t>;      // of any alignment, as Some is
  template <int V>
  using Loose = Bits<V> __attribute__((aligned(sizeof(T))));
  template <int V>
  __device__ __forceinline__ uint32_t load(uint32_t byte) const { return *(const __attribute__((address_space(1))) Loose<V>*)(at + byte); }
  template <int V>
  __device__ __forceinline__ void store(uint32_t byte, const float (&x)[V]) const {
    Some<T, V> s;
#pragma unroll
    for (int i = 0; i < V; ++i) s.v[i] = static_cast<T>(x[i]);
    *(__attribute__((address_space(1))) Loose<V>*)(at + byte) = __builtin_bit_cast(Bits<V>, s);
  }
  // (opaque, or the lane's offset is added first and every row's address is one of vector registers)
  __device__ __forceinline__ void move_by(int64_t bytes) {
    at += bytes;
    asm("" : "+s"(at));
  }
  __device__ __forceinline__ void move() { move_by(step); }
};
// R rows of it; of fewer (not WHOLE) the last one again: what is made of those is left out.
template <bool WHOLE, int R, int V, typename E>
__device__ __forceinline__ void load_rows(const Rows<E>& from, int first, int b, int rows, uint32_t byte, uint32_t (&x)[R]) {
  Run<E> run(from, first, b);
  asm("" : "+s"(run.at));
#pragma unroll
  for (int j = 0; j < R; ++j) {
    x[j] = run.template load<V>(byte);
    if (j + 1 < R) run.move_by(WHOLE || j + 1 < rows ? run.step : 0);
  }
}

// The instructions of two rows stay together: the compiler starts all rows of a run at once, which takes more registers than there are.
__device__ __forceinline__ void apart(int row) {
  if (row % 2 == 0) __builtin_amdgcn_sched_barrier(0);
}

// The channel of place `at` of a workgroup's 64 V, D where it has none.
template <int V>
__device__ __forceinline__ int channel_of(int column, int at, int D) {
  const Own<V> own(column, at / V, D);
  return own.on ? own.d + at % V : D;
}
// 1 - exp(-x) for x >= 0, given e2 = exp(-x / 2): below 1/4, where the difference would lose bits, x times (1 - exp(-x)) / x
// interpolated at the five Chebyshev nodes of [0, 1/4]: the polynomial is within 2^-27.6 of it, what fp32 makes of it within 2^-23.3.
__device__ __forceinline__ float one_minus(float e2, float x) {
  const float p = fmaf(fmaf(fmaf(fmaf(7.51360599e-3f, x, -4.14906554e-2f), x, 0.166651085f), x, -0.499999523f), x, 1.0f);
  return x < 0.25f ? x * p : fmaf(-e2, e2, 1.0f);
}

// A channel's parameters as a step's gates take them.  Activations of 16 bits have their biases and log2(e) in one multiply-add
// in front of the exponential; float32 ones are added up and go through the corrected functions.
template <typename E>
struct Channel {
  float r_bias, i_bias, decay, of_exp;
  __device__ __forceinline__ static float gate(float x, float bias) {
    if constexpr (kExact<E>) return sigmoid<E>(x + bias);
    else return __builtin_amdgcn_rcpf(1.0f + exp2_fast(fmaf(x, -kLog2e, bias)));
  }
  __device__ __forceinline__ float rho(float r) const { return gate(r, r_bias); }
  __device__ __forceinline__ float iota(float i) const { return gate(i, i_bias); }
  __device__ __forceinline__ float a(float rho) const {
    if constexpr (kExact<E>) return exp_of<true>(-decay * rho);
    else return exp2_fast(of_exp * rho);
  }
  // 1 - a^2
  __device__ __forceinline__ float m2(float a, float rho) const { return one_minus(a, (decay + decay) * rho); }
};

// A lane's channels.  All of it is asked for together: a branch around a bias that may not be there would wait for it (T = 30000,
// B = 1, D = 2048: 150 us instead of 134).
template <typename E, int V>
__device__ __forceinline__ void channels_of(const Layer<E>& l, int d, Channel<E> (&channel)[V]) {
  const Some<float, V> decay = load_some<float, V>(l.decay + d), r = load_some<float, V>(l.r_bias + d), i = load_some<float, V>(l.i_bias + d);
  const float scale = kExact<E> ? 1.0f : -kLog2e;
#pragma unroll
  for (int c = 0; c < V; ++c)
    channel[c] = Channel<E>{__uint_as_float(__float_as_uint(r.v[c]) & l.r_mask) * scale,
                            __uint_as_float(__float_as_uint(i.v[c]) & l.i_mask) * scale, decay.v[c], decay.v[c] * -kLog2e};
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

// The state that comes into a tile: `mine` are this tile's words, the same for a wave, `at` a lane's place in them, `step` the words to
// the next tile, `tiles` how many lie in front of it (the farthest one's words become settled without waiting for any other).  Every
// word that is waited for comes, unless another call at the same time works in the same workspace: then the wait ends after
// kLooks looks, of a microsecond and more each, and channels whose state was not found get NaN.
constexpr int kLooks = 1 << 24;
__device__ __forceinline__ float look_back(const uint64_t* mine, uint32_t at, int64_t step, int tiles, int most = kLooks) {
  constexpr int WINDOW = 4;
  int far = 0;                                 // windows behind this one that hold no settled word
  uint64_t w[WINDOW];
  auto window = [&](int k) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < WINDOW; ++j) {
      const int back = k * WINDOW + j + 1;
      w[j] = peek(mine - step * (back <= tiles ? back : tiles) + at);
    }
  };
  bool again = true;
  for (int looks = 0; again && looks < most; ++looks) {
    window(far);
    bool wait = false, found = false;
#pragma unroll
    for (int j = 0; j < WINDOW; ++j) {
      wait |= !found && w[j] == kEmpty;
      found |= is_settled(w[j]);
    }
    const bool stay = __any(wait), on = !__all(found);
    if (stay) __builtin_amdgcn_s_sleep(1);
    else far += on;
    again = stay || on;
  }
  float h = NAN;                               // of a wait that was given up; every other has found a state
  for (;; --far) {
#pragma unroll
    for (int j = WINDOW - 1; j >= 0; --j) h = through(w[j], h);
    if (far == 0) return h;
    window(far - 1);
  }
}

// The tiles of a column of a sample, which wait for each other, are one chain; the chains are dealt out to eight queues, one a compute
// die, and a workgroup takes the next tile of its own die's queue (hardware register XCC_ID, id 20), or of another's when
// that is done: words that were left on this die are found in its L2.  Where a workgroup runs is no more than a preference: each takes
// exactly one of as many tiles as there are workgroups, and a queue hands its tiles out in the order of its chains' waits.
constexpr int kQueues = 8, kTicketStride = 32, kTicketBytes = kQueues * kTicketStride * 4;
__device__ __forceinline__ int2 take(int* tickets, int chains, int each, int tiles) {        // (chain, number of its tile)
  const int own = __builtin_amdgcn_s_getreg(20 | 3 << 11) & (kQueues - 1);
  for (int k = 0; k < kQueues; ++k) {
    const int q = (own + k) & (kQueues - 1), first = q * each, n = chains - first < each ? chains - first : each;
    if (n < 1) continue;
    const int t = __hip_atomic_fetch_add(tickets + q * kTicketStride, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t < n * tiles) return make_int2(first + t % n, t / n);
  }
  return make_int2(-1, 0);                     // not reached
}

// Chains of a queue.  Columns of one die alone fall into few of its L2's channels where rows lie a power of two apart, so few chains
// are one queue, whose tiles are neighbours in memory: T = 30000, B = 1 bf16, D = 2048 and 4096 (16 and 32 chains): 131 and 235 us,
// 141 and 249 in eight queues; T = 512, D = 4096, 64 chains: 18 and 17; T = 1000, B = 16, D = 330 fp32, 96 chains: 30 and 23.
static inline int chains_of_queue(int chains) { return chains >= 64 ? bppsa_ceil_div(chains, kQueues) : chains; }

// Empties the words of a call and its tickets, which lie in front of them.
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
