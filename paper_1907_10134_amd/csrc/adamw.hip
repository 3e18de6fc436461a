// One AdamW update of many tensors by one launch, moments in 32 or in 8 bits.
#include <cfloat>
#include <cmath>

#include "ssm_common.h"

namespace {

using ssm::bf16_t;

constexpr int kThreads = 256;
constexpr int kBlock = BPPSA_ADAMW_BLOCK;
constexpr int kPiece = BPPSA_ADAMW_PIECE;
static_assert(kBlock == BPPSA_WAVE * 4, "a wave holds a block, four values a lane");

struct Step {
  float beta1, one_minus_beta1, beta2, one_minus_beta2, per_correct1, per_root_correct2, eps, lr;
  double lr_exact;
  uint32_t seed;
};

// The number that decides which way a place of a tensor is rounded: two rounds of multiply and fold.
__device__ __forceinline__ uint32_t folded(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xBB67AE85u;
  x = (x ^ (x >> 16)) * 0x3C6EF373u;
  return x ^ (x >> 15);
}
__device__ __forceinline__ float chance(uint32_t x) { return (float)(x >> 8) * 0x1p-24f; }      // [0, 1)

// q >= 0 in units of its block's scale, on the grid of e4m3 below or above it by chance.
__device__ __forceinline__ float up_or_down(float q, float up) {
  // 2^(floor(log2 q) - 3), the spacing of e4m3 at q (2^-9 below 2^-6), from the exponent bits
  const uint32_t e = __float_as_uint(fmaxf(q, 0x1p-6f)) & 0x7F800000u;
  const float unit = __uint_as_float(e - (3u << 23)), per = __uint_as_float(0x7F000000u - (e - (3u << 23)));
  const float low = floorf(q * per) * unit;
  return (q - low) * per + up >= 1.0f ? low + unit : low;
}
// The root of v: above zero stays above zero.
__device__ __forceinline__ float held_root(float q, uint32_t x) {
  const float chosen = up_or_down(q, chance(x));
  return q > 0.0f ? fminf(fmaxf(chosen, 0x1p-9f), 448.0f) : q;
}

// m: to the nearest, which the conversion does, where that cannot stop it from decaying.  A value that nothing feeds loses
// 1 - beta1 of itself a step.  At beta1 <= 15/16 that is more than half the grid's spacing from 2^-6 on, where a value has 8 to 15
// spacings; below, where the spacing stays 2^-9, it is not: 4 spacings at 0.9 are 3.6, and 4 again, for ever, over a root
// that goes on falling, and so a weight without a gradient would move by up to a third of lr a step.  A magnitude that has
// become smaller there goes up or down by chance instead, and so reaches zero; at a larger beta1 (LONG) every value does.
__device__ __forceinline__ float chance_of_m(uint32_t x) { return chance(x * 0x9E3779B1u); }
__device__ __forceinline__ float held_m(float q, uint32_t x) { return copysignf(up_or_down(fabsf(q), chance_of_m(x)), q); }
__device__ __forceinline__ float held_small_m(float q, uint32_t x) {     // below 2^-6
  return copysignf(floorf(fmaf(fabsf(q), 0x1p9f, chance_of_m(x))) * 0x1p-9f, q);
}

template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

// Four values in a row; `full`: all four exist and the address is aligned for one access.
template <typename T>
__device__ __forceinline__ void get4(const T* p, int n, bool full, T (&v)[4]) {
  if (full) {
    const Pack<T, 4> x = *reinterpret_cast<const Pack<T, 4>*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : T(0);
  }
}
template <typename T>
__device__ __forceinline__ void put4(T* p, int n, bool full, const T (&v)[4]) {
  if (full) {
    Pack<T, 4> x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = v[i];
    *reinterpret_cast<Pack<T, 4>*>(p) = x;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}

// Largest magnitude of a wave's values by their bits, so that a NaN among them wins.
__device__ __forceinline__ float wave_largest(const float (&x)[4]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
  for (int k = 32; k; k >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, k));
  return __uint_as_float(m);
}

__device__ __forceinline__ float scale_of(float largest) {
  return (largest < 0x1p-100f ? 0x1p-100f : largest) * (1.0f / 448.0f);
}

__device__ __forceinline__ void unpack(uint32_t w, float (&x)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
}
__device__ __forceinline__ float within(float q) { return q > 448.0f ? 448.0f : (q < -448.0f ? -448.0f : q); }   // keeps NaN
__device__ __forceinline__ uint32_t pack(const float (&q)[4]) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(within(q[0]), within(q[1]), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(within(q[2]), within(q[3]), w, true);
}

// What a lane has of a block: four values of everything.
template <typename G, bool EIGHT>
struct Held {
  G g[4];
  float theta[4];
  std::conditional_t<EIGHT, uint8_t, float> m[4], v[4];
  float m_scale, v_scale;
  __device__ __forceinline__ void get(const bppsa_adamw_tensor& t, int64_t i, int n, bool full) {
    typedef std::conditional_t<EIGHT, uint8_t, float> M;
    get4(static_cast<const G*>(t.grad) + i, n, full, g);
    get4(t.theta + i, n, full, theta);
    get4(static_cast<const M*>(t.m) + i, n, full, m);
    get4(static_cast<const M*>(t.v) + i, n, full, v);
    if (EIGHT) m_scale = t.m_scale[i / kBlock], v_scale = t.v_scale[i / kBlock];
  }
};

// One block by one wave.
template <typename G, bool EIGHT, bool LONG>
__device__ __forceinline__ void update(const bppsa_adamw_tensor& t, const Held<G, EIGHT>& x, int64_t i, int n, bool full, int lane,
                                       float keep, uint32_t tensor, const Step& c) {
  float theta[4], m[4], v[4], root[4], was[4];
  if constexpr (EIGHT) {
    unpack(__builtin_bit_cast(uint32_t, x.m), m);
    unpack(__builtin_bit_cast(uint32_t, x.v), v);
#pragma unroll
    for (int k = 0; k < 4; ++k) was[k] = m[k] *= x.m_scale, v[k] *= x.v_scale, v[k] *= v[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = x.m[k], v[k] = x.v[k];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float g = static_cast<float>(x.g[k]);
    m[k] = fmaf(c.one_minus_beta1, g, c.beta1 * m[k]);
    v[k] = fmaf(c.one_minus_beta2, g * g, c.beta2 * v[k]);
    root[k] = sqrtf(v[k]);
    // v_rcp_f32 is good to one step: 2^-23 of an update that is itself added to theta
    const float update = (m[k] * c.per_correct1) * __builtin_amdgcn_rcpf(fmaf(root[k], c.per_root_correct2, c.eps));
    theta[k] = fmaf(x.theta[k], keep, -c.lr * update);
  }
  put4(t.theta + i, n, full, theta);
  if (t.copy) {
    bf16_t small[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) small[k] = static_cast<bf16_t>(theta[k]);
    put4(static_cast<bf16_t*>(t.copy) + i, n, full, small);
  }
  if constexpr (EIGHT) {
    const float sm = scale_of(wave_largest(m)), sv = scale_of(wave_largest(root));
    const float im = 1.0f / sm, iv = 1.0f / sv;
    const uint32_t place = c.seed * 0x9E3779B1u + tensor * 0x6A09E667u + (uint32_t)i;
    uint32_t number[4];
    bool any = false, by_chance[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      number[k] = folded(place + k);
      root[k] = held_root(root[k] * iv, number[k]);
      by_chance[k] = fabsf(m[k]) < fminf(fabsf(was[k]), 0x1p-6f * sm);
      m[k] *= im;
      any |= by_chance[k];
    }
    // hardly a value of a block is so small.  19 layers of width 76: 11.86 us, 11.65 without, 12.3 with held_m() here for both
    if (LONG || any)
#pragma unroll
      for (int k = 0; k < 4; ++k) m[k] = LONG ? held_m(m[k], number[k]) : by_chance[k] ? held_small_m(m[k], number[k]) : m[k];
    put4(static_cast<uint8_t*>(t.m) + i, n, full, __builtin_bit_cast(Pack<uint8_t, 4>, pack(m)).v);
    put4(static_cast<uint8_t*>(t.v) + i, n, full, __builtin_bit_cast(Pack<uint8_t, 4>, pack(root)).v);
    if (lane == 0) t.m_scale[i / kBlock] = sm, t.v_scale[i / kBlock] = sv;
  } else {
    put4(static_cast<float*>(t.m) + i, n, full, m);
    put4(static_cast<float*>(t.v) + i, n, full, v);
  }
}

// A workgroup takes a piece; a wave four blocks of it in a row, four values a lane, and asks for all of a full piece's
// before it works on the first (a block at a time: 1190 and 854 us instead of 1107 and 638 for 210 M parameters with bf16
// gradients and copies, moments in 32 and in 8 bits).  Bound by memory, 5.3 TB/s.
template <typename G, bool EIGHT, bool LONG>
__global__ void __launch_bounds__(kThreads)
adamw_kernel(const bppsa_adamw_tensor* __restrict__ tensors, const bppsa_adamw_piece* __restrict__ pieces, const Step c) {
  const bppsa_adamw_piece piece = pieces[blockIdx.x];
  const bppsa_adamw_tensor t = tensors[piece.tensor];
  const int64_t first = (int64_t)piece.piece * kPiece;
  const int count = (int)(t.n - first < kPiece ? t.n - first : kPiece);
  constexpr int BLOCKS = kPiece / kBlock / (kThreads / BPPSA_WAVE);
  const int lane = threadIdx.x & 63, start = (threadIdx.x >> 6) * BLOCKS * kBlock;
  const float keep = (float)(1.0 - c.lr_exact * t.decay);
  const bool aligned = (((uintptr_t)t.theta | ((uintptr_t)t.grad * (16 / (sizeof(G) * 4))) |
                         (EIGHT ? ((uintptr_t)t.m | (uintptr_t)t.v) * 4 : (uintptr_t)t.m | (uintptr_t)t.v) |
                         (uintptr_t)t.copy * 2) & 15) == 0;
  if (aligned && count == kPiece) {
    Held<G, EIGHT> x[BLOCKS];
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) x[j].get(t, first + start + j * kBlock + lane * 4, 4, true);
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j)
      update<G, EIGHT, LONG>(t, x[j], first + start + j * kBlock + lane * 4, 4, true, lane, keep, (uint32_t)piece.tensor, c);
    return;
  }
  for (int at = start; at < count && at < start + BLOCKS * kBlock; at += kBlock) {
    const int64_t i = first + at + lane * 4;
    const int n = count - at - lane * 4;       // values that are left for this lane
    Held<G, EIGHT> x;
    x.get(t, i, n, aligned && n >= 4);
    update<G, EIGHT, LONG>(t, x, i, n, aligned && n >= 4, lane, keep, (uint32_t)piece.tensor, c);
  }
}

}  // namespace

extern "C" int64_t bppsa_adamw_pieces(int n_tensors, const int64_t* n, bppsa_adamw_piece* pieces) {
  if (n_tensors < 1 || !n) return 0;
  int64_t count = 0;
  for (int k = 0; k < n_tensors; ++k) {
    if (n[k] < 0 || n[k] > (int64_t)1 << 40) return 0;
    for (int64_t p = 0; p * kPiece < n[k]; ++p, ++count)
      if (pieces) pieces[count] = bppsa_adamw_piece{k, (int32_t)p};
  }
  return count;
}

extern "C" bppsa_status bppsa_adamw_step(int n_tensors, const bppsa_adamw_tensor* tensors, int64_t n_pieces,
                                         const bppsa_adamw_piece* pieces, int grad_type, int state_bits, int step, double lr,
                                         double beta1, double beta2, double eps, uint32_t seed, void* stream) {
  if (n_tensors < 1 || !tensors || n_pieces < 1 || !pieces || step < 1) return BPPSA_EINVAL;
  if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !std::isfinite((float)lr)) return BPPSA_EINVAL;
  if (!((float)eps >= FLT_MIN) || !std::isfinite((float)eps)) return BPPSA_EINVAL;       // v_rcp_f32 takes no less
  if (state_bits != 32 && state_bits != 8) return BPPSA_EUNSUPPORTED;
  if (n_pieces >= 1 << 24) return BPPSA_EOVERFLOW;       // a launch has fewer than 2^32 threads
  const Step c{(float)beta1, (float)(1 - beta1), (float)beta2, (float)(1 - beta2), (float)(1 / (1 - std::pow(beta1, step))),
               (float)(1 / std::sqrt(1 - std::pow(beta2, step))), (float)eps, (float)lr, lr, seed};
  return ssm::by_type(grad_type, [&](auto g) -> bppsa_status {
    using G = decltype(g);
    const auto kernel = state_bits == 32 ? adamw_kernel<G, false, false> : beta1 > 0.9375 ? adamw_kernel<G, true, true> : adamw_kernel<G, true, false>;
    kernel<<<(unsigned)n_pieces, kThreads, 0, (hipStream_t)stream>>>(tensors, pieces, c);
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
