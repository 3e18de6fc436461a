// The loss of a student against a teacher's top logits, and its gradient for the student's logits.
//
// With q = softmax(x / tau) over the vocabulary, shares p of the teacher's entries (c_k, t_k) and, where the teacher's normaliser
// is given, the share p0 = 1 - sum p of all other tokens, which the student gives q0 = sum of q over them,
//     soft = sum_k p_k log(p_k / q[c_k]) + p0 log(p0 / q0),      tau dsoft/dx = q M - p on the entries,  q (M - p0 / q0) elsewhere,
// M = sum p + p0, p0 / q0 = 0 without the normaliser.  The other part, -log softmax(x)[target], has the gradient
// softmax(x) - 1[target].  What is made of the K entries alone is made in 64 bits: there are few of them, and the parts of a
// divergence cancel.
#include "ssm_common.h"

namespace {

using namespace ssm;

struct Entries {                   // of the teacher, [T,B,K]
  const void* logits;
  const int32_t* index;
  int K, type;
};
__device__ __forceinline__ float entry_logit(const Entries& e, int64_t at) {
  if (e.type == BPPSA_F32) return static_cast<const float*>(e.logits)[at];
  if (e.type == BPPSA_BF16) return static_cast<float>(static_cast<const bf16_t*>(e.logits)[at]);
  return static_cast<float>(static_cast<const f16_t*>(e.logits)[at]);
}

template <typename E>
struct Loss {
  Rows<const E> x;
  Rows<E> dx;
  Entries top;
  const float *top_norm, *weight;
  const int32_t* targets;
  float* loss;
  int B, V;
  float tau, hard;
};

constexpr int kMost = BPPSA_DISTIL_MAX_K;

// exp(d scale), to_log2 = scale log2(e).  The difference to the largest is exact or nearly so; float32 logits take the corrected exponential.
template <typename E>
__device__ __forceinline__ float exponential(float d, float scale, float to_log2) {
  if constexpr (kExact<E>) return exp_of<true>(d * scale);
  else return exp2_fast(d * to_log2);
}

// Eight 16-bit or four 32-bit logits as they were loaded, and the value of one.
template <typename E>
struct Chunk {
  static constexpr int N = 16 / sizeof(E);
  uint32_t w[4];
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[k]);
    else if constexpr (std::is_same_v<E, bf16_t>) return __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
    else return static_cast<float>(__builtin_bit_cast(E, (uint16_t)(k & 1 ? w[k / 2] >> 16 : w[k / 2])));
  }
};
// What lies behind the row's end counts as minus infinity, which has no share.
template <typename E>
__device__ __forceinline__ Chunk<E> load_chunk(const E* x, int at, int V) {
  constexpr int N = Chunk<E>::N;
  if (at + N <= V) return __builtin_bit_cast(Chunk<E>, load_some<E, N>(x + at));
  Some<E, N> s;
#pragma unroll
  for (int k = 0; k < N; ++k) s.v[k] = at + k < V ? x[at + k] : static_cast<E>(-INFINITY);
  return __builtin_bit_cast(Chunk<E>, s);
}
template <typename E>
__device__ __forceinline__ void store_chunk(E* x, int at, int V, const float (&v)[Chunk<E>::N]) {
  constexpr int N = Chunk<E>::N;
  if (at + N <= V) return store_some<E, N>(x + at, v);
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (at + k < V) store(x + at + k, v[k]);
}

template <int WAVES, int N>
struct Share {                     // of the waves, N values each
  double v[N][WAVES];
};
// Sums of N values over the workgroup, in the same order for all of its threads.
template <int WAVES, int N>
__device__ __forceinline__ void sum_over_threads(double (&v)[N], Share<WAVES, N>& share) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) v[i] += __shfl_xor(v[i], k);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) < N) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if ((threadIdx.x & 63) == i) share.v[i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = share.v[i][0];
#pragma unroll
      for (int k = 1; k < WAVES; ++k) v[i] += share.v[i][k];
    }
  }
}

// One workgroup a row.  CHUNKS > 0: the row is read once, into registers (16 bytes a lane and chunk), and its largest value, its sums
// and its gradient are made of those; 0: a row too long for that is read three times.  SECOND: the data's own token has a
// softmax of its own, at another temperature.
template <typename E, int WAVES, int CHUNKS, bool SECOND>
__global__ void __launch_bounds__(WAVES * 64)
distil_kernel(const Loss<E> l) {
  constexpr int N = Chunk<E>::N, THREADS = WAVES * 64, STEP = THREADS * N, HELD = CHUNKS ? CHUNKS : 1;
  extern __shared__ uint32_t is_entry[];       // a bit a token, where the other tokens are a class
  __shared__ Share<WAVES, 2> of_max;
  __shared__ Share<WAVES, 5> of_sum;
  __shared__ int place[kMost];
  __shared__ float p[kMost], at_place[kMost];
  const int64_t row = blockIdx.x;
  const int t = (int)(row / l.B), b = (int)(row % l.B), K = l.top.K, first = threadIdx.x * N;
  const float weight = l.weight ? l.weight[row] : 1.0f;
  E* const dx = l.dx.data ? l.dx.at(t, b) : nullptr;
  if (weight == 0.0f) {
    if (threadIdx.x == 0) l.loss[row] = 0.0f;
    const float zero[N] = {};
    if (dx)
      for (int v = first; v < l.V; v += STEP) store_chunk<E>(dx, v, l.V, zero);
    return;
  }
  const E* const x = l.x.at(t, b);
  const bool tail = l.top_norm != nullptr;
  const float scale = 1.0f / l.tau, to_log2 = scale * kLog2e;
  // the entries' indices and logits are asked for first, then the row, then the row's logits of the entries
  constexpr int ENTRIES = (kMost + THREADS - 1) / THREADS;
  int c[ENTRIES];
  double logit[ENTRIES];
#pragma unroll
  for (int i = 0; i < ENTRIES; ++i) {
    const int k = threadIdx.x + i * THREADS;
    c[i] = -1, logit[i] = -INFINITY;
    if (k < K) c[i] = l.top.index[row * K + k], logit[i] = (double)entry_logit(l.top, row * K + k);
  }
  const int target = l.targets && l.hard != 0.0f ? l.targets[row] : -1;
  const bool known = target >= 0 && target < l.V;
  Chunk<E> held[HELD];
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k)
        if (k * STEP < l.V) f(held[k], first + k * STEP);
    } else {
      for (int v = first; v < l.V; v += STEP) f(load_chunk(x, v, l.V), v);
    }
  };
  if constexpr (CHUNKS > 0)
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k)
      if (k * STEP < l.V) held[k] = load_chunk(x, first + k * STEP, l.V);
  float at_c[ENTRIES];
  const float at_target = known ? (float)x[target] : 0.0f;
  double top = -INFINITY;
#pragma unroll
  for (int i = 0; i < ENTRIES; ++i) {
    const int k = threadIdx.x + i * THREADS;
    if (c[i] >= l.V || logit[i] == -INFINITY) c[i] = -1;
    at_c[i] = c[i] >= 0 ? (float)x[c[i]] : 0.0f;
    logit[i] = c[i] >= 0 ? logit[i] / (double)l.tau : -INFINITY;
    top = fmax(top, logit[i]);
    if (k < K) place[k] = c[i], at_place[k] = at_c[i];
  }
  if (tail) {
    for (int v = threadIdx.x; v < (l.V + 31) / 32; v += THREADS) is_entry[v] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i)
      if (c[i] >= 0) atomicOr(&is_entry[c[i] / 32], 1u << c[i] % 32);
  }
  float m = -INFINITY;
  each([&](const Chunk<E>& x, int) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < N; ++k) m = fmaxf(m, x[k]);
  });
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) m = fmaxf(m, __shfl_xor(m, k)), top = fmax(top, __shfl_xor(top, k));
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) of_max.v[0][threadIdx.x >> 6] = (double)m, of_max.v[1][threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WAVES; ++k) m = fmaxf(m, (float)of_max.v[0][k]), top = fmax(top, of_max.v[1][k]);
  } else {
    __syncthreads();
  }
  const double norm = tail ? (double)l.top_norm[row] : top;

  float s = 0.0f, s1 = 0.0f, rest = 0.0f;
  each([&](const Chunk<E>& x, int at) __attribute__((always_inline)) {
    float e[N], sum = 0.0f, sum1 = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      e[k] = exponential<E>(x[k] - m, scale, to_log2), sum += e[k];
      if (SECOND) sum1 += exponential<E>(x[k] - m, 1.0f, kLog2e);
    }
    s += sum, s1 += sum1;
    if (tail) {
      const uint32_t bits = at < l.V ? is_entry[at / 32] >> at % 32 : 0;
      float others = 0.0f;
#pragma unroll
      for (int k = 0; k < N; ++k) others += bits >> k & 1 ? 0.0f : e[k];
      rest += others;
    }
  });
  // the entries' shares, before they are divided by their sum where they are all there is, and what they leave of the divergence
  double share[ENTRIES], sums[5] = {(double)s, (double)s1, (double)rest, 0.0, 0.0};
#pragma unroll
  for (int i = 0; i < ENTRIES; ++i) {
    share[i] = c[i] >= 0 ? exp(logit[i] - norm) : 0.0;
    sums[3] += share[i];
    if (share[i] > 0.0) sums[4] += share[i] * ((logit[i] - norm) - ((double)at_c[i] - (double)m) * (double)scale);
  }
  sum_over_threads<WAVES, 5>(sums, of_sum);
  const double all = sums[3], over = tail || !(all > 0.0) ? 1.0 : 1.0 / all, total = all * over;
  const double p0 = tail && sums[2] > 0.0 ? fmax(0.0, 1.0 - all) : 0.0;
  if (threadIdx.x < 64) {
    const double log_s = log(sums[0]);
    double soft = sums[4] * over + total * log_s;
    if (!tail && all > 0.0) soft -= log(all);
    if (p0 > 0.0) soft += p0 * (log(p0) - log(sums[2]) + log_s);
    const double ce = known ? (double)m - (double)at_target + (SECOND ? log(sums[1]) : log_s) : 0.0;
    if (threadIdx.x == 0)
      l.loss[row] = (float)((double)weight * ((1.0 - (double)l.hard) * (double)l.tau * (double)l.tau * soft + (double)l.hard * ce));
  }
  if (!dx) return;
  const float of_soft = weight * (1.0f - l.hard) * l.tau, hard = known ? weight * l.hard : 0.0f;
  const float one = (float)(1.0 / sums[0]), of_e1 = SECOND ? (float)((double)hard / sums[1]) : 0.0f, of_e = SECOND ? 0.0f : hard * one;
  const float M = (float)(total + p0), ratio = p0 > 0.0 ? (float)(p0 * sums[0] / sums[2]) : 0.0f;
  const float elsewhere = fmaf(of_soft * (M - ratio), one, of_e), inside = fmaf(of_soft * M, one, of_e);
  each([&](const Chunk<E>& x, int at) __attribute__((always_inline)) {
    float g[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      g[k] = elsewhere * exponential<E>(x[k] - m, scale, to_log2);
      if (SECOND) g[k] = fmaf(of_e1, exponential<E>(x[k] - m, 1.0f, kLog2e), g[k]);
    }
    if (at < l.V) store_chunk<E>(dx, at, l.V, g);
  });
#pragma unroll
  for (int i = 0; i < ENTRIES; ++i)
    if (threadIdx.x + i * THREADS < K) p[threadIdx.x + i * THREADS] = (float)(share[i] * over);
  __syncthreads();                 // behind it the places of the entries and of the target are written again
  auto again = [&](int at, float value, float coefficient, float own) __attribute__((always_inline)) {
    float g = coefficient * exponential<E>(value - m, scale, to_log2) - own;
    if (SECOND) g = fmaf(of_e1, exponential<E>(value - m, 1.0f, kLog2e), g);
    store(dx + at, g);
  };
#pragma unroll
  for (int i = 0; i < ENTRIES; ++i)
    if (c[i] >= 0) {
      float own = c[i] == target ? hard : 0.0f;
      for (int k = 0; k < K; ++k) own += place[k] == c[i] ? of_soft * p[k] : 0.0f;
      again(c[i], at_c[i], inside, own);
    }
  if (threadIdx.x == THREADS - 1 && known) {
    bool entry = false;
    for (int k = 0; k < K; ++k) entry |= place[k] == target;
    if (!entry) again(target, at_target, elsewhere, hard);
  }
}

}  // namespace

extern "C" bppsa_status bppsa_distil(const bppsa_distil_rows* r, float* loss, const bppsa_rows* dlogits, void* stream) {
  if (!r || r->T < 1 || r->B < 1 || r->V < 1 || r->K < 1) return BPPSA_EINVAL;
  if (!r->logits.data || !r->top_logits || !r->top_index || !loss) return BPPSA_EINVAL;
  if (!(r->temperature > 0x1p-20f && r->temperature < 0x1p20f) || !(r->hard >= 0.0f && r->hard <= 1.0f)) return BPPSA_EINVAL;
  if (r->hard != 0.0f && !r->targets) return BPPSA_EINVAL;
  if (dlogits && !writable(*dlogits, r->T, r->B)) return BPPSA_EINVAL;
  if (dlogits && dlogits->data == r->logits.data &&
      ((r->T > 1 && dlogits->stride_t != r->logits.stride_t) || (r->B > 1 && dlogits->stride_b != r->logits.stride_b))) return BPPSA_EINVAL;
  if (r->K > kMost || r->type < BPPSA_F32 || r->type > BPPSA_F16 || r->top_type < BPPSA_F32 || r->top_type > BPPSA_F16)
    return BPPSA_EUNSUPPORTED;
  if (bppsa_mul_overflows(r->T, r->B, r->V, 1) || r->V > BPPSA_DISTIL_MAX_V || (int64_t)r->T * r->B >= 1 << 22) return BPPSA_EOVERFLOW;
  return by_type(r->type, [&](auto e) {
    using E = decltype(e);
    const Loss<E> l{rows_of<const E>(r->logits), dlogits ? rows_of<E>(*dlogits) : Rows<E>{}, Entries{r->top_logits, r->top_index, r->K, r->top_type},
                    r->top_norm, r->weight, r->targets, loss, r->B, r->V, r->temperature, r->hard};
    const auto run = [&](auto waves, auto chunks) {
      const size_t bits = l.top_norm ? (size_t)bppsa_ceil_div(l.V, 32) * sizeof(uint32_t) : 0;
      const auto kernel = l.hard != 0.0f && l.tau != 1.0f ? distil_kernel<E, waves.value, chunks.value, true>
                                                          : distil_kernel<E, waves.value, chunks.value, false>;
      kernel<<<(unsigned)(r->T * r->B), waves.value * 64, bits, (hipStream_t)stream>>>(l);
    };
    constexpr int N = Chunk<E>::N;
    const auto fits = [&](int waves, int chunks) { return l.V <= waves * 64 * N * chunks; };
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    typedef std::integral_constant<int, 4> Four;
    typedef std::integral_constant<int, 8> Eight;
    typedef std::integral_constant<int, 16> Sixteen;
    if (fits(1, 1)) run(One{}, One{});
    else if (fits(4, 2)) run(Four{}, Two{});
    else if (fits(4, 8)) run(Four{}, Eight{});
    else if (fits(8, 8)) run(Eight{}, Eight{});
    else if (fits(16, 8)) run(Sixteen{}, Eight{});
    else if (fits(16, 16)) run(Sixteen{}, Sixteen{});
    else run(Sixteen{}, None{});
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
