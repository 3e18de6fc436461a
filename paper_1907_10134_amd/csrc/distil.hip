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

// One workgroup a row, which is read for its largest value, for the sums and for the gradient.
constexpr int kThreads = 256;
template <typename F>
__device__ __forceinline__ float over_threads(float v, float (&share)[kThreads / 64], F&& f) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v = f(v, __shfl_xor(v, k));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) share[threadIdx.x >> 6] = v;
  __syncthreads();
  v = share[0];
  for (int k = 1; k < kThreads / 64; ++k) v = f(v, share[k]);
  return v;
}
__device__ __forceinline__ double sum_over_threads(double v, double (&share)[kThreads / 64]) {
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) share[threadIdx.x >> 6] = v;
  __syncthreads();
  v = share[0];
  for (int k = 1; k < kThreads / 64; ++k) v += share[k];
  return v;
}

template <typename E>
__global__ void __launch_bounds__(kThreads)
distil_kernel(const Loss<E> l) {
  __shared__ float fshare[kThreads / 64];
  __shared__ double dshare[kThreads / 64];
  __shared__ int place[kMost];
  __shared__ double p[kMost];
  const int64_t row = blockIdx.x;
  const int t = (int)(row / l.B), b = (int)(row % l.B), K = l.top.K;
  const float weight = l.weight ? l.weight[row] : 1.0f;
  E* const dx = l.dx.data ? l.dx.at(t, b) : nullptr;
  if (weight == 0.0f) {
    if (threadIdx.x == 0) l.loss[row] = 0.0f;
    if (dx)
      for (int v = threadIdx.x; v < l.V; v += kThreads) store(dx + v, 0.0f);
    return;
  }
  const E* const x = l.x.at(t, b);
  const auto plus = [](float a, float c) { return a + c; };
  const auto larger = [](float a, float c) { return fmaxf(a, c); };
  const float scale = 1.0f / l.tau;
  // the entries
  double top = -INFINITY, mine = 0.0;
  int c = -1;
  if (threadIdx.x < K) {
    c = l.top.index[row * K + threadIdx.x];
    const double logit = (double)entry_logit(l.top, row * K + threadIdx.x) / (double)l.tau;
    if (c < 0 || c >= l.V || logit == -INFINITY) c = -1;
    else top = logit;
    place[threadIdx.x] = c;
  }
  if (l.top_norm) {
    mine = c >= 0 ? exp(top - (double)l.top_norm[row]) : 0.0;
  } else {
    const double largest = (double)over_threads((float)top, fshare, larger);      // any value near it serves
    mine = c >= 0 ? exp(top - largest) : 0.0;
    const double all = sum_over_threads(mine, dshare);
    mine = all > 0.0 ? mine / all : mine;
  }
  const double total = sum_over_threads(mine, dshare);
  if (threadIdx.x < K) p[threadIdx.x] = mine;
  const float at_c = c >= 0 ? (float)x[c] : 0.0f;
  const int target = l.targets && l.hard != 0.0f ? l.targets[row] : -1;
  const bool known = target >= 0 && target < l.V;
  const float at_target = known ? (float)x[target] : 0.0f;
  __syncthreads();

  float m = -INFINITY, s = 0.0f, s1 = 0.0f, rest = 0.0f;
  for (int v = threadIdx.x; v < l.V; v += kThreads) m = fmaxf(m, (float)x[v]);
  m = over_threads(m, fshare, larger);
  for (int v = threadIdx.x; v < l.V; v += kThreads) {
    const float d = (float)x[v] - m, e = exp_of<kExact<E>>(d * scale);
    s += e;
    if (known) s1 += exp_of<kExact<E>>(d);
    if (l.top_norm) {
      bool in = false;
      for (int k = 0; k < K; ++k) in |= place[k] == v;
      rest += in ? 0.0f : e;
    }
  }
  s = over_threads(s, fshare, plus);
  if (known) s1 = over_threads(s1, fshare, plus);
  if (l.top_norm) rest = over_threads(rest, fshare, plus);
  const double log_s = log((double)s);
  const double p0 = l.top_norm && rest > 0.0f ? fmax(0.0, 1.0 - total) : 0.0;
  double soft = mine > 0.0 ? mine * (log(mine) - ((double)at_c - (double)m) * (double)scale + log_s) : 0.0;
  soft = sum_over_threads(soft, dshare);
  if (p0 > 0.0) soft += p0 * (log(p0) - log((double)rest) + log_s);
  if (threadIdx.x == 0) {
    const double ce = known ? (double)m - (double)at_target + log((double)s1) : 0.0;
    l.loss[row] = (float)((double)weight * ((1.0 - (double)l.hard) * (double)l.tau * (double)l.tau * soft + (double)l.hard * ce));
  }
  if (!dx) return;
  const float of_soft = weight * (1.0f - l.hard) * l.tau, of_hard = known ? weight * l.hard / s1 : 0.0f;
  const float M = (float)(total + p0), ratio = p0 > 0.0 ? (float)(p0 * (double)s / (double)rest) : 0.0f;
  const float elsewhere = of_soft * (M - ratio) / s, inside = of_soft * M / s;
  for (int v = threadIdx.x; v < l.V; v += kThreads) {
    const float d = (float)x[v] - m;
    float g = elsewhere * exp_of<kExact<E>>(d * scale);
    if (known) g = fmaf(of_hard, exp_of<kExact<E>>(d), g) - (v == target ? weight * l.hard : 0.0f);
    store(dx + v, g);
  }
  __syncthreads();                 // the entries' places are written again
  if (c >= 0) {
    double all = 0.0;
    for (int k = 0; k < K; ++k) all += place[k] == c ? p[k] : 0.0;
    const float d = at_c - m;
    float g = inside * exp_of<kExact<E>>(d * scale) - of_soft * (float)all;
    if (known) g = fmaf(of_hard, exp_of<kExact<E>>(d), g) - (c == target ? weight * l.hard : 0.0f);
    store(dx + c, g);
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
    distil_kernel<E><<<(unsigned)(r->T * r->B), kThreads, 0, (hipStream_t)stream>>>(l);
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
