// The short causal convolution in front of the selective scan.
#include "ssm_common.h"

namespace {

using namespace ssm;

constexpr int kSpan = 64;        // steps of a workgroup

template <typename E>
struct Conv {
  Rows<const E> x;
  const float *weight, *bias;
  const E* state0;
  const int32_t* lengths;
  int T, B, D, silu;
};

template <typename E>
Conv<E> conv_of(const bppsa_conv& c) {
  return Conv<E>{rows_of<const E>(c.x), c.weight, c.bias, static_cast<const E*>(c.state0), c.lengths, c.T, c.B, c.D, c.silu};
}

// Input t of a sample, t from -(W-1): the carried state in front of the first, nothing behind its end.
template <typename E, int W>
__device__ __forceinline__ float input(const Conv<E>& c, int t, int b, int d, int len) {
  if (t >= len) return 0.0f;
  if (t >= 0) return load(c.x.at(t, b) + d);
  return c.state0 ? load(c.state0 + ((int64_t)b * (W - 1) + t + W - 1) * c.D + d) : 0.0f;
}

// One thread a channel and span of steps, the window in registers.
template <typename E, int W>
__global__ void __launch_bounds__(64)
conv_kernel(const Conv<E> c, Rows<E> y, E* __restrict__ state_last) {
  const int d = blockIdx.x * 64 + threadIdx.x, b = blockIdx.y, t0 = blockIdx.z * kSpan;
  if (d >= c.D) return;
  const int len = clamp_length(c.lengths, b, c.T), t1 = t0 + kSpan < c.T ? t0 + kSpan : c.T;
  float w[W], seen[W];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    w[k] = c.weight[(int64_t)d * W + k];
    seen[k] = k ? input<E, W>(c, t0 - W + k, b, d, len) : 0.0f;
  }
  const float bias = c.bias ? c.bias[d] : 0.0f;
  for (int t = t0; t < t1; ++t) {
#pragma unroll
    for (int k = 0; k + 1 < W; ++k) seen[k] = seen[k + 1];
    seen[W - 1] = input<E, W>(c, t, b, d, len);
    float p = bias;
#pragma unroll
    for (int k = 0; k < W; ++k) p = fmaf(w[k], seen[k], p);
    store(y.at(t, b) + d, t < len ? (c.silu ? p * sigmoid<E>(p) : p) : 0.0f);
  }
  if (state_last && blockIdx.z == 0)
#pragma unroll
    for (int k = 0; k + 1 < W; ++k)
      store(state_last + ((int64_t)b * (W - 1) + k) * c.D + d, input<E, W>(c, len - (W - 1) + k, b, d, len));
}

// dL/dp[t], p recomputed from its window.
template <typename E, int W>
__device__ __forceinline__ float outer(const Conv<E>& c, const Rows<const E>& dy, int t, int b, int d, int len, const float (&w)[W],
                                       float bias, float (&seen)[W]) {
#pragma unroll
  for (int k = 0; k + 1 < W; ++k) seen[k] = seen[k + 1];
  seen[W - 1] = input<E, W>(c, t, b, d, len);
  if (t >= len) return 0.0f;
  const float g = load(dy.at(t, b) + d);
  if (!c.silu) return g;
  float p = bias;
#pragma unroll
  for (int k = 0; k < W; ++k) p = fmaf(w[k], seen[k], p);
  const float sg = sigmoid<E>(p);
  return g * sg * fmaf(p, 1.0f - sg, 1.0f);
}

// dx[t] = sum_k w[k] dp[t + W-1 - k].  A span forms the dp of its steps, and of W-1 behind it for its last dx; its sums of
// dweight and dbias go to parts [span][b][W+1][D].  The first span also has the gradient of the carried state: dx at
// t = -(W-1)..-1.
template <typename E, int W>
__global__ void __launch_bounds__(64)
conv_backward_kernel(const Conv<E> c, Rows<const E> dy, Rows<E> dx, E* __restrict__ dstate0, float* __restrict__ parts) {
  const int d = blockIdx.x * 64 + threadIdx.x, b = blockIdx.y, t0 = blockIdx.z * kSpan;
  if (d >= c.D) return;
  const int len = clamp_length(c.lengths, b, c.T), t1 = t0 + kSpan < c.T ? t0 + kSpan : c.T;
  float w[W], seen[W], dp[W], dw[W], db = 0.0f;
#pragma unroll
  for (int k = 0; k < W; ++k) {
    w[k] = c.weight[(int64_t)d * W + k];
    seen[k] = k ? input<E, W>(c, t0 - W + k, b, d, len) : 0.0f;
    dp[k] = dw[k] = 0.0f;
  }
  const float bias = c.bias ? c.bias[d] : 0.0f;
  // at step t dp[j] holds dL/dp[t - (W-1) + j]; it completes dx[t - (W-1)]
  for (int t = t0; t < t1 + W - 1; ++t) {
#pragma unroll
    for (int k = 0; k + 1 < W; ++k) dp[k] = dp[k + 1];
    dp[W - 1] = outer<E, W>(c, dy, t, b, d, len, w, bias, seen);
    if (t < t1) {
      db += dp[W - 1];
#pragma unroll
      for (int k = 0; k < W; ++k) dw[k] = fmaf(dp[W - 1], seen[k], dw[k]);
    }
    const int at = t - (W - 1);
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < W; ++k) sum = fmaf(w[k], dp[W - 1 - k], sum);
    if (at >= t0) {
      store(dx.at(at, b) + d, at < len ? sum : 0.0f);
    } else if (t0 == 0 && dstate0) {
      store(dstate0 + ((int64_t)b * (W - 1) + t) * c.D + d, sum);
    }
  }
  float* out = parts + ((int64_t)blockIdx.z * c.B + b) * (W + 1) * c.D + d;
#pragma unroll
  for (int k = 0; k < W; ++k) out[(int64_t)k * c.D] = dw[k];
  out[(int64_t)W * c.D] = db;
}

template <int W>
__global__ void __launch_bounds__(256)
join_weights_kernel(const float* __restrict__ parts, int count, int D, float* __restrict__ dweight, float* __restrict__ dbias) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)(W + 1) * D;
  if (i >= all) return;
  float sum = 0.0f;
  for (int k = 0; k < count; ++k) sum += parts[k * all + i];
  const int tap = (int)(i / D), d = (int)(i - (int64_t)tap * D);
  if (tap < W) dweight[(int64_t)d * W + tap] = sum;
  else if (dbias) dbias[d] = sum;
}

template <typename E, int W>
__global__ void __launch_bounds__(64)
conv_step_kernel(const Conv<E> c, Rows<E> y, E* __restrict__ state, int slots_in_state, const int32_t* __restrict__ slots) {
  const int d = blockIdx.x * 64 + threadIdx.x, b = blockIdx.y;
  if (d >= c.D) return;
  const int slot = slots ? slots[b] : b;
  if (slot < 0 || slot >= slots_in_state) {
    store(y.at(0, b) + d, 0.0f);
    return;
  }
  E* s = state + (int64_t)slot * (W - 1) * c.D + d;
  const E* x = c.x.at(0, b) + d;
  float p = c.bias ? c.bias[d] : 0.0f;
  E seen[W];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    seen[k] = k < W - 1 ? s[(int64_t)k * c.D] : *x;
    p = fmaf(c.weight[(int64_t)d * W + k], load(&seen[k]), p);
  }
#pragma unroll
  for (int k = 0; k + 1 < W; ++k) s[(int64_t)k * c.D] = seen[k + 1];
  store(y.at(0, b) + d, c.silu ? p * sigmoid<E>(p) : p);
}

template <typename F>
bppsa_status by_width(int W, F&& f) {
  switch (W) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    default: return f(std::integral_constant<int, 4>{});
  }
}

bppsa_status check_conv(const bppsa_conv* c) {
  if (!c || c->T < 1 || c->B < 1 || c->D < 1 || c->W < 1 || !c->x.data || !c->weight) return BPPSA_EINVAL;
  if (c->W < 2 || c->W > BPPSA_SSM_MAX_W || c->type < BPPSA_F32 || c->type > BPPSA_F16) return BPPSA_EUNSUPPORTED;
  if (bppsa_mul_overflows(c->T, c->B, c->D, 2) || c->B > 65535 || c->T > 65535 * kSpan) return BPPSA_EOVERFLOW;
  return BPPSA_OK;
}

}  // namespace

extern "C" bppsa_status bppsa_ssm_conv(const bppsa_conv* conv, const bppsa_rows* y, void* state_last, void* stream) {
  BPPSA_TRY(check_conv(conv));
  if (!y || !writable(*y, conv->T, conv->B)) return BPPSA_EINVAL;
  return by_type(conv->type, [&](auto e) {
    using E = decltype(e);
    return by_width(conv->W, [&](auto w) {
      conv_kernel<E, w.value><<<dim3(bppsa_ceil_div(conv->D, 64), conv->B, bppsa_ceil_div(conv->T, kSpan)), 64, 0,
                                (hipStream_t)stream>>>(conv_of<E>(*conv), rows_of<E>(*y), static_cast<E*>(state_last));
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}

extern "C" size_t bppsa_ssm_conv_backward_workspace_bytes(int T, int B, int D, int W) {
  if (T < 1 || B < 1 || D < 1 || W < 2 || W > BPPSA_SSM_MAX_W) return 0;
  return (size_t)bppsa_ceil_div(T, kSpan) * B * (W + 1) * D * sizeof(float);
}

extern "C" bppsa_status bppsa_ssm_conv_backward(const bppsa_conv* conv, const bppsa_rows* dy, const bppsa_rows* dx,
                                                float* dweight, float* dbias, void* dstate0, void* workspace,
                                                size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_conv(conv));
  if (!dy || !dy->data || !dx || !writable(*dx, conv->T, conv->B) || !dweight) return BPPSA_EINVAL;
  if (!workspace || workspace_bytes < bppsa_ssm_conv_backward_workspace_bytes(conv->T, conv->B, conv->D, conv->W))
    return BPPSA_EWORKSPACE;
  if ((uintptr_t)workspace & 255) return BPPSA_EINVAL;
  const hipStream_t s = (hipStream_t)stream;
  float* parts = static_cast<float*>(workspace);
  return by_type(conv->type, [&](auto e) {
    using E = decltype(e);
    return by_width(conv->W, [&](auto w) {
      constexpr int W = w.value;
      const int spans = bppsa_ceil_div(conv->T, kSpan);
      conv_backward_kernel<E, W><<<dim3(bppsa_ceil_div(conv->D, 64), conv->B, spans), 64, 0, s>>>(
          conv_of<E>(*conv), rows_of<const E>(*dy), rows_of<E>(*dx), static_cast<E*>(dstate0), parts);
      join_weights_kernel<W><<<(unsigned)(((int64_t)(W + 1) * conv->D + 255) / 256), 256, 0, s>>>(
          parts, spans * conv->B, conv->D, dweight, dbias);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}

extern "C" bppsa_status bppsa_ssm_conv_step(const bppsa_conv* conv, const bppsa_rows* y, void* state, int slots_in_state,
                                            const int32_t* slots, void* stream) {
  BPPSA_TRY(check_conv(conv));
  if (!y || !writable(*y, 1, conv->B) || !state || slots_in_state < 1 || conv->state0 || conv->lengths) return BPPSA_EINVAL;
  if (conv->T != 1 || (!slots && conv->B > slots_in_state)) return BPPSA_ESHAPE;
  return by_type(conv->type, [&](auto e) {
    using E = decltype(e);
    return by_width(conv->W, [&](auto w) {
      conv_step_kernel<E, w.value><<<dim3(bppsa_ceil_div(conv->D, 64), conv->B), 64, 0, (hipStream_t)stream>>>(
          conv_of<E>(*conv), rows_of<E>(*y), static_cast<E*>(state), slots_in_state, slots);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}
