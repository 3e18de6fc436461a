// The short causal convolution in front of the selective scan.
#include <algorithm>

#include "ssm_common.h"

namespace {

using namespace ssm;

// The forward kernels are bound by memory; the backward one is not: 25 us at T = 1000, B = 16, D = 641, W = 4, f16, whose bytes
// would take 10, with 706 vector instructions for 16 values, of which 147 move the windows on and 61 make row addresses.
// A thread takes V neighbouring channels (16 bytes forward, 8 backward, where a window of inputs and one of gradients and the
// sums of the weights' gradients have to stay in registers too) and a span of steps, the window of the last W inputs in
// registers.  The last thread of a row starts early enough to have V channels too and repeats some of its neighbour's, with
// the same results; fewer than V channels go one to a thread.
// T = 4096, B = 4, D = 4096, W = 4, bf16: forward 49 us (5.4 TB/s) on the same buffers again, 57 on others each time; with 8
// bytes a lane 71, with 128 registers, which spills, 84.
constexpr int kAhead = 4;        // rows that are asked for together
constexpr int kTogether = 4;     // spans of a workgroup of the backward pass

template <typename E>
struct Conv {
  Rows<const E> x;
  const float *weight, *bias;
  const E* state0;
  const int32_t* lengths;
  int T, B, D, silu, span;
};

template <typename E>
Conv<E> conv_of(const bppsa_conv& c, int span) {
  return Conv<E>{rows_of<const E>(c.x), c.weight, c.bias, static_cast<const E*>(c.state0), c.lengths, c.T, c.B, c.D, c.silu, span};
}

template <int V, int W>
struct Taps {
  float w[V][W], bias[V];
  template <typename E>
  __device__ __forceinline__ Taps(const Conv<E>& c, int d) {
    const Some<float, V * W> all = load_some<float, V * W>(c.weight + (int64_t)d * W);
    Some<float, V> b = {};
    if (c.bias) b = load_some<float, V>(c.bias + d);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      bias[i] = b.v[i];
#pragma unroll
      for (int k = 0; k < W; ++k) w[i][k] = all.v[i * W + k];
    }
  }
  __device__ __forceinline__ float sum(const float (&seen)[W][V], int i) const {
    float p = bias[i];
#pragma unroll
    for (int k = 0; k < W; ++k) p = fmaf(w[i][k], seen[k][i], p);
    return p;
  }
};

// Input t of a sample, t from -(W-1): the carried state in front of the first, nothing behind its end.
template <typename E, int W, int V>
__device__ __forceinline__ void input(const Conv<E>& c, int t, int b, int d, int len, float (&x)[V]) {
  Some<E, V> s = {};
  if (t >= 0 && t < len) s = load_some<E, V>(c.x.at(t, b) + d);
  else if (t < 0 && c.state0) s = load_some<E, V>(c.state0 + ((int64_t)b * (W - 1) + t + W - 1) * c.D + d);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (float)s.v[i];
}

// Which channels and which span a thread has: threads are counted through the channels of a span and on to the next span, so
// that a row of few or odd channels leaves no lanes idle.
struct Place {
  int d, span;
  bool real;
};
__device__ __forceinline__ Place place_of(int64_t thread, int D, int V, int spans) {
  const int across = (D + V - 1) / V, first = (int)(thread % across) * V;
  const int64_t span = thread / across;
  return Place{first + V <= D ? first : D - V, (int)(span < spans ? span : 0), span < spans};
}

template <typename E, int W, int V>
__global__ void __launch_bounds__(64)
conv_kernel(const Conv<E> c, Rows<E> y, E* __restrict__ state_last) {
  const Place at = place_of((int64_t)blockIdx.x * 64 + threadIdx.x, c.D, V, (c.T + c.span - 1) / c.span);
  const int d = at.d, b = blockIdx.y, t0 = at.span * c.span;
  if (!at.real) return;
  const int len = clamp_length(c.lengths, b, c.T), t1 = t0 + c.span < c.T ? t0 + c.span : c.T, stop = t1 < len ? t1 : len;
  if (state_last && t0 == 0)
#pragma unroll
    for (int k = 0; k + 1 < W; ++k) {
      float x[V];
      input<E, W, V>(c, len - (W - 1) + k, b, d, len, x);
      store_some<E, V>(state_last + ((int64_t)b * (W - 1) + k) * c.D + d, x);
    }
  float seen[W][V];
  if (t0 < stop) {
    const Taps<V, W> taps(c, d);
#pragma unroll
    for (int k = 1; k < W; ++k) input<E, W, V>(c, t0 - W + k, b, d, len, seen[k]);
    const E* from = c.x.at(t0, b) + d;
    E* to = y.at(t0, b) + d;
    for (int t = t0; t < stop; t += kAhead) {
      Some<E, V> x[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) x[j] = load_some<E, V>(from + (t + j < stop ? j : stop - 1 - t) * c.x.st);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
          for (int k = 0; k + 1 < W; ++k) seen[k][i] = seen[k + 1][i];
          seen[W - 1][i] = (float)x[j].v[i];
          const float p = taps.sum(seen, i);
          out[i] = c.silu ? p * sigmoid<E>(p) : p;
        }
        if (t + j < stop) store_some<E, V>(to + j * y.st, out);
      }
      from += kAhead * c.x.st, to += kAhead * y.st;
    }
  }
  const float zero[V] = {};
  for (int t = t0 > len ? t0 : len; t < t1; ++t) store_some<E, V>(y.at(t, b) + d, zero);
}

// dx[t] = sum_k w[k] dp[t + W-1 - k], dp = dL/dp with p recomputed from its window.  A span forms the dp of its steps, and of
// W-1 behind it for its last dx.  The four waves of a workgroup take a span each and add their sums of dweight and dbias,
// which go to parts [four spans][b][W+1][D].  The first span also has the gradient of the carried state: dx at
// t = -(W-1)..-1.
template <typename E, int W, int V>
__global__ void __launch_bounds__(64 * kTogether)
conv_backward_kernel(const Conv<E> c, Rows<const E> dy, Rows<E> dx, E* __restrict__ dstate0, float* __restrict__ parts) {
  __shared__ float share[kTogether - 1][(W + 1) * V][64];
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6;
  // threads behind the last channel repeat the last ones', with the same results
  const int first = (blockIdx.x * 64 + lane) * V, d = first + V <= c.D ? first : c.D - V;
  const int b = blockIdx.y, t0 = (blockIdx.z * kTogether + q) * c.span;
  const int len = clamp_length(c.lengths, b, c.T), t1 = t0 + c.span < c.T ? t0 + c.span : c.T;
  float seen[W][V], dp[W][V] = {}, dw[W + 1][V] = {};
  const Taps<V, W> taps(c, d);
#pragma unroll
  for (int k = 1; k < W; ++k) input<E, W, V>(c, t0 - W + k, b, d, len, seen[k]);
  // at step t dp[j] holds dL/dp[t - (W-1) + j]; it completes dx[t - (W-1)]
  for (int t = t0; t0 < t1 && t < t1 + W - 1; t += kAhead) {
    Some<E, V> x[kAhead] = {}, go[kAhead] = {};
    if (len)
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int at = t + j < len ? t + j : len - 1;
        x[j] = load_some<E, V>(c.x.at(at, b) + d), go[j] = load_some<E, V>(dy.at(at, b) + d);
      }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int now = t + j, done = now - (W - 1);
      if (now >= t1 + W - 1) break;
      float out[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int k = 0; k + 1 < W; ++k) seen[k][i] = seen[k + 1][i], dp[k][i] = dp[k + 1][i];
        seen[W - 1][i] = now < len ? (float)x[j].v[i] : 0.0f;
        float g = now < len ? (float)go[j].v[i] : 0.0f;
        if (c.silu) {
          const float p = taps.sum(seen, i), sg = sigmoid<E>(p);
          g *= sg * fmaf(p, 1.0f - sg, 1.0f);
        }
        dp[W - 1][i] = g;
        const float mine = now < t1 ? g : 0.0f;
        dw[W][i] += mine;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) {
          dw[k][i] = fmaf(mine, seen[k][i], dw[k][i]);
          sum = fmaf(taps.w[i][k], dp[W - 1 - k][i], sum);
        }
        out[i] = done < len ? sum : 0.0f;
      }
      if (done >= t0) {
        store_some<E, V>(dx.at(done, b) + d, out);
      } else if (t0 == 0 && dstate0) {
        store_some<E, V>(dstate0 + ((int64_t)b * (W - 1) + now) * c.D + d, out);
      }
    }
  }
  if (q)
#pragma unroll
    for (int k = 0; k <= W; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) share[q - 1][k * V + i][lane] = dw[k][i];
  __syncthreads();
  if (q) return;
#pragma unroll
  for (int k = 0; k <= W; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j + 1 < kTogether; ++j) dw[k][i] += share[j][k * V + i][lane];
  float* to = parts + ((int64_t)blockIdx.z * c.B + b) * (W + 1) * c.D + d;
#pragma unroll
  for (int k = 0; k <= W; ++k) store_some<float, V>(to + (int64_t)k * c.D, dw[k]);
}

// The parts in order: sixteen waves a share each, then the shares.
template <int W>
__global__ void __launch_bounds__(1024)
join_weights_kernel(const float* __restrict__ parts, int count, int D, float* __restrict__ dweight, float* __restrict__ dbias) {
  __shared__ float share[16][64];
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane, all = (int64_t)(W + 1) * D;
  const int each = (count + 15) / 16, last = (q + 1) * each < count ? (q + 1) * each : count;
  float sum = 0.0f;
  if (i < all)
#pragma unroll 8
    for (int k = q * each; k < last; ++k) sum += parts[k * all + i];
  share[q][lane] = sum;
  __syncthreads();
  if (q || i >= all) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) sum += share[k][lane];
  const int tap = (int)(i / D), d = (int)(i - (int64_t)tap * D);
  if (tap < W) dweight[(int64_t)d * W + tap] = sum;
  else if (dbias) dbias[d] = sum;
}

template <typename E, int W, int V>
__global__ void __launch_bounds__(64)
conv_step_kernel(const Conv<E> c, Rows<E> y, E* __restrict__ state, int slots_in_state, const int32_t* __restrict__ slots) {
  const int d = (blockIdx.x * 64 + threadIdx.x) * V, b = blockIdx.y;     // V divides D: a window that two threads move is moved twice
  if (d >= c.D) return;
  const int slot = slots ? slots[b] : b;
  float out[V] = {};
  if (slot >= 0 && slot < slots_in_state) {
    E* s = state + (int64_t)slot * (W - 1) * c.D + d;
    Some<E, V> held[W];
#pragma unroll
    for (int k = 0; k < W; ++k) held[k] = load_some<E, V>(k < W - 1 ? s + (int64_t)k * c.D : c.x.at(0, b) + d);
    const Taps<V, W> taps(c, d);
    float seen[W][V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int k = 0; k < W; ++k) seen[k][i] = (float)held[k].v[i];
      const float p = taps.sum(seen, i);
      out[i] = c.silu ? p * sigmoid<E>(p) : p;
    }
#pragma unroll
    for (int k = 0; k + 1 < W; ++k) *reinterpret_cast<Some<E, V>*>(s + (int64_t)k * c.D) = held[k + 1];
  }
  store_some<E, V>(y.at(0, b) + d, out);
}

// Steps of a span: 64, or fewer, to 8, while the device would have less than `waves` a SIMD; every span reads W-1 rows twice.
// Forward at T = 4096, B = 4, D = 4096: 60.8 us in spans of 32 (four waves), 69.5 in spans of 64.
int span_of(int T, int64_t threads_a_step, int waves) {
  int span = 64;
  while (span > 8 && threads_a_step * bppsa_ceil_div(T, span) < (int64_t)bppsa_compute_units() * 256 * waves) span /= 2;
  return span;
}
// Channels of a thread.
template <typename E>
constexpr int kWide = 16 / sizeof(E);
template <typename E>
constexpr int kNarrow = 8 / sizeof(E);
int waves_for(int D, int V) { return bppsa_ceil_div(bppsa_ceil_div(D, V), 64); }
int backward_width(int D, int type) {
  const int V = type == BPPSA_F32 ? kNarrow<float> : kNarrow<bf16_t>;
  return D >= V ? V : 1;
}
int backward_span(int T, int B, int D, int type) { return span_of(T, (int64_t)B * bppsa_ceil_div(D, backward_width(D, type)), 2); }

template <typename F>
bppsa_status by_width(int W, F&& f) {
  switch (W) {
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    default: return f(std::integral_constant<int, 4>{});
  }
}

bool too_large(int T, int B, int D) {
  return bppsa_mul_overflows(T, B, D, 2) || B > 65535 || T > 65535 * 64 || D > 1 << 24;
}

bppsa_status check_conv(const bppsa_conv* c) {
  if (!c || c->T < 1 || c->B < 1 || c->D < 1 || c->W < 1 || !c->x.data || !c->weight) return BPPSA_EINVAL;
  if (c->W < 2 || c->W > BPPSA_SSM_MAX_W || c->type < BPPSA_F32 || c->type > BPPSA_F16) return BPPSA_EUNSUPPORTED;
  return too_large(c->T, c->B, c->D) ? BPPSA_EOVERFLOW : BPPSA_OK;
}

}  // namespace

extern "C" bppsa_status bppsa_ssm_conv(const bppsa_conv* conv, const bppsa_rows* y, void* state_last, void* stream) {
  BPPSA_TRY(check_conv(conv));
  if (!y || !writable(*y, conv->T, conv->B) || (state_last && state_last == conv->state0)) return BPPSA_EINVAL;
  return by_type(conv->type, [&](auto e) {
    using E = decltype(e);
    return by_width(conv->W, [&](auto w) {
      auto run = [&](auto v) {
        constexpr int V = v.value;
        const int across = bppsa_ceil_div(conv->D, V), span = span_of(conv->T, (int64_t)conv->B * across, 4);
        const int64_t threads = (int64_t)across * bppsa_ceil_div(conv->T, span);
        conv_kernel<E, w.value, V><<<dim3((unsigned)((threads + 63) / 64), conv->B), 64, 0, (hipStream_t)stream>>>(
            conv_of<E>(*conv, span), rows_of<E>(*y), static_cast<E*>(state_last));
        BPPSA_CHECK_LAUNCH();
        return BPPSA_OK;
      };
      return conv->D >= kWide<E> ? run(std::integral_constant<int, kWide<E>>{}) : run(std::integral_constant<int, 1>{});
    });
  });
}

extern "C" size_t bppsa_ssm_conv_backward_workspace_bytes(int T, int B, int D, int W) {
  if (T < 1 || B < 1 || D < 1 || W < 2 || W > BPPSA_SSM_MAX_W || too_large(T, B, D)) return 0;
  // the type is not asked for: the shorter spans of the two
  const int span = std::min(backward_span(T, B, D, BPPSA_F32), backward_span(T, B, D, BPPSA_BF16));
  return (size_t)bppsa_ceil_div(T, span * kTogether) * B * (W + 1) * D * sizeof(float);
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
      const int span = backward_span(conv->T, conv->B, conv->D, conv->type), spans = bppsa_ceil_div(conv->T, span * kTogether);
      auto run = [&](auto v) {
        constexpr int V = v.value;
        conv_backward_kernel<E, W, V><<<dim3(waves_for(conv->D, V), conv->B, spans), 64 * kTogether, 0, s>>>(
            conv_of<E>(*conv, span), rows_of<const E>(*dy), rows_of<E>(*dx), static_cast<E*>(dstate0), parts);
      };
      if (backward_width(conv->D, conv->type) == 1) run(std::integral_constant<int, 1>{});
      else run(std::integral_constant<int, kNarrow<E>>{});
      join_weights_kernel<W><<<(unsigned)(((int64_t)(W + 1) * conv->D + 63) / 64), 1024, 0, s>>>(parts, spans * conv->B, conv->D,
                                                                                               dweight, dbias);
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
      auto run = [&](auto v) {
        constexpr int V = v.value;
        conv_step_kernel<E, w.value, V><<<dim3(waves_for(conv->D, V), conv->B), 64, 0, (hipStream_t)stream>>>(
            conv_of<E>(*conv, 1), rows_of<E>(*y), static_cast<E*>(state), slots_in_state, slots);
        BPPSA_CHECK_LAUNCH();
        return BPPSA_OK;
      };
      return conv->D % 4 == 0 ? run(std::integral_constant<int, 4>{}) : run(std::integral_constant<int, 1>{});
    });
  });
}
