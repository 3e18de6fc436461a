// The gated recurrence, forward: over sequences, and the step of single tokens.
#include "gated_parts.h"

namespace {

using namespace gated;

// One thread a lane's channels of a sample, one step after the other.
template <typename E, int V, bool GATE>
__global__ void __launch_bounds__(64)
gated_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states) {
  const Own<V> own(blockIdx.x, threadIdx.x, l.D);
  const int b = blockIdx.y, d = own.d, len = clamp_length(l.lengths, b, l.T);
  if (!own.on) return;
  float decay[V], rb[V], ib[V], h[V];
  parameter(l.decay, d, decay), parameter(l.r_bias, d, rb), parameter(l.i_bias, d, ib);
  parameter(l.h0 ? l.h0 + (int64_t)b * l.D : nullptr, d, h);
  for (int t = 0; t < l.T; ++t) {
    float out[V] = {};
    if (states && t % kKept == 0)
      for (int c = 0; c < V; ++c) states[((int64_t)(t / kKept) * l.B + b) * l.D + d + c] = h[c];
    if (t < len) {
      const auto x = load_some<E, V>(l.x.at(t, b) + d), r = load_some<E, V>(l.r.at(t, b) + d), i = load_some<E, V>(l.i.at(t, b) + d);
      Some<E, V> z = {};
      if (GATE) z = load_some<E, V>(l.z.at(t, b) + d);
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const Gates g = gates_of<E>((float)r.v[c] + rb[c], (float)i.v[c] + ib[c], decay[c]);
        h[c] = fmaf(g.a, h[c], __builtin_amdgcn_sqrtf(g.m2) * g.iota * (float)x.v[c]);
        out[c] = GATE ? h[c] * (float)z.v[c] * sigmoid<E>((float)z.v[c]) : h[c];
      }
    }
    store_some<E, V>(y.at(t, b) + d, out);
  }
  if (h_last) store_some<float, V>(h_last + (int64_t)b * l.D + d, h);
}

// One token.  A thread has a lane's channels of one row of the batch; bound by the launch and one round of loads.
template <typename E, int V>
__global__ void __launch_bounds__(64)
gated_step_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ state, int slots_in_state, const int32_t* __restrict__ slots) {
  const int b = blockIdx.x / l.columns;
  const Own<V> own(blockIdx.x % l.columns, threadIdx.x, l.D);
  if (!own.on) return;
  const int d = own.d;
  int slot = slots ? slots[b] : b;
  float out[V] = {};
  if (slot < 0 || slot >= slots_in_state) return store_some<E, V>(y.at(0, b) + d, out);
  float decay[V], rb[V], ib[V], h[V];
  float* const at = state + (int64_t)slot * l.D + d;
  parameter(l.decay, d, decay), parameter(l.r_bias, d, rb), parameter(l.i_bias, d, ib), parameter(at, 0, h);
  const auto x = load_some<E, V>(l.x.at(0, b) + d), r = load_some<E, V>(l.r.at(0, b) + d), i = load_some<E, V>(l.i.at(0, b) + d);
  Some<E, V> z = {};
  if (l.z.data) z = load_some<E, V>(l.z.at(0, b) + d);
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const Gates g = gates_of<E>((float)r.v[c] + rb[c], (float)i.v[c] + ib[c], decay[c]);
    h[c] = fmaf(g.a, h[c], __builtin_amdgcn_sqrtf(g.m2) * g.iota * (float)x.v[c]);
    out[c] = l.z.data ? h[c] * (float)z.v[c] * sigmoid<E>((float)z.v[c]) : h[c];
  }
  // in place: what is repeated has been read before or behind the neighbour's update, and is not stored
  if (own.repeated) {
    for (int c = own.repeated; c < V; ++c) at[c] = h[c], store(y.at(0, b) + d + c, out[c]);
    return;
  }
  store_some<float, V>(at, h);
  store_some<E, V>(y.at(0, b) + d, out);
}

}  // namespace

extern "C" size_t bppsa_gated_scan_states_bytes(int T, int B, int D) {
  return sizes_ok(T, B, D) ? (size_t)bppsa_ceil_div(T, kKept) * B * D * sizeof(float) : 0;
}

extern "C" size_t bppsa_gated_scan_workspace_bytes(int T, int B, int D) { return 0; }

extern "C" bppsa_status bppsa_gated_scan(const bppsa_gated* layer, const bppsa_rows* y, float* h_last, void* states,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, layer->T, layer->B) || (h_last && h_last == layer->h0) || ((uintptr_t)states & 15)) return BPPSA_EINVAL;
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, bppsa_gated_scan_workspace_bytes(layer->T, layer->B, layer->D)));
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    return by_width(layer->D, [&](auto width) {
      constexpr int V = width.value;
      const Layer<E> l = layer_of<E>(*layer, 64 * V);
      const auto kernel = l.z.data ? gated_kernel<E, V, true> : gated_kernel<E, V, false>;
      kernel<<<dim3(l.columns, l.B), 64, 0, (hipStream_t)stream>>>(l, rows_of<E>(*y), h_last, static_cast<float*>(states));
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}

extern "C" bppsa_status bppsa_gated_scan_step(const bppsa_gated* layer, const bppsa_rows* y, float* state, int slots_in_state,
                                              const int32_t* slots, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, 1, layer->B) || !state || slots_in_state < 1 || layer->h0 || layer->lengths) return BPPSA_EINVAL;
  if (layer->T != 1 || (!slots && layer->B > slots_in_state)) return BPPSA_ESHAPE;
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    return by_width(layer->D, [&](auto width) {
      constexpr int V = width.value;
      const Layer<E> l = layer_of<E>(*layer, 64 * V);
      gated_step_kernel<E, V><<<(unsigned)(l.columns * l.B), 64, 0, (hipStream_t)stream>>>(l, rows_of<E>(*y), state, slots_in_state, slots);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}
