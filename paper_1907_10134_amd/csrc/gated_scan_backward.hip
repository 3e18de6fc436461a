// The gated recurrence's gradients.
//
// With q = dy silu(z) and g[t] = dL/dh[t] = q + a[t+1] g[t+1], the walk from the end carries w[t] = a[t] g[t], and with
//     s = g (a^2 iota x rho / m - rho a h[t-1])
//     dx = g m iota,  di = g m x iota (1 - iota),  dr = decay (1 - rho) s,  dz = dy h silu'(z),
// ddecay, the biases' gradients are the sums of s, dr and di over samples and time.
#include "gated_parts.h"

namespace {

using namespace gated;

template <typename E>
struct Grads {
  Rows<E> dx, dr, di, dz;
  float *parts, *dh0;              // parts: of ddecay, dr_bias and di_bias, [part][3][D]
};

// One thread a lane's channels of a sample, the states of kKept steps found again from the one kept before them.
template <typename E, int V, bool GATE>
__global__ void __launch_bounds__(64)
gated_backward_kernel(const Layer<E> l, Rows<const E> dy, const float* __restrict__ dh_last, const float* __restrict__ states,
                      const Grads<E> o) {
  const Own<V> own(blockIdx.x, threadIdx.x, l.D);
  const int b = blockIdx.y, d = own.d, len = clamp_length(l.lengths, b, l.T);
  if (!own.on) return;
  float decay[V], rb[V], ib[V], w[V], sums[3][V] = {}, zero[V] = {};
  parameter(l.decay, d, decay), parameter(l.r_bias, d, rb), parameter(l.i_bias, d, ib);
  parameter(dh_last ? dh_last + (int64_t)b * l.D : nullptr, d, w);
  for (int t = len; t < l.T; ++t) {
    store_some<E, V>(o.dx.at(t, b) + d, zero), store_some<E, V>(o.dr.at(t, b) + d, zero), store_some<E, V>(o.di.at(t, b) + d, zero);
    if (GATE) store_some<E, V>(o.dz.at(t, b) + d, zero);
  }
  for (int tile = (len + kKept - 1) / kKept - 1; tile >= 0; --tile) {
    const int first = tile * kKept, end = first + kKept < len ? first + kKept : len;
    float before[kKept][V], h[V];
    parameter(states + ((int64_t)tile * l.B + b) * l.D, d, h);
    for (int t = first; t < end; ++t) {
      const auto x = load_some<E, V>(l.x.at(t, b) + d), r = load_some<E, V>(l.r.at(t, b) + d), i = load_some<E, V>(l.i.at(t, b) + d);
      for (int c = 0; c < V; ++c) {
        before[t - first][c] = h[c];
        const Gates g = gates_of<E>((float)r.v[c] + rb[c], (float)i.v[c] + ib[c], decay[c]);
        h[c] = fmaf(g.a, h[c], __builtin_amdgcn_sqrtf(g.m2) * g.iota * (float)x.v[c]);
      }
    }
    for (int t = end - 1; t >= first; --t) {
      const auto x_ = load_some<E, V>(l.x.at(t, b) + d), r = load_some<E, V>(l.r.at(t, b) + d), i = load_some<E, V>(l.i.at(t, b) + d);
      const auto go = load_some<E, V>(dy.at(t, b) + d);
      Some<E, V> z_ = {};
      if (GATE) z_ = load_some<E, V>(l.z.at(t, b) + d);
      float dx[V], dr[V], di[V], dz[V];
      for (int c = 0; c < V; ++c) {
        const Gates g = gates_of<E>((float)r.v[c] + rb[c], (float)i.v[c] + ib[c], decay[c]);
        const float x = (float)x_.v[c], root = g.m2 > 0x1p-120f ? __builtin_amdgcn_rsqf(g.m2) : 0.0f, m = g.m2 * root;
        float q = (float)go.v[c];
        if (GATE) {
          const float z = (float)z_.v[c], sg = sigmoid<E>(z), now = fmaf(g.a, before[t - first][c], m * g.iota * x);
          dz[c] = q * now * sg * fmaf(z, 1.0f - sg, 1.0f);
          q *= z * sg;
        }
        const float gh = q + w[c];
        w[c] = g.a * gh;
        const float s = w[c] * g.rho * (g.a * g.iota * x * root - before[t - first][c]);
        dx[c] = gh * m * g.iota;
        di[c] = dx[c] * x * (1.0f - g.iota);
        dr[c] = decay[c] * (1.0f - g.rho) * s;
        sums[0][c] += s, sums[1][c] += dr[c], sums[2][c] += di[c];
      }
      store_some<E, V>(o.dx.at(t, b) + d, dx), store_some<E, V>(o.dr.at(t, b) + d, dr), store_some<E, V>(o.di.at(t, b) + d, di);
      if (GATE) store_some<E, V>(o.dz.at(t, b) + d, dz);
    }
  }
  if (o.dh0) store_some<float, V>(o.dh0 + (int64_t)b * l.D + d, w);
  for (int k = 0; k < 3; ++k) store_some<float, V>(o.parts + ((int64_t)b * 3 + k) * l.D + d, sums[k]);
}

// The sums over parts, in order: sixteen waves a sixteenth each, then those.  In 64 bits, which cost nothing beside the loads.
struct Joined {
  float *ddecay, *dr_bias, *di_bias;
};
constexpr int kJoining = 16;
__global__ void __launch_bounds__(kJoining * 64)
gated_join_kernel(const float* __restrict__ parts, int D, int64_t n, const Joined to) {
  __shared__ double share[kJoining][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t i = (int64_t)blockIdx.x * 64 + lane, each = (n + kJoining - 1) / kJoining;
  const int64_t last = (w + 1) * each < n ? (w + 1) * each : n;
  double sum = 0.0;
  if (i < 3 * (int64_t)D)
#pragma unroll 8
    for (int64_t k = w * each; k < last; ++k) sum += (double)parts[k * 3 * D + i];
  share[w][lane] = sum;
  __syncthreads();
  if (w || i >= 3 * (int64_t)D) return;
  for (int k = 1; k < kJoining; ++k) sum += share[k][lane];
  float* const out = i < D ? to.ddecay : i < 2 * (int64_t)D ? to.dr_bias : to.di_bias;
  if (out) out[i % D] = (float)sum;
}

}  // namespace

extern "C" size_t bppsa_gated_scan_backward_workspace_bytes(int T, int B, int D) {
  return sizes_ok(T, B, D) ? bppsa_align_up((size_t)B * 3 * D * sizeof(float), 256) : 0;
}

extern "C" bppsa_status bppsa_gated_scan_backward(const bppsa_gated* layer, const bppsa_rows* dy, const float* dh_last,
                                                  const void* states, const bppsa_gated_grads* grads, void* workspace,
                                                  size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!dy || !dy->data || !states || ((uintptr_t)states & 15) || !grads || !grads->ddecay) return BPPSA_EINVAL;
  if (!writable(grads->dx, layer->T, layer->B) || !writable(grads->dr, layer->T, layer->B) || !writable(grads->di, layer->T, layer->B))
    return BPPSA_EINVAL;
  if (!layer->z.data != !grads->dz.data || (layer->z.data && !writable(grads->dz, layer->T, layer->B))) return BPPSA_EINVAL;
  if (dh_last && dh_last == grads->dh0) return BPPSA_EINVAL;
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, bppsa_gated_scan_backward_workspace_bytes(layer->T, layer->B, layer->D)));
  const hipStream_t s = (hipStream_t)stream;
  float* const parts = static_cast<float*>(workspace);
  BPPSA_TRY(by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    return by_width<E>(layer->D, [&](auto width) {
      constexpr int V = width.value;
      const Layer<E> l = layer_of<E>(*layer, 64 * V);
      const Grads<E> o{rows_of<E>(grads->dx), rows_of<E>(grads->dr), rows_of<E>(grads->di), rows_of<E>(grads->dz), parts, grads->dh0};
      const auto kernel = l.z.data ? gated_backward_kernel<E, V, true> : gated_backward_kernel<E, V, false>;
      kernel<<<dim3(l.columns, l.B), 64, 0, s>>>(l, rows_of<const E>(*dy), dh_last, static_cast<const float*>(states), o);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  }));
  gated_join_kernel<<<bppsa_ceil_div(3 * layer->D, 64), kJoining * 64, 0, s>>>(
      parts, layer->D, layer->B, Joined{grads->ddecay, grads->dr_bias, grads->di_bias});
  BPPSA_CHECK_LAUNCH();
  return BPPSA_OK;
}
