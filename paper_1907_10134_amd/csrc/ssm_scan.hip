// The selective scan: forward over sequences, its gradients, and the step of single tokens.
#include "ssm_common.h"

namespace {

using namespace ssm;

constexpr int kTile = 64;        // channels of a workgroup, one a lane, all of one group of B and C
constexpr int kStates = 8;       // steps between two states kept for the backward pass

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

// One thread a channel, its states in registers, one step after the other.
template <typename E, int NP>
__global__ void __launch_bounds__(kTile)
scan_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states) {
  const int g = blockIdx.x / l.tiles, in = (blockIdx.x % l.tiles) * kTile + threadIdx.x, b = blockIdx.y;
  if (in >= l.wide) return;
  const int d = g * l.wide + in, len = clamp_length(l.lengths, b, l.T);
  const int64_t bd = (int64_t)b * l.D + d;
  float h[NP], A2[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    A2[n] = n < l.N ? l.A[(int64_t)d * l.N + n] * kLog2e : 0.0f;
    h[n] = n < l.N && l.h0 ? l.h0[bd * l.N + n] : 0.0f;
  }
  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f, skip = l.skip ? l.skip[d] : 0.0f;
  for (int t = 0; t < len; ++t) {
    if (states && t % kStates == 0)
#pragma unroll
      for (int n = 0; n < NP; ++n)
        if (n < l.N) states[((int64_t)(t / kStates) * l.B * l.D + bd) * l.N + n] = h[n];
    const float u = load(l.u.at(t, b) + d), s = softplus(load(l.dt.at(t, b) + d) + bias), su = s * u;
    const E *Bt = l.Bm.at(t, b) + g * l.N, *Ct = l.Cm.at(t, b) + g * l.N;
    float sum = skip * u;
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if (n < l.N) {
        h[n] = fmaf(exp2_fast(s * A2[n]), h[n], su * load(Bt + n));
        sum = fmaf(load(Ct + n), h[n], sum);
      }
    if (l.z.data) {
      const float z = load(l.z.at(t, b) + d);
      sum *= z * sigmoid(z);
    }
    store(y.at(t, b) + d, sum);
  }
  for (int t = len; t < l.T; ++t) store(y.at(t, b) + d, 0.0f);
  if (h_last)
#pragma unroll
    for (int n = 0; n < NP; ++n)
      if (n < l.N) h_last[bd * l.N + n] = h[n];
}

template <typename E>
struct Grads {
  Rows<E> du, ddt, dz;
  float *bc, *dA, *dskip, *ddt_bias, *dh0;     // bc, dA, dskip and ddt_bias are partial sums, see Partials
};

// Sums that more than one workgroup has a part of: of dB and dC [tiles][T][B][G][2N], one part a tile of channels; of dA
// [B][D][N], dskip and ddt_bias [B][D], one a sample.
struct Partials {
  size_t bc, dA, dskip, ddt_bias, bytes;
  Partials(int64_t T, int64_t B, int64_t D, int64_t N, int64_t G) {
    const int64_t tiles = (D / G + kTile - 1) / kTile;
    size_t at = 0;
    auto take = [&](int64_t n) { const size_t o = at; at += bppsa_align_up((size_t)n * sizeof(float), 256); return o; };
    bc = take(tiles * T * B * G * 2 * N), dA = take(B * D * N), dskip = take(B * D), ddt_bias = take(B * D);
    bytes = at;
  }
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int k = 32; k; k >>= 1) v += __shfl_xor(v, k);
  return v;
}

template <typename E, int NP>
__global__ void __launch_bounds__(kTile)
scan_backward_kernel(const Layer<E> l, Rows<const E> dy, const float* __restrict__ states, const Grads<E> o) {
  const int g = blockIdx.x / l.tiles, tile = blockIdx.x % l.tiles, in = tile * kTile + threadIdx.x, b = blockIdx.y;
  const bool on = in < l.wide;                 // lanes beyond the group's last channel take part in the sums with zeros
  const int d = on ? g * l.wide + in : g * l.wide, len = clamp_length(l.lengths, b, l.T);
  const int64_t bd = (int64_t)b * l.D + d;
  float A2[NP], A[NP], carry[NP], dA[NP];
#pragma unroll
  for (int n = 0; n < NP; ++n) {
    A[n] = n < l.N ? l.A[(int64_t)d * l.N + n] : 0.0f;
    A2[n] = A[n] * kLog2e;
    carry[n] = dA[n] = 0.0f;
  }
  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f, skip = l.skip ? l.skip[d] : 0.0f;
  float dskip = 0.0f, dbias = 0.0f;
  float* bc = o.bc + (int64_t)tile * l.T * l.B * l.G * 2 * l.N;
  for (int t = len; t < l.T; ++t) {
    if (on) {
      store(o.du.at(t, b) + d, 0.0f), store(o.ddt.at(t, b) + d, 0.0f);
      if (o.dz.data) store(o.dz.at(t, b) + d, 0.0f);
    }
    for (int n = threadIdx.x; n < 2 * l.N; n += kTile) bc[(((int64_t)t * l.B + b) * l.G + g) * 2 * l.N + n] = 0.0f;
  }
  for (int k = (len + kStates - 1) / kStates - 1; k >= 0; --k) {
    float h[kStates + 1][NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) h[0][n] = n < l.N ? states[((int64_t)k * l.B * l.D + bd) * l.N + n] : 0.0f;
    const int steps = len - k * kStates < kStates ? len - k * kStates : kStates;
    for (int i = 0; i < steps; ++i) {
      const int t = k * kStates + i;
      const float s = softplus(load(l.dt.at(t, b) + d) + bias), su = s * load(l.u.at(t, b) + d);
      const E* Bt = l.Bm.at(t, b) + g * l.N;
#pragma unroll
      for (int n = 0; n < NP; ++n)
        h[i + 1][n] = n < l.N ? fmaf(exp2_fast(s * A2[n]), h[i][n], su * load(Bt + n)) : 0.0f;
    }
    for (int i = steps - 1; i >= 0; --i) {
      const int t = k * kStates + i;
      const float u = load(l.u.at(t, b) + d), raw = load(l.dt.at(t, b) + d) + bias, s = softplus(raw), su = s * u;
      const E *Bt = l.Bm.at(t, b) + g * l.N, *Ct = l.Cm.at(t, b) + g * l.N;
      const float go = load(dy.at(t, b) + d), z = l.z.data ? load(l.z.at(t, b) + d) : 0.0f;
      const float sg = sigmoid(z), q = l.z.data ? go * z * sg : go;
      float s1 = 0.0f, s2 = 0.0f, plain = skip * u;
#pragma unroll
      for (int n = 0; n < NP; ++n)
        if (n < l.N) {
          const float Bn = load(Bt + n), Cn = load(Ct + n);
          const float gh = fmaf(q, Cn, carry[n]);
          carry[n] = exp2_fast(s * A2[n]) * gh;
          const float ga = carry[n] * h[i][n];
          plain = fmaf(Cn, h[i + 1][n], plain);
          s1 = fmaf(gh, Bn, s1);
          s2 = fmaf(ga, A[n], s2);
          dA[n] = fmaf(ga, s, dA[n]);
          const float sumB = wave_sum(on ? gh * su : 0.0f), sumC = wave_sum(on ? h[i + 1][n] * q : 0.0f);
          if (threadIdx.x == 0) {
            float* at = bc + (((int64_t)t * l.B + b) * l.G + g) * 2 * l.N;
            at[n] = sumB, at[l.N + n] = sumC;
          }
        }
      const float ddt = fmaf(u, s1, s2) * sigmoid(raw);
      dbias += ddt;
      dskip = fmaf(q, u, dskip);
      if (on) {
        store(o.du.at(t, b) + d, fmaf(s, s1, skip * q)), store(o.ddt.at(t, b) + d, ddt);
        if (o.dz.data) store(o.dz.at(t, b) + d, go * plain * sg * fmaf(z, 1.0f - sg, 1.0f));
      }
    }
  }
  if (!on) return;
#pragma unroll
  for (int n = 0; n < NP; ++n)
    if (n < l.N) {
      o.dA[bd * l.N + n] = dA[n];
      if (o.dh0) o.dh0[bd * l.N + n] = carry[n];
    }
  o.dskip[bd] = dskip, o.ddt_bias[bd] = dbias;
}

// dB and dC from the tiles' parts, in the tiles' order.
template <typename E>
__global__ void __launch_bounds__(256)
join_bc_kernel(const float* __restrict__ bc, int tiles, int64_t rows, int N, E* __restrict__ dBm, E* __restrict__ dCm) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = rows * 2 * N;
  if (i >= all) return;
  float sum = 0.0f;
  for (int k = 0; k < tiles; ++k) sum += bc[k * all + i];
  const int64_t row = i / (2 * N);
  const int n = (int)(i - row * 2 * N);
  store((n < N ? dBm : dCm) + row * N + (n < N ? n : n - N), sum);
}

__global__ void __launch_bounds__(256)
join_kernel(const float* __restrict__ parts, int count, int64_t n, float* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float sum = 0.0f;
  for (int k = 0; k < count; ++k) sum += parts[k * n + i];
  out[i] = sum;
}

template <typename E>
__global__ void __launch_bounds__(kTile)
scan_step_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ state, int slots_in_state, const int32_t* __restrict__ slots) {
  const int d = blockIdx.x * kTile + threadIdx.x, b = blockIdx.y;
  if (d >= l.D) return;
  const int slot = slots ? slots[b] : b;
  if (slot < 0 || slot >= slots_in_state) {
    store(y.at(0, b) + d, 0.0f);
    return;
  }
  const int g = d / l.wide;
  const float u = load(l.u.at(0, b) + d), s = softplus(load(l.dt.at(0, b) + d) + (l.dt_bias ? l.dt_bias[d] : 0.0f));
  const E *Bt = l.Bm.at(0, b) + g * l.N, *Ct = l.Cm.at(0, b) + g * l.N;
  float* h = state + ((int64_t)slot * l.D + d) * l.N;
  float sum = l.skip ? l.skip[d] * u : 0.0f;
  for (int n = 0; n < l.N; ++n) {
    const float v = fmaf(exp2_fast(s * l.A[(int64_t)d * l.N + n] * kLog2e), h[n], s * u * load(Bt + n));
    h[n] = v;
    sum = fmaf(load(Ct + n), v, sum);
  }
  if (l.z.data) {
    const float z = load(l.z.at(0, b) + d);
    sum *= z * sigmoid(z);
  }
  store(y.at(0, b) + d, sum);
}

template <typename F>
bppsa_status by_states(int N, F&& f) {
  if (N <= 4) return f(std::integral_constant<int, 4>{});
  if (N <= 8) return f(std::integral_constant<int, 8>{});
  if (N <= 16) return f(std::integral_constant<int, 16>{});
  if (N <= 32) return f(std::integral_constant<int, 32>{});
  return f(std::integral_constant<int, 64>{});
}

bool sizes_ok(int T, int B, int D, int N, int G) {
  return T > 0 && B > 0 && D > 0 && N > 0 && G > 0 && N <= BPPSA_SSM_MAX_N && D % G == 0;
}

bppsa_status check_layer(const bppsa_ssm* l) {
  if (!l || l->T < 1 || l->B < 1 || l->D < 1 || l->N < 1 || l->G < 1) return BPPSA_EINVAL;
  if (!l->u.data || !l->dt.data || !l->Bm.data || !l->Cm.data || !l->A) return BPPSA_EINVAL;
  if (l->D % l->G) return BPPSA_ESHAPE;
  if (l->N > BPPSA_SSM_MAX_N || l->type < BPPSA_F32 || l->type > BPPSA_F16) return BPPSA_EUNSUPPORTED;
  if (bppsa_mul_overflows(l->T, l->B, l->D, 2) || bppsa_mul_overflows(l->B, l->D, l->N, 1) || l->B > 65535)
    return BPPSA_EOVERFLOW;
  return BPPSA_OK;
}

bppsa_status check_workspace(const void* workspace, size_t have, size_t need) {
  if (need && (!workspace || have < need)) return BPPSA_EWORKSPACE;
  return need && ((uintptr_t)workspace & 255) ? BPPSA_EINVAL : BPPSA_OK;
}

}  // namespace

extern "C" size_t bppsa_ssm_scan_states_bytes(int T, int B, int D, int N) {
  if (!sizes_ok(T, B, D, N, 1)) return 0;
  return (size_t)bppsa_ceil_div(T, kStates) * B * D * N * sizeof(float);
}

extern "C" size_t bppsa_ssm_scan_workspace_bytes(int T, int B, int D, int N, int G) { return 0; }

extern "C" bppsa_status bppsa_ssm_scan(const bppsa_ssm* layer, const bppsa_rows* y, float* h_last, void* states,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, layer->T, layer->B)) return BPPSA_EINVAL;
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, bppsa_ssm_scan_workspace_bytes(layer->T, layer->B, layer->D, layer->N, layer->G)));
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    const Layer<E> l = layer_of<E>(*layer);
    return by_states(l.N, [&](auto np) {
      scan_kernel<E, np.value><<<dim3(l.G * l.tiles, l.B), kTile, 0, (hipStream_t)stream>>>(l, rows_of<E>(*y), h_last,
                                                                                          static_cast<float*>(states));
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}

extern "C" size_t bppsa_ssm_scan_backward_workspace_bytes(int T, int B, int D, int N, int G) {
  return sizes_ok(T, B, D, N, G) ? Partials(T, B, D, N, G).bytes : 0;
}

extern "C" bppsa_status bppsa_ssm_scan_backward(const bppsa_ssm* layer, const bppsa_rows* dy, const void* states,
                                                const bppsa_ssm_grads* grads, void* workspace, size_t workspace_bytes,
                                                void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!dy || !dy->data || !states || !grads || !grads->dBm || !grads->dCm || !grads->dA) return BPPSA_EINVAL;
  if (!writable(grads->du, layer->T, layer->B) || !writable(grads->ddt, layer->T, layer->B)) return BPPSA_EINVAL;
  if (!layer->z.data != !grads->dz.data || (layer->z.data && !writable(grads->dz, layer->T, layer->B))) return BPPSA_EINVAL;
  const Partials at(layer->T, layer->B, layer->D, layer->N, layer->G);
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, at.bytes));
  const hipStream_t s = (hipStream_t)stream;
  return by_type(layer->type, [&](auto e) -> bppsa_status {
    using E = decltype(e);
    const Layer<E> l = layer_of<E>(*layer);
    auto part = [&](size_t o) { return reinterpret_cast<float*>(static_cast<char*>(workspace) + o); };
    const Grads<E> o{rows_of<E>(grads->du), rows_of<E>(grads->ddt), rows_of<E>(grads->dz), part(at.bc), part(at.dA),
                     part(at.dskip), part(at.ddt_bias), grads->dh0};
    BPPSA_TRY(by_states(l.N, [&](auto np) {
      scan_backward_kernel<E, np.value><<<dim3(l.G * l.tiles, l.B), kTile, 0, s>>>(
          l, rows_of<const E>(*dy), static_cast<const float*>(states), o);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    }));
    const int64_t rows = (int64_t)l.T * l.B * l.G;
    join_bc_kernel<E><<<(unsigned)((rows * 2 * l.N + 255) / 256), 256, 0, s>>>(
        o.bc, l.tiles, rows, l.N, static_cast<E*>(grads->dBm), static_cast<E*>(grads->dCm));
    auto join = [&](const float* parts, int64_t n, float* out) {
      if (out) join_kernel<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(parts, l.B, n, out);
    };
    join(o.dA, (int64_t)l.D * l.N, grads->dA), join(o.dskip, l.D, grads->dskip), join(o.ddt_bias, l.D, grads->ddt_bias);
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}

extern "C" bppsa_status bppsa_ssm_scan_step(const bppsa_ssm* layer, const bppsa_rows* y, float* state, int slots_in_state,
                                            const int32_t* slots, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, 1, layer->B) || !state || slots_in_state < 1 || layer->h0 || layer->lengths) return BPPSA_EINVAL;
  if (layer->T != 1 || (!slots && layer->B > slots_in_state)) return BPPSA_ESHAPE;
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    const Layer<E> l = layer_of<E>(*layer);
    scan_step_kernel<E><<<dim3(bppsa_ceil_div(l.D, kTile), l.B), kTile, 0, (hipStream_t)stream>>>(l, rows_of<E>(*y), state,
                                                                                                slots_in_state, slots);
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
