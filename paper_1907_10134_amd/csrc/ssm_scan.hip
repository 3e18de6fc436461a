// The selective scan, forward: over sequences, and the step of single tokens.
#include "ssm_scan_parts.h"

namespace {

using namespace ssm;

// One workgroup: 64 channels, one sample, one span, in passes of PASS steps.  In each pass a wave turns ROWS of the steps
// into (s, s u) in LDS for all waves, all waves walk the PASS steps of their states and leave their share of the sum over
// the states in LDS, and each wave finishes its ROWS of outputs.  Inputs of the next pass are prepared and outputs of the
// last one finished beside a pass, so there is one barrier a pass.
// Bound by issue: a step of four states takes 4 exp (two slots each), 16 products and multiply-adds, two LDS accesses.
template <typename E, int WAVES, bool SUMMARY, bool GATE>
__global__ void __launch_bounds__(WAVES * 64)
scan_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states, const float* __restrict__ coef,
            const Summary sum, const Spans spans) {
  constexpr int PASS = kKept, ROWS = (PASS + WAVES - 1) / WAVES;   // a wave prepares and finishes ROWS steps
  __shared__ float2 step_in[2][PASS][kTile];
  __shared__ float share[SUMMARY ? 1 : 2][SUMMARY ? 1 : WAVES][SUMMARY ? 1 : PASS][kTile];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int count = SUMMARY ? spans.count - 1 : spans.count;       // nothing asks for the last span's summary
  const int span = blockIdx.x % count, tile = blockIdx.x / count, g = tile / l.tiles, b = blockIdx.y;
  const int in = tile % l.tiles * kTile + lane;
  const bool on = in < l.wide;
  const int d = g * l.wide + (on ? in : 0);              // lanes without a channel compute the group's first, and store nothing
  const int len = clamp_length(l.lengths, b, l.T), t0 = span * spans.steps;
  const int t1 = t0 + spans.steps < l.T ? t0 + spans.steps : l.T, stop = t1 < len ? t1 : len;

  float A2[kHeld], h[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int n = w * kHeld + i;
    A2[i] = n < l.N ? l.A[(int64_t)d * l.N + n] * kLog2e : 0.0f;
    h[i] = !SUMMARY && n < l.N && l.h0 ? l.h0[((int64_t)b * l.D + d) * l.N + n] : 0.0f;
  }
  if (!SUMMARY && stop > t0)
    for (int k = 0; k < span; ++k) {
      const float4 end = *reinterpret_cast<const float4*>(sum.ends + state_at(k, l.B, b, WAVES, w, l.D, d));
      const float s = sum.sums[((int64_t)k * l.B + b) * l.D + d];
      h[0] = fmaf(exp2_fast(A2[0] * s), h[0], end.x), h[1] = fmaf(exp2_fast(A2[1] * s), h[1], end.y);
      h[2] = fmaf(exp2_fast(A2[2] * s), h[2], end.z), h[3] = fmaf(exp2_fast(A2[3] * s), h[3], end.w);
    }

  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f, skip = l.skip ? l.skip[d] : 0.0f;
  const uint32_t byte = (uint32_t)d * sizeof(E);
  E u[ROWS], dt[ROWS], z[ROWS], u_was[ROWS], z_was[ROWS];
  float total = 0.0f;
  // Steps behind the last one read the last one's row and count as steps of size zero.  The values stay as they are loaded
  // until they are needed: a conversion here would wait for each load by itself.
  auto fetch = [&](int first) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int t = first + w * ROWS + r, at = t < stop ? t : stop - 1;
      u[r] = element(l.u.at(at, b), byte), dt[r] = element(l.dt.at(at, b), byte);
      if (GATE) z[r] = element(l.z.at(at, b), byte);
    }
  };
  auto prepare = [&](int first, int buffer) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (w * ROWS + r >= PASS) break;
      const bool real = first + w * ROWS + r < stop;
      const float s = real ? softplus<E>((float)dt[r] + bias) : 0.0f;
      if (SUMMARY) total += s;
      step_in[buffer][w * ROWS + r][lane] = make_float2(s, real ? s * (float)u[r] : 0.0f);
    }
  };
  auto finish = [&](int first, int buffer) {
    float v[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int row = w * ROWS + r < PASS ? w * ROWS + r : 0;
      v[r] = skip * (float)u_was[r];
#pragma unroll
      for (int k = 0; k < WAVES; ++k) v[r] += share[buffer][k][row][lane];
      if (GATE) v[r] *= (float)z_was[r] * sigmoid<E>((float)z_was[r]);
    }
    if (!on) return;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int t = first + w * ROWS + r;
      if (w * ROWS + r < PASS && t < stop) element(y.at(t, b), byte) = static_cast<E>(v[r]);
    }
  };

  const int padded = (l.T + kPad - 1) / kPad * kPad;
  const int passes = stop > t0 ? (stop - t0 + PASS - 1) / PASS : 0;
  const float* from = coef + ((((int64_t)b * l.G + g) * WAVES + w) * padded + t0) * 2 * kHeld;
  Coef now, next;
  if (passes) {
    fetch(t0);
    prepare(t0, 0);
    now.ask(from);
  }
  __syncthreads();
  for (int p = 0; p < passes; ++p) {
    const int first = t0 + p * PASS, buffer = p & 1;
    float2 in_now[kBatch], in_next[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) in_now[i] = step_in[buffer][i][lane];
    if (!SUMMARY && p) finish(first - PASS, buffer ^ 1);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) u_was[r] = u[r], z_was[r] = z[r];
    if (p + 1 < passes) fetch(first + PASS);
#pragma unroll
    for (int j = 0; j < PASS; j += kBatch) {
      wait_for_scalars();
      next.ask(from + (j + kBatch < PASS || p + 1 < passes ? j + kBatch : 0) * 2 * kHeld);
      if (j + kBatch < PASS)
#pragma unroll
        for (int i = 0; i < kBatch; ++i) in_next[i] = step_in[buffer][j + kBatch + i][lane];
      __builtin_amdgcn_sched_barrier(0);
      if (!SUMMARY && states && j % kKept == 0 && on && first + j < stop)
        *reinterpret_cast<float4*>(states + state_at((first + j) / kKept, l.B, b, WAVES, w, l.D, d)) = make_float4(h[0], h[1], h[2], h[3]);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
          h[k] = fmaf(exp2_fast(in_now[i].x * A2[k]), h[k], in_now[i].y * now.B(i, k));
          if (!SUMMARY) v = k ? fmaf(now.C(i, k), h[k], v) : now.C(i, k) * h[k];
        }
        if (!SUMMARY) share[buffer][w][j + i][lane] = v;
      }
      __builtin_amdgcn_sched_barrier(0);
      now = next;
#pragma unroll
      for (int i = 0; i < kBatch; ++i) in_now[i] = in_next[i];
    }
    from += PASS * 2 * kHeld;
    if (p + 1 < passes) prepare(first + PASS, buffer ^ 1);
    __syncthreads();
  }
  if (!SUMMARY && passes) finish(t0 + (passes - 1) * PASS, (passes - 1) & 1);

  if constexpr (SUMMARY) {
    // every wave has the steps of its rows
    static_assert(sizeof(step_in) >= WAVES * kTile * sizeof(float));
    float* totals = &step_in[0][0][0].x;
    totals[w * kTile + lane] = total;
    __syncthreads();
    if (!on) return;
    *reinterpret_cast<float4*>(sum.ends + state_at(span, l.B, b, WAVES, w, l.D, d)) = make_float4(h[0], h[1], h[2], h[3]);
    if (w == 0) {
      for (int k = 1; k < WAVES; ++k) total += totals[k * kTile + lane];
      sum.sums[((int64_t)span * l.B + b) * l.D + d] = total;
    }
  } else {
    if (!on) return;
    for (int t = (t0 > len ? t0 : len) + w; t < t1; t += WAVES) store(y.at(t, b) + d, 0.0f);
    if (h_last && (len ? t0 < len && len <= t1 : span == 0))
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (w * kHeld + i < l.N) h_last[((int64_t)b * l.D + d) * l.N + w * kHeld + i] = h[i];
  }
}

// The workspace of a forward call: Bm and Cm as floats, and the spans' summaries.
struct Scratch {
  size_t coef, ends, sums, bytes;
  Spans spans;
  Scratch(int T, int B, int D, int N, int G) : spans(spans_of(T, B, D, N, G, 6)) {
    Arena take;
    coef = take(coef_floats(T, B, N, G));
    const int64_t parts = spans.count > 1 ? (int64_t)spans.count * B * D : 0;
    ends = take(parts * waves_of(N) * kHeld), sums = take(parts);
    bytes = take.at;
  }
};

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
  const float u = load(l.u.at(0, b) + d), s = softplus<E>(load(l.dt.at(0, b) + d) + (l.dt_bias ? l.dt_bias[d] : 0.0f));
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
    sum *= z * sigmoid<E>(z);
  }
  store(y.at(0, b) + d, sum);
}

}  // namespace

extern "C" size_t bppsa_ssm_scan_states_bytes(int T, int B, int D, int N) {
  if (!sizes_ok(T, B, D, N, 1)) return 0;
  return (size_t)bppsa_ceil_div(T, kKept) * B * D * waves_of(N) * kHeld * sizeof(float);
}

extern "C" size_t bppsa_ssm_scan_workspace_bytes(int T, int B, int D, int N, int G) {
  return sizes_ok(T, B, D, N, G) ? Scratch(T, B, D, N, G).bytes : 0;
}

extern "C" bppsa_status bppsa_ssm_scan(const bppsa_ssm* layer, const bppsa_rows* y, float* h_last, void* states,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, layer->T, layer->B)) return BPPSA_EINVAL;
  const Scratch at(layer->T, layer->B, layer->D, layer->N, layer->G);
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, at.bytes));
  const hipStream_t s = (hipStream_t)stream;
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    const Layer<E> l = layer_of<E>(*layer);
    auto part = [&](size_t o) { return reinterpret_cast<float*>(static_cast<char*>(workspace) + o); };
    launch_coef(l, part(at.coef), s);
    const Summary sum{part(at.ends), part(at.sums)};
    return by_waves(waves_of(l.N), [&](auto waves) {
      constexpr int W = waves.value;
      if (at.spans.count > 1)
        scan_kernel<E, W, true, false><<<dim3(l.G * l.tiles * (at.spans.count - 1), l.B), W * 64, 0, s>>>(
            l, Rows<E>{}, nullptr, nullptr, part(at.coef), sum, at.spans);
      const auto kernel = l.z.data ? scan_kernel<E, W, false, true> : scan_kernel<E, W, false, false>;
      kernel<<<dim3(l.G * l.tiles * at.spans.count, l.B), W * 64, 0, s>>>(l, rows_of<E>(*y), h_last, static_cast<float*>(states),
                                                                        part(at.coef), sum, at.spans);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
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
