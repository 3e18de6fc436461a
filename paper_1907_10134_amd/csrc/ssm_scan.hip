// The selective scan: forward over sequences, its gradients, and the step of single tokens.
#include "ssm_scan_parts.h"

namespace {

using namespace ssm;

// A long sequence with few channels is cut into spans.  A first launch scans each span from a state of zero and keeps
// only where that ends and the sum of its steps; a channel's decay over a span is exp(A sum), so that the second launch
// can join the spans in front of its own in a few multiply-adds and scan it from its true start.
struct Summary {
  float *ends, *sums;              // [span][b][wave][d][4], [span][b][d]
};

// Steps of a pass: a multiple of kKept that divides kPad.
constexpr int pass_of(int waves) { return waves > 2 && waves <= 8 ? 16 : 8; }

// One workgroup: 64 channels, one sample, one span, in passes of PASS steps.  In each pass a wave turns ROWS of the steps
// into (s, s u) in LDS for all waves, all waves walk the PASS steps of their states and leave their share of the sum over
// the states in LDS, and each wave finishes its ROWS of outputs.  Inputs of the next pass are prepared and outputs of the
// last one finished beside a pass, so there is one barrier a pass.
// Bound by issue: a step of four states takes 4 exp (two slots each), 16 products and multiply-adds, two LDS accesses.
template <typename E, int WAVES, bool SUMMARY, bool GATE>
__global__ void __launch_bounds__(WAVES * 64)
scan_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states, const float* __restrict__ coef,
            const Summary sum, const Spans spans) {
  constexpr int PASS = pass_of(WAVES), ROWS = (PASS + WAVES - 1) / WAVES;   // a wave prepares and finishes ROWS steps
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

// Spans: as many as give every SIMD some four waves, none shorter than 64 steps (a multiple of 32), 64 at most.
Spans spans_of(int T, int B, int D, int N, int G) {
  const int64_t waves = (int64_t)G * bppsa_ceil_div(D / G, kTile) * B * waves_of(N);
  int64_t count = (int64_t)bppsa_compute_units() * 4 * 3 / waves;
  if (count > T / 64) count = T / 64;
  if (count > 64) count = 64;
  if (count < 2) return Spans{1, T};
  const int steps = bppsa_ceil_div(bppsa_ceil_div(T, (int)count), kPad) * kPad;
  return Spans{bppsa_ceil_div(T, steps), steps};
}

// The workspace of a forward call: Bm and Cm as floats, and the spans' summaries.
struct Scratch {
  size_t coef, ends, sums, bytes;
  Spans spans;
  Scratch(int T, int B, int D, int N, int G) : spans(spans_of(T, B, D, N, G)) {
    size_t at = 0;
    auto take = [&](int64_t n) { const size_t o = at; at += bppsa_align_up((size_t)n * sizeof(float), 256); return o; };
    coef = take(coef_floats(T, B, N, G));
    const int64_t parts = spans.count > 1 ? (int64_t)spans.count * B * D : 0;
    ends = take(parts * waves_of(N) * kHeld), sums = take(parts);
    bytes = at;
  }
};

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
scan_backward_kernel(const Layer<E> l, Rows<const E> dy, const float* __restrict__ states, int waves, const Grads<E> o) {
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
  for (int k = (len + kKept - 1) / kKept - 1; k >= 0; --k) {
    float h[kKept + 1][NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) h[0][n] = n < l.N ? states[state_at(k, l.B, b, waves, n / kHeld, l.D, d) + n % kHeld] : 0.0f;
    const int steps = len - k * kKept < kKept ? len - k * kKept : kKept;
    for (int i = 0; i < steps; ++i) {
      const int t = k * kKept + i;
      const float s = softplus<E>(load(l.dt.at(t, b) + d) + bias), su = s * load(l.u.at(t, b) + d);
      const E* Bt = l.Bm.at(t, b) + g * l.N;
#pragma unroll
      for (int n = 0; n < NP; ++n)
        h[i + 1][n] = n < l.N ? fmaf(exp2_fast(s * A2[n]), h[i][n], su * load(Bt + n)) : 0.0f;
    }
    for (int i = steps - 1; i >= 0; --i) {
      const int t = k * kKept + i;
      const float u = load(l.u.at(t, b) + d), raw = load(l.dt.at(t, b) + d) + bias, s = softplus<E>(raw), su = s * u;
      const E *Bt = l.Bm.at(t, b) + g * l.N, *Ct = l.Cm.at(t, b) + g * l.N;
      const float go = load(dy.at(t, b) + d), z = l.z.data ? load(l.z.at(t, b) + d) : 0.0f;
      const float sg = sigmoid<E>(z), q = l.z.data ? go * z * sg : go;
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
      const float ddt = fmaf(u, s1, s2) * sigmoid<E>(raw);
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
          l, rows_of<const E>(*dy), static_cast<const float*>(states), waves_of(l.N), o);
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
