// The selective scan, forward: over sequences, and the step of single tokens.
#include "ssm_scan_parts.h"

namespace {

using namespace ssm;

// One workgroup: 64 channels, one sample, one span, in passes of PASS steps.  In each pass a wave turns ROWS of the steps
// into (s, s u) in LDS for all waves, all waves walk the PASS steps of their states and leave their share of the sum over
// the states in LDS, and each wave finishes its ROWS of outputs.  Inputs of the next pass are prepared and outputs of the
// last one finished beside a pass, so there is one barrier a pass.
// Bound by issue: a step of four states takes 4 exp (two slots each) and 16 products and multiply-adds, a step and channel some
// 45 slots beside them for softplus, gate and sums.  T = 30000, B = 1, D = 2048, N = 16, bf16, gated: 310 us with the
// vector unit 88 % busy (and 228 us, 84 %, for the summaries) by a counter that shows 94 % for nothing but one exp and four
// multiply-adds in turn; 0.49 GB of inputs and outputs would take 96 us.
template <typename E, int WAVES, int H, bool SUMMARY, bool GATE>
__global__ void __launch_bounds__(WAVES * 64, WAVES <= 12 ? 6 : 4)      // at least so many waves a SIMD
scan_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states, const Summary sum,
            const Spans spans) {
  constexpr int PASS = kKept, ROWS = (PASS + WAVES - 1) / WAVES;   // a wave prepares and finishes ROWS steps
  constexpr bool ALL = PASS % WAVES == 0;                          // none has fewer
  __shared__ float2 step_in[2][PASS][kTile];
  __shared__ alignas(16) float coef[2][PASS][WAVES][2 * H];
  __shared__ float share[SUMMARY ? 1 : 2][SUMMARY ? 1 : WAVES][SUMMARY ? 1 : PASS][kTile];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // neighbours in the grid, which go to different dies, are tiles of a span: spans may lie behind a sample's end
  const int tile = blockIdx.x % (l.G * l.tiles), span = blockIdx.x / (l.G * l.tiles), g = tile / l.tiles, b = blockIdx.y;
  const int in = tile % l.tiles * kTile + lane;
  const bool on = in < l.wide;
  const int d = g * l.wide + (on ? in : 0);              // lanes without a channel compute the group's first, and store nothing
  const int len = clamp_length(l.lengths, b, l.T), t0 = span * spans.steps;
  const int t1 = t0 + spans.steps < l.T ? t0 + spans.steps : l.T, stop = t1 < len ? t1 : len;

  if (!SUMMARY && on)
    for (int t = (t0 > len ? t0 : len) + w; t < t1; t += WAVES) store(y.at(t, b) + d, 0.0f);

  float A2[H], h[H];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int n = w * H + i;
    A2[i] = n < l.N ? l.A[(int64_t)d * l.N + n] * kLog2e : 0.0f;
    h[i] = !SUMMARY && n < l.N && l.h0 ? l.h0[((int64_t)b * l.D + d) * l.N + n] : 0.0f;
  }
  if (!SUMMARY && stop > t0)
    join_spans(sum, 0, 1, span, l.B, b, WAVES, w, l.D, d, A2, h);

  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f, skip = l.skip ? l.skip[d] : 0.0f;
  const uint32_t byte = (uint32_t)d * sizeof(E);
  const int mine = w * ROWS;                             // this wave's first step of a pass
  Walk<const E> at_u(l.u, t0 + mine, b, byte, PASS), at_dt(l.dt, t0 + mine, b, byte, PASS), at_z(l.z, t0 + mine, b, byte, PASS);
  Walk<E> at_y(y, t0 + mine, b, byte, PASS);
  float* at_states = SUMMARY || !states ? nullptr : states + state_at(H, t0 / kKept, l.B, b, WAVES, w, l.D, d);
  Coef<E, H> at_coef(l, WAVES, threadIdx.x, t0, b, g);
  // What a wave fetches for a pass, two passes ahead: one is not enough for a device that is not full.  The values stay as
  // they are loaded until they are needed: a conversion here would wait for each load by itself.
  struct Fetched {
    uint32_t u[ROWS], dt[ROWS], z[ROWS], coef;
  } raw0, raw1;
  uint32_t u_was[ROWS], z_was[ROWS];
  float total = 0.0f;
  auto fetch = [&](int first, Fetched& x) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      uint32_t a = 0, b = 0, c = 0;
      if ((ALL || mine + r < PASS) && first + mine + r < stop) {
        a = at_u.bits(r), b = at_dt.bits(r);
        if (GATE) c = at_z.bits(r);
      }
      x.u[r] = a, x.dt[r] = b, x.z[r] = c;
    }
    x.coef = at_coef.fetch(stop - first);
    at_u.move(), at_dt.move(), at_coef.move(1);
    if (GATE) at_z.move();
  };
  auto prepare = [&](int first, int buffer, const Fetched& x) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (!ALL && mine + r >= PASS) break;
      float s = softplus<E>(value<E>(x.dt[r]) + bias);
      s = first + mine + r < stop ? s : 0.0f;            // u is zero there
      if (SUMMARY) total += s;
      step_in[buffer][mine + r][lane] = make_float2(s, s * value<E>(x.u[r]));
    }
    if (64 * H >= 256 || threadIdx.x < WAVES * PASS * 2 * H) (&coef[buffer][0][0][0])[threadIdx.x] = value<E>(x.coef);
  };
  auto finish = [&](int first, int buffer) __attribute__((always_inline)) {
    float v[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int row = (ALL || mine + r < PASS) ? mine + r : 0;
      v[r] = skip * value<E>(u_was[r]);
#pragma unroll
      for (int k = 0; k < WAVES; ++k) v[r] += share[buffer][k][row][lane];
      if (GATE) v[r] *= value<E>(z_was[r]) * sigmoid<E>(value<E>(z_was[r]));
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if ((ALL || mine + r < PASS) && first + mine + r < stop && on) at_y.put(r, v[r]);
    at_y.move();
  };

  const int passes = stop > t0 ? (stop - t0 + PASS - 1) / PASS : 0;
  auto pass = [&](int p, auto parity) __attribute__((always_inline)) {
    constexpr int buffer = parity.value;
    Fetched &here = pick<buffer>(raw0, raw1), &there = pick<buffer>(raw1, raw0);
    const int first = t0 + p * PASS;
    if (!SUMMARY && p) finish(first - PASS, buffer ^ 1);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) u_was[r] = here.u[r], z_was[r] = here.z[r];
    fetch(first + 2 * PASS, here);               // nothing, behind the last pass
    if (!SUMMARY && states) {
      if (on) put(at_states, h);
      at_states += (int64_t)l.B * WAVES * l.D * H;
    }
#pragma unroll
    for (int i = 0; i < PASS; ++i) {
      float Bm[H], Cm[H], v = 0.0f;
      two_by_two(i);
      const float2 in_ = step_in[buffer][i][lane];
      get(coef[buffer][i][w], Bm);
      if (!SUMMARY) get(coef[buffer][i][w] + H, Cm);
#pragma unroll
      for (int k = 0; k < H; ++k) {
        h[k] = fmaf(exp2_fast(in_.x * A2[k]), h[k], in_.y * Bm[k]);
        if (!SUMMARY) v = k ? fmaf(Cm[k], h[k], v) : Cm[k] * h[k];
      }
      if (!SUMMARY) share[buffer][w][i][lane] = v;
    }
    now(h);
    prepare(first + PASS, buffer ^ 1, there);    // a pass that no one walks, behind the last one
    __syncthreads();
  };
  if (passes) {
    fetch(t0, raw0);
    fetch(t0 + PASS, raw1);
    prepare(t0, 0, raw0);
  }
  __syncthreads();
  constexpr std::integral_constant<int, 0> even;
  constexpr std::integral_constant<int, 1> odd;
  int p = 0;
  for (; p + 1 < passes; p += 2) pass(p, even), pass(p + 1, odd);
  if (p < passes) pass(p, even);
  if (!SUMMARY && passes) finish(t0 + (passes - 1) * PASS, (passes - 1) & 1);

  if constexpr (SUMMARY) {
    // every wave has the steps of its rows
    static_assert(sizeof(step_in) >= WAVES * kTile * sizeof(float));
    float* totals = &step_in[0][0][0].x;
    totals[w * kTile + lane] = total;
    __syncthreads();
    if (!on) return;
    put(sum.ends + state_at(H, span, l.B, b, WAVES, w, l.D, d), h);
    if (w == 0) {
      for (int k = 1; k < WAVES; ++k) total += totals[k * kTile + lane];
      sum.sums[((int64_t)span * l.B + b) * l.D + d] = total;
    }
  } else {
    if (!on) return;
    if (h_last && (len ? t0 < len && len <= t1 : span == 0))
#pragma unroll
      for (int i = 0; i < H; ++i)
        if (w * H + i < l.N) h_last[((int64_t)b * l.D + d) * l.N + w * H + i] = h[i];
  }
}

constexpr int kWavesWanted = 6;  // of a SIMD, by spans: as many as fit
// The workspace of a forward call: the spans' summaries.
struct Scratch {
  size_t ends, sums, bytes;
  Scratch(int T, int B, int D, int N, int G) {
    Arena take;
    const int most = most_spans(T, B, D, N, G, kWavesWanted);
    const int64_t parts = most > 1 ? (int64_t)most * B * D : 0;
    ends = take(parts * padded_of(N)), sums = take(parts);
    bytes = take.at;
  }
};

// One token.  A thread holds four states of a channel, 2^LANES neighbouring lanes a channel, for kStreams rows of the batch
// one after the other, so that A is read once for all of them and their states are on their way together.  Bound by the
// states' memory: 16 bytes a lane, read and written in place.  VECTOR: N is a multiple of 4 and state and A lie on 16 bytes.
constexpr int kStreams = 2, kHeld = 4;       // B = 64, D = 4096, N = 16: 11.0 us with one, 10.8 with two, 11.3 with four
template <typename E, int LANES, bool VECTOR>
__global__ void __launch_bounds__(256)
scan_step_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ state, int slots_in_state, const int32_t* __restrict__ slots) {
  const int d = blockIdx.x * (256 >> LANES) + (threadIdx.x >> LANES), n = (threadIdx.x & ((1 << LANES) - 1)) * kHeld;
  if (d >= l.D) return;                        // all lanes of a channel alike
  const bool any = n < l.N;
  auto get = [&](const float* p) {
    if (VECTOR) return any ? *reinterpret_cast<const float4*>(p) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    return make_float4(any ? p[0] : 0.0f, n + 1 < l.N ? p[1] : 0.0f, n + 2 < l.N ? p[2] : 0.0f, n + 3 < l.N ? p[3] : 0.0f);
  };
  const float4 A = get(l.A + (int64_t)d * l.N + n);
  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f, skip = l.skip ? l.skip[d] : 0.0f;
  const int g = d / l.wide, b0 = blockIdx.y * kStreams;
  int slot[kStreams];
  float4 h[kStreams];
  E u[kStreams], dt[kStreams], z[kStreams], Bm[kStreams][kHeld], Cm[kStreams][kHeld];
#pragma unroll
  for (int r = 0; r < kStreams; ++r) {
    const int b = b0 + r < l.B ? b0 + r : l.B - 1;
    slot[r] = slots ? slots[b] : b;
    if (slot[r] < 0 || slot[r] >= slots_in_state) slot[r] = -1;
  }
#pragma unroll
  for (int r = 0; r < kStreams; ++r) {
    const int b = b0 + r < l.B ? b0 + r : l.B - 1;
    h[r] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (slot[r] >= 0) h[r] = get(state + ((int64_t)slot[r] * l.D + d) * l.N + n);
    u[r] = *(l.u.at(0, b) + d), dt[r] = *(l.dt.at(0, b) + d), z[r] = l.z.data ? *(l.z.at(0, b) + d) : E(0.0f);
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const int at = g * l.N + (n + k < l.N ? n + k : 0);
      Bm[r][k] = *(l.Bm.at(0, b) + at), Cm[r][k] = *(l.Cm.at(0, b) + at);
    }
  }
#pragma unroll
  for (int r = 0; r < kStreams; ++r) {
    if (b0 + r >= l.B) break;
    const float x = (float)u[r], s = softplus<E>((float)dt[r] + bias), su = s * x, s2 = s * kLog2e;
    float4 v;
    v.x = fmaf(exp2_fast(s2 * A.x), h[r].x, su * (float)Bm[r][0]), v.y = fmaf(exp2_fast(s2 * A.y), h[r].y, su * (float)Bm[r][1]);
    v.z = fmaf(exp2_fast(s2 * A.z), h[r].z, su * (float)Bm[r][2]), v.w = fmaf(exp2_fast(s2 * A.w), h[r].w, su * (float)Bm[r][3]);
    float sum = any ? (float)Cm[r][0] * v.x : 0.0f;
    sum = n + 1 < l.N ? fmaf((float)Cm[r][1], v.y, sum) : sum;
    sum = n + 2 < l.N ? fmaf((float)Cm[r][2], v.z, sum) : sum;
    sum = n + 3 < l.N ? fmaf((float)Cm[r][3], v.w, sum) : sum;
#pragma unroll
    for (int k = 1; k < 1 << LANES; k <<= 1) sum += __shfl_xor(sum, k);
    if (slot[r] >= 0) {
      float* to = state + ((int64_t)slot[r] * l.D + d) * l.N + n;
      if (VECTOR) {
        if (any) *reinterpret_cast<float4*>(to) = v;
      } else {
        if (any) to[0] = v.x;
        if (n + 1 < l.N) to[1] = v.y;
        if (n + 2 < l.N) to[2] = v.z;
        if (n + 3 < l.N) to[3] = v.w;
      }
    }
    if (n == 0) {
      sum = fmaf(skip, x, sum);
      if (l.z.data) sum *= (float)z[r] * sigmoid<E>((float)z[r]);
      store(y.at(0, b0 + r) + d, slot[r] >= 0 ? sum : 0.0f);
    }
  }
}

}  // namespace

extern "C" size_t bppsa_ssm_scan_states_bytes(int T, int B, int D, int N) {
  if (!sizes_ok(T, B, D, N, 1)) return 0;
  return (size_t)bppsa_ceil_div(T, kKept) * B * D * padded_of(N) * sizeof(float);
}

extern "C" size_t bppsa_ssm_scan_workspace_bytes(int T, int B, int D, int N, int G) {
  return sizes_ok(T, B, D, N, G) ? Scratch(T, B, D, N, G).bytes : 0;
}

extern "C" bppsa_status bppsa_ssm_scan(const bppsa_ssm* layer, const bppsa_rows* y, float* h_last, void* states,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, layer->T, layer->B) || (h_last && h_last == layer->h0) || !states_ok(states)) return BPPSA_EINVAL;
  const Scratch at(layer->T, layer->B, layer->D, layer->N, layer->G);
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, at.bytes));
  const Spans spans = spans_of(layer->T, layer->B, layer->D, layer->N, layer->G, kWavesWanted, layer->lengths != nullptr);
  const hipStream_t s = (hipStream_t)stream;
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    const Layer<E> l = layer_of<E>(*layer);
    auto part = [&](size_t o) { return reinterpret_cast<float*>(static_cast<char*>(workspace) + o); };
    const Summary sum{part(at.ends), part(at.sums)};
    return by_states(l.N, [&](auto waves, auto held) {
      constexpr int W = waves.value, H = held.value;
      if (spans.count > 1)                  // nothing asks for the last span's summary
        scan_kernel<E, W, H, true, false><<<dim3(l.G * l.tiles * (spans.count - 1), l.B), W * 64, 0, s>>>(
            l, Rows<E>{}, nullptr, nullptr, sum, spans);
      const auto kernel = l.z.data ? scan_kernel<E, W, H, false, true> : scan_kernel<E, W, H, false, false>;
      kernel<<<dim3(l.G * l.tiles * spans.count, l.B), W * 64, 0, s>>>(l, rows_of<E>(*y), h_last,
                                                                        static_cast<float*>(states), sum, spans);
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
    const bool vector = l.N % kHeld == 0 && (((uintptr_t)state | (uintptr_t)l.A) & 15) == 0;
    auto run = [&](auto lanes, auto v) {
      constexpr int L = lanes.value;
      scan_step_kernel<E, L, v.value><<<dim3(bppsa_ceil_div(l.D, 256 >> L), bppsa_ceil_div(l.B, kStreams)), 256, 0,
                                        (hipStream_t)stream>>>(l, rows_of<E>(*y), state, slots_in_state, slots);
    };
    auto by_lanes = [&](auto v) {
      if (l.N <= 4) run(std::integral_constant<int, 0>{}, v);
      else if (l.N <= 8) run(std::integral_constant<int, 1>{}, v);
      else if (l.N <= 16) run(std::integral_constant<int, 2>{}, v);
      else if (l.N <= 32) run(std::integral_constant<int, 3>{}, v);
      else run(std::integral_constant<int, 4>{}, v);
    };
    if (vector) by_lanes(std::true_type{});
    else by_lanes(std::false_type{});
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
