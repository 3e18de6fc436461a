// The selective scan's gradients.
//
// With q = dy silu(z) and g[t] = dL/dh[t] = q C[t] + a[t+1] g[t+1], the walk from the end carries w[t] = a[t] g[t], and per
// state
//     dB[t] += g s u, dC[t] += h q (sums over the channels), dA += w h[t-1] s (over time and samples),
//     du = s sum_n g B + skip q,  ddt = (u sum_n g B + sum_n w h[t-1] A) sigmoid(raw),
//     dz = dy (sum_n C h + skip u) silu'(z).
// The forward call kept the states every kKept steps, so h and a of a pass of so many steps are found again in registers.
#include "ssm_scan_parts.h"

namespace {

using namespace ssm;

template <typename E>
struct Grads {
  Rows<E> du, ddt, dz;
  float *bc, *dA, *dskip, *ddt_bias, *dh0;     // all but dh0 parts of sums, see Scratch
};

constexpr int PASS = kKept;
// Passes after which the sums over time go to their totals and start again: 512 steps in a row, then the totals, keep a span of any
// length as exact as fp32 sums of that many terms.
constexpr int kRun = 64;

// Sums over the wave's 64 lanes of the 2 H products (dB and dC of H states) of each of 8 steps.  A level halves the registers
// and doubles the lanes that are summed: two registers exchange halves and are added, one slot a register and level, 126
// in all at H = 4, where 64 full sums would take 384.  At the end a lane has one product, at H = 2 the same one as its
// neighbour: the bits of its number say which, from the highest on dB or dC, state, step (lowest bit first each).
// The levels of one step run as soon as its products are there.
__device__ __forceinline__ float swap32_add(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float swap16_add(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Lanes 0-7 of a row of 16: a summed with lanes 8-15; lanes 8-15: b.  (A DPP read of a register needs two wait states behind
// the write of it, which the compiler does not count inside asm.)
__device__ __forceinline__ float half_row_add(float a, float b) {
  float t;
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %1, %1 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
      "v_add_f32_dpp %0, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xc"
      : "=&v"(t) : "v"(a), "v"(b));
  return t;
}
// Even fours of lanes: a summed with the next four; odd ones: b with the four before.
__device__ __forceinline__ float four_add(float a, float b) {
  float t;
  asm("s_nop 1\n\t"
      "v_add_f32_dpp %0, %1, %1 row_shl:4 row_mask:0xf bank_mask:0x5\n\t"
      "v_add_f32_dpp %0, %2, %2 row_shr:4 row_mask:0xf bank_mask:0xa"
      : "=&v"(t) : "v"(a), "v"(b));
  return t;
}
template <int QUAD_PERM>
__device__ __forceinline__ float in_four_add(float a, float b, bool second) {
  const float keep = second ? b : a, give = second ? a : b;
  return keep + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(give), QUAD_PERM, 0xf, 0xf, true));
}
struct Product {
  int of_C, state, step;
  bool first;                      // of the lanes that have it
};
__device__ __forceinline__ Product product_of_lane(int lane, int held) {
  auto bit = [&](int k) { return lane >> k & 1; };
  if (held == 4) return Product{bit(5), bit(4) | bit(3) << 1, bit(2) | bit(1) << 1 | bit(0) << 2, true};
  return Product{bit(5), bit(4), bit(3) | bit(2) << 1 | bit(1) << 2, !bit(0)};
}
// The levels over the steps.
template <int H>
__device__ __forceinline__ float over_steps(const float (&x)[PASS], int lane) {
  const bool odd = lane & 1, high = lane & 2;
  if constexpr (H == 4) {
    const float low = in_four_add<0x4E>(four_add(x[0], x[1]), four_add(x[2], x[3]), high);
    const float top = in_four_add<0x4E>(four_add(x[4], x[5]), four_add(x[6], x[7]), high);
    return in_four_add<0xB1>(low, top, odd);
  } else {
    const float low = four_add(half_row_add(x[0], x[1]), half_row_add(x[2], x[3]));
    const float top = four_add(half_row_add(x[4], x[5]), half_row_add(x[6], x[7]));
    const float v = in_four_add<0x4E>(low, top, high);
    return in_four_add<0xB1>(v, v, odd);
  }
}

// Where a span's walk from its end with nothing carried in arrives, and the sum of its steps; the cut and the passes are
// those of the main kernel below.
template <typename E, int WAVES, int H, bool GATE>
__global__ void __launch_bounds__(WAVES * 64, WAVES <= 12 ? 6 : 4)
scan_backward_summary_kernel(const Layer<E> l, Rows<const E> dy, const Summary sum, const Spans spans) {
  constexpr int ROWS = (PASS + WAVES - 1) / WAVES;
  constexpr bool ALL = PASS % WAVES == 0;
  __shared__ float2 step_in[2][PASS][kTile];             // (s, q)
  __shared__ alignas(16) float coef[2][PASS][WAVES][2 * H];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = blockIdx.x % (l.G * l.tiles), span = blockIdx.x / (l.G * l.tiles) + 1, g = tile / l.tiles, b = blockIdx.y;
  const int in = tile % l.tiles * kTile + lane;
  const bool on = in < l.wide;
  const int d = g * l.wide + (on ? in : 0);
  const int len = clamp_length(l.lengths, b, l.T), t0 = span * spans.steps;
  const int t1 = t0 + spans.steps < l.T ? t0 + spans.steps : l.T, stop = t1 < len ? t1 : len;
  float A2[H], carry[H], total = 0.0f;
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int n = w * H + i;
    A2[i] = n < l.N ? l.A[(int64_t)d * l.N + n] * kLog2e : 0.0f;
    carry[i] = 0.0f;
  }
  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f;
  const uint32_t byte = (uint32_t)d * sizeof(E);
  const int mine = w * ROWS, passes = stop > t0 ? (stop - t0 + PASS - 1) / PASS : 0, last = t0 + (passes - 1) * PASS;
  Walk<const E> at_dt(l.dt, last + mine, b, byte, -PASS), at_dy(dy, last + mine, b, byte, -PASS), at_z(l.z, last + mine, b, byte, -PASS);
  Coef<E, H> at_coef(l, WAVES, threadIdx.x, last, b, g);
  struct Fetched {                                       // two passes ahead, as in the forward kernel
    uint32_t dt[ROWS], go[ROWS], z[ROWS], coef;
  } raw0, raw1;
  auto fetch = [&](int first, Fetched& x) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      uint32_t a = 0, b = 0, c = 0;
      if ((ALL || mine + r < PASS) && first >= t0 && first + mine + r < stop) {
        a = at_dt.bits(r), b = at_dy.bits(r);
        if (GATE) c = at_z.bits(r);
      }
      x.dt[r] = a, x.go[r] = b, x.z[r] = c;
    }
    x.coef = at_coef.fetch(first >= t0 ? stop - first : 0);
    at_dt.move(), at_dy.move(), at_coef.move(-1);
    if (GATE) at_z.move();
  };
  auto prepare = [&](int first, int buffer, const Fetched& x) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (!ALL && mine + r >= PASS) break;
      float s = softplus<E>(value<E>(x.dt[r]) + bias), q = value<E>(x.go[r]);
      s = first >= t0 && first + mine + r < stop ? s : 0.0f;      // q is zero there
      if (GATE) q *= value<E>(x.z[r]) * sigmoid<E>(value<E>(x.z[r]));
      total += s;
      step_in[buffer][mine + r][lane] = make_float2(s, q);
    }
    if (64 * H >= 256 || threadIdx.x < WAVES * PASS * 2 * H) (&coef[buffer][0][0][0])[threadIdx.x] = value<E>(x.coef);
  };
  auto pass = [&](int k, auto parity) __attribute__((always_inline)) {                  // the k-th from the end
    constexpr int buffer = parity.value;
    Fetched &here = pick<buffer>(raw0, raw1), &there = pick<buffer>(raw1, raw0);
    const int first = last - k * PASS;
    fetch(first - 2 * PASS, here);               // nothing, in front of the span
#pragma unroll
    for (int i = PASS - 1; i >= 0; --i) {
      float Cm[H];
      two_by_two(i + 1);
      const float2 in_ = step_in[buffer][i][lane];
      get(coef[buffer][i][w] + H, Cm);
#pragma unroll
      for (int j = 0; j < H; ++j) carry[j] = exp2_fast(in_.x * A2[j]) * fmaf(in_.y, Cm[j], carry[j]);
    }
    now(carry);
    prepare(first - PASS, buffer ^ 1, there);    // a pass that no one walks, in front of it
    __syncthreads();
  };
  if (passes) {
    fetch(last, raw0);
    fetch(last - PASS, raw1);
    prepare(last, 0, raw0);
  }
  __syncthreads();
  constexpr std::integral_constant<int, 0> even;
  constexpr std::integral_constant<int, 1> odd;
  int k = 0;
  for (; k + 1 < passes; k += 2) pass(k, even), pass(k + 1, odd);
  if (k < passes) pass(k, even);
  static_assert(sizeof(step_in) >= WAVES * kTile * sizeof(float));
  float* totals = &step_in[0][0][0].x;
  totals[w * kTile + lane] = total;
  __syncthreads();
  if (!on) return;
  put(sum.ends + state_at(H, span, l.B, b, WAVES, w, l.D, d), carry);
  if (w == 0) {
    for (int k = 1; k < WAVES; ++k) total += totals[k * kTile + lane];
    sum.sums[((int64_t)span * l.B + b) * l.D + d] = total;
  }
}

// The cut of the work is the forward kernel's; the passes run from the span's end.  In a pass every wave first finds a and h
// of its states, then walks back; the sums over the states go through LDS (s1 = sum g B, s2 = sum w h A, and with a gate
// sum C h), those over the channels through registers.
// Bound by issue: a step of four states takes 20 slots to find a and h again, 36 for the walk back and 16 for the sums over
// channels, a step and channel some 130 beside them.  T = 4096, B = 4, D = 4096, N = 16, bf16, gated: 874 us with the vector
// unit 88 % busy (and 218 us, 87 %, for the summaries); its 1.6 GB would take 0.31 ms.
template <typename E, int WAVES, int H, bool GATE>
__global__ void __launch_bounds__(WAVES * 64, WAVES <= 12 ? 3 : 4)
scan_backward_kernel(const Layer<E> l, Rows<const E> dy, const float* __restrict__ states, const Summary sum, const Spans spans,
                     const Grads<E> o) {
  // sixteen waves have 128 registers each, not enough for a and h of eight steps: in two halves, the first four steps walked twice
  constexpr int ROWS = (PASS + WAVES - 1) / WAVES, SUMS = GATE ? 3 : 2, HALVES = WAVES > 12 ? 2 : 1;
  constexpr bool ALL = PASS % WAVES == 0;
  __shared__ float2 step_in[2][PASS][kTile];             // (s, s u)
  __shared__ float step_q[2][PASS][kTile];
  __shared__ alignas(16) float coef[2][PASS][WAVES][2 * H];
  __shared__ float share[SUMS][WAVES][PASS][kTile];
  __shared__ float2 totals[WAVES][kTile];                // of dskip and ddt_bias, every wave those of its rows
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = blockIdx.x % (l.G * l.tiles), span = blockIdx.x / (l.G * l.tiles), g = tile / l.tiles, b = blockIdx.y;
  const int in = tile % l.tiles * kTile + lane;
  const bool on = in < l.wide;                           // lanes without a channel count in the sums with s u = q = 0
  const int d = g * l.wide + (on ? in : 0);
  const int len = clamp_length(l.lengths, b, l.T), t0 = span * spans.steps;
  const int t1 = t0 + spans.steps < l.T ? t0 + spans.steps : l.T, stop = t1 < len ? t1 : len;

  if (on)
    for (int t = (t0 > len ? t0 : len) + w; t < t1; t += WAVES) {
      store(o.du.at(t, b) + d, 0.0f), store(o.ddt.at(t, b) + d, 0.0f);
      if (GATE) store(o.dz.at(t, b) + d, 0.0f);
    }

  float A[H], A2[H], carry[H], dA[H];
#pragma unroll
  for (int i = 0; i < H; ++i) {
    const int n = w * H + i;
    A[i] = n < l.N ? l.A[(int64_t)d * l.N + n] : 0.0f;
    A2[i] = A[i] * kLog2e;
    carry[i] = dA[i] = 0.0f;
  }
  if (stop > t0) join_spans(sum, spans.count - 1, -1, spans.count - 1 - span, l.B, b, WAVES, w, l.D, d, A2, carry);

  const float bias = l.dt_bias ? l.dt_bias[d] : 0.0f, skip = l.skip ? l.skip[d] : 0.0f;
  const uint32_t byte = (uint32_t)d * sizeof(E);
  float dskip = 0.0f, dbias = 0.0f;
  totals[w][lane] = make_float2(0.0f, 0.0f);
  const int mine = w * ROWS, passes = stop > t0 ? (stop - t0 + PASS - 1) / PASS : 0, last = t0 + (passes - 1) * PASS;
  Walk<const E> at_u(l.u, last + mine, b, byte, -PASS), at_dt(l.dt, last + mine, b, byte, -PASS), at_dy(dy, last + mine, b, byte, -PASS), at_z(l.z, last + mine, b, byte, -PASS);
  Walk<E> at_du(o.du, last + mine, b, byte, -PASS), at_ddt(o.ddt, last + mine, b, byte, -PASS), at_dz(o.dz, last + mine, b, byte, -PASS);
  const float* at_states = states + state_at(H, last / kKept, l.B, b, WAVES, w, l.D, d);
  Coef<E, H> at_coef(l, WAVES, threadIdx.x, last, b, g);
  uint32_t u[ROWS], dt[ROWS], go[ROWS], z[ROWS], raw_coef;
  struct Row {                                           // of a step: what its outputs are made of
    float s, u, q, slope, gate;                          // slope: sigmoid(raw), gate: dy silu'(z)
  } row[ROWS], was[ROWS];
  float kept[H];
  auto fetch = [&](int first) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      uint32_t a = 0, b = 0, c = 0, e = 0;
      if ((ALL || mine + r < PASS) && first + mine + r < stop) {
        a = at_u.bits(r), b = at_dt.bits(r), c = at_dy.bits(r);
        if (GATE) e = at_z.bits(r);
      }
      u[r] = a, dt[r] = b, go[r] = c, z[r] = e;
    }
    raw_coef = at_coef.fetch(stop - first);
    get(at_states, kept);
    at_u.move(), at_dt.move(), at_dy.move(), at_coef.move(-1);
    if (GATE) at_z.move();
    at_states -= (int64_t)l.B * WAVES * l.D * H;
  };
  auto prepare = [&](int first, int buffer) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (!ALL && mine + r >= PASS) break;
      const bool real = on && first + mine + r < stop;
      const float raw = value<E>(dt[r]) + bias;
      Row v{softplus<E>(raw), value<E>(u[r]), value<E>(go[r]), sigmoid<E>(raw), 0.0f};
      if (GATE) {
        const float x = value<E>(z[r]), sg = sigmoid<E>(x);
        v.gate = v.q * sg * fmaf(x, 1.0f - sg, 1.0f);
        v.q *= x * sg;                                   // silu(z) first, as the forward pass has it
      }
      if (!real) v.s = v.u = v.q = 0.0f;
      row[r] = v;
      step_in[buffer][mine + r][lane] = make_float2(v.s, v.s * v.u);
      step_q[buffer][mine + r][lane] = v.q;
    }
    if (64 * H >= 256 || threadIdx.x < WAVES * PASS * 2 * H) (&coef[buffer][0][0][0])[threadIdx.x] = value<E>(raw_coef);
  };
  auto finish = [&](int first) __attribute__((always_inline)) {
    float du[ROWS], ddt[ROWS], dz[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int i = (ALL || mine + r < PASS) ? mine + r : 0;
      const Row v = was[r];
      float s1 = 0.0f, s2 = 0.0f, plain = skip * v.u;
#pragma unroll
      for (int k = 0; k < WAVES; ++k) {
        s1 += share[0][k][i][lane], s2 += share[1][k][i][lane];
        if (GATE) plain += share[SUMS - 1][k][i][lane];
      }
      du[r] = fmaf(v.s, s1, skip * v.q);
      ddt[r] = fmaf(v.u, s1, s2) * v.slope;
      dz[r] = v.gate * plain;
      if ((ALL || mine + r < PASS) && first + mine + r < stop) dbias += ddt[r], dskip = fmaf(v.q, v.u, dskip);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if ((ALL || mine + r < PASS) && first + mine + r < stop && on) {
        at_du.put(r, du[r]), at_ddt.put(r, ddt[r]);
        if (GATE) at_dz.put(r, dz[r]);
      }
    at_du.move(), at_ddt.move();
    if (GATE) at_dz.move();
  };

  // adds the sums so far to their totals, of dA in memory that no one else has (in LDS they would cost N = 8 a workgroup a
  // compute unit: 726 us instead of 654 at T = 4096, B = 4, D = 4096)
  auto total = [&](bool first) __attribute__((always_inline)) {
    if (on) {
      float before[H] = {}, *at_dA = o.dA + state_at(H, span, l.B, b, WAVES, w, l.D, d);
      if (!first) get(at_dA, before);
#pragma unroll
      for (int i = 0; i < H; ++i) before[i] += dA[i], dA[i] = 0.0f;
      put(at_dA, before);
    }
    const float2 before = totals[w][lane];
    totals[w][lane] = make_float2(before.x + dskip, before.y + dbias);
    dskip = dbias = 0.0f;
  };

  float* at_bc = o.bc + (((((int64_t)(tile % l.tiles) * l.B + b) * l.G + g) * ((l.T + PASS - 1) / PASS) + last / PASS) * WAVES + w) * 64;
  if (passes) {
    fetch(last);
    prepare(last, (passes - 1) & 1);
  }
  __syncthreads();
  for (int p = passes - 1; p >= 0; --p) {
    const int first = t0 + p * PASS, buffer = p & 1;
    if (p + 1 < passes) finish(first + PASS);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) was[r] = row[r];
    float start[H], step_sum[PASS];
#pragma unroll
    for (int k = 0; k < H; ++k) start[k] = kept[k];
    if (p) fetch(first - PASS);
#pragma unroll
    for (int half = HALVES - 1; half >= 0; --half) {
      constexpr int STEPS = PASS / HALVES;
      float a[STEPS][H], h[STEPS + 1][H];
      auto step = [&](int i, float (&decay)[H], const float (&before)[H], float (&after)[H]) __attribute__((always_inline)) {
        float Bm[H];
        two_by_two(i);
        const float2 in_ = step_in[buffer][i][lane];
        get(coef[buffer][i][w], Bm);
#pragma unroll
        for (int k = 0; k < H; ++k) {
          decay[k] = exp2_fast(in_.x * A2[k]);
          after[k] = fmaf(decay[k], before[k], in_.y * Bm[k]);
        }
      };
#pragma unroll
      for (int k = 0; k < H; ++k) h[0][k] = start[k];
      if (half)
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          float decay[H];
          step(i, decay, h[0], h[0]);
        }
#pragma unroll
      for (int i = 0; i < STEPS; ++i) step(half * STEPS + i, a[i], h[i], h[i + 1]);
      // the last pass's shares have been read: a second barrier a pass instead of a second set of them, whose LDS would let
      // eight waves on a compute unit instead of twelve (1105 us against 925 at T = 4096, B = 4, D = 4096)
      if (half == HALVES - 1) __syncthreads();
#pragma unroll
      for (int j = STEPS - 1; j >= 0; --j) {
        const int i = half * STEPS + j;
        float Bm[H], Cm[H], s1 = 0.0f, s2 = 0.0f, plain = 0.0f, pair[H];
        two_by_two(i + 1);
        const float2 in_ = step_in[buffer][i][lane];
        get(coef[buffer][i][w], Bm), get(coef[buffer][i][w] + H, Cm);
        const float q = step_q[buffer][i][lane];
#pragma unroll
        for (int k = 0; k < H; ++k) {
          const float gh = fmaf(q, Cm[k], carry[k]);
          carry[k] = a[j][k] * gh;
          const float through = carry[k] * h[j][k];
          s1 = k ? fmaf(gh, Bm[k], s1) : gh * Bm[k];
          s2 = k ? fmaf(through, A[k], s2) : through * A[k];
          dA[k] = fmaf(through, in_.x, dA[k]);
          if (GATE) plain = k ? fmaf(Cm[k], h[j + 1][k], plain) : Cm[k] * h[j + 1][k];
          pair[k] = swap32_add(gh * in_.y, h[j + 1][k] * q);
        }
        if constexpr (H == 4) step_sum[i] = half_row_add(swap16_add(pair[0], pair[1]), swap16_add(pair[2], pair[3]));
        else step_sum[i] = swap16_add(pair[0], pair[1]);
        share[0][w][i][lane] = s1, share[1][w][i][lane] = s2;
        if (GATE) share[SUMS - 1][w][i][lane] = plain;
      }
    }
    at_bc[lane] = over_steps<H>(step_sum, lane);
    at_bc -= WAVES * 64;
    if (p) prepare(first - PASS, buffer ^ 1);
    // here: beside finish() the kernels of sixteen waves would spill 66 values, not 13 (T = 2048, B = 4, D = 2048, N = 64: 1034 us,
    // 1663 without this branch and with 46)
    if (p && p % kRun == 0) total(p == (passes - 1) / kRun * kRun);
    __syncthreads();
  }
  if (passes) finish(t0);
  total(passes <= kRun);
  __syncthreads();
  if (!on) return;
  if (w == 0) {
    float2 sum = totals[0][lane];
    for (int k = 1; k < WAVES; ++k) sum.x += totals[k][lane].x, sum.y += totals[k][lane].y;
    const int64_t part = (int64_t)span * l.B + b;
    o.dskip[part * l.D + d] = sum.x, o.ddt_bias[part * l.D + d] = sum.y;
  }
  if (o.dh0 && span == 0)
#pragma unroll
    for (int i = 0; i < H; ++i)
      if (w * H + i < l.N) o.dh0[((int64_t)b * l.D + d) * l.N + w * H + i] = carry[i];
}

// The sums over parts.  The first workgroups have dB and dC, the tiles' parts in the tiles' order, a thread the place of a lane
// of the main kernel; the others dA, dskip and ddt_bias, the parts of the samples and spans, in order: four waves a
// quarter each, then the quarters.
struct Joined {
  void *dBm, *dCm;
  float *dA, *dskip, *ddt_bias;
  int64_t places;                              // of dB and dC: the parts of one tile
  int first_groups, waves, held, parts;        // workgroups for dB and dC; waves of the main kernel and their states; samples times spans
};
template <typename E>
__global__ void __launch_bounds__(256)
join_kernel(const Layer<E> l, const Grads<E> o, const Joined to) {
  if ((int)blockIdx.x < to.first_groups) {
    const int passes = (l.T + PASS - 1) / PASS;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < to.places; i += (int64_t)to.first_groups * 256) {
      const Product product = product_of_lane((int)(i & 63), to.held);
      const int w = (int)(i / 64 % to.waves), t = (int)(i / 64 / to.waves % passes) * PASS + product.step;
      const int64_t bg = i / 64 / to.waves / passes;
      const int g = (int)(bg % l.G), b = (int)(bg / l.G), n = w * to.held + product.state;
      if (t >= l.T || n >= l.N || !product.first) continue;
      float sum = 0.0f;
      if (t < clamp_length(l.lengths, b, l.T)) {
#pragma unroll 8
        for (int k = 0; k < l.tiles; ++k) sum += o.bc[k * to.places + i];
      }
      store(static_cast<E*>(product.of_C ? to.dCm : to.dBm) + (((int64_t)t * l.B + b) * l.G + g) * l.N + n, sum);
    }
    return;
  }
  __shared__ float quarter[4][64];
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, of_dA = to.waves * to.held * l.D;
  const int i = ((int)blockIdx.x - to.first_groups) * 64 + lane, all = of_dA + 2 * l.D;
  const float* from = i < of_dA ? o.dA + i : i < of_dA + l.D ? o.dskip + (i - of_dA) : o.ddt_bias + (i - of_dA - l.D);
  const int64_t step = i < of_dA ? of_dA : l.D;
  const int each = (to.parts + 3) / 4, last = (q + 1) * each < to.parts ? (q + 1) * each : to.parts;
  float sum = 0.0f;
  if (i < all)
#pragma unroll 8
    for (int k = q * each; k < last; ++k) sum += from[k * step];
  quarter[q][lane] = sum;
  __syncthreads();
  if (q || i >= all) return;
  sum = (quarter[0][lane] + quarter[1][lane]) + (quarter[2][lane] + quarter[3][lane]);
  if (i < of_dA) {
    const int w = i / (to.held * l.D), d = i / to.held % l.D, n = w * to.held + i % to.held;
    if (n < l.N) to.dA[(int64_t)d * l.N + n] = sum;
  } else if (i < of_dA + l.D) {
    if (to.dskip) to.dskip[i - of_dA] = sum;
  } else if (to.ddt_bias) {
    to.ddt_bias[i - of_dA - l.D] = sum;
  }
}

// bc: parts of dB and dC [tile of the group][b][g][pass][w][64 lanes]; dA, dskip, ddt_bias: one part a span and sample.
// Three waves fit a SIMD.  Where that is twelve spans and more, so many at a time do, each with few spans to join (T = 4096, B
// = 16, D = 64: 122 us, 146 with eight waves a SIMD; T = 2000, B = 4, D = 400: 95 and 107); with fewer, rounds of shorter
// spans (T = 4096, B = 4, D = 4096 with summaries: 1217 us in three spans, 1160 in eight).
int waves_wanted(int D, int N, int G, int B) {
  const int64_t have = (int64_t)G * bppsa_ceil_div(D / G, kTile) * B * waves_of(N);
  return bppsa_compute_units() * 4 * 3 / have >= 12 ? 3 : 8;
}
struct Scratch {
  size_t ends, sums, bc, dA, dskip, ddt_bias, bytes;
  int64_t bc_floats;                           // of one tile
  Scratch(int T, int B, int D, int N, int G) {
    const int most = most_spans(T, B, D, N, G, waves_wanted(D, N, G, B));
    const int64_t waves = waves_of(N), tiles = bppsa_ceil_div(D / G, kTile), parts = (int64_t)most * B * D;
    bc_floats = (int64_t)B * G * ((T + PASS - 1) / PASS) * waves * 64;
    Arena take;
    ends = take(most > 1 ? parts * padded_of(N) : 0), sums = take(most > 1 ? parts : 0);
    bc = take(tiles * bc_floats);
    dA = take(parts * padded_of(N)), dskip = take(parts), ddt_bias = take(parts);
    bytes = take.at;
  }
};

}  // namespace

extern "C" size_t bppsa_ssm_scan_backward_workspace_bytes(int T, int B, int D, int N, int G) {
  return sizes_ok(T, B, D, N, G) ? Scratch(T, B, D, N, G).bytes : 0;
}

extern "C" bppsa_status bppsa_ssm_scan_backward(const bppsa_ssm* layer, const bppsa_rows* dy, const void* states,
                                                const bppsa_ssm_grads* grads, void* workspace, size_t workspace_bytes,
                                                void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!dy || !dy->data || !states || !states_ok(states) || !grads || !grads->dBm || !grads->dCm || !grads->dA) return BPPSA_EINVAL;
  if (!writable(grads->du, layer->T, layer->B) || !writable(grads->ddt, layer->T, layer->B)) return BPPSA_EINVAL;
  if (!layer->z.data != !grads->dz.data || (layer->z.data && !writable(grads->dz, layer->T, layer->B))) return BPPSA_EINVAL;
  const Scratch at(layer->T, layer->B, layer->D, layer->N, layer->G);
  // the joining launch: more places of dB and dC than 2^28 are taken in turns, the parameters' sums are not
  const int64_t first = std::min<int64_t>((at.bc_floats + 255) / 256, 1 << 20);
  const int64_t groups = first + ((padded_of(layer->N) + 2) * (int64_t)layer->D + 63) / 64;
  if (groups >= 1 << 24) return BPPSA_EOVERFLOW;
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, at.bytes));
  const Spans spans = spans_of(layer->T, layer->B, layer->D, layer->N, layer->G,
                               waves_wanted(layer->D, layer->N, layer->G, layer->B), layer->lengths != nullptr);
  const hipStream_t s = (hipStream_t)stream;
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    const Layer<E> l = layer_of<E>(*layer);
    const int waves = waves_of(l.N);
    auto part = [&](size_t o) { return reinterpret_cast<float*>(static_cast<char*>(workspace) + o); };
    const Grads<E> o{rows_of<E>(grads->du), rows_of<E>(grads->ddt), rows_of<E>(grads->dz), part(at.bc), part(at.dA),
                     part(at.dskip), part(at.ddt_bias), grads->dh0};
    const Summary sum{part(at.ends), part(at.sums)};
    const Rows<const E> out = rows_of<const E>(*dy);
    auto walk = [&](auto waves_, auto held, auto gate) {
      constexpr int W = waves_.value, H = held.value;
      constexpr bool GATE = gate.value;
      if (spans.count > 1)
        scan_backward_summary_kernel<E, W, H, GATE><<<dim3(l.G * l.tiles * (spans.count - 1), l.B), W * 64, 0, s>>>(
            l, out, sum, spans);
      scan_backward_kernel<E, W, H, GATE><<<dim3(l.G * l.tiles * spans.count, l.B), W * 64, 0, s>>>(
          l, out, static_cast<const float*>(states), sum, spans, o);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    };
    BPPSA_TRY(by_states(l.N, [&](auto w, auto h) { return l.z.data ? walk(w, h, std::true_type{}) : walk(w, h, std::false_type{}); }));
    const Joined to{grads->dBm, grads->dCm, grads->dA, grads->dskip, grads->ddt_bias, at.bc_floats, (int)first, waves, held_of(l.N),
                    spans.count * l.B};
    join_kernel<E><<<(unsigned)groups, 256, 0, s>>>(l, o, to);
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
