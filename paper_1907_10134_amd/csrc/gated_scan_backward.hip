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

// The tiles run from the end, kKept steps each, joined as those of the forward pass are: a word says what a tile does to the
// gradient that comes in from behind.  A run's states are found again from the one kept before its tile and the shares of the
// runs in front of it, so a tile's inputs are read once.
//
// Bound by memory: T = 4096, B = 4, D = 4096 bf16 with a gate 257 us, 1.25 GB at 4.9 TB/s, the vector unit busy for 75 % of it.  Five values
// a step and channel stay in registers, so runs are of eight steps; fp32 without a gate leaves registers for three workgroups a
// unit (T = 1000, B = 16, D = 330: 33 us), the others for two; 10 to 70 scalars are spilled.
template <typename E, int V, bool GATE, bool JOINED>
__global__ void __launch_bounds__(kWaves * 64, sizeof(E) == 4 && !GATE ? 6 : 4)
gated_backward_kernel(const Layer<E> l, Rows<const E> dy, const float* __restrict__ dh_last, const float* __restrict__ states,
                      const Grads<E> o, int* tickets, uint64_t* words, int tiles, int each) {
  constexpr int R = kRunBack;
  // product of the decays, state from zero, gradient from zero; a lane's channels 64 apart, so that a wave's accesses lie side by side (T =
  // 4096, B = 4, D = 4096 bf16 without a gate, both passes: 321 us, 335 with them next to each other)
  __shared__ float4 runs[kWaves][64 * V];
  __shared__ float2 border[64 * V];                   // the state before the tile, the gradient behind it
  __shared__ float sums[3][kWaves][64 * V];
  __shared__ int2 taken;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int chain = blockIdx.x, tile = 0;
  if (JOINED) {
    if (threadIdx.x == 0) taken = take(tickets, l.columns * l.B, each, tiles);
    lds_barrier();
    chain = __builtin_amdgcn_readfirstlane(taken.x), tile = tiles - 1 - __builtin_amdgcn_readfirstlane(taken.y);
    if (chain < 0) return;
  }
  const int column = chain % l.columns, b = chain / l.columns;
  const Own<V> own(column, lane, l.D);
  const int d = own.d, len = clamp_length(l.lengths, b, l.T), t0 = tile * kKept, first = t0 + w * R;
  const int last_tile = (len + kKept - 1) / kKept - 1;
  // behind an end
  if (own.on)
    for (int t = first > len ? first : len; t < first + R && t < l.T; ++t) {
      const float zero[V] = {};
      store_some<E, V>(o.dx.at(t, b) + d, zero), store_some<E, V>(o.dr.at(t, b) + d, zero), store_some<E, V>(o.di.at(t, b) + d, zero);
      if (GATE) store_some<E, V>(o.dz.at(t, b) + d, zero);
    }
  if (len == 0 && tile == 0 && w == 0 && o.dh0 && own.on)
    for (int c = 0; c < V; ++c) o.dh0[(int64_t)b * l.D + d + c] = dh_last ? dh_last[(int64_t)b * l.D + d + c] : 0.0f;

  uint32_t x[R], go[R], z[R];
  float a[R][V], e[R][V], rho[R][V], iota[R][V], sum[3][V] = {};
  const int rows = len - first < R ? len - first : R;
  const uint32_t byte = (uint32_t)d * sizeof(E);
  Channel<E> channel[V];
  if (rows > 0) channels_of(l, d, channel);
  auto gather = [&](auto all) __attribute__((always_inline)) {
    constexpr bool WHOLE = all.value;
    uint32_t r[R], i[R];
    load_rows<WHOLE, R, V>(l.r, first, b, rows, byte, r), load_rows<WHOLE, R, V>(l.i, first, b, rows, byte, i), load_rows<WHOLE, R, V>(l.x, first, b, rows, byte, x);
    load_rows<WHOLE, R, V>(dy, first, b, rows, byte, go);
    if (GATE) load_rows<WHOLE, R, V>(l.z, first, b, rows, byte, z);
    float product[V], end[V], back[V];
#pragma unroll
    for (int c = 0; c < V; ++c) product[c] = 1.0f, end[c] = back[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      apart(j);
#pragma unroll
      for (int c = 0; c < V; ++c) {
        rho[j][c] = channel[c].rho(part<E>(r[j], c)), iota[j][c] = channel[c].iota(part<E>(i[j], c));
        a[j][c] = channel[c].a(rho[j][c]);
        e[j][c] = __builtin_amdgcn_sqrtf(channel[c].m2(a[j][c], rho[j][c])) * iota[j][c] * part<E>(x[j], c);
        float q = part<E>(go[j], c);
        if (GATE) q *= part<E>(z[j], c) * sigmoid<E>(part<E>(z[j], c));
        if (!WHOLE && j >= rows) a[j][c] = 1.0f, e[j][c] = q = 0.0f;
        product[c] *= a[j][c], end[c] = fmaf(a[j][c], end[c], e[j][c]), back[c] = fmaf(product[c], q, back[c]);
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) runs[w][c * 64 + lane] = make_float4(product[c], end[c], back[c], 0.0f);
  };
  if (rows == R) gather(std::true_type{});
  else if (rows > 0) gather(std::false_type{});
  else
#pragma unroll
    for (int c = 0; c < V; ++c) runs[w][c * 64 + lane] = make_float4(1.0f, 0.0f, 0.0f, 0.0f);
  lds_barrier();
  if (w < V && t0 < len) {                   // the tile's own share, a channel a lane
    const uint32_t at = w * 64 + lane;
    const int channel = d + w;
    const float kept = states[((int64_t)tile * l.B + b) * l.D + channel];      // asked for before the wait, by lanes without a channel too
    float p = 1.0f, s = 0.0f, in = 0.0f;
#pragma unroll
    for (int k = kWaves - 1; k >= 0; --k) {
      const float4 run = runs[k][at];
      p *= run.x, s = fmaf(run.x, s, run.z);
    }
    if (tile == last_tile && dh_last && own.on) in = dh_last[(int64_t)b * l.D + channel];
    if (JOINED) {
      const int64_t step = (int64_t)l.B * l.columns * 64 * V;
      uint64_t* const mine = words + tile * step + ((int64_t)b * l.columns + column) * 64 * V;
      if (tile < last_tile) leave(mine + at, word_of(p, s)), in = look_back(mine, at, -step, last_tile - tile);
      leave(mine + at, settled(through(word_of(p, s), in)));
    }
    border[at] = make_float2(kept, in);
  }
  lds_barrier();
  if (rows > 0 && own.on) {
    float h[V], g[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
      const float2 both = border[c * 64 + lane];
      h[c] = both.x, g[c] = both.y;
    }
    for (int k = 0; k < w; ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float4 run = runs[k][c * 64 + lane];
        h[c] = fmaf(run.x, h[c], run.y);
      }
    for (int k = kWaves - 1; k > w; --k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float4 run = runs[k][c * 64 + lane];
        g[c] = fmaf(run.x, g[c], run.z);
      }
    // the states before each step, in the place of what enters
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float before = h[c];
        h[c] = fmaf(a[j][c], h[c], e[j][c]);
        e[j][c] = before;
      }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      as_loaded(x[j]), as_loaded(go[j]);
      if (GATE) as_loaded(z[j]);
    }
    Run<E> to_x(o.dx, first, b), to_r(o.dr, first, b), to_i(o.di, first, b), to_z(GATE ? o.dz : o.dx, first, b);
    const int64_t last = rows - 1;
    to_x.move_by(last * to_x.step), to_r.move_by(last * to_r.step), to_i.move_by(last * to_i.step);
    if (GATE) to_z.move_by(last * to_z.step);
#pragma unroll
    for (int j = R - 1; j >= 0; --j) {
      apart(j + 1);
      float dx[V], dr[V], di[V], dz[V];
      if (j >= rows) continue;
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float of_x = part<E>(x[j], c), m2 = channel[c].m2(a[j][c], rho[j][c]), root = m2 > 0x1p-120f ? __builtin_amdgcn_rsqf(m2) : 0.0f, m = m2 * root;
        float q = part<E>(go[j], c);
        if (GATE) {
          const float of_z = part<E>(z[j], c), sg = sigmoid<E>(of_z), q_sg = q * sg;
          dz[c] = q_sg * h[c] * fmaf(of_z, 1.0f - sg, 1.0f);
          q = q_sg * of_z;
        }
        const float gh = q + g[c];
        g[c] = a[j][c] * gh;
        const float s = g[c] * rho[j][c] * fmaf(a[j][c] * iota[j][c] * of_x, root, -e[j][c]);
        dx[c] = gh * m * iota[j][c];
        di[c] = dx[c] * fmaf(-of_x, iota[j][c], of_x);
        dr[c] = channel[c].decay * fmaf(-rho[j][c], s, s);
        h[c] = e[j][c];
        sum[0][c] += s, sum[1][c] += dr[c], sum[2][c] += di[c];
      }
      to_x.store(byte, dx), to_r.store(byte, dr), to_i.store(byte, di);
      to_x.move_by(-to_x.step), to_r.move_by(-to_r.step), to_i.move_by(-to_i.step);
      if (GATE) to_z.store(byte, dz), to_z.move_by(-to_z.step);
    }
    if (o.dh0 && first == 0)
#pragma unroll
      for (int c = 0; c < V; ++c) o.dh0[(int64_t)b * l.D + d + c] = g[c];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int c = 0; c < V; ++c) sums[k][w][lane * V + c] = sum[k][c];
  lds_barrier();
  for (int at = threadIdx.x; at < 3 * 64 * V; at += kWaves * 64) {
    const int k = at / (64 * V), place = at % (64 * V), channel = channel_of<V>(column, place, l.D);
    float all = 0.0f;
#pragma unroll
    for (int n = 0; n < kWaves; ++n) all += sums[k][n][place];
    if (channel < l.D) o.parts[(((int64_t)tile * l.B + b) * 3 + k) * l.D + channel] = all;
  }
}

// The sums over parts, in order: sixteen waves a sixteenth each, then those.  In 64 bits, which cost nothing beside the loads.  Bound by
// the launch and two rounds of loads (256 parts of 4096 channels: 5 us).  A workgroup has all parts of 64 sums: few channels of many parts are
// left to few workgroups (4096 parts of 16 channels: 13 us, of a call of 181).
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

// The words of the widest workgroups, or of one channel a lane, whichever are more, then the parts.
extern "C" size_t bppsa_gated_scan_backward_workspace_bytes(int T, int B, int D) {
  if (!sizes_ok(T, B, D)) return 0;
  const int tiles = bppsa_ceil_div(T, kKept);
  return words_bytes(tiles, B, bppsa_ceil_div(D, 128), 2) + bppsa_align_up((size_t)tiles * B * 3 * D * sizeof(float), 256);
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
  const int tiles = bppsa_ceil_div(layer->T, kKept);
  char* const base = static_cast<char*>(workspace);
  float* const parts = reinterpret_cast<float*>(base + words_bytes(tiles, layer->B, bppsa_ceil_div(layer->D, 128), 2));
  BPPSA_TRY(by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    return by_width<E>(layer->D, [&](auto width) {
      constexpr int V = width.value;
      const Layer<E> l = layer_of<E>(*layer, 64 * V);
      const Grads<E> o{rows_of<E>(grads->dx), rows_of<E>(grads->dr), rows_of<E>(grads->di), rows_of<E>(grads->dz), parts, grads->dh0};
      const int total = tiles * l.B * l.columns;
      const auto run = [&](auto gate, auto joined) {
        constexpr bool GATE = gate.value, JOINED = joined.value;
        gated_backward_kernel<E, V, GATE, JOINED><<<total, kWaves * 64, 0, s>>>(
            l, rows_of<const E>(*dy), dh_last, static_cast<const float*>(states), o, reinterpret_cast<int*>(base),
            reinterpret_cast<uint64_t*>(base + kTicketBytes), tiles, chains_of_queue(l.columns * l.B));
      };
      constexpr std::true_type yes;
      constexpr std::false_type no;
      if (tiles > 1) {
        empty_words(workspace, words_bytes(tiles, l.B, l.columns, V), s);
        l.z.data ? run(yes, yes) : run(no, yes);
      } else {
        l.z.data ? run(yes, no) : run(no, no);
      }
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  }));
  gated_join_kernel<<<bppsa_ceil_div(3 * layer->D, 64), kJoining * 64, 0, s>>>(
      parts, layer->D, (int64_t)tiles * layer->B, Joined{grads->ddecay, grads->dr_bias, grads->di_bias});
  BPPSA_CHECK_LAUNCH();
  return BPPSA_OK;
}
