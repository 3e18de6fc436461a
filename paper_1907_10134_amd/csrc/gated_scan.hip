// The gated recurrence, forward: over sequences, and the step of single tokens.
#include "gated_parts.h"

namespace {

using namespace gated;

// A workgroup takes a tile of 8 R steps of 64 V channels.  Each wave has a run of the steps in registers: it turns them into decays
// and what enters, finds what its run does to a state, and when the state before it is known walks them again.  The gate is asked for
// while the tile waits for that state.
//
// Bound by memory (calls with the words' emptying, gated): T = 4096, B = 4, D = 4096 bf16 132 us, 5.1 TB/s; T = 30000, B = 1, D = 2048 130 us;
// T = 4096, B = 4, D = 2048 fp32 105 us without a gate, 5.1 TB/s; less where tiles are few: T = 1000, B = 16, D = 641 fp16 28.7 us,
// 768 workgroups where 512 run at once.  Two workgroups a unit is what 16-bit runs of two channels have registers for, fp32 ones of one channel
// leave three.  Runs of eight steps, in the same session: 147, 162, 106 and 28.8 us, and with registers for a third workgroup 135, 149, 106 and
// 27.2: a twentieth less where tiles are few, a seventh more where they are many.  No vector register is spilled; scalars are, 2 to
// 93 of them, each a write and a read of a lane.
template <typename E, int V, int R, bool GATE, bool JOINED>
__global__ void __launch_bounds__(kWaves * 64, sizeof(E) == 4 ? 6 : 4)
gated_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states, int* tickets, uint64_t* words, int tiles, int each) {
  __shared__ float2 runs[kWaves][64 * V];
  __shared__ float before[64 * V];
  __shared__ int2 taken;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int chain = blockIdx.x, tile = 0;
  if (JOINED) {
    if (threadIdx.x == 0) taken = take(tickets, l.columns * l.B, each, tiles);
    lds_barrier();
    chain = __builtin_amdgcn_readfirstlane(taken.x), tile = __builtin_amdgcn_readfirstlane(taken.y);
    if (chain < 0) return;
  }
  const int column = chain % l.columns, b = chain / l.columns;
  const Own<V> own(column, lane, l.D);
  const int d = own.d, len = clamp_length(l.lengths, b, l.T), t0 = tile * kWaves * R, first = t0 + w * R;
  // behind an end
  if (own.on)
    for (int t = first > len ? first : len; t < first + R && t < l.T; ++t) {
      const float zero[V] = {};
      store_some<E, V>(y.at(t, b) + d, zero);
    }
  if (len == 0 && tile == 0 && w == 0 && h_last && own.on)
    for (int c = 0; c < V; ++c) h_last[(int64_t)b * l.D + d + c] = l.h0 ? l.h0[(int64_t)b * l.D + d + c] : 0.0f;

  float a[R][V], e[R][V];
  const int rows = len - first < R ? len - first : R;
  const uint32_t byte = (uint32_t)d * sizeof(E);
  // a run with an end in it is another copy of the code: with its conditions in this one there are too few scalar registers
  auto gather = [&](auto all) __attribute__((always_inline)) {
    constexpr bool WHOLE = all.value;
    Channel<E> channel[V];
    channels_of(l, d, channel);
    uint32_t x[R], r[R], i[R];
    load_rows<WHOLE, R, V>(l.r, first, b, rows, byte, r), load_rows<WHOLE, R, V>(l.i, first, b, rows, byte, i), load_rows<WHOLE, R, V>(l.x, first, b, rows, byte, x);
    float product[V], end[V];
#pragma unroll
    for (int c = 0; c < V; ++c) product[c] = 1.0f, end[c] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      apart(j);
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float rho = channel[c].rho(part<E>(r[j], c)), iota = channel[c].iota(part<E>(i[j], c));
        a[j][c] = channel[c].a(rho), e[j][c] = __builtin_amdgcn_sqrtf(channel[c].m2(a[j][c], rho)) * iota * part<E>(x[j], c);
        if (!WHOLE && j >= rows) a[j][c] = 1.0f, e[j][c] = 0.0f;
        product[c] *= a[j][c], end[c] = fmaf(a[j][c], end[c], e[j][c]);
      }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) runs[w][lane * V + c] = make_float2(product[c], end[c]);
  };
  if (rows == R) gather(std::true_type{});
  else if (rows > 0) gather(std::false_type{});
  else
#pragma unroll
    for (int c = 0; c < V; ++c) runs[w][lane * V + c] = make_float2(1.0f, 0.0f);
  lds_barrier();
  uint32_t z[R];                // asked for now and used when the tile is joined
  if (GATE && rows == R) load_rows<true, R, V>(l.z, first, b, rows, byte, z);
  else if (GATE && rows > 0) load_rows<false, R, V>(l.z, first, b, rows, byte, z);
  if (w < V && t0 < len) {                   // the tile's own share, a channel a lane
    const uint32_t at = w * 64 + lane;
    float p = 1.0f, s = 0.0f, in = 0.0f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float2 run = runs[k][at];
      p *= run.x, s = fmaf(run.x, s, run.y);
    }
    if (tile == 0 && l.h0) {
      const int channel = channel_of<V>(column, at, l.D);
      if (channel < l.D) in = l.h0[(int64_t)b * l.D + channel];
    }
    if (JOINED) {
      const int64_t step = (int64_t)l.B * l.columns * 64 * V;
      uint64_t* const mine = words + tile * step + ((int64_t)b * l.columns + column) * 64 * V;
      if (tile) leave(mine + at, word_of(p, s)), in = look_back(mine, at, step, tile);
      leave(mine + at, settled(through(word_of(p, s), in)));
    }
    before[at] = in;
  }
  lds_barrier();
  if (rows > 0 && own.on) {
    if (GATE)
#pragma unroll
      for (int j = 0; j < R; ++j) as_loaded(z[j]);
    float h[V];
#pragma unroll
    for (int c = 0; c < V; ++c) h[c] = before[lane * V + c];
    for (int k = 0; k < w; ++k)
#pragma unroll
      for (int c = 0; c < V; ++c) {
        const float2 run = runs[k][lane * V + c];
        h[c] = fmaf(run.x, h[c], run.y);
      }
    if (states && first % kKept == 0)
#pragma unroll
      for (int c = 0; c < V; ++c) states[((int64_t)(first / kKept) * l.B + b) * l.D + d + c] = h[c];
    Run<E> to(y, first, b);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float out[V];
#pragma unroll
      for (int c = 0; c < V; ++c) {
        h[c] = fmaf(a[j][c], h[c], e[j][c]);
        out[c] = GATE ? h[c] * (part<E>(z[j], c) * sigmoid<E>(part<E>(z[j], c))) : h[c];
      }
      if (j < rows) to.store(byte, out);
      to.move();
    }
    if (h_last && len <= first + R)
#pragma unroll
      for (int c = 0; c < V; ++c) h_last[(int64_t)b * l.D + d + c] = h[c];
  }
}

// One token.  A thread has a lane's channels of one row of the batch; bound by the launch and one round of loads.
template <typename E, int V, bool GATE>
__global__ void __launch_bounds__(64)
gated_step_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ state, int slots_in_state, const int32_t* __restrict__ slots) {
  const int b = blockIdx.x / l.columns;
  const Own<V> own(blockIdx.x % l.columns, threadIdx.x, l.D);
  if (!own.on) return;
  const int d = own.d, slot = slots ? slots[b] : b;
  float out[V] = {};
  if (slot < 0 || slot >= slots_in_state) return store_some<E, V>(y.at(0, b) + d, out);
  float* const at = state + (int64_t)slot * l.D + d;
  Channel<E> channel[V];
  channels_of(l, d, channel);
  const auto was = load_some<float, V>(at);
  const auto x = load_some<E, V>(l.x.at(0, b) + d), r = load_some<E, V>(l.r.at(0, b) + d), i = load_some<E, V>(l.i.at(0, b) + d);
  Some<E, V> z = {};
  if (GATE) z = load_some<E, V>(l.z.at(0, b) + d);
  float h[V];
#pragma unroll
  for (int c = 0; c < V; ++c) {
    const float rho = channel[c].rho((float)r.v[c]), iota = channel[c].iota((float)i.v[c]), a = channel[c].a(rho);
    h[c] = fmaf(a, was.v[c], __builtin_amdgcn_sqrtf(channel[c].m2(a, rho)) * iota * (float)x.v[c]);
    out[c] = GATE ? h[c] * ((float)z.v[c] * sigmoid<E>((float)z.v[c])) : h[c];
  }
  // in place: what is repeated has been read before or behind the neighbour's update, and is not stored
  if (own.repeated) {
#pragma unroll
    for (int c = 0; c < V; ++c)
      if (c >= own.repeated) at[c] = h[c], store(y.at(0, b) + d + c, out[c]);
    return;
  }
  store_some<float, V>(at, h);
  store_some<E, V>(y.at(0, b) + d, out);
}

// A wave's wait by itself, on words that the caller fills in: [tiles][64], the first tile's first.
__global__ void __launch_bounds__(64)
gated_wait_kernel(const uint64_t* words, int tiles, int looks, float* __restrict__ h) {
  h[threadIdx.x] = look_back(words + (int64_t)tiles * 64, threadIdx.x, 64, tiles, looks);
}

}  // namespace

extern "C" size_t bppsa_gated_scan_states_bytes(int T, int B, int D) {
  return sizes_ok(T, B, D) ? (size_t)bppsa_ceil_div(T, kKept) * B * D * sizeof(float) : 0;
}

// of the widest workgroups, 16-bit ones, or of one channel a lane, whichever is more
extern "C" size_t bppsa_gated_scan_workspace_bytes(int T, int B, int D) {
  if (!sizes_ok(T, B, D)) return 0;
  const int tiles = bppsa_ceil_div(T, kTile);
  return words_bytes(tiles, B, bppsa_ceil_div(D, 128), 2);
}

extern "C" bppsa_status bppsa_gated_scan(const bppsa_gated* layer, const bppsa_rows* y, float* h_last, void* states,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  BPPSA_TRY(check_layer(layer));
  if (!y || !writable(*y, layer->T, layer->B) || (h_last && h_last == layer->h0) || ((uintptr_t)states & 15)) return BPPSA_EINVAL;
  BPPSA_TRY(check_workspace(workspace, workspace_bytes, bppsa_gated_scan_workspace_bytes(layer->T, layer->B, layer->D)));
  const hipStream_t s = (hipStream_t)stream;
  return by_type(layer->type, [&](auto e) {
    using E = decltype(e);
    return by_width<E>(layer->D, [&](auto width) {
      constexpr int V = width.value;
      const Layer<E> l = layer_of<E>(*layer, 64 * V);
      const int tiles = bppsa_ceil_div(l.T, kTile), total = tiles * l.B * l.columns;
      const auto run = [&](auto steps, auto gate, auto joined) {
        gated_kernel<E, V, steps.value, gate.value, joined.value><<<total, kWaves * 64, 0, s>>>(
            l, rows_of<E>(*y), h_last, static_cast<float*>(states), static_cast<int*>(workspace),
            reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + kTicketBytes), tiles, chains_of_queue(l.columns * l.B));
      };
      constexpr std::integral_constant<int, kRun> whole;
      constexpr std::integral_constant<int, kRun / 2> half;
      constexpr std::true_type yes;
      constexpr std::false_type no;
      if (tiles > 1) {
        empty_words(workspace, words_bytes(tiles, l.B, l.columns, V), s);
        l.z.data ? run(whole, yes, yes) : run(whole, no, yes);
      } else if (l.T > kTile / 2) {
        l.z.data ? run(whole, yes, no) : run(whole, no, no);
      } else {                       // T = 16, B = 2, D = 40 fp32: 3.8 us, 5.6 by runs of sixteen steps
        l.z.data ? run(half, yes, no) : run(half, no, no);
      }
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
    return by_width<E>(layer->D, [&](auto width) {
      constexpr int V = width.value;
      const Layer<E> l = layer_of<E>(*layer, 64 * V);
      const auto kernel = l.z.data ? gated_step_kernel<E, V, true> : gated_step_kernel<E, V, false>;
      kernel<<<(unsigned)(l.columns * l.B), 64, 0, (hipStream_t)stream>>>(l, rows_of<E>(*y), state, slots_in_state, slots);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}

extern "C" bppsa_status bppsa_gated_wait_diag(const uint64_t* words, int tiles, int looks, float* h, void* stream) {
  if (!words || ((uintptr_t)words & 7) || tiles < 1 || looks < 1 || looks > kLooks || !h) return BPPSA_EINVAL;
  gated_wait_kernel<<<1, 64, 0, (hipStream_t)stream>>>(words, tiles, looks, h);
  BPPSA_CHECK_LAUNCH();
  return BPPSA_OK;
}
