// The gated recurrence, forward: over sequences, and the step of single tokens.
#include "gated_parts.h"

namespace {

using namespace gated;

// A workgroup takes tiles of kTile steps of 64 V channels, one after the other.  Each wave has a run of the steps in registers:
// it turns them into decays and what enters, finds what its run does to a state, and when the state before it is known walks
// them again.  Outputs of a tile are on their way while the next one's inputs are asked for.
template <typename E, int V, bool GATE, bool JOINED>
__global__ void __launch_bounds__(kWaves * 64, 4)
gated_kernel(const Layer<E> l, Rows<E> y, float* __restrict__ h_last, float* __restrict__ states, int* ticket, uint64_t* words,
             int total) {
  constexpr int R = kRun;
  __shared__ float2 runs[2][kWaves][64 * V];
  __shared__ float before[2][64 * V];
  __shared__ int taken[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = blockIdx.x;
  if (JOINED) {
    if (threadIdx.x == 0) taken[1] = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    id = __builtin_amdgcn_readfirstlane(taken[1]);
  }
  for (int parity = 0; id < total; parity ^= 1) {
    int next = total;
    if (JOINED && threadIdx.x == 0) next = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const int column = id % l.columns, b = id / l.columns % l.B, tile = id / l.columns / l.B;
    const Own<V> own(column, lane, l.D);
    const int d = own.d, len = clamp_length(l.lengths, b, l.T), t0 = tile * kTile, first = t0 + w * R;
    // behind an end
    if (own.on)
      for (int t = first > len ? first : len; t < first + R && t < l.T; ++t) {
        const float zero[V] = {};
        store_some<E, V>(y.at(t, b) + d, zero);
      }
    if (len == 0 && tile == 0 && w == 0 && h_last && own.on)
      for (int c = 0; c < V; ++c) h_last[(int64_t)b * l.D + d + c] = l.h0 ? l.h0[(int64_t)b * l.D + d + c] : 0.0f;

    float a[R][V], e[R][V], h[V];
    Some<E, V> z[GATE ? R : 1];
    float product[V], end[V];
#pragma unroll
    for (int c = 0; c < V; ++c) product[c] = 1.0f, end[c] = 0.0f;
    if (first < len) {
      Some<E, V> x[R], r[R], i[R];
      float decay[V], rb[V], ib[V];
      parameter(l.decay, d, decay), parameter(l.r_bias, d, rb), parameter(l.i_bias, d, ib);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int t = first + j < len ? first + j : len - 1;
        r[j] = load_some<E, V>(l.r.at(t, b) + d), i[j] = load_some<E, V>(l.i.at(t, b) + d), x[j] = load_some<E, V>(l.x.at(t, b) + d);
        if (GATE) z[j] = load_some<E, V>(l.z.at(t, b) + d);
      }
#pragma unroll
      for (int j = 0; j < R; ++j)
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const Gates g = gates_of<E>((float)r[j].v[c] + rb[c], (float)i[j].v[c] + ib[c], decay[c]);
          const bool real = first + j < len;
          a[j][c] = real ? g.a : 1.0f;
          e[j][c] = real ? __builtin_amdgcn_sqrtf(g.m2) * g.iota * (float)x[j].v[c] : 0.0f;
          product[c] *= a[j][c], end[c] = fmaf(a[j][c], end[c], e[j][c]);
        }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) runs[parity][w][lane * V + c] = make_float2(product[c], end[c]);
    lds_barrier();
    if (w < V && t0 < len) {                   // the tile's own share, a channel a lane
      const int at = w * 64 + lane;
      float p = 1.0f, s = 0.0f, in = 0.0f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float2 run = runs[parity][k][at];
        p *= run.x, s = fmaf(run.x, s, run.y);
      }
      if (tile == 0 && l.h0) {
        const int channel = channel_of<V>(column, at, l.D);
        if (channel < l.D) in = l.h0[(int64_t)b * l.D + channel];
      }
      if (JOINED) {
        const int64_t step = (int64_t)l.B * l.columns * 64 * V;
        uint64_t* const mine = words + tile * step + ((int64_t)b * l.columns + column) * 64 * V + at;
        if (tile) leave(mine, word_of(p, s)), in = look_back(mine, step, tile);
        leave(mine, settled(through(word_of(p, s), in)));
      }
      before[parity][at] = in;
    }
    if (JOINED && threadIdx.x == 0) taken[parity] = next;
    lds_barrier();
    if (first < len) {
      if (GATE)
#pragma unroll
        for (int j = 0; j < R; ++j) as_loaded(z[j]);
#pragma unroll
      for (int c = 0; c < V; ++c) h[c] = before[parity][lane * V + c];
      for (int k = 0; k < w; ++k)
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float2 run = runs[parity][k][lane * V + c];
          h[c] = fmaf(run.x, h[c], run.y);
        }
      if (states && first % kKept == 0 && own.on)
#pragma unroll
        for (int c = 0; c < V; ++c) states[((int64_t)(first / kKept) * l.B + b) * l.D + d + c] = h[c];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float out[V];
#pragma unroll
        for (int c = 0; c < V; ++c) {
          h[c] = fmaf(a[j][c], h[c], e[j][c]);
          out[c] = GATE ? h[c] * ((float)z[j].v[c] * sigmoid<E>((float)z[j].v[c])) : h[c];
        }
        if (first + j < len && own.on) store_some<E, V>(y.at(first + j, b) + d, out);
      }
      if (h_last && own.on && len <= first + R)
#pragma unroll
        for (int c = 0; c < V; ++c) h_last[(int64_t)b * l.D + d + c] = h[c];
    }
    id = JOINED ? __builtin_amdgcn_readfirstlane(taken[parity]) : total;
  }
}

constexpr int kResident = 2;     // workgroups of a compute unit

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
      const auto run = [&](auto gate, auto joined) {
        constexpr bool GATE = gate.value, JOINED = joined.value;
        const int groups = JOINED ? std::min(total, bppsa_compute_units() * kResident) : total;
        gated_kernel<E, V, GATE, JOINED><<<groups, kWaves * 64, 0, s>>>(
            l, rows_of<E>(*y), h_last, static_cast<float*>(states), static_cast<int*>(workspace),
            reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + kTicketBytes), total);
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
      gated_step_kernel<E, V><<<(unsigned)(l.columns * l.B), 64, 0, (hipStream_t)stream>>>(l, rows_of<E>(*y), state, slots_in_state, slots);
      BPPSA_CHECK_LAUNCH();
      return BPPSA_OK;
    });
  });
}
