// The loss of a student against a teacher's top logits, and its gradient for the student's logits.
//
// With q = softmax(x / tau) over the vocabulary, shares p of the teacher's entries (c_k, t_k) and, where the teacher's normaliser
// is given, the share p0 = 1 - sum p of all other tokens, which the student gives q0 = sum of q over them,
//     soft = sum_k p_k log(p_k / q[c_k]) + p0 log(p0 / q0),      tau dsoft/dx = q M - p on the entries,  q (M - p0 / q0) elsewhere,
// M = sum p + p0, p0 / q0 = 0 without the normaliser.  The other part, -log softmax(x)[target], has the gradient
// softmax(x) - 1[target].  What is made of the K entries alone is made in 64 bits: there are few of them, and the parts of a
// divergence cancel.
#include "logits.h"
#include "lanes.h"

namespace {

using namespace logits;

struct Entries {                   // of the teacher, [T,B,K]
  const void* logits;
  const int32_t* index;
  int K, type;
};
// as it is stored, and its value: whoever asks for it does not wait for it
__device__ __forceinline__ uint32_t entry_bits(const Entries& e, int64_t at) {
  if (e.type == BPPSA_F32) return static_cast<const uint32_t*>(e.logits)[at];
  return static_cast<const uint16_t*>(e.logits)[at];
}
__device__ __forceinline__ float entry_logit(const Entries& e, uint32_t bits) {
  if (e.type == BPPSA_F32) return __uint_as_float(bits);
  if (e.type == BPPSA_BF16) return __uint_as_float(bits << 16);
  return static_cast<float>(__builtin_bit_cast(f16_t, (uint16_t)bits));
}

template <typename E>
struct Loss {
  Rows<const E> x;
  Rows<E> dx;
  Entries top;
  const float *top_norm, *weight;
  const int32_t* targets;
  float* loss;
  int B, V;
  float tau, hard;
  double scale;                    // 1 / tau
};

constexpr int kMost = BPPSA_DISTIL_MAX_K;

// A value that is the same in all lanes, in a scalar register: the rows of sixteen waves have no vector register to spare.
__device__ __forceinline__ float scalar(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }

// What the waves of a row tell each other, each by its first lane.
template <int WAVES>
struct Share {
  float largest[WAVES], sums[3][WAVES];
  float top[WAVES];
  double shares[WAVES], terms[WAVES];
};
// One workgroup a row.  CHUNKS > 0: the row is read once, into registers (16 bytes a lane and chunk), and its largest value, its sums
// and its gradient are made of those; 0: a row too long for that is read three times.  SECOND: the data's own token has a
// softmax of its own, at another temperature.  TAIL: all other tokens are one more class.
//
// Bound by memory: 8192 rows of 32768 bf16 with two softmaxes 210 us, 5.1 TB/s, the vector unit busy for 92 % of that (two exponentials
// a logit and softmax: to keep them takes twice the registers of a 16-bit row).  Short rows are bound by what a row takes besides its
// logits, the entries' shares in 64 bits and seven sums over a wave or more (16000 rows of 4001 fp16: 62 us, 4.2 TB/s; 65536 of 100 fp32
// 47 us, 1.3 TB/s; 262144 of 16 fp32 167 us).  Rows that are read three times: 1024 of 150001 bf16 252 us, of 128001 fp32 395.
//
// As many waves a SIMD as the registers of the row let, and no more: two workgroups of sixteen waves are worth the 4 to
// 10 vector registers that most of them spill (2048 rows of 65536 bf16 with two softmaxes: 137 to 143 us, 172 by one workgroup a unit; with
// the others as one more class 119 and 151), four of eight instead of three are not (4096 rows of 32001 bf16: 130 us, 119).
template <typename E, int WAVES, int CHUNKS, bool SECOND, bool TAIL>
__global__ void __launch_bounds__(WAVES * 64, CHUNKS == 16 ? 4 : WAVES == 16 ? 8 : 6)
distil_kernel(const Loss<E> l) {
  constexpr int N = Chunk<E>::N, THREADS = WAVES * 64, STEP = THREADS * N, HELD = CHUNKS ? CHUNKS : 1;
  extern __shared__ uint32_t is_entry[];       // a bit a token
  __shared__ Share<WAVES> of;
  // of the entries: the place (-1: does not count), the student's logit there, the teacher's, the share
  __shared__ int place[kMost];
  __shared__ float at_place[kMost], logit[kMost], p[kMost];
  __shared__ float at_target;
  __shared__ int twice;
  const int64_t row = blockIdx.x;
  const int t = (int)(row / l.B), b = (int)(row % l.B), K = l.top.K, first = threadIdx.x * N;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // the entries are dealt out to the first threads; what is made in 64 bits is left to waves that have some
  const int with_entries = (K + 63) / 64 < WAVES ? (K + 63) / 64 : WAVES;
  const bool entries = wave < with_entries;
  const float weight = l.weight ? l.weight[row] : 1.0f;
  E* const dx = l.dx.data ? l.dx.at(t, b) : nullptr;
  if (weight == 0.0f) {
    if (threadIdx.x == 0) l.loss[row] = 0.0f;
    const float zero[N] = {};
    if (dx)
      for (int v = first; v < l.V; v += STEP) store_chunk<E>(dx, v, l.V, zero);
    return;
  }
  const E* const x = l.x.at(t, b);
  const float top_norm = TAIL ? l.top_norm[row] : 0.0f;
  const float scale = (float)l.scale;
  const int target = l.targets && l.hard != 0.0f ? l.targets[row] : -1;
  const bool known = target >= 0 && target < l.V;
  // the entries are asked for first, then the row, then the row's logits of the entries; nothing of it in a branch of its own, which would
  // wait for it
  constexpr int ENTRIES = (kMost + THREADS - 1) / THREADS;
  int c[ENTRIES];
  uint32_t raw[ENTRIES];
  if (entries)
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
      const int k = threadIdx.x + i * THREADS;
      const int64_t at = row * K + (k < K ? k : K - 1);
      if (wave * 64 + i * THREADS < K) c[i] = l.top.index[at], raw[i] = entry_bits(l.top, at);
    }
  // f(chunk, its first token less the thread's, how many of its tokens are a neighbour's, whether the step is whole).  A step in which not all of the
  // workgroup's chunks are whole is apart from the others: there is code for its ends but once.  The last chunk of a row begins early
  // enough to be loaded whole, and what it shares with the one before it is made minus infinity.
  Chunk<E> held[HELD], end;
  const int steps = l.V / STEP, end_at = first + steps * STEP, last = l.V - N, end_from = end_at < last ? end_at : last;
  const bool ends = CHUNKS > 0 && steps * STEP < l.V;
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (CHUNKS > 0) {
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        __builtin_amdgcn_sched_barrier(0);
        if (k < steps) f(held[k], k * STEP, 0, std::true_type{});
      }
      if (ends) f(end, end_from - first, end_at - end_from, std::false_type{});
    } else {
      for (int v = 0; first + v < l.V; v += STEP) f(load_chunk(x, first + v, l.V), v, 0, std::true_type{});
    }
  };
  if constexpr (CHUNKS > 0) {
    // 16-bit chunks behind the last whole one are left out, of fp32 ones that is read again: as each has less or more room than it needs, the
    // other way takes some of the row out of registers (2048 rows of 40000 bf16 82 us, 95; of 32000 fp32 with two softmaxes 130, 202)
    if (sizeof(E) == 2 || steps > 0)
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k)
        if (sizeof(E) == 4 || k < steps) held[k] = load_whole(x + (k < steps ? k : steps - 1) * STEP, first * sizeof(E));
    if (ends) end = load_whole(x, end_from * sizeof(E));
  }
  // between two passes: the compiler would keep what the first made of the row for the second, in several times the registers
  auto forget = [&]() __attribute__((always_inline)) {
    if constexpr (CHUNKS > 0)
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) asm volatile("" : "+v"(held[k].w));
    asm volatile("" : "+v"(end.w));
  };
  const E of_target = x[known ? target : 0];
  E of_entry[ENTRIES];
  float top = -INFINITY;
  if (entries)
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i) {
      const int k = threadIdx.x + i * THREADS;
      if (wave * 64 + i * THREADS >= K) continue;
      const float value = entry_logit(l.top, raw[i]);
      if (k >= K || c[i] >= l.V || value == -INFINITY) c[i] = -1;
      of_entry[i] = x[c[i] >= 0 ? c[i] : 0];
      if (c[i] >= 0) top = fmaxf(top, value);
      if (k < K) place[k] = c[i], logit[k] = value;
    }
  // an index that comes twice finds its bit set
  for (int v = threadIdx.x; v <= (l.V + 31) / 32; v += THREADS) is_entry[v] = 0;
  if (threadIdx.x == 0) twice = 0;
  __syncthreads();
  if (entries)
    for (int k = threadIdx.x; k < K; k += THREADS)
      if (place[k] >= 0 && atomicOr(&is_entry[place[k] / 32], 1u << place[k] % 32) >> place[k] % 32 & 1) twice = 1;
  float m = -INFINITY;
  end.leave_out(end_at - end_from);
  each([&](const Chunk<E>& x, int, int, auto) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < N; ++k) m = fmaxf(m, x[k]);
  });
  m = lanes::largest(m);
  if (entries) {
    top = lanes::largest(top);
#pragma unroll
    for (int i = 0; i < ENTRIES; ++i)
      if (threadIdx.x + i * THREADS < K) at_place[threadIdx.x + i * THREADS] = static_cast<float>(of_entry[i]);
  }
  if (threadIdx.x == 0) at_target = static_cast<float>(of_target);
  if (lane == 0) of.largest[wave] = m, of.top[wave] = top;
  __syncthreads();
  if (WAVES > 1) {
    m = lanes::largest(lane < WAVES ? of.largest[lane % WAVES] : -INFINITY);
    if (entries) top = lanes::largest(lane < with_entries ? of.top[lane % WAVES] : -INFINITY);
  }

  forget();
  const Exponential<E> of_tau(m, scale), of_one(m, 1.0f);
  float s = 0.0f, s1 = 0.0f, rest = 0.0f;
  each([&](const Chunk<E>& x, int at, int, auto) __attribute__((always_inline)) {
    float e[N], sum = 0.0f, sum1 = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      e[k] = of_tau(x[k]), sum += e[k];
      if (SECOND) sum1 += of_one(x[k]);
    }
    s += sum, s1 += sum1;
    if (TAIL) {
      const int from = first + at;
      const uint32_t bits = (uint32_t)(((uint64_t)is_entry[from / 32 + 1] << 32 | is_entry[from / 32]) >> from % 32);
      float others = 0.0f;
#pragma unroll
      for (int k = 0; k < N; ++k) others += __uint_as_float(__float_as_uint(e[k]) & ~(uint32_t)__builtin_amdgcn_sbfe((int)bits, k, 1));
      rest += others;
    }
  });
  s = lanes::sum(s);
  if (SECOND) s1 = lanes::sum(s1);
  if (TAIL) rest = lanes::sum(rest);
  // the entries' shares, before they are divided by their sum where they are all there is, and what they leave of the divergence
  double shares = 0.0, terms = 0.0;
  if (entries) {
    for (int k = threadIdx.x; k < K; k += THREADS) {
      if (place[k] < 0) continue;
      // the difference in 64 bits, its exponential in 32, corrected by what the difference loses there; what is NaN stays it
      const double over = TAIL ? (double)logit[k] * l.scale - (double)top_norm : ((double)logit[k] - (double)top) * l.scale;
      const float near = (float)over, e = exp_of<true>(near), share = e == 0.0f ? 0.0f : fmaf(e, (float)(over - (double)near), e);
      shares += (double)share, p[k] = share;
      if (share != 0.0f) terms += (double)share * (over - ((double)at_place[k] - (double)m) * l.scale);
    }
    shares = lanes::sum(shares), terms = lanes::sum(terms);
  }
  if (lane == 0) of.sums[0][wave] = s, of.sums[1][wave] = s1, of.sums[2][wave] = rest, of.shares[wave] = shares, of.terms[wave] = terms;
  __syncthreads();
  if (WAVES > 1) {               // a lane a wave
    s = lanes::sum(lane < WAVES ? of.sums[0][lane % WAVES] : 0.0f);
    if (SECOND) s1 = lanes::sum(lane < WAVES ? of.sums[1][lane % WAVES] : 0.0f);
    if (TAIL) rest = lanes::sum(lane < WAVES ? of.sums[2][lane % WAVES] : 0.0f);
    shares = lanes::sum(lane < with_entries ? of.shares[lane % WAVES] : 0.0);
    if (wave == 0) terms = lanes::sum(lane < with_entries ? of.terms[lane % WAVES] : 0.0);
  }
  s = scalar(s), s1 = scalar(s1), rest = scalar(rest);
  const bool any = shares != 0.0;
  const double p0 = TAIL && rest > 0.0f ? fmax(0.0, 1.0 - shares) : 0.0;
  const float over = any && !TAIL ? 1.0f / (float)shares : 1.0f;
  if (dx) {
    const float of_soft = weight * (1.0f - l.hard) * l.tau, hard = known ? weight * l.hard : 0.0f;
    const float one = 1.0f / s, of_e1 = SECOND ? scalar(hard / s1) : 0.0f, of_e = SECOND ? 0.0f : hard * one;
    const float M = (TAIL ? (float)shares : shares > 0.0 ? 1.0f : (float)shares) + (float)p0;
    // where the student gives the others next to nothing, p0 / q0 and with it elsewhere would be out of range, which the product with their
    // exponentials is not: these are lifted first, and elsewhere is as much smaller
    const bool far = TAIL && p0 > 0.0 && rest < 0x1p-64f;
    const float lift = far ? 0x1p64f : 1.0f, drop = far ? 0x1p-64f : 1.0f, ratio = p0 > 0.0 ? (float)p0 * (s / (rest * lift)) : 0.0f;
    const float elsewhere = scalar(fmaf(of_soft * fmaf(M, drop, -ratio), one, of_e * drop)), inside = scalar(fmaf(of_soft * M, one, of_e));
    const auto lifted = [&](float e) { return TAIL ? e * lift : e; };
    forget();
    each([&](const Chunk<E>& x, int at, int shared, auto whole) __attribute__((always_inline)) {
      float g[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        g[k] = elsewhere * lifted(of_tau(x[k]));
        if (SECOND) g[k] = fmaf(of_e1, of_one(x[k]), g[k]);
      }
      if constexpr (CHUNKS == 0) store_chunk<E>(dx, first + at, l.V, g);
      else if constexpr (whole.value) store_whole(dx + at, first * sizeof(E), g);
      else if (shared == 0) store_whole(dx, (first + at) * sizeof(E), g);
      else
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (k >= shared) store(dx + first + at + k, g[k]);
    });
    __syncthreads();               // behind it the places of the entries and of the target are written again
    auto again = [&](int at, float e, float value, float coefficient, float own) __attribute__((always_inline)) {
      float g = coefficient * e - own;
      if (SECOND) g = fmaf(of_e1, of_one(value), g);
      store(dx + at, g);
    };
    if (entries)
      for (int k = threadIdx.x; k < K; k += THREADS) {
        const int c = place[k];
        if (c < 0) continue;
        float own = p[k];
        if (twice) {
          own = 0.0f;
          for (int i = 0; i < K; ++i) own += place[i] == c ? p[i] : 0.0f;
        }
        again(c, of_tau(at_place[k]), at_place[k], inside, of_soft * (own * over) + (c == target ? hard : 0.0f));
      }
    if (threadIdx.x == THREADS - 1 && known) {
      if (!(is_entry[target / 32] >> target % 32 & 1)) again(target, lifted(of_tau(at_target)), at_target, elsewhere, hard);
    }
  }
  // last, when the row's registers are free
  if (wave == 0) {
    double soft = 0.0, ce = 0.0, log_s = 0.0;
    if (TAIL || (known && !SECOND)) log_s = log_of(s) - of_tau.log_off();
    if (TAIL) soft = terms + (shares + p0) * log_s + (p0 > 0.0 ? p0 * (log_of((float)p0) - log_of(rest) + of_tau.log_off()) : 0.0);
    else if (any) soft = terms / shares + log_of(s) - log_of((float)shares) - of_tau.log_off();
    if (known) ce = (double)m - (double)at_target + (SECOND ? log_of(s1) - of_one.log_off() : log_s);
    if (threadIdx.x == 0)
      l.loss[row] = (float)((double)weight * ((1.0 - (double)l.hard) * (double)l.tau * (double)l.tau * soft + (double)l.hard * ce));
  }
}

}  // namespace

extern "C" bppsa_status bppsa_distil(const bppsa_distil_rows* r, float* loss, const bppsa_rows* dlogits, void* stream) {
  if (!r || r->T < 1 || r->B < 1 || r->V < 1 || r->K < 1) return BPPSA_EINVAL;
  if (!r->logits.data || !r->top_logits || !r->top_index || !loss) return BPPSA_EINVAL;
  if (!(r->temperature > 0x1p-20f && r->temperature < 0x1p20f) || !(r->hard >= 0.0f && r->hard <= 1.0f)) return BPPSA_EINVAL;
  if (r->hard != 0.0f && !r->targets) return BPPSA_EINVAL;
  if (dlogits && !writable(*dlogits, r->T, r->B)) return BPPSA_EINVAL;
  if (dlogits && dlogits->data == r->logits.data &&
      ((r->T > 1 && dlogits->stride_t != r->logits.stride_t) || (r->B > 1 && dlogits->stride_b != r->logits.stride_b))) return BPPSA_EINVAL;
  if (r->K > kMost || r->type < BPPSA_F32 || r->type > BPPSA_F16 || r->top_type < BPPSA_F32 || r->top_type > BPPSA_F16)
    return BPPSA_EUNSUPPORTED;
  if (bppsa_mul_overflows(r->T, r->B, r->V, 1) || r->V > BPPSA_DISTIL_MAX_V || (int64_t)r->T * r->B >= 1 << 22) return BPPSA_EOVERFLOW;
  return by_type(r->type, [&](auto e) {
    using E = decltype(e);
    const Loss<E> l{rows_of<const E>(r->logits), dlogits ? rows_of<E>(*dlogits) : Rows<E>{}, Entries{r->top_logits, r->top_index, r->K, r->top_type},
                    r->top_norm, r->weight, r->targets, loss, r->B, r->V, r->temperature, r->hard, 1.0 / (double)r->temperature};
    const auto run = [&](auto waves, auto chunks) {
      const size_t bits = ((size_t)bppsa_ceil_div(l.V, 32) + 1) * sizeof(uint32_t);
      const bool second = l.hard != 0.0f && l.tau != 1.0f;
      const auto kernel = l.top_norm ? second ? distil_kernel<E, waves.value, chunks.value, true, true> : distil_kernel<E, waves.value, chunks.value, false, true>
                                     : second ? distil_kernel<E, waves.value, chunks.value, true, false> : distil_kernel<E, waves.value, chunks.value, false, false>;
      kernel<<<(unsigned)(r->T * r->B), waves.value * 64, bits, (hipStream_t)stream>>>(l);
    };
    constexpr int N = Chunk<E>::N;
    const auto fits = [&](int waves, int chunks) { return l.V <= waves * 64 * N * chunks; };
    typedef std::integral_constant<int, 0> None;
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    typedef std::integral_constant<int, 4> Four;
    typedef std::integral_constant<int, 8> Eight;
    typedef std::integral_constant<int, 16> Sixteen;
    // The fewest waves that hold a row in as many chunks as their registers take, and fewer chunks where rows are short: each line
    // measured with it and with the next one in its place.  65536 rows of 300 bf16 and 16 entries 59 and 61 us; of 50 entries, with the others as
    // one more class, 16384 of 3000 48 and 55, 8192 of 5000 39 and 47, 8192 of 10000 65 and 92, 4096 of 32001 119 and 156; of 64 2048 of 65536
    // 119 and 156, and 1024 of 131072 with two softmaxes, the longest that registers hold, 154 and 189.  (Rows that fill their line's chunks
    // gain less, at worst nothing.)
    if (l.V < N) run(One{}, None{});
    else if (fits(1, 4)) run(One{}, Four{});
    else if (fits(1, 8)) run(One{}, Eight{});
    else if (fits(2, 8)) run(Two{}, Eight{});
    else if (fits(4, 8)) run(Four{}, Eight{});
    else if (fits(8, 8)) run(Eight{}, Eight{});
    else if (fits(16, 8)) run(Sixteen{}, Eight{});
    else if (fits(16, 16)) run(Sixteen{}, Sixteen{});
    else run(Sixteen{}, None{});
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}
