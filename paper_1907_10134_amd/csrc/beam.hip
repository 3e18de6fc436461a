// One step of a beam search: the selection over beams and vocabulary, and the move of the beams' states.
//
// A beam's candidates are its score plus log softmax of its logits.  Within a beam the logits alone decide the order (larger
// first, of equal ones the lower token); the beams' lists are merged by their sums in 64 bits (of equal ones the lower beam): sums
// of different beams may lie next to each other, and a selection that turned on a rounding would differ from run to run of a
// model with other sizes of a batch.
#include <algorithm>

#include "logits.h"
#include "lanes.h"

namespace {

using namespace logits;

constexpr int kThreads = 256, kEach = 32, kPiece = kThreads * kEach, kFound = 1024;
constexpr int kMostBeams = BPPSA_BEAM_MAX_W, kMostPieces = 64;
static_assert(kMostPieces * kPiece == BPPSA_BEAM_MAX_V);

// What a piece of a row leaves: its largest value, the sum of exponentials relative to that and its first W logits.
struct Pieces {
  float* largest;                  // [row][piece]
  double* sum;
  uint64_t* key;                   // [row][piece][W], 0 where there are fewer
  int count;
};

// Ascending with the value, and of equal values descending with the place; never 0.
__device__ __forceinline__ uint64_t key_of(float v, int place) {
  const uint32_t u = __float_as_uint(v + 0.0f);          // no -0, which is equal to 0
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~place;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ int place_of(uint64_t key) { return (int)~(uint32_t)key; }

// Ascending with the value; 0 for none.
__device__ __forceinline__ uint64_t order_of(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v + 0.0);
  return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}

template <typename E>
struct Beams {
  Rows<const E> logits;            // [B][W][V], the sequences' stride first
  const float* scores;
  const uint8_t* finished;
  const int32_t* slots;
  int B, W, V, end;
};
template <typename E>
__device__ __forceinline__ bool alive(const Beams<E>& s, int row) {
  return fabsf(s.scores[row]) < INFINITY && !(s.finished && s.finished[row]);
}

// One workgroup a piece of a row, whose values stay in registers.  A bound that W of 64 columns of the piece pass, by their
// largest values, is no larger than the W-th largest value; so few values pass it (some 10 of 8192 normal ones at W = 8) that each
// can count those in front of it.  Where more than kFound do, equal ones that is, they are taken one after the other.
//
// 512 rows of 131072 bf16, W = 8: 38 us, 3.5 TB/s, about 26 of them the read itself, 6 the bound and the values behind it, 5 the
// exponentials.  Eight workgroups a unit have 64 vector registers each; 14 to 16 more are spilled, 60 to 64 bytes a lane (8.2 MB are written,
// 0.6 of them results).  The next piece's read beside that, two pieces a workgroup in registers, has fewer waves: 66 us a call instead of 46.
template <typename E>
__global__ void __launch_bounds__(kThreads, 8)
beam_piece_kernel(const Beams<E> s, const Pieces out) {
  constexpr int N = Chunk<E>::N, LOADS = kEach / N, STEP = kThreads * N;
  __shared__ float of_column[kThreads / 64][64];
  __shared__ double sums[kThreads / 64];
  __shared__ uint64_t found[kFound];
  __shared__ int n_found;
  const int piece = blockIdx.x % out.count, row = blockIdx.x / out.count, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (!alive(s, row)) return;
  const E* const from = s.logits.at(row / s.W, row % s.W) + (int64_t)piece * kPiece;
  const int left = s.V - piece * kPiece, first = threadIdx.x * N;           // tokens from the piece's first on
  Chunk<E> held[LOADS];
  if (left >= kPiece) {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) held[k] = load_whole(from + k * STEP, first * sizeof(E));
  } else {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) held[k] = load_chunk(from, first + k * STEP, left);
  }
  float of_chunk[LOADS], m = -INFINITY;
#pragma unroll
  for (int k = 0; k < LOADS; ++k) {
    of_chunk[k] = -INFINITY;
#pragma unroll
    for (int j = 0; j < N; ++j) of_chunk[k] = fmaxf(of_chunk[k], held[k][j]);
    m = fmaxf(m, of_chunk[k]);
  }
  if (threadIdx.x == 0) n_found = 0;
  of_column[wave][lane] = m;
  __syncthreads();
  const int64_t at = (int64_t)row * out.count + piece;
  uint64_t* const to = out.key + at * s.W;
  float column = m;
#pragma unroll
  for (int k = 0; k < kThreads / 64; ++k) column = fmaxf(column, of_column[k][lane]);
  const float top = lanes::largest(column);
  // as high a bound as W columns pass, within a 128th of the columns' range
  const bool none = top == -INFINITY;          // no token has a share: the first ones come first
  float bound = none ? INFINITY : -INFINITY;
  if (!none && __popcll(__ballot(column > -INFINITY)) >= s.W) {
    float over = top;
    bound = -lanes::largest(column > -INFINITY ? -column : -INFINITY);
#pragma unroll 1
    for (int k = 0; k < 7; ++k) {
      const float half = 0.5f * bound + 0.5f * over;
      if (__popcll(__ballot(column >= half)) >= s.W) bound = half;
      else over = half;
    }
  }
  const float zero = none ? 0.0f : top;
  float e = 0.0f;
#pragma unroll
  for (int k = 0; k < LOADS; ++k) {
    float part = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) part += exp2_fast((held[k][j] - zero) * kLog2e);         // the largest is 1, exactly
    e += part;
  }
  if (m >= bound)
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      if (of_chunk[k] < bound) continue;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (held[k][j] >= bound && first + k * STEP + j < left) {
          const int at = atomicAdd(&n_found, 1);
          if (at < kFound) found[at] = key_of(held[k][j], piece * kPiece + first + k * STEP + j);
        }
    }
  const double sum = lanes::sum((double)e);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  const int n = n_found;
  if (threadIdx.x == 0) {
    double all = sums[0];
    for (int k = 1; k < kThreads / 64; ++k) all += sums[k];
    out.largest[at] = zero, out.sum[at] = all;
  }
  if (none) {
    if (threadIdx.x < s.W) to[threadIdx.x] = (int)threadIdx.x < left ? key_of(-INFINITY, piece * kPiece + threadIdx.x) : 0;
    return;
  }
  if (n <= kFound) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const uint64_t mine = found[i];
      int before = 0;
#pragma unroll 8
      for (int k = 0; k < n; ++k) before += found[k] > mine;
      if (before < s.W) to[before] = mine;
    }
    if (threadIdx.x >= n && threadIdx.x < s.W) to[threadIdx.x] = 0;
    return;
  }
  uint64_t last = ~(uint64_t)0;
  for (int i = 0; i < s.W; ++i) {
    uint64_t best = 0;
#pragma unroll
    for (int k = 0; k < LOADS; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const uint64_t key = first + k * STEP + j < left ? key_of(held[k][j], piece * kPiece + first + k * STEP + j) : 0;
        if (key < last && key > best) best = key;
      }
    best = lanes::largest(best);
    __syncthreads();
    if (lane == 0) found[wave] = best;
    __syncthreads();
    for (int k = 0; k < kThreads / 64; ++k) best = found[k] > best ? found[k] : best;
    if (threadIdx.x == 0) to[i] = best;
    last = best;
  }
}

// One workgroup a sequence: a wave merges the pieces' lists of a beam, then the first one the beams' lists.  Bound by the chain of what it
// waits for (W = 8, 16 pieces: 8 us; by comparisons of 32 bits, 64 where those are equal: B = 16, W = 32 74 us a call, 85 by 64 at once).
struct Choice {
  float* scores;
  int32_t *parents, *tokens, *slots, *sources;
  uint8_t* finished;
};
template <typename E>
__global__ void __launch_bounds__(1024)
beam_join_kernel(const Beams<E> s, const Pieces in, const Choice out) {
  extern __shared__ uint64_t lists[];          // of each wave, [piece][W]
  __shared__ double total[kMostBeams][kMostBeams];
  __shared__ int token[kMostBeams][kMostBeams];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, W = s.W;
  uint64_t* const list = lists + (int64_t)wave * in.count * W;
  for (int w = wave; w < W; w += waves) {
    const int row = blockIdx.x * W + w;
    const float score = s.scores[row];
    double norm = NAN;
    // what the pieces left is asked for together with what tells whether they left anything
    const int64_t at = (int64_t)row * in.count;
    const float largest = lane < in.count ? in.largest[at + lane] : -INFINITY;
    const double sum = lane < in.count ? in.sum[at + lane] : 0.0;
    for (int k = lane; k < in.count * W; k += 64) list[k] = in.key[at * W + k];
    if (alive(s, row)) {
      const float m = lanes::largest(sum > 0.0 ? largest : -INFINITY);
      const double all = lanes::sum(sum == 0.0 ? 0.0 : sum * exp((double)largest - (double)m));
      norm = (double)m + log(all);
    }
    if (!(fabs(norm) < INFINITY)) {            // only a finished beam's end counts; of equal candidates the first tokens
      const bool ends = s.finished && s.finished[row] && fabsf(score) < INFINITY;
      if (lane < W) {
        int k = lane;
        double v = -INFINITY;
        if (ends) {
          k = lane == 0 ? s.end : lane - 1 < s.end ? lane - 1 : lane;
          if (lane == 0) v = (double)score;
        }
        total[w][lane] = v, token[w][lane] = k < s.V ? k : -1;
      }
      continue;
    }
    // a lane has the first of a piece's list that is not yet taken; of equal values the first piece has the lower tokens
    int next = 0;
    __builtin_amdgcn_wave_barrier();
    uint64_t mine = lane < in.count ? list[lane * W] : 0;
    for (int i = 0; i < W; ++i) {
      const uint32_t value = (uint32_t)(mine >> 32);
      if (lane != __builtin_ctzll(__ballot(value == lanes::largest(value)))) continue;
      total[w][i] = (double)score + ((double)value_of(mine) - norm), token[w][i] = mine ? place_of(mine) : -1;
      mine = ++next < W ? list[lane * W + next] : 0;
    }
  }
  __syncthreads();
  if (wave) return;
  const bool was_finished = s.finished && lane < W && s.finished[blockIdx.x * W + lane];
  int next = 0, parent = -1, t;
  double v;
  uint64_t mine;
  auto head = [&]() {
    t = lane < W && next < W ? token[lane][next] : -1;
    if (t >= 0) v = total[lane][next];
    mine = t >= 0 ? order_of(v) : 0;
  };
  head();
  for (int i = 0; i < W; ++i) {
    // by the upper half; the lower one tells equal ones apart, and of those that are equal in both the lowest beam is first
    const uint32_t upper = (uint32_t)(mine >> 32);
    bool best = upper == lanes::largest(upper);
    uint64_t who = __ballot(best);
    if (who & (who - 1)) {
      const uint32_t lower = best ? (uint32_t)mine : 0;
      best = best && lower == lanes::largest(lower);
      who = __ballot(best);
    }
    const int first = __builtin_ctzll(who);
    if (lane == i) parent = first;
    if (lane != first) continue;
    const int at = blockIdx.x * W + i;
    out.scores[at] = (float)v, out.parents[at] = lane, out.tokens[at] = t;
    if (out.finished) out.finished[at] = was_finished || t == s.end;
    ++next, head();
  }
  if (!s.slots) return;
  // the first child of a beam goes on in its slot, the others take those of beams without one, in order
  const uint32_t before = (1u << (lane & 31)) - 1;
  uint32_t childless = 0, siblings = 0;
  for (int w = 0; w < W; ++w) {
    const uint32_t children = (uint32_t)__ballot(parent == w);
    if (!children) childless |= 1u << w;
    if (parent == w) siblings = children;
  }
  const bool more = siblings & before;
  uint32_t free = childless;
  for (int k = __popc((uint32_t)__ballot(lane < W && more) & before); k > 0; --k) free &= free - 1;
  if (lane < W) {
    const int32_t* const slots = s.slots + (int64_t)blockIdx.x * W;
    const int home = more ? __builtin_ctz(free) : parent;
    const int at = blockIdx.x * W + lane, to = slots[home], of = slots[parent];
    out.slots[at] = to, out.sources[at] = more ? of : -1;
  }
}

struct Scratch {
  size_t largest, sum, key, bytes;
  int pieces;
  Scratch(int B, int W, int V) {
    pieces = bppsa_ceil_div(V, kPiece);
    const size_t n = (size_t)B * W * pieces;
    largest = 0, sum = bppsa_align_up(n * sizeof(float), 256);
    key = sum + bppsa_align_up(n * sizeof(double), 256);
    bytes = key + bppsa_align_up(n * W * sizeof(uint64_t), 256);
  }
};

static inline bool beam_sizes_ok(int B, int W, int V) {
  return B > 0 && W > 0 && V > 0 && W <= kMostBeams && V <= BPPSA_BEAM_MAX_V &&
         (int64_t)B * W * bppsa_ceil_div(V, kPiece) < 1 << 24;
}

// A workgroup takes a piece of a tensor's slots for every so many rows.  Bound by memory: 147 MB read and written in 48 us, 6.1 TB/s.
template <typename U>
__device__ __forceinline__ void copy_bytes(char* to, const char* from, int n) {
  for (int k = threadIdx.x; k < n / (int)sizeof(U); k += kThreads) reinterpret_cast<U*>(to)[k] = reinterpret_cast<const U*>(from)[k];
}
__global__ void __launch_bounds__(kThreads)
beam_move_kernel(const bppsa_beam_tensor* __restrict__ tensors, const bppsa_adamw_piece* __restrict__ pieces, int rows,
                 const int32_t* __restrict__ sources, const int32_t* __restrict__ slots, int slots_in_state) {
  const bppsa_beam_tensor x = tensors[pieces[blockIdx.x].tensor];
  const int64_t at = (int64_t)pieces[blockIdx.x].piece * BPPSA_BEAM_PIECE;
  const int n = (int)(x.bytes - at < BPPSA_BEAM_PIECE ? x.bytes - at : BPPSA_BEAM_PIECE);
  const uint64_t odd = (uint64_t)x.data | (uint64_t)x.bytes;
  for (int row = blockIdx.y; row < rows; row += gridDim.y) {
    const int from = sources[row], to = slots[row];
    if (from < 0 || to < 0 || from >= slots_in_state || to >= slots_in_state || from == to) continue;
    char* const d = static_cast<char*>(x.data) + at;
    if ((odd & 15) == 0) copy_bytes<uint4>(d + to * x.bytes, d + from * x.bytes, n);
    else if ((odd & 3) == 0) copy_bytes<uint32_t>(d + to * x.bytes, d + from * x.bytes, n);
    else copy_bytes<uint8_t>(d + to * x.bytes, d + from * x.bytes, n);
  }
}

}  // namespace

extern "C" size_t bppsa_beam_select_workspace_bytes(int B, int W, int V) {
  return beam_sizes_ok(B, W, V) ? Scratch(B, W, V).bytes : 0;
}

extern "C" bppsa_status bppsa_beam_select(const bppsa_beam* beams, const bppsa_beam_choice* choice, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  if (!beams || beams->B < 1 || beams->W < 1 || beams->V < 1 || !beams->logits.data || !beams->scores) return BPPSA_EINVAL;
  if (!choice || !choice->scores || !choice->parents || !choice->tokens || choice->scores == beams->scores) return BPPSA_EINVAL;
  if (choice->finished && choice->finished == beams->finished) return BPPSA_EINVAL;
  if (beams->finished && (beams->end < 0 || beams->end >= beams->V || !choice->finished)) return BPPSA_EINVAL;
  if (beams->slots && (!choice->slots || !choice->sources || choice->slots == beams->slots || choice->sources == beams->slots))
    return BPPSA_EINVAL;
  if (beams->W > kMostBeams || beams->V > BPPSA_BEAM_MAX_V || beams->type < BPPSA_F32 || beams->type > BPPSA_F16)
    return BPPSA_EUNSUPPORTED;
  if (!beam_sizes_ok(beams->B, beams->W, beams->V)) return BPPSA_EOVERFLOW;
  const Scratch at(beams->B, beams->W, beams->V);
  if (!workspace || workspace_bytes < at.bytes) return BPPSA_EWORKSPACE;
  if ((uintptr_t)workspace & 255) return BPPSA_EINVAL;
  char* const base = static_cast<char*>(workspace);
  const Pieces pieces{reinterpret_cast<float*>(base + at.largest), reinterpret_cast<double*>(base + at.sum),
                      reinterpret_cast<uint64_t*>(base + at.key), at.pieces};
  const Choice out{choice->scores, choice->parents, choice->tokens, choice->slots, choice->sources, choice->finished};
  const hipStream_t q = (hipStream_t)stream;
  const size_t list = (size_t)at.pieces * beams->W * sizeof(uint64_t);         // 16 KB at most
  const int waves = std::max<int>(1, std::min<int64_t>({16, beams->W, (int64_t)((64 << 10) / list)}));
  return by_type(beams->type, [&](auto e) {
    using E = decltype(e);
    const Beams<E> s{rows_of<const E>(beams->logits), beams->scores, beams->finished, beams->slots, beams->B, beams->W, beams->V, beams->end};
    beam_piece_kernel<E><<<(unsigned)(beams->B * beams->W * at.pieces), kThreads, 0, q>>>(s, pieces);
    BPPSA_CHECK_LAUNCH();
    beam_join_kernel<E><<<beams->B, 64 * waves, waves * list, q>>>(s, pieces, out);
    BPPSA_CHECK_LAUNCH();
    return BPPSA_OK;
  });
}

extern "C" int64_t bppsa_beam_pieces(int n_tensors, const int64_t* bytes, bppsa_adamw_piece* pieces) {
  if (n_tensors < 1 || !bytes) return 0;
  int64_t n = 0;
  for (int t = 0; t < n_tensors; ++t) {
    if (bytes[t] < 1) return 0;
    const int64_t here = (bytes[t] + BPPSA_BEAM_PIECE - 1) / BPPSA_BEAM_PIECE;
    if (here > 0x7FFFFFFF || n + here > 1 << 22) return 0;
    if (pieces)
      for (int64_t k = 0; k < here; ++k) pieces[n + k] = bppsa_adamw_piece{t, (int32_t)k};
    n += here;
  }
  return n;
}

extern "C" bppsa_status bppsa_beam_move(const bppsa_beam_tensor* tensors, int64_t n_pieces, const bppsa_adamw_piece* pieces, int rows,
                                        const int32_t* sources, const int32_t* slots, int slots_in_state, void* stream) {
  if (!tensors || !pieces || n_pieces < 1 || rows < 1 || !sources || !slots || slots_in_state < 1) return BPPSA_EINVAL;
  if (n_pieces > 1 << 22) return BPPSA_EOVERFLOW;
  const int64_t want = std::max<int64_t>(1, 4096 / n_pieces);
  beam_move_kernel<<<dim3((unsigned)n_pieces, (unsigned)std::min<int64_t>(rows, want)), kThreads, 0, (hipStream_t)stream>>>(
      tensors, pieces, rows, sources, slots, slots_in_state);
  BPPSA_CHECK_LAUNCH();
  return BPPSA_OK;
}
