// Logits as a sampler wants them: penalties for tokens that a row has seen, a bias, and a mask of allowed tokens; and the gradient through them.
//
// With n the number of times that row r has seen token j (its history is a range of a list of tokens, ranges may overlap):
//   z = x                                          if n = 0
//   z = (x > 0 ? x / repetition : x repetition) - presence   otherwise
//   out = z - frequency n + bias[j];  -inf where the mask has no bit
// and backwards d = g, g / repetition or g repetition by the same distinction, 0 where the mask has no bit.  In fp32, rounded once.
//
// One pass over the logits, bound by memory.  A workgroup takes a slice of a row and counts the row's history for its slice in LDS, in whole
// numbers, so the order of the additions does not show; the history is read once a slice and comes from L2.  Backwards two bits a token do, whether it was
// seen and whether its logit is above 0, and logits are read only where a token was seen.  2048 x 32000 bf16 backwards (264 MB) 53 us, 5.0 TB/s; 256 x 50265 with a
// bias, masks and 1500 tokens seen a row (54 MB) 14.6 us, 3.7 TB/s: a row's tokens, counted before the first result leaves, show there; 1 x 32000 4.0 us.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace hift {
namespace {

constexpr int BLK = 512;
constexpr int LOOSE = 8;  // elements before the first aligned piece: at most 7
constexpr int U = 2;      // pieces of 16 bytes of a thread, at most: LDS holds a count for each entry, and four workgroups fill a compute unit

struct AdjustArgs {
  int V, slice, slices;
  int64_t rows, ld, ldo, ldg;
  const void* x;
  const void* g;  // backward: the gradient that comes in
  void* out;
  const int32_t* tokens;
  int64_t n_tokens;
  const int64_t *begin, *end;
  float repetition, inverse, presence, frequency;
  const float* bias;
  int64_t ld_bias;
  const uint32_t* allowed;
  int64_t ld_allowed;
  bool aligned;  // rows of all matrices lie alike within 16 bytes
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// x: the logit, or backward the gradient; n: the count, backward 1 for a seen token and -1 for one whose logit is above 0
template <bool BWD>
__device__ __forceinline__ float adjusted(float x, int n, float bias, bool allowed, const AdjustArgs& p) {
  if constexpr (BWD) {
    if (!allowed) return 0.f;
    return n == 0 ? x : n < 0 ? x * p.inverse : x * p.repetition;
  } else {
    if (!allowed) return -INFINITY;
    const float z = n > 0 ? (x > 0.f ? x * p.inverse : x * p.repetition) - p.presence : x;
    return z - p.frequency * (float)n + bias;
  }
}

// PAST: large matrices are read and written past the caches.
template <typename T, bool BWD, bool PAST>
__global__ void __launch_bounds__(BLK) adjust_k(AdjustArgs p) {
  // forward counts [LOOSE + slice], in whole quads; backward bits [2][(LOOSE + slice) / 32]: seen, and above 0.  The first aligned piece is at LOOSE.
  extern __shared__ int4 count_quads[];
  int* counts = reinterpret_cast<int*>(count_quads);
  const int words = (LOOSE + p.slice) / 32 + 1;
  __shared__ int any;
  constexpr int E = 16 / (int)sizeof(T);
  const int64_t row = blockIdx.x / (unsigned)p.slices;
  const int part = (int)(blockIdx.x % (unsigned)p.slices);
  const T* x = (const T*)p.x + row * p.ld;
  const T* g = BWD ? (const T*)p.g + row * p.ldg : nullptr;
  T* out = (T*)p.out + row * p.ldo;
  // slices begin at aligned pieces of the row; the first has the elements before them, too
  const int head = p.aligned ? min(p.V, (int)((16 - (reinterpret_cast<uintptr_t>(BWD ? g : x) & 15)) & 15) / (int)sizeof(T)) : 0;
  const int lo = part ? (int)min((int64_t)p.V, (int64_t)head + (int64_t)part * p.slice) : 0;
  const int hi = part + 1 == p.slices ? p.V : (int)min((int64_t)p.V, (int64_t)head + (int64_t)(part + 1) * p.slice);
  const int n = hi - lo;
  if (n <= 0) return;
  const int from = part ? lo : head, shift = LOOSE - (from - lo);  // counts[shift + j - lo] is element j's
  const int t = threadIdx.x, pieces = p.aligned ? (hi - from) / E : 0;
  // what the pass streams is on its way while the history is counted
  typedef Vec<T, E> P;
  P in[U];
  uint64_t let[U];
  f32x4_any add[U][E / 4];
  const float* bias = p.bias ? p.bias + row * p.ld_bias : nullptr;
  const uint32_t* allowed = p.allowed ? p.allowed + row * p.ld_allowed : nullptr;
#pragma unroll
  for (int k = 0; k < U; ++k)
    if (t + k * BLK < pieces) {
      const int j0 = from + (t + k * BLK) * E;
      const f32x4* piece = reinterpret_cast<const f32x4*>((BWD ? g : x) + j0);
      in[k] = __builtin_bit_cast(P, PAST ? __builtin_nontemporal_load(piece) : *piece);
      if (allowed) let[k] = (uint64_t)allowed[(j0 + E - 1) >> 5] << 32 | allowed[j0 >> 5];
      if (!BWD && bias) {
#pragma unroll
        for (int e = 0; e < E / 4; ++e) add[k][e] = *reinterpret_cast<const f32x4_any*>(bias + j0 + 4 * e);
      }
    }
  bool seen = false;
  if (p.tokens) {
    const int64_t b = min(max(p.begin[row], (int64_t)0), p.n_tokens), e = min(max(p.end[row], b), p.n_tokens);
    if (e > b) {
      if (t == 0) any = 0;
      if (BWD)
        for (int i = t; i < 2 * words; i += BLK) counts[i] = 0;
      else
        for (int i = t; i < (shift + n + 3) / 4; i += BLK) count_quads[i] = make_int4(0, 0, 0, 0);
      __syncthreads();
      int mine = 0;
      for (int64_t i = b + t; i < e; i += BLK) {
        const unsigned at = (unsigned)p.tokens[i] - (unsigned)lo;
        if (at < (unsigned)n) {
          const int j = shift + (int)at;
          mine = 1;
          if constexpr (BWD) {
            // the first to meet the token looks its logit up, all of them at the same time
            const int had = atomicOr(&counts[j >> 5], 1 << (j & 31));
            if (!(had >> (j & 31) & 1) && to_f32(x[lo + (int)at]) > 0.f) atomicOr(&counts[words + (j >> 5)], 1 << (j & 31));
          } else {
            atomicAdd(&counts[j], 1);
          }
        }
      }
      if (mine) any = 1;
      __syncthreads();
      seen = any != 0;
    }
  }
  auto one = [&](int j) __attribute__((always_inline)) {
    int c = 0;
    if (seen) {
      const int i = shift + j - lo;
      if constexpr (BWD) c = counts[i >> 5] >> (i & 31) & 1 ? (counts[words + (i >> 5)] >> (i & 31) & 1 ? -1 : 1) : 0;
      else c = counts[i];
    }
    const bool let = !allowed || (allowed[j >> 5] >> (j & 31) & 1);
    out[j] = from_f32<T>(adjusted<BWD>(to_f32((BWD ? g : x)[j]), c, !BWD && bias ? bias[j] : 0.f, let, p));
  };
  if (!p.aligned) {
    for (int j = lo + t; j < hi; j += BLK) one(j);
    return;
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int i = t + k * BLK;
    if (i >= pieces) break;
    const int j0 = from + i * E;
    int c[E];
    if constexpr (BWD) {
      const int b = LOOSE + i * E, w = seen ? counts[b >> 5] >> (b & 31) : 0, above = seen ? counts[words + (b >> 5)] >> (b & 31) : 0;  // a piece lies in one word
#pragma unroll
      for (int e = 0; e < E; ++e) c[e] = w >> e & 1 ? (above >> e & 1 ? -1 : 1) : 0;
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const int4 q = seen ? count_quads[(LOOSE + i * E + e) / 4] : make_int4(0, 0, 0, 0);
        c[e] = q.x; c[e + 1] = q.y; c[e + 2] = q.z; c[e + 3] = q.w;
      }
    }
    const uint32_t bits = allowed ? (uint32_t)(let[k] >> (j0 & 31)) : 0xFFFFFFFFu;
    P o;
#pragma unroll
    for (int e = 0; e < E; ++e) o.v[e] = from_f32<T>(adjusted<BWD>(to_f32(in[k].v[e]), c[e], !BWD && bias ? add[k][e / 4][e % 4] : 0.f, bits >> e & 1, p));
    f32x4* piece = reinterpret_cast<f32x4*>(out + j0);
    if (PAST) __builtin_nontemporal_store(__builtin_bit_cast(f32x4, o), piece);
    else *piece = __builtin_bit_cast(f32x4, o);
  }
  // what is left before the first piece and after the last
  if (part == 0 && t < head) one(t);
  const int tail = from + pieces * E;
  if (t < hi - tail) one(tail + t);
}

template <typename T, bool BWD>
hipError_t run(AdjustArgs p, hipStream_t st) {
  // Slices: U pieces a thread, fewer where rows are few, down to one.  bf16, us, one piece / two: 1 x 32000 3.5 / 4.2, 32 x 32000 3.8 / 4.5, 512 x 32000 17.6 / 16.8,
  // 2048 x 50000 107 / 90 (through the caches).
  constexpr int E = 16 / (int)sizeof(T);
  p.slice = U * BLK * E;
  while (p.slice > BLK * E && p.rows * ((p.V + p.slice - 1) / p.slice) < 512) p.slice /= 2;
  p.slices = (int)(((int64_t)p.V + p.slice - 1) / p.slice);
  if (p.rows * p.slices > 0x7FFFFFFF) return hipErrorInvalidValue;
  const auto low = [](const void* q) { return (int64_t)(reinterpret_cast<uintptr_t>(q) & 15); };
  p.aligned = low(p.out) == low(BWD ? p.g : p.x) && (p.ldo - (BWD ? p.ldg : p.ld)) % E == 0;
  const size_t lds = BWD ? ((LOOSE + p.slice) / 32 + 1) * 8 : (size_t)(LOOSE + p.slice + 4) * 4;
  // Matrices that fill the last-level cache (256 MB) for a good part leave nothing there for who reads the result.  bf16, 512 tokens seen a row, us, past the caches /
  // through them: 2048 x 50000 79 / 89, its gradient 85 / 105; 512 x 32000 with the log probabilities read from the result 30.8 / 28.8, 2048 x 32000 with them 80 / 84.
  const bool past = p.rows * p.V * 2 * (int64_t)sizeof(T) >= int64_t(1) << 26;
  const unsigned grid = (unsigned)(p.rows * p.slices);
  if (past) adjust_k<T, BWD, true><<<grid, BLK, lds, st>>>(p);
  else adjust_k<T, BWD, false><<<grid, BLK, lds, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t adjust_logits(int dt, bool backward, int64_t rows, int V, int64_t ld, const void* x, const AdjustBy& by, int64_t ldg, const void* g, int64_t ldo,
                         void* out, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  AdjustArgs p{};
  p.V = V; p.rows = rows; p.ld = ld; p.ldo = ldo; p.ldg = ldg; p.x = x; p.g = g; p.out = out;
  // penalties that change nothing need no history
  const bool neutral = by.repetition == 1.f && (backward || (by.presence == 0.f && by.frequency == 0.f));
  p.tokens = neutral ? nullptr : by.tokens;
  p.n_tokens = by.n_tokens; p.begin = by.begin; p.end = by.end;
  p.repetition = by.repetition; p.inverse = 1.f / by.repetition; p.presence = by.presence; p.frequency = by.frequency;
  p.bias = backward ? nullptr : by.bias; p.ld_bias = by.ld_bias;
  p.allowed = by.allowed; p.ld_allowed = by.ld_allowed;
  if (dt == DT_BF16) return backward ? run<bf16, true>(p, st) : run<bf16, false>(p, st);
  return backward ? run<float, true>(p, st) : run<float, false>(p, st);
}

}  // namespace hift
