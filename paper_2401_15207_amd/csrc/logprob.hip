// Log probabilities of given tokens with the entropy of each row and its most probable alternatives, and the gradient of both.
//
// Row r of the logits x, scale s (the reciprocal of a temperature), z = s x, m = max z, S = sum exp(z - m):
//   logp_j = (z_j - m) - ln S,   p_j = exp(logp_j),   H = ln S - sum exp(z - m) (z - m) / S
//   d/dz_j of logp_y = 1(j = y) - p_j,   of H = -p_j (logp_j + H)
// All of it is formed in 32 bits from logits of either type; exponentials are powers of two of z log2(e).
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace hift {
namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr double LN2 = 0.69314718055994530942;
constexpr int CANDIDATES = 1024;  // entries that may be at or above a row's threshold before it goes the slow way

struct LogprobArgs {
  int V, top;
  int64_t ld;
  const void* logits;
  const int32_t* targets;
  float scale;
  float *logp, *entropy, *stats, *top_logp;
  int32_t* top_ids;
};

// Values as whole numbers of the same order: NaN of either sign above everything, -0 equal to 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
// Larger value first, then smaller id.
__device__ __forceinline__ uint64_t top_key(float x, int id) { return (uint64_t)ordered(x) << 32 | (0xFFFFFFFFu - (uint32_t)id); }
__device__ __forceinline__ int key_id(uint64_t k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// A row seen by a workgroup of NT threads: pieces of 16 bytes from its first aligned element on, thread t taking t, t + NT, ..., and the
// elements before and after them (fewer than a piece at either end), one each for the first threads.
template <typename T, int NT>
struct RowOf {
  static constexpr int E = 16 / (int)sizeof(T);
  const T* x;
  int V, head, pieces, tail;
  __device__ RowOf(const T* row, int V_) : x(row), V(V_) {
    head = min(V, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T));
    pieces = (V - head) / E;
    tail = V - head - pieces * E;
  }
  // the one element outside the pieces that is thread t's, or -1
  __device__ int loose(int t) const { return t < head ? t : t < head + tail ? V - tail + (t - head) : -1; }
  // f(value, id) for every element of thread t
  template <class F>
  __device__ __forceinline__ void each(int t, F f) const {
    for (int i = t; i < pieces; i += NT) {
      const Vec<T, E> v = *reinterpret_cast<const Vec<T, E>*>(x + head + (int64_t)i * E);
#pragma unroll
      for (int e = 0; e < E; ++e) f(to_f32(v.v[e]), head + i * E + e);
    }
    const int l = loose(t);
    if (l >= 0) f(to_f32(x[l]), l);
  }
};

template <int NW>
__device__ __forceinline__ uint64_t block_max64(uint64_t v, uint64_t* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t w = __shfl_xor((unsigned long long)v, o, 64);
    v = w > v ? w : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) v = red[i] > v ? red[i] : v;
  return v;
}

// One workgroup a row.
// The alternatives: the k-th largest of the maxima of 64 disjoint parts of the row is at most its k-th largest entry, and few entries are
// at or above it (the parts interleave); those are collected and each counts how many of them precede it.  Rows where they are more than
// the list holds, or that hold NaN or +inf, take the largest key below the one before, k times.
template <typename T, int NT>
__global__ void __launch_bounds__(NT) logprob_k(LogprobArgs a) {
  constexpr int NW = NT / 64;
  __shared__ float red[NW], parts[64];
  __shared__ uint64_t red64[NW], cand[CANDIDATES];
  __shared__ float tau_s;
  __shared__ int count;
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x;
  const T* x = reinterpret_cast<const T*>(a.logits) + r * a.ld;
  const RowOf<T, NT> row(x, a.V);

  float mine = -INFINITY;
  row.each(t, [&](float v, int) { mine = fmaxf(mine, v); });
  const float mx = block_max<NW>(mine, red);
  const float c = a.scale * LOG2E;
  const float m2 = mx == -INFINITY ? 0.f : mx * c;
  float s = 0.f, u = 0.f;
  row.each(t, [&](float v, int) {
    const float d = fmaf(v, c, -m2), e = __builtin_amdgcn_exp2f(d);
    s += e;
    u = fmaf(e, fmaxf(d, -1024.f), u);  // (0 times the -inf of a masked entry)
  });
  s = block_sum<NW>(s, red);
  u = block_sum<NW>(u, red);
  // m2 is the rounded maximum in powers of two; the sum that goes with the rounded maximum itself:
  const float m = mx == -INFINITY ? 0.f : mx * a.scale;
  const float ln_s = s > 0.f ? (float)(log((double)s) + ((double)m2 * LN2 - (double)m)) : s == 0.f ? -INFINITY : s;
  if (t == 0) {
    if (a.logp) {
      const int y = a.targets[r];
      a.logp[r] = y < 0 || y >= a.V ? 0.f : s == 0.f ? -INFINITY : fmaf(to_f32(x[y]), a.scale, -m) - ln_s;
    }
    if (a.entropy) a.entropy[r] = s == 0.f ? 0.f : (float)(log((double)s) - LN2 * (double)u / (double)s);
    if (a.stats) {
      a.stats[2 * r] = m;
      a.stats[2 * r + 1] = ln_s;
    }
  }
  const int k = a.top;
  if (k == 0) return;
  float* top_logp = a.top_logp + r * k;
  int32_t* top_ids = a.top_ids + r * k;
  auto put = [&](int at, float v, int id) {
    top_ids[at] = id;
    top_logp[at] = s == 0.f ? -INFINITY : fmaf(v, a.scale, -m) - ln_s;
  };

  // threshold
  float part = mine;
#pragma unroll
  for (int o = 1; o < NT / 64; o <<= 1) part = fmaxf(part, __shfl_xor(part, o, 64));
  if (t % (NT / 64) == 0) parts[t / (NT / 64)] = part;
  if (t == 0) count = 0;
  __syncthreads();
  if (t < 64) {
    const float p = parts[t];
    int before = 0;
    for (int j = 0; j < 64; ++j) before += parts[j] > p || (parts[j] == p && j < t);
    if (before == k - 1) tau_s = p;
  }
  __syncthreads();
  const float tau = tau_s;
  const bool plain = s < INFINITY;  // neither NaN nor +inf in the row
  if (plain && mine >= tau)
    row.each(t, [&](float v, int id) {
      if (v >= tau && v > -INFINITY) {
        const int at = atomicAdd(&count, 1);
        if (at < CANDIDATES) cand[at] = top_key(v, id);
      }
    });
  __syncthreads();
  const int n = count;
  if (plain && n <= CANDIDATES) {
    for (int i = t; i < n; i += NT) {
      const uint64_t key = cand[i];
      int before = 0;
      for (int j = 0; j < n; ++j) before += cand[j] > key;
      if (before < k) put(before, unordered(key >> 32), key_id(key));
    }
    if (n < k && t < 64) {  // fewer entries than asked for are above -inf: the first masked ones follow
      int at = n;
      for (int base = 0; at < k && base < a.V; base += 64) {
        const bool masked = base + t < a.V && to_f32(x[base + t]) == -INFINITY;
        const uint64_t b = __ballot(masked);
        const int to = at + __popcll(b & ((1ull << t) - 1));
        if (masked && to < k) put(to, -INFINITY, base + t);
        at += __popcll(b);
      }
    }
    return;
  }
  uint64_t last = ~0ull;
  for (int i = 0; i < k; ++i) {
    uint64_t best = 0;
    row.each(t, [&](float v, int id) {
      const uint64_t key = top_key(v, id);
      if (key < last && key > best) best = key;
    });
    last = block_max64<NW>(best, red64);
    if (t == 0) {
      const int id = key_id(last);
      put(i, to_f32(x[id]), id);
    }
  }
}

struct LogprobBwdArgs {
  int V, parts;
  int64_t ld, ldd;
  const void* logits;
  const int32_t* targets;
  float scale;
  const float *stats, *entropy, *d_logp, *d_entropy;
  void* dlogits;
  int zero_to;  // entries [V, zero_to) of a row of the gradient are set to 0
};

constexpr int BWD_THREADS = 256;

// `parts` workgroups a row.  An element is read and written by one thread, so the gradient may take the logits' place.
template <typename T, int E>
__global__ void __launch_bounds__(BWD_THREADS) logprob_bwd_k(LogprobBwdArgs a) {
  const int64_t r = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  const T* x = reinterpret_cast<const T*>(a.logits) + r * a.ld;
  T* dx = reinterpret_cast<T*>(a.dlogits) + r * a.ldd;
  const float m = a.stats[2 * r], ln_s = a.stats[2 * r + 1];
  const int y = a.targets ? a.targets[r] : -1;
  const bool has = y >= 0 && y < a.V;
  const float g = has && a.d_logp ? a.d_logp[r] : 0.f;
  const float h = a.d_entropy ? a.d_entropy[r] : 0.f;
  const float gh = a.d_entropy ? fmaf(h, a.entropy[r], g) : g;
  const bool empty = ln_s == -INFINITY;  // nothing but masked entries: no gradient
  auto one = [&](float v, int j) {
    const float lp = fmaf(v, a.scale, -m) - ln_s;
    const float p = __builtin_amdgcn_exp2f(lp * LOG2E);
    float d = -p * fmaf(h, fmaxf(lp, -1024.f), gh);  // (0 times the -inf of a masked entry)
    if (j == y) d += g;
    return empty ? 0.f : d * a.scale;
  };
  const int head = E == 1 ? 0 : min(a.V, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T));
  const int pieces = (a.V - head) / E;
  for (int i = part * BWD_THREADS + threadIdx.x; i < pieces; i += a.parts * BWD_THREADS) {
    const int at = head + i * E;
    Vec<T, E> v = *reinterpret_cast<const Vec<T, E>*>(x + at);
#pragma unroll
    for (int e = 0; e < E; ++e) v.v[e] = from_f32<T>(one(to_f32(v.v[e]), at + e));
    *reinterpret_cast<Vec<T, E>*>(dx + at) = v;
  }
  if (part != 0) return;
  const int t = threadIdx.x, tail = a.V - head - pieces * E;
  const int l = t < head ? t : t < head + tail ? a.V - tail + (t - head) : -1;
  if (l >= 0) dx[l] = from_f32<T>(one(to_f32(x[l]), l));
  for (int j = a.V + t; j < a.zero_to; j += BWD_THREADS) dx[j] = from_f32<T>(0.f);
}

template <typename T>
hipError_t launch_logprob(int64_t rows, const LogprobArgs& a, hipStream_t st) {
  logprob_k<T, 512><<<(uint32_t)rows, 512, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_logprob_bwd(int64_t rows, LogprobBwdArgs a, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  // pieces of 16 bytes where a row of the gradient lies in them as its row of logits does
  const uintptr_t off = reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.dlogits);
  const bool alike = (off & 15) == 0 && (rows == 1 || (a.ld - a.ldd) * (int64_t)sizeof(T) % 16 == 0);
  const int per = BWD_THREADS * (alike ? E : 1) * 4;
  a.parts = (int)std::min<int64_t>((a.V + per - 1) / per, std::max<int64_t>(1, (int64_t(1) << 23) / rows));
  const uint32_t grid = (uint32_t)(rows * a.parts);
  if (alike) logprob_bwd_k<T, E><<<grid, BWD_THREADS, 0, st>>>(a);
  else logprob_bwd_k<T, 1><<<grid, BWD_THREADS, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t token_logprob(int dt, int64_t rows, int V, int64_t ld, const void* logits, const int32_t* targets, float scale, int top, float* logp,
                         float* entropy, float* stats, float* top_logp, int32_t* top_ids, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  const LogprobArgs a{V, top, ld, logits, targets, scale, logp, entropy, stats, top_logp, top_ids};
  return dt == DT_BF16 ? launch_logprob<bf16>(rows, a, st) : launch_logprob<float>(rows, a, st);
}

hipError_t token_logprob_bwd(int dt, int64_t rows, int V, int64_t ld, const void* logits, const int32_t* targets, float scale, const float* stats,
                             const float* entropy, const float* d_logp, const float* d_entropy, int64_t ldd, void* dlogits, int zero_to, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  const LogprobBwdArgs a{V, 1, ld, ldd, logits, targets, scale, stats, entropy, d_logp, d_entropy, dlogits, zero_to};
  return dt == DT_BF16 ? launch_logprob_bwd<bf16>(rows, a, st) : launch_logprob_bwd<float>(rows, a, st);
}

}  // namespace hift
