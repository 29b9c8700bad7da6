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
constexpr float LN2_HI = 0.69314718246459960938f, LN2_LO = -1.904654299957767e-9f;  // ln 2 = LN2_HI + LN2_LO
constexpr float LOWEST = -3.402823466e38f;
constexpr int CANDIDATES = 1024;  // entries that may be at or above a row's threshold before it goes the slow way

// Near rows, whose largest z is at most NEAR from 0, are summed against references that are rounded products: z's rounding shows in what is summed, by
// 2^-24 of the largest z.  In the others, far ones, every z is rounded and the largest subtracted from it first, which is exact where it matters.
constexpr float NEAR = 4096.f;
__device__ __forceinline__ bool is_near(float m) { return fabsf(m) <= NEAR; }
// z of a far row.  Beyond fp32's range a finite logit's z is the largest number of its sign.
__device__ __forceinline__ float far_z(float x, float scale) {
  const float z = x * scale;
  return fabsf(x) <= -LOWEST ? fminf(fmaxf(z, LOWEST), -LOWEST) : z;
}
// z - m in a row whose largest z is m
__device__ __forceinline__ float below(float x, float scale, float m, bool near) { return near ? fmaf(x, scale, -m) : far_z(x, scale) - m; }

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

// A row seen by a workgroup of NT threads: pieces of 16 bytes from its first aligned element on, thread t taking t, t + NT, ..., U at a time,
// and the elements before and after them (fewer than a piece at either end), one each for the first threads.
template <typename T>
struct Piece {
  static constexpr int E = 16 / (int)sizeof(T);
  hift_u32x4 w;
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
  }
};
template <typename T, int NT>
struct RowOf {
  static constexpr int E = Piece<T>::E, U = 4;
  const T* x;
  int V, t, head, pieces, loose_id;
  float loose;
  __device__ __forceinline__ RowOf(const T* row, int V_) : x(row), V(V_), t(threadIdx.x) {
    head = min(V, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T));
    pieces = (V - head) / E;
    const int tail = V - head - pieces * E;
    loose_id = t < head ? t : t < head + tail ? V - tail + (t - head) : -1;
    loose = loose_id >= 0 ? to_f32(x[loose_id]) : -INFINITY;
  }
  // pieces i, i + NT, ..; those past the end as -inf
  __device__ __forceinline__ void load(Piece<T> (&p)[U], int i) const {
    constexpr uint32_t MASKED = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
#pragma unroll
    for (int k = 0; k < U; ++k) {
      p[k].w = hift_u32x4{MASKED, MASKED, MASKED, MASKED};
      if (i + k * NT < pieces) p[k].w = *reinterpret_cast<const hift_u32x4*>(x + head + (int64_t)(i + k * NT) * E);
    }
  }
  // f(value, id) for every element of the thread
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    for (int i = t; i < pieces; i += NT) {
      const Piece<T> p{*reinterpret_cast<const hift_u32x4*>(x + head + (int64_t)i * E)};
#pragma unroll
      for (int e = 0; e < E; ++e) f(p.at(e), head + i * E + e);
    }
    if (loose_id >= 0) f(loose, loose_id);
  }
};

// Within a row of 16 lanes by DPP, across rows by lane swaps: all 64 lanes receive the result.  `group` receives what the 2^STEPS lanes
// around each have by themselves.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, false));
}
template <int STEPS, class Op>
__device__ __forceinline__ float wave_all(float v, Op op, float* group = nullptr) {
  if (STEPS == 0 && group) *group = v;
  v = op(v, dpp<0xB1>(v));   // the other lane of two
  if (STEPS == 1 && group) *group = v;
  v = op(v, dpp<0x4E>(v));   // the other two of four
  if (STEPS == 2 && group) *group = v;
  v = op(v, dpp<0x141>(v));  // the other four of eight (mirrored)
  if (STEPS == 3 && group) *group = v;
  v = op(v, dpp<0x140>(v));  // the other eight of sixteen (mirrored)
  if (STEPS == 4 && group) *group = v;
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

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

// Where a part's largest entry lies in powers of two: what its sums refer to.  Not below -2^24: a large finite mask (-1e10, the type's lowest) has no
// c x that fp32 could hold to within a few powers of two, or at all, and a near row's largest entry is far above; parts without entries
// start there too.
__device__ __forceinline__ float reference_of(float largest, float c) { return fmaxf(largest * c, -16777216.f); }

// Sums of a part of a row against a reference: s = sum 2^d, u = sum 2^d d.  A masked entry has d = -inf and adds 0.
struct Sums {
  float s = 0.f, u = 0.f;
  __device__ __forceinline__ void add(float d) {
    const float e = __builtin_amdgcn_exp2f(d);
    s += e;
    u = fmaf(e, fmaxf(d, -1024.f), u);
  }
  __device__ __forceinline__ void add(float x, float c, float m2) { add(fmaf(x, c, -m2)); }
  // the same against a reference larger by `by` (0 or more)
  __device__ __forceinline__ void shift(float by) {
    const float f = __builtin_amdgcn_exp2f(-by);
    u = f * fmaf(-by, s, u);
    s *= f;
  }
};

// One workgroup a row, one pass over it.  Every wavefront forms its sums against its own largest entry; the first one joins them.  Far rows take
// another pass, against the row's largest (that is all that a mask costs which is not -inf, and only where a row holds nothing else: half of each row at
// the type's lowest value, 2048 x 32000 bf16, 35 us, without 34).
// Bound: the logits' way from memory once rows are many (4096 x 50272 fp32 138 us, 6.0 TB/s; 2048 x 32000 bf16 with 8 alternatives 32 us, 4.1
// TB/s: one exponential and two multiply-adds an entry take as long as its two bytes); the chain of loads, reductions and barriers for one
// (1 x 32000 with 20 alternatives 6 us).  Rows are not split over workgroups: one of 128000 takes 13 us, a launch that joins parts 4 more.
// The alternatives: the k-th largest of the maxima of 64 disjoint parts of the row is at most its k-th largest entry, and few entries are
// at or above it (the parts interleave: 20 of 64 maxima exceed it where about 24 entries do); those are collected and each counts how
// many of them precede it.  Rows where they are more than the list holds, or that hold NaN or +inf, take the largest key below the one
// before, k times.
template <typename T, int NT>
__global__ void __launch_bounds__(NT, NT == 1024 ? 4 : 8) logprob_k(LogprobArgs a) {
  constexpr int NW = NT / 64, STEPS = NT == 64 ? 0 : NT == 256 ? 2 : NT == 512 ? 3 : 4;
  __shared__ float wave_m[NW], wave_s[NW], wave_u[NW];
  __shared__ uint32_t parts[64];
  __shared__ uint64_t red64[NW], cand[CANDIDATES];
  __shared__ float tau_s, ln_s_s, s_s;
  __shared__ int count, look_count, looks[NT];
  const int64_t r = blockIdx.x;
  const int t = threadIdx.x, lane = t & 63;
  const T* x = reinterpret_cast<const T*>(a.logits) + r * a.ld;
  typedef RowOf<T, NT> Row;
  const Row row(x, a.V);
  const float c = a.scale * LOG2E;
  const auto max2 = [](float p, float q) { return fmaxf(p, q); };
  const auto sum2 = [](float p, float q) { return p + q; };

  // One pass: the next pieces are on their way while the sums take the present ones; where those hold a new largest entry the sums are
  // shifted first.  Which pieces held it, and the largest of all others, spare nearly every thread the look for its alternatives.
  float mine = row.loose, second = -INFINITY, group;
  int best = -1;
  float m2 = reference_of(mine, c);
  Sums q;
  if (row.loose_id >= 0) q.add(row.loose, c, m2);
  Piece<T> now[Row::U], next[Row::U];
  if (t < row.pieces) row.load(now, t);
  for (int i = t; i < row.pieces; i += Row::U * NT) {
    if (i + Row::U * NT < row.pieces) row.load(next, i + Row::U * NT);
    float most = -INFINITY;
#pragma unroll
    for (int k = 0; k < Row::U; ++k)
#pragma unroll
      for (int e = 0; e < Row::E; ++e) most = fmaxf(most, now[k].at(e));
    // (the compiler would keep all elements as floats from the one look to the other)
#pragma unroll
    for (int k = 0; k < Row::U; ++k) asm volatile("" : "+v"(now[k].w));
    if (most > mine) {
      const float to = reference_of(most, c);
      q.shift(to - m2);
      second = mine;
      mine = most;
      m2 = to;
      best = i;
    } else {
      second = fmaxf(second, most);
    }
#pragma unroll
    for (int k = 0; k < Row::U; ++k)
#pragma unroll
      for (int e = 0; e < Row::E; ++e) q.add(now[k].at(e), c, m2);
#pragma unroll
    for (int k = 0; k < Row::U; ++k) now[k] = next[k];
  }
  const float wm = wave_all<STEPS>(mine, max2, &group);
  q.shift(reference_of(wm, c) - m2);
  q.s = wave_all<0>(q.s, sum2);
  q.u = wave_all<0>(q.u, sum2);
  const int k = a.top;
  if (lane == 0) {
    wave_m[t >> 6] = wm;
    wave_s[t >> 6] = q.s;
    wave_u[t >> 6] = q.u;
  }
  // 26 bits of the order suffice for a threshold; the rest makes the 64 of them different
  if (t % (NT / 64) == 0) parts[t / (NT / 64)] = (ordered(group) & ~63u) | (63 - t / (NT / 64));
  if (t == 0) count = look_count = 0;
  __syncthreads();
  float mx = wave_m[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) mx = fmaxf(mx, wave_m[w]);
  const float m = mx == -INFINITY ? 0.f : far_z(mx, a.scale);
  const bool near = is_near(m);
  if (!near) {  // (+inf too: it gives NaN here)
    Sums f;
    row.each([&](float v, int) { f.add((far_z(v, a.scale) - m) * LOG2E); });
    f.s = wave_all<0>(f.s, sum2);
    f.u = wave_all<0>(f.u, sum2);
    if (lane == 0) {
      wave_s[t >> 6] = f.s;
      wave_u[t >> 6] = f.u;
    }
    __syncthreads();
  }
  if (t < 64) {
    const float m2 = reference_of(mx, c);
    Sums all;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      Sums p;
      p.s = wave_s[w];
      p.u = wave_u[w];
      if (near) p.shift(m2 - reference_of(wave_m[w], c));
      all.s += p.s;
      all.u += p.u;
    }
    const float s = all.s < INFINITY ? all.s : NAN;
    // a near row's m2 is the rounded maximum in powers of two; ln S is given for the rounded maximum itself
    const float ln = __builtin_amdgcn_logf(s) * LN2_HI;
    const float ln_s = s > 0.f ? ln + (near ? fmaf(m2, LN2_LO, fmaf(m2, LN2_HI, -m)) : 0.f) : s == 0.f ? -INFINITY : s;
    if (t == 0) {
      if (a.logp) {
        const int y = a.targets[r];
        a.logp[r] = y < 0 || y >= a.V ? 0.f : s == 0.f ? -INFINITY : below(to_f32(x[y]), a.scale, m, near) - ln_s;
      }
      if (a.entropy) a.entropy[r] = s == 0.f ? 0.f : ln - LN2_HI * (all.u / s);
      if (a.stats) {
        a.stats[2 * r] = m;
        a.stats[2 * r + 1] = ln_s;
      }
      ln_s_s = ln_s;
      s_s = s;
    }
  }
  if (k > 0 && (NW > 1 ? t >= 64 && t < 128 : true)) {  // (meanwhile)
    const uint32_t p = parts[lane];
    int before = 0;
#pragma unroll
    for (int j = 0; j < 64; ++j) before += parts[j] > p;
    if (before == k - 1) tau_s = (p & ~63u) <= ordered(-INFINITY) ? LOWEST : unordered(p & ~63u);  // (masked entries are never at or above it)
  }
  if (k == 0) return;
  __syncthreads();
  const float s = s_s, ln_s = ln_s_s, tau = tau_s;
  float* top_logp = a.top_logp + r * k;
  int32_t* top_ids = a.top_ids + r * k;
  auto put = [&](int at, float v, int id) {
    top_ids[at] = id;
    top_logp[at] = s == 0.f ? -INFINITY : below(v, a.scale, m, near) - ln_s;
  };
  const bool plain = s < INFINITY;  // neither NaN nor +inf in the row
  const auto collect = [&](float v, int id) {
    if (v >= tau) {
      const int at = atomicAdd(&count, 1);
      if (at < CANDIDATES) cand[at] = top_key(v, id);
    }
  };
  if (plain && mine >= tau) {
    if (second >= tau || best < 0) row.each(collect);
    else looks[atomicAdd(&look_count, 1)] = best;
  }
  __syncthreads();
  // the few threads' pieces, a lane an element
  constexpr int G = Row::U * Row::E;
  for (int j = t / G; j < look_count; j += NT / G) {
    const int i = looks[j] + t % G / Row::E * NT;
    const int id = row.head + i * Row::E + t % Row::E;
    if (i < row.pieces) collect(to_f32(x[id]), id);
  }
  __syncthreads();
  const int n = count;
  if (plain && n <= CANDIDATES) {
    if (n <= 64) {
      if (t >= 64) return;
      const uint64_t key = t < n ? cand[t] : 0;
      int before = 0;
      for (int j = 0; j < n; ++j) {
        const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), j) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)key, j);
        before += other > key;
      }
      if (t < n && before < k) put(before, unordered(key >> 32), key_id(key));
    } else {
      for (int i = t; i < n; i += NT) {
        const uint64_t key = cand[i];
        int before = 0;
        for (int j = 0; j < n; ++j) before += cand[j] > key;
        if (before < k) put(before, unordered(key >> 32), key_id(key));
      }
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
    row.each([&](float v, int id) {
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
// Bound: the way from and to memory (2048 x 32000 bf16 52 us, 5.0 TB/s; 1000 x 50265 42 us, 4.8 TB/s).
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
  const bool near = is_near(m);          // (as the forward pass formed m and ln S)
  auto one = [&](float v, int j) {
    const float lp = below(v, a.scale, m, near) - ln_s;
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
  // Threads so that one batch of a thread's loads, four pieces, takes most of a row.  Few rows: the more threads the shorter the chain (1 x
  // 1000 entries in bf16: 4.5 us with 256, 5.1 with 64; 256 x 10000: 5.8 with 512, 7.2 with 256; 64 x 32000: 7.3 with 1024, 9.3 with 512;
  // but 64 x 16300: 5.8 with 512, 7.2 with 1024).  Many rows fill the chip by themselves, and joining the wavefronts' parts costs more
  // (2048 x 1000: 6.9 with 64, 8.4 with 256; 2048 x 8000: 11.3 with 256, 16.1 with 512; 2048 x 32000: 32 with 512, 37 with 1024).
  const int pieces = a.V / (16 / (int)sizeof(T));
  const uint32_t grid = (uint32_t)rows;
#define ROW(NT) logprob_k<T, NT><<<grid, NT, 0, st>>>(a)
  if (pieces <= 48 || (pieces <= 256 && rows > 512)) ROW(64);
  else if (pieces <= 1024) ROW(256);
  else if (pieces <= 2200 || rows > 256) ROW(512);
  else ROW(1024);  // a row a compute unit at most
#undef ROW
  return hipGetLastError();
}

template <typename T>
hipError_t launch_logprob_bwd(int64_t rows, LogprobBwdArgs a, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  // pieces of 16 bytes where a row of the gradient lies in them as its row of logits does (2048 x 32000 in bf16: 44 us, element by element
  // 127; in fp32 96 and 163)
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
