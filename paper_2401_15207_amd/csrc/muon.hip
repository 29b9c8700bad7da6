// Orthogonalisation of matrices by Newton-Schulz steps, and the update of a group's matrices with it.
//
//   X = U / max(|U|_F, eps);  steps times:  A = X X^T,  B = a I + b A + c A^2,  X <- B X     (X the wide one of U and U^T)
//   update:  M <- mu M + G,  U = G + mu M,  W <- (1 - lr wd) W - lr 0.2 sqrt(max(rows, cols)) X
//
// Precision: a rounding of X before step k is multiplied by up to a^(steps - k) (3.44^5 = 485) where singular values are small, so neither
// bf16 nor one fp16 number holds enough.  Every factor is kept as the sum of two fp16 numbers, high and low (22 bits; see ns_plan.h for
// the scales), and a product is three matrix instructions, high high + high low + low high, summed in fp32: results as exact as fp32
// products give them, at a third of the fp16 rate instead of an eleventh of it.
// Factors lie in the matrix instruction's register order: blocks of 32 rows x 16 k, 1 KB of high and 1 KB of low numbers, lane l of a
// wavefront holding row l % 32 and k 8 (l / 32) .. +7 of it, so that a fragment is one contiguous load; blocks along k follow each other.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "ns_plan.h"

namespace hift {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A factor of rows x k entries (multiples of 32 and 16): block (row / 32, k / 16) starts 1024 ((row / 32) (k total / 16) + k / 16) numbers in.
struct Factor {
  _Float16* p;
  int kb;  // blocks along k
  __device__ __forceinline__ _Float16* block(int rb, int b) const { return p + ((int64_t)rb * kb + b) * 1024; }
};

struct NsMatrix {
  int64_t rows, cols, ld_src, ld_dst;
  const void* src;      // U, or the gradient
  float* momentum;      // the update's buffer M, or null
  void* dst;            // where X goes, or null
  float* master;        // the update's weights, or null
  bf16* copy;           // ... and their rounded copy, or null
  float factor;         // lr 0.2 sqrt(max(rows, cols))
  int n, m;             // short and long side, filled up
  int tall;             // rows > cols: X is U^T
  _Float16 *x, *xt, *xt2, *a, *b;  // X [n, m], X^T [m, n] now and after the step, A and B [n, n]
  double* norm_parts;
  int* small;           // how many powers of two X is below 1 at the start (norms below eps; ns_start_k)
  int block0;           // first workgroup of the launch that works on it
};
struct NsTable {
  int count;
  NsMatrix m[NS_TABLE];
};
static_assert(sizeof(NsTable) < 3500, "kernel arguments");

__device__ __forceinline__ const NsMatrix& matrix_of(const NsTable& t, int block) {
  int i = 0;
  while (i + 1 < t.count && block >= t.m[i + 1].block0) ++i;
  return t.m[i];
}

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

// ---- norm ----------------------------------------------------------------------------------
// Sums of squares in 64 bits (an entry's square may pass fp32's range either way), NS_NORM_PARTS of them a matrix; with a momentum buffer,
// that is updated on the way.
template <typename T>
__global__ void __launch_bounds__(256) ns_norm_k(NsTable t, float mu) {
  __shared__ double red[4];
  const NsMatrix& q = matrix_of(t, blockIdx.x);
  const int part = blockIdx.x - q.block0;
  double s = 0.0;
  const int64_t per = (q.rows + NS_NORM_PARTS - 1) / NS_NORM_PARTS;
  const int64_t r1 = min(q.rows, (part + 1) * per);
  for (int64_t r = part * per; r < r1; ++r)
    for (int64_t c = threadIdx.x; c < q.cols; c += 256) {
      float u = to_f32(reinterpret_cast<const T*>(q.src)[r * q.ld_src + c]);
      if (q.momentum) {
        const float g = u;
        float* mp = q.momentum + r * q.cols + c;
        const float m = fmaf(mu, *mp, g);
        *mp = m;
        u = fmaf(mu, m, g);
      }
      s += (double)u * u;
    }
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) q.norm_parts[part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// ---- U -> X and X^T in fragment order --------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) ns_start_k(NsTable t, float mu, float eps, float scale) {
  __shared__ float tile[64][65];
  __shared__ double red[4];
  const NsMatrix& q = matrix_of(t, blockIdx.x);
  const int th = threadIdx.x, lane = th & 63;
  static_assert(NS_NORM_PARTS == 256, "one part a thread");
  double s = q.norm_parts[th];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) red[th >> 6] = s;
  __syncthreads();
  const double norm = sqrt((red[0] + red[1]) + (red[2] + red[3]));
  // A norm below eps leaves X that small.  Its factors are stored a power of two larger then: X times 2^small, and after k steps, each of
  // which lets X grow by less than 2^growth, times 2^(small - k growth) as long as that is above 1.
  const int below = norm > 0.0 && norm < (double)eps ? min((int)floor(log2((double)eps / norm)), 200) : 0;
  const double by = ldexp((double)scale, below) / (norm < (double)eps ? (double)eps : norm);  // (a norm that is no number stays one)
  if (blockIdx.x == q.block0 && th == 0) *q.small = below;
  // sides as they lie in memory, filled up
  const int R = q.tall ? q.m : q.n, C = q.tall ? q.n : q.m;
  const int tiles_c = C / 64, id = blockIdx.x - q.block0;
  const int64_t r0 = (int64_t)(id / tiles_c) * 64, c0 = (int64_t)(id % tiles_c) * 64;
  for (int i = th >> 6; i < 64; i += 4) {
    const int64_t r = r0 + i, c = c0 + lane;
    float v = 0.f;
    if (r < q.rows && c < q.cols) {
      v = to_f32(reinterpret_cast<const T*>(q.src)[r * q.ld_src + c]);
      if (q.momentum) v = fmaf(mu, q.momentum[r * q.cols + c], v);
      v = (float)((double)v * by);
    }
    tile[i][lane] = v;
  }
  __syncthreads();
  // as a factor of rows R and k C, and as one of rows C and k R
  const Factor along{q.tall ? q.xt : q.x, C / 16}, across{q.tall ? q.x : q.xt, R / 16};
  for (int b = th >> 6; b < 8; b += 4) {  // 2 x 4 blocks of 32 x 16
    const int rb = b >> 2, kb = b & 3, i = rb * 32 + (lane & 31), k = kb * 16 + 8 * (lane >> 5);
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(tile[i][k + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16* p = along.block((int)(r0 / 32) + rb, (int)(c0 / 16) + kb) + lane * 8;
    *reinterpret_cast<half8*>(p) = hi;
    *reinterpret_cast<half8*>(p + 512) = lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(tile[k + e][i], h, l);
      hi[e] = h; lo[e] = l;
    }
    p = across.block((int)(c0 / 32) + rb, (int)(r0 / 16) + kb) + lane * 8;
    *reinterpret_cast<half8*>(p) = hi;
    *reinterpret_cast<half8*>(p + 512) = lo;
  }
}

// ---- products --------------------------------------------------------------------------------
// C[i][j] = sum_k P[i][k] Q[j][k] of two factors, in tiles of 128 x 128.
//   NS_GRAM   A = X X^T           upper tiles; both halves are written
//   NS_POLY   B = a I + b A + c A A
//   NS_APPLY  X^T and X of the next step from B and X^T
//   NS_LAST   X into dst, or into the update of the weights
enum { NS_GRAM, NS_POLY, NS_APPLY, NS_LAST };
struct NsStep {
  float unscale;        // of the sums
  float out_scale;      // of the factor that is written
  float ca, cb, cc;     // NS_POLY: coefficients, b's with A's scale taken out
  float decay;          // NS_LAST: 1 - lr wd
  int grown, growth;    // powers of two that X may have grown by before this step, and in it
};

// Where accumulator i of lane l lies in its 32 x 32 block: column l % 32 and row 8 (i / 4) + 4 (l / 32) + i % 4.
__device__ __forceinline__ int acc_row(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

// v: entries [i0 ..][j0 ..] of a 32 x 32 block, as a factor of rows j and k i (four consecutive k of a lane at a time) ...
__device__ __forceinline__ void put_rows_j(const Factor& f, int i0, int j0, const f32x16& v, int lane) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    half4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 h, l;
      split(v[4 * g + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16* p = f.block(j0 / 32, i0 / 16 + (g >> 1)) + ((lane & 31) + 32 * (g & 1)) * 8 + 4 * (lane >> 5);
    *reinterpret_cast<half4*>(p) = hi;
    *reinterpret_cast<half4*>(p + 512) = lo;
  }
}
// ... and as one of rows i and k j
__device__ __forceinline__ void put_rows_i(const Factor& f, int i0, int j0, const f32x16& v, int lane) {
  const int j = lane & 31;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    _Float16 h, l;
    split(v[i], h, l);
    _Float16* p = f.block(i0 / 32, j0 / 16 + (j >> 4)) + (acc_row(i, lane) + 32 * ((j >> 3) & 1)) * 8 + (j & 7);
    p[0] = h;
    p[512] = l;
  }
}

template <int MODE, typename OUT>
__global__ void __launch_bounds__(256) ns_product_k(NsTable t, NsStep st) {
  const NsMatrix& q = matrix_of(t, blockIdx.x);
  int id = blockIdx.x - q.block0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Factor P, Q;
  int ti, tj;
  if (MODE == NS_GRAM || MODE == NS_POLY) {
    P.p = Q.p = MODE == NS_GRAM ? q.x : q.a;
    P.kb = Q.kb = (MODE == NS_GRAM ? q.m : q.n) / 16;
    ti = 0;
    const int tiles = q.n / 128;
    while (id >= tiles - ti) { id -= tiles - ti; ++ti; }
    tj = ti + id;
  } else {
    const Factor b{q.b, q.n / 16}, x{q.xt, q.n / 16};
    const bool turn = MODE == NS_LAST && q.tall;  // dst's columns along the lanes
    P = turn ? x : b;
    Q = turn ? b : x;
    const int across = (turn ? q.n : q.m) / 128;
    ti = id / across;
    tj = id % across;
  }
  const int small = *q.small, up = max(0, small - st.grown);  // X is stored times 2^up
  const int i0 = ti * 128 + (wave >> 1) * 64, j0 = tj * 128 + (wave & 1) * 64;

  f32x16 acc[2][2] = {};
  for (int k = 0; k < P.kb; ++k) {
    half8 ph[2], pl[2], qh[2], ql[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const _Float16* p = P.block(i0 / 32 + b, k) + lane * 8;
      ph[b] = *reinterpret_cast<const half8*>(p);
      pl[b] = *reinterpret_cast<const half8*>(p + 512);
      p = Q.block(j0 / 32 + b, k) + lane * 8;
      qh[b] = *reinterpret_cast<const half8*>(p);
      ql[b] = *reinterpret_cast<const half8*>(p + 512);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl[x], qh[y], acc[x][y], 0, 0, 0);
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[x], ql[y], acc[x][y], 0, 0, 0);
        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ph[x], qh[y], acc[x][y], 0, 0, 0);
      }
  }

#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      f32x16 v = acc[x][y];
      const int i = i0 + 32 * x, j = j0 + 32 * y;
      if (MODE == NS_POLY) {
        // A at the same place: rows j, k i of a symmetric factor
        const Factor a{q.a, q.n / 16};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const _Float16* p = a.block(j / 32, i / 16 + (g >> 1)) + ((lane & 31) + 32 * (g & 1)) * 8 + 4 * (lane >> 5);
          const half4 hi = *reinterpret_cast<const half4*>(p), lo = *reinterpret_cast<const half4*>(p + 512);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool diagonal = i + acc_row(4 * g + e, lane) == j + (lane & 31);
            v[4 * g + e] = (fmaf(st.cc, v[4 * g + e], st.cb * ((float)hi[e] + (float)lo[e])) + (diagonal ? st.ca : 0.f)) * st.out_scale;
          }
        }
      } else if (MODE != NS_LAST) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = ldexpf(v[e] * st.unscale * st.out_scale, MODE == NS_GRAM ? -2 * up : max(0, small - st.grown - st.growth) - up);
      }
      if (MODE == NS_GRAM || MODE == NS_POLY) {
        const Factor out{MODE == NS_GRAM ? q.a : q.b, q.n / 16};
        put_rows_j(out, i, j, v, lane);
        if (ti != tj) put_rows_i(out, i, j, v, lane);
      } else if (MODE == NS_APPLY) {
        put_rows_j(Factor{q.xt2, q.n / 16}, i, j, v, lane);
        put_rows_i(Factor{q.x, q.m / 16}, i, j, v, lane);
      } else {
        const int64_t c = j + (lane & 31);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int64_t r = i + acc_row(e, lane);
          if (r >= q.rows || c >= q.cols) continue;
          const float o = ldexpf(v[e] * st.unscale, -up);
          if (q.master) {
            float* w = q.master + r * q.cols + c;
            const float nw = fmaf(-q.factor, o, st.decay * *w);
            *w = nw;
            if (q.copy) q.copy[r * q.cols + c] = from_f32<bf16>(nw);
          } else {
            reinterpret_cast<OUT*>(q.dst)[r * q.ld_dst + c] = from_f32<OUT>(o);
          }
        }
      }
    }
}

// Gives every matrix of the table its workgroups; blocks(q): how many.
template <class F>
uint32_t spread(NsTable& t, F blocks) {
  int64_t at = 0;
  for (int i = 0; i < t.count; ++i) {
    t.m[i].block0 = (int)at;
    at += blocks(t.m[i]);
  }
  return (uint32_t)at;
}

hipError_t steps_of(NsTable& t, int dt_src, int dt_dst, const NsRun& run, hipStream_t st) {
  const uint32_t parts = spread(t, [](const NsMatrix&) { return NS_NORM_PARTS; });
  if (dt_src == DT_BF16) ns_norm_k<bf16><<<parts, 256, 0, st>>>(t, run.mu);
  else ns_norm_k<float><<<parts, 256, 0, st>>>(t, run.mu);
  double r = 1.001;  // the norm is at least the largest singular value, but for rounding
  NsScales s;
  if (!ns_scales(run.co, r, &s)) return hipErrorInvalidValue;
  const int growth = ns_growth(run.co);
  const uint32_t squares = spread(t, [](const NsMatrix& q) { return (int64_t)(q.n / 64) * (q.m / 64); });
  if (dt_src == DT_BF16) ns_start_k<bf16><<<squares, 256, 0, st>>>(t, run.mu, run.eps, s.x);
  else ns_start_k<float><<<squares, 256, 0, st>>>(t, run.mu, run.eps, s.x);
  for (int k = 0; k < run.steps; ++k) {
    if (!ns_scales(run.co, r, &s)) return hipErrorInvalidValue;
    NsStep p{};
    p.grown = k * growth;
    p.growth = growth;
    p.unscale = 1.f / (s.x * s.x);
    p.out_scale = s.a;
    const uint32_t half = spread(t, [](const NsMatrix& q) { return (int64_t)(q.n / 128) * (q.n / 128 + 1) / 2; });
    ns_product_k<NS_GRAM, float><<<half, 256, 0, st>>>(t, p);
    p.ca = (float)run.co[0];
    p.cb = (float)run.co[1] / s.a;
    p.cc = (float)run.co[2] / (s.a * s.a);
    p.out_scale = s.b;
    ns_product_k<NS_POLY, float><<<half, 256, 0, st>>>(t, p);
    p.unscale = 1.f / (s.b * s.x);
    const uint32_t whole = spread(t, [](const NsMatrix& q) { return (int64_t)(q.n / 128) * (q.m / 128); });
    r = std::max(s.r_next, 1.0);  // (and what norms below eps are stored as)
    if (k + 1 < run.steps) {
      NsScales next;
      if (!ns_scales(run.co, r, &next)) return hipErrorInvalidValue;
      p.out_scale = next.x;
      ns_product_k<NS_APPLY, float><<<whole, 256, 0, st>>>(t, p);
      for (int i = 0; i < t.count; ++i) std::swap(t.m[i].xt, t.m[i].xt2);
    } else {
      p.decay = run.decay;
      if (dt_dst == DT_BF16) ns_product_k<NS_LAST, bf16><<<whole, 256, 0, st>>>(t, p);
      else ns_product_k<NS_LAST, float><<<whole, 256, 0, st>>>(t, p);
    }
  }
  return hipGetLastError();
}

}  // namespace

bool ns_coefficients_hold(const double (&co)[3], int steps) {
  if (!(co[0] >= 1.0)) return false;
  double r = 1.001;
  for (int k = 0; k < steps; ++k) {
    NsScales s;
    if (!ns_scales(co, r, &s)) return false;
    r = std::max(s.r_next, 1.0);
  }
  return true;
}

size_t ns_workspace(const NsItem* items, int count) {
  return ns_workspace_bytes(count, [&](int i, int64_t* r, int64_t* c) { *r = items[i].rows; *c = items[i].cols; });
}

hipError_t newton_schulz(const NsItem* items, int count, int dt_src, int dt_dst, const NsRun& run, void* workspace, hipStream_t st) {
  const auto shape = [&](int i, int64_t* r, int64_t* c) { *r = items[i].rows; *c = items[i].cols; };
  for (int at = 0; at < count;) {
    const int n = ns_together(at, count, shape);
    NsTable t{};
    unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
    for (int i = at; i < at + n; ++i) {
      const NsItem& it = items[i];
      if (it.rows == 0 || it.cols == 0) continue;
      NsMatrix& q = t.m[t.count++];
      q.rows = it.rows; q.cols = it.cols; q.ld_src = it.ld_src; q.ld_dst = it.ld_dst;
      q.src = it.src; q.momentum = it.momentum; q.dst = it.dst; q.master = it.master; q.copy = (bf16*)it.copy;
      q.factor = (float)(run.lr * 0.2 * sqrt((double)std::max(it.rows, it.cols)));
      q.tall = it.rows > it.cols;
      q.n = (int)ns_up(std::min(it.rows, it.cols));
      q.m = (int)ns_up(std::max(it.rows, it.cols));
      auto take = [&](int64_t entries) {
        _Float16* p = reinterpret_cast<_Float16*>(ws);
        ws += entries * 4;
        return p;
      };
      q.x = take((int64_t)q.n * q.m);
      q.xt = take((int64_t)q.n * q.m);
      q.xt2 = take((int64_t)q.n * q.m);
      q.a = take((int64_t)q.n * q.n);
      q.b = take((int64_t)q.n * q.n);
      q.norm_parts = reinterpret_cast<double*>(ws);
      ws += NS_NORM_PARTS * 8;
      q.small = reinterpret_cast<int*>(ws);
      ws += 16;
    }
    if (t.count > 0) {
      const hipError_t e = steps_of(t, dt_src, dt_dst, run, st);
      if (e != hipSuccess) return e;
    }
    at += n;
  }
  return hipSuccess;
}

}  // namespace hift
