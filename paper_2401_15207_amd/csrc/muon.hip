// Orthogonalisation of matrices by Newton-Schulz steps, and the update of a group's matrices with it.
//
//   X = U / max(|U|_F, eps);  steps times:  A = X X^T,  B = a I + b A + c A^2,  X <- B X     (X the wide one of U and U^T)
//   update:  M <- mu M + G,  U = G + mu M,  W <- (1 - lr wd) W - lr 0.2 sqrt(max(rows, cols)) X
//
// Precision: a rounding of X before step k is multiplied by up to a^(steps - k) (3.44^5 = 485) where singular values are small, so neither
// bf16 nor one fp16 number holds enough.  Every factor is kept as the sum of two fp16 numbers, high and low (22 bits; see ns_plan.h for
// the scales), and a product is three matrix instructions, high high + high low + low high, summed in fp32: results as exact as fp32
// products give them, at a third of the fp16 rate instead of an eleventh of it.
// Results in bf16 take the same products.  Single numbers for A, for A A or for the last B X leave roundings that no sum averages out where the
// entries of a matrix round alike: simulated in 64 bits, diagonal, block-repeated and equal-magnitude matrices come out 2e-3 to 6e-3 off in the
// 2-norm after five steps and up to 0.2 after sixteen, which is more than the rounding to bf16.
// Factors lie in the matrix instruction's register order: blocks of 32 rows x 16 k, 1 KB of high or of low numbers, lane l of a wavefront
// holding row l % 32 and k 8 (l / 32) .. +7 of it, so that a fragment is one contiguous load; blocks along k follow each other, high and
// low ones apart.
#include <limits.h>
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "ns_plan.h"

namespace hift {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A factor of rows x k entries (multiples of 32 and 16): for every 32 rows the blocks of their high numbers along k, then those of the low ones.
struct Factor {
  _Float16* p;
  int kb;  // blocks along k
  __device__ __forceinline__ _Float16* block(int rb, int b) const { return p + ((int64_t)rb * 2 * kb + b) * 512; }
  __device__ __forceinline__ int low() const { return kb * 512; }  // from a high number to its low one
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
  int parts;            // workgroups that share the k range of one of its tiles
  int tile0, tiles;     // of its product's tiles, those from tile0 on
  int alone;            // workgroups before it that share nothing, if it is the launch's last round
};
// first[i]: the first workgroup of a launch that works on matrix i; from `count` on, beyond all of them.
struct NsTable {
  int first[NS_TABLE];
  int count;
  NsMatrix m[NS_TABLE];
};
static_assert(sizeof(NsTable) < 3500, "kernel arguments");

// (all of `first` in one load and a comparison each: a search would wait for memory at every step)
__device__ __forceinline__ int matrix_of(const NsTable& t, int block) {
  int i = 0;
#pragma unroll
  for (int j = 1; j < NS_TABLE; ++j) i += block >= t.first[j];
  return __builtin_amdgcn_readfirstlane(i);
}

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

// One entry's square, its momentum updated on the way
template <typename T>
__device__ __forceinline__ double norm_entry(const NsMatrix& q, int64_t at, int64_t at_momentum, float mu) {
  float u = to_f32(reinterpret_cast<const T*>(q.src)[at]);
  if (q.momentum) {
    const float m = fmaf(mu, q.momentum[at_momentum], u);
    q.momentum[at_momentum] = m;
    u = fmaf(mu, m, u);
  }
  return (double)u * u;
}

// ---- norm ----------------------------------------------------------------------------------
// Sums of squares in 64 bits (an entry's square may pass fp32's range either way), NS_NORM_PARTS of them a matrix; with a momentum buffer,
// that is updated on the way.  Bound: memory, 2.4 GB of gradients and momentum of a layer 4096 wide in 540 us.  Parts of fixed size in a
// fixed order, so that a norm has the same bits in every list.
template <typename T>
__global__ void __launch_bounds__(256) ns_norm_k(NsTable t, float mu, unsigned* shared) {
  __shared__ double red[4];
  const int at = matrix_of(t, blockIdx.x), part = blockIdx.x - t.first[at];
  const NsMatrix& q = t.m[at];
  if (blockIdx.x == 0)  // the counters of shared tiles; who counts last leaves 0 again
    for (int i = threadIdx.x; i < NS_SHARED_UNITS; i += 256) shared[i] = 0;
  double s = 0.0;
  constexpr int E = 16 / (int)sizeof(T), U = 4;
  const int64_t all = q.rows * q.cols;
  if (q.ld_src == q.cols && ((reinterpret_cast<uintptr_t>(q.src) | reinterpret_cast<uintptr_t>(q.momentum)) & 15) == 0) {
    // one run of pieces of 16 bytes, U of them a thread on their way at a time (202 M entries with momentum: 0.77 -> 0.53 ms against rows of entries)
    const int64_t pieces = all / E, per = (pieces + NS_NORM_PARTS - 1) / NS_NORM_PARTS, end = min(pieces, (part + 1) * per);
    const T* src = reinterpret_cast<const T*>(q.src);
    for (int64_t i = part * per + threadIdx.x; i < end; i += U * 256) {
      Vec<T, E> g[U];
      Vec<float, E> m[U];
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i + k * 256 < end) {
          g[k] = *reinterpret_cast<const Vec<T, E>*>(src + (i + k * 256) * E);
          if (q.momentum) m[k] = *reinterpret_cast<const Vec<float, E>*>(q.momentum + (i + k * 256) * E);
        }
#pragma unroll
      for (int k = 0; k < U; ++k)
        if (i + k * 256 < end) {
          float u[E];
#pragma unroll
          for (int e = 0; e < E; ++e) {
            u[e] = to_f32(g[k].v[e]);
            if (q.momentum) {
              m[k].v[e] = fmaf(mu, m[k].v[e], u[e]);
              u[e] = fmaf(mu, m[k].v[e], u[e]);
            }
            s += (double)u[e] * u[e];
          }
          if (q.momentum) *reinterpret_cast<Vec<float, E>*>(q.momentum + (i + k * 256) * E) = m[k];
        }
    }
    const int64_t left = pieces * E + threadIdx.x;
    if (part == NS_NORM_PARTS - 1 && left < all) s += norm_entry<T>(q, left, left, mu);
  } else {
    const int64_t per = (q.rows + NS_NORM_PARTS - 1) / NS_NORM_PARTS, r1 = min(q.rows, (part + 1) * per);
    for (int64_t r = part * per; r < r1; ++r)
      for (int64_t c = threadIdx.x; c < q.cols; c += 256) s += norm_entry<T>(q, r * q.ld_src + c, r * q.cols + c, mu);
  }
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) q.norm_parts[part] = (red[0] + red[1]) + (red[2] + red[3]);
}

// What U is multiplied with to become X, times X's scale; returns `small`: a norm below eps leaves X that many powers of two below 1.  Its
// factors are stored a power of two larger then: X times 2^small, and after k steps, each of which lets X grow by less than 2^growth, times
// 2^(small - k growth) as long as that is above 1.
__device__ __forceinline__ int start_scale(double sum_of_squares, float eps, float scale, double* by) {
  const double norm = sqrt(sum_of_squares);
  const int small = norm > 0.0 && norm < (double)eps ? min((int)floor(log2((double)eps / norm)), 200) : 0;
  *by = ldexp((double)scale, small) / (norm < (double)eps ? (double)eps : norm);  // (a norm that is no number stays one)
  return small;
}

// ---- U -> X and X^T in fragment order --------------------------------------------------------
// Squares of 64 x 64 through LDS, so that both orders leave in whole blocks.  Bound: memory, 1.6 GB read and 1.6 written of a layer 4096
// wide in 670 us; the square is requested before the norm's parts are summed.
template <typename T>
__global__ void __launch_bounds__(256) ns_start_k(NsTable t, float mu, float eps, float scale) {
  __shared__ float tile[64][65];
  __shared__ double red[4];
  const int at = matrix_of(t, blockIdx.x), id = blockIdx.x - t.first[at];
  const NsMatrix& q = t.m[at];
  const int th = threadIdx.x, lane = th & 63;
  // sides as they lie in memory, filled up
  const int R = q.tall ? q.m : q.n, C = q.tall ? q.n : q.m;
  const int tiles_c = C / 64;
  const int64_t r0 = (int64_t)(id / tiles_c) * 64, c0 = (int64_t)(id % tiles_c) * 64;
  // the tile is on its way while the norm's parts are summed
  float v[16], m[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t r = r0 + i * 4 + (th >> 6), c = c0 + lane;
    const bool in = r < q.rows && c < q.cols;
    v[i] = in ? to_f32(reinterpret_cast<const T*>(q.src)[r * q.ld_src + c]) : 0.f;
    m[i] = in && q.momentum ? q.momentum[r * q.cols + c] : 0.f;
  }
  static_assert(NS_NORM_PARTS == 256, "one part a thread");
  double s = q.norm_parts[th];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) red[th >> 6] = s;
  __syncthreads();
  double by;
  const int small = start_scale((red[0] + red[1]) + (red[2] + red[3]), eps, scale, &by);
  if (id == 0 && th == 0) *q.small = small;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float u = q.momentum ? fmaf(mu, m[i], v[i]) : v[i];
    tile[i * 4 + (th >> 6)][lane] = (float)((double)u * by);
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
    *reinterpret_cast<half8*>(p + along.low()) = lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split(tile[k + e][i], h, l);
      hi[e] = h; lo[e] = l;
    }
    p = across.block((int)(c0 / 32) + rb, (int)(r0 / 16) + kb) + lane * 8;
    *reinterpret_cast<half8*>(p) = hi;
    *reinterpret_cast<half8*>(p + across.low()) = lo;
  }
}

// ---- products --------------------------------------------------------------------------------
// C[i][j] = sum_k P[i][k] Q[j][k] of two factors, tile by tile (which tiles: ns_plan.h).
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
  unsigned char* shared;  // where workgroups that share a tile meet: a counter for each tile, and their sums
  int grown, growth;    // powers of two that X may have grown by before this step, and in it
};

// Where accumulator i of lane l lies in its 32 x 32 block: column l % 32 and row 8 (i / 4) + 4 (l / 32) + i % 4.
__device__ __forceinline__ int acc_row(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

constexpr int TURN_PITCH = 36;  // words: the turned block's rows are read in 16-byte pieces

// v: entries [i0 ..][j0 ..] of a 32 x 32 block, into a factor of rows j and k i (four consecutive k of a lane at a time) and, if
// `other`, turned around in LDS into one of rows i and k j.
__device__ __forceinline__ void put_block(const Factor& rows_j, const Factor& rows_i, bool other, int i0, int j0, const f32x16& v, uint32_t* turned,
                                          int lane) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    half4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 h, l;
      split(v[4 * g + e], h, l);
      hi[e] = h; lo[e] = l;
      typedef _Float16 half2 __attribute__((ext_vector_type(2)));
      const half2 both = {h, l};
      turned[acc_row(4 * g + e, lane) * TURN_PITCH + (lane & 31)] = __builtin_bit_cast(uint32_t, both);
    }
    _Float16* p = rows_j.block(j0 / 32, i0 / 16 + (g >> 1)) + ((lane & 31) + 32 * (g & 1)) * 8 + 4 * (lane >> 5);
    *reinterpret_cast<half4*>(p) = hi;
    *reinterpret_cast<half4*>(p + rows_j.low()) = lo;
  }
  if (!other) return;
  __builtin_amdgcn_wave_barrier();  // (a wavefront's own LDS accesses stay in order)
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint32_t* row = turned + (lane & 31) * TURN_PITCH + b * 16 + 8 * (lane >> 5);
    uint32_t w[8], hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = row[e];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      hi[e] = (w[2 * e] & 0xFFFFu) | w[2 * e + 1] << 16;
      lo[e] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xFFFF0000u);
    }
    _Float16* p = rows_i.block(i0 / 32, j0 / 16 + b) + lane * 8;
    *reinterpret_cast<hift_u32x4*>(p) = hift_u32x4{hi[0], hi[1], hi[2], hi[3]};
    *reinterpret_cast<hift_u32x4*>(p + rows_i.low()) = hift_u32x4{lo[0], lo[1], lo[2], lo[3]};
  }
  __builtin_amdgcn_wave_barrier();
}

// Four consecutive k of a lane's row of a factor of rows j and k i, where put_block leaves accumulators 4 g .. 4 g + 3
__device__ __forceinline__ const _Float16* at_block(const Factor& rows_j, int i0, int j0, int g, int lane) {
  return rows_j.block(j0 / 32, i0 / 16 + (g >> 1)) + ((lane & 31) + 32 * (g & 1)) * 8 + 4 * (lane >> 5);
}

// Tiles of 256 x 256 by 2 x 4 wavefronts, of 128 x 128 and 64 x 64 by 2 x 2.  Both operands travel into LDS with direct-to-LDS loads, as they
// lie, into a ring of stages of 16 to 64 k; a stage's fragments are read into registers under the products of the stage before.
// What bounds it, a layer 4096 wide with 11008 in its feed-forward block (256 x 256): A 1.97 ms, 1340 TFLOP/s by the matrix instructions of the
// upper tiles, B 1.25 (1220; 4 rounds of 3.7), X 3.8 (1320; 12 rounds and a shared one), the last X with the update 4.1 (1210): the matrix pipe,
// of which a large fp16 product reaches 1500.  A layer 1024 wide (128 x 128): 65, 37, 81 and 86 us (with the update 105), each one round or two of
// tiles.
// DEEP: the ring of a launch that gives a compute unit one workgroup at most.  That one waits for memory by itself: a stage of 16 KB takes
// the time of its requests' latency over the stages in flight, so the ring takes most of the LDS.
template <int SIDE, bool DEEP>
struct NsTile {
  static constexpr int WI = 2, WJ = SIDE == 256 ? 4 : 2, NW = WI * WJ;
  static constexpr int BI = SIDE / 32 / WI, BJ = SIDE / 32 / WJ;   // blocks of 32 x 32 a wavefront
  static constexpr int KS = SIDE == 64 ? 4 : 1;                    // blocks along k of a stage
  static constexpr int PN = SIDE / 32 * KS * 2, PIECES = 2 * PN;   // KB of P in a stage, and of both
  static constexpr int LOADS = PIECES / NW;                        // load instructions a wavefront and stage, 1 KB each
  static constexpr int STAGE = PIECES * 1024, RING = SIDE == 256 || (SIDE == 64 && DEEP) ? 4 : SIDE == 64 ? 2 : DEEP ? 8 : 3, LDS = RING * STAGE;
  static_assert(PIECES % NW == 0 && LDS <= 160 * 1024 && NW * 32 * TURN_PITCH * 4 <= LDS, "blocks turn in the ring");
};

// entry (row, c) of the result o: into dst, or into the update of the weights (w: what that one is)
template <typename OUT>
__device__ __forceinline__ void put_result(const NsMatrix& q, int64_t row, int64_t c, float o, float decay, float w) {
  if (row >= q.rows || c >= q.cols) return;
  if (q.master) {
    const float nw = fmaf(-q.factor, o, decay * w);
    q.master[row * q.cols + c] = nw;
    if (q.copy) q.copy[row * q.cols + c] = from_f32<bf16>(nw);
  } else {
    reinterpret_cast<OUT*>(q.dst)[row * q.ld_dst + c] = from_f32<OUT>(o);
  }
}

template <int SIDE, int MODE, bool DEEP, typename OUT>
__global__ void __launch_bounds__((64 * NsTile<SIDE, DEEP>::NW), (DEEP && SIDE < 256 ? 1 : 2)) ns_product_k(NsTable t, NsStep st) {
  typedef NsTile<SIDE, DEEP> T;
  constexpr int BI = T::BI, BJ = T::BJ, RING = T::RING, KS = T::KS;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int at = matrix_of(t, blockIdx.x), block0 = t.first[at];
  const NsMatrix& q = t.m[at];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroups are dealt round-robin to the 8 XCDs (every matrix starts at a multiple of 8): each XCD gets a contiguous run of tiles, so
  // that those it works on at a time share operands in its L2.
  constexpr bool SYM = MODE == NS_GRAM || MODE == NS_POLY;
  const bool turn = MODE == NS_LAST && q.tall;  // dst's columns along the lanes
  const int side_i = (turn ? q.m : q.n) / SIDE, side_j = (SYM || turn ? q.n : q.m) / SIDE;
  const int units = q.tiles * q.parts;
  int id = blockIdx.x - block0;
  id = (id & 7) * ((units + 7) >> 3) + (id >> 3);
  if (id >= units) return;
  const int unit = block0 + id - q.alone, part = id % q.parts;
  id = q.tile0 + id / q.parts;
  Factor P, Q;
  int ti, tj;
  if (SYM) {
    P.p = Q.p = MODE == NS_GRAM ? q.x : q.a;
    P.kb = Q.kb = (MODE == NS_GRAM ? q.m : q.n) / 16;
    ti = 0;
    while (id >= side_i - ti) { id -= side_i - ti; ++ti; }
    tj = ti + id;
  } else {
    const Factor b{q.b, q.n / 16}, x{q.xt, q.n / 16};
    P = turn ? x : b;
    Q = turn ? b : x;
    // down bands of 4 tile rows
    const int band = id / (4 * side_j), in_band = id - band * 4 * side_j, rows = min(4, side_i - band * 4);
    ti = band * 4 + in_band % rows;
    tj = in_band / rows;
  }
  const int small = *q.small, up = max(0, small - st.grown);  // X is stored times 2^up
  const int all = P.kb / KS, first = all * part / q.parts, stages = all * (part + 1) / q.parts;  // this workgroup's: [first, stages)

  const uint64_t pa = reinterpret_cast<uint64_t>(P.block(ti * (SIDE / 32), 0)), qa = reinterpret_cast<uint64_t>(Q.block(tj * (SIDE / 32), 0));
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(smem), voff = lane * 16;
  auto slot = [](int s) __attribute__((always_inline)) { return RING & (RING - 1) ? s % RING : s & (RING - 1); };
  auto request = [&](int s) __attribute__((always_inline)) {
    const uint32_t at = lds0 + (uint32_t)slot(s) * T::STAGE;
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) {
      const int load = wave * T::LOADS + i;
      const bool is_q = load >= T::PN;
      const int in = is_q ? load - T::PN : load, rb = in / (KS * 2), rest = in % (KS * 2);
      const uint64_t base = is_q ? qa : pa;
      const hift_u32x4 rsrc = {(uint32_t)base, (uint32_t)(base >> 32) & 0xFFFFu, 0xFFFFFFF0u, 0x00020000u};
      const uint32_t soff = (((uint32_t)rb * 2 + rest % 2) * P.kb + s * KS + rest / 2) * 1024u;
      load_to_lds_b128(rsrc, at + (uint32_t)load * 1024, voff, soff);
    }
  };
  const int wi = wave / T::WJ, wj = wave % T::WJ;
  half8 p[2][KS][BI][2], r[2][KS][BJ][2];  // fragments of two stages: high and low numbers
  auto read = [&](int to, int s) __attribute__((always_inline)) {
    const unsigned char* at = smem + slot(s) * T::STAGE + lane * 16;
#pragma unroll
    for (int k = 0; k < KS; ++k) {
#pragma unroll
      for (int b = 0; b < BI; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) p[to][k][b][h] = *reinterpret_cast<const half8*>(at + (((wi * BI + b) * KS + k) * 2 + h) * 1024);
#pragma unroll
      for (int b = 0; b < BJ; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) r[to][k][b][h] = *reinterpret_cast<const half8*>(at + (T::PN + ((wj * BJ + b) * KS + k) * 2 + h) * 1024);
    }
  };
  f32x16 acc[BI][BJ] = {};
  auto multiply = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int h = 2; h >= 0; --h)  // low high, high low, high high
#pragma unroll
        for (int x = 0; x < BI; ++x)
#pragma unroll
          for (int y = 0; y < BJ; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[c][k][x][h == 2], r[c][k][y][h == 1], acc[x][y], 0, 0, 0);
  };
#pragma unroll
  for (int s = 0; s < RING; ++s)
    if (first + s < stages) request(first + s);
  if (first + RING <= stages) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * T::LOADS) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  read(0, first);
  // Past the wait the stage after s has landed (all but the younger stages' requests), and past the barrier s's buffer, whose fragments every
  // wavefront has, is free for the stage a whole ring further on.  Near the end fewer requests are in flight: there the wait is for all.
  auto stage = [&](int s, int c, bool tail) __attribute__((always_inline)) {
    if (!tail) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 2) * T::LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    read(c ^ 1, s + 1);  // (past the end: what the ring holds, and never multiplied)
    if (!tail || s + RING < stages) request(s + RING);
    multiply(c);
    __builtin_amdgcn_sched_barrier(0);
  };
  int s = first;
  for (; s + 1 + RING < stages; s += 2) {
    stage(s, 0, false);
    stage(s + 1, 1, false);
  }
  for (; s < stages; s += 2) {
    stage(s, 0, true);
    if (s + 1 < stages) stage(s + 1, 1, true);
  }

  if (q.parts > 1) {
    // Every one of them leaves its sums in memory and counts itself in; the one that finds all others counted adds them up in their order
    // (its own too: the result must not depend on who came last) and goes on.  Nobody waits.  They run on different XCDs, so the sums go past the
    // L2s both ways (device scope).
    constexpr int SC1 = 16, BYTES = SIDE * SIDE * 4;
    int* is_last = reinterpret_cast<int*>(smem);
    unsigned* count = reinterpret_cast<unsigned*>(st.shared) + (unit - part);
    const __amdgpu_buffer_rsrc_t sums = __builtin_amdgcn_make_buffer_rsrc(st.shared + NS_SHARED_UNITS * 4 + (int64_t)(unit - part) * BYTES, 0, q.parts * BYTES, 0x00020000);
    const int mine = threadIdx.x * 16;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int x = 0; x < BI; ++x)
#pragma unroll
      for (int y = 0; y < BJ; ++y)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 v = {acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(hift_u32x4, v), sums, mine + part * BYTES, ((x * BJ + y) * 4 + g) * T::NW * 1024, SC1);
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this lane's sums have reached memory
    __syncthreads();
    if (threadIdx.x == 0) {
      const unsigned before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      *is_last = before == (unsigned)q.parts - 1;
      if (*is_last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!*is_last) return;
    constexpr int ROWS = SIDE == 256 ? 1 : BI;  // of blocks at a time, for their registers
#pragma unroll
    for (int x0 = 0; x0 < BI; x0 += ROWS)
      for (int u = 0; u < q.parts; ++u) {  // a part's sums are all requested before the first is added
        f32x4 v[ROWS][BJ][4];
#pragma unroll
        for (int x = 0; x < ROWS; ++x)
#pragma unroll
          for (int y = 0; y < BJ; ++y)
#pragma unroll
            for (int g = 0; g < 4; ++g)
              v[x][y][g] = __builtin_bit_cast(
                  f32x4, __builtin_amdgcn_raw_buffer_load_b128(sums, mine + u * BYTES, (((x0 + x) * BJ + y) * 4 + g) * T::NW * 1024, SC1));
#pragma unroll
        for (int x = 0; x < ROWS; ++x)
#pragma unroll
          for (int y = 0; y < BJ; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[x0 + x][y][e] = u == 0 ? v[x][y][e >> 2][e & 3] : acc[x0 + x][y][e] + v[x][y][e >> 2][e & 3];
      }
  }

  __syncthreads();  // the ring is free: nothing is on its way there either
  uint32_t* turned = reinterpret_cast<uint32_t*>(smem) + wave * 32 * TURN_PITCH;
  // What a block of the epilogue reads is requested before the block before it is written: the wait for a load would take in the stores
  // before it.
  struct Ahead { half4 hi[4], lo[4]; f32x16 w; };
  const Factor f{q.a, q.n / 16};
  const auto block_i = [&](int b) __attribute__((always_inline)) { return ti * SIDE + (wi * BI + b / BJ) * 32; };
  const auto block_j = [&](int b) __attribute__((always_inline)) { return tj * SIDE + (wj * BJ + b % BJ) * 32; };
  const auto ahead = [&](Ahead& n, int b) __attribute__((always_inline)) {
    const int i = block_i(b), j = block_j(b);
    if (MODE == NS_POLY)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const _Float16* p = at_block(f, i, j, g, lane);
        n.hi[g] = *reinterpret_cast<const half4*>(p);
        n.lo[g] = *reinterpret_cast<const half4*>(p + f.low());
      }
    if (MODE == NS_LAST && q.master)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t row = i + acc_row(e, lane), c = j + (lane & 31);
        n.w[e] = row < q.rows && c < q.cols ? q.master[row * q.cols + c] : 0.f;
      }
  };
  Ahead next;
  ahead(next, 0);
#pragma unroll
  for (int b = 0; b < BI * BJ; ++b) {
    f32x16 v = acc[b / BJ][b % BJ];
    const int i = block_i(b), j = block_j(b);
    const Ahead now = next;
    if (b + 1 < BI * BJ) ahead(next, b + 1);
    if (MODE == NS_POLY) {
      // A at the same place: rows j, k i of a symmetric factor
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float entry = (float)now.hi[g][e] + (float)now.lo[g][e];
          const bool diagonal = i + acc_row(4 * g + e, lane) == j + (lane & 31);
          v[4 * g + e] = (fmaf(st.cc, v[4 * g + e], st.cb * entry) + (diagonal ? st.ca : 0.f)) * st.out_scale;
        }
    }
    if (MODE == NS_GRAM || MODE == NS_APPLY) {
      const int power = MODE == NS_GRAM ? -2 * up : max(0, small - st.grown - st.growth) - up;
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = ldexpf(v[e] * st.unscale * st.out_scale, power);
    }
    if (SYM) {
      const Factor out{MODE == NS_GRAM ? q.a : q.b, q.n / 16};
      put_block(out, out, ti != tj, i, j, v, turned, lane);
    } else if (MODE == NS_APPLY) {
      put_block(Factor{q.xt2, q.n / 16}, Factor{q.x, q.m / 16}, true, i, j, v, turned, lane);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) put_result<OUT>(q, i + acc_row(e, lane), j + (lane & 31), ldexpf(v[e] * st.unscale, -up), st.decay, now.w[e]);
    }
  }
}

// ---- matrices that fit a compute unit's LDS ---------------------------------------------------
// All steps in one launch, a workgroup a matrix: X, X^T and A (in whose place B goes) stay in LDS, in the same order as in memory, sides filled
// up to multiples of 32.  What bounds the launches above for such matrices is their number and each one's way to memory and back: six
// matrices of 64 x 64 to 256 x 64 take 82 us in 17 launches, 55 here.
struct NsSteps {
  int steps, growth;
  float mu, eps, decay;
  float ca, cb, cc;
  float x[NS_STEPS_MAX + 1], a[NS_STEPS_MAX], b[NS_STEPS_MAX];  // scales
};
constexpr int SMALL_WAVES = 8, SMALL_TILES = NS_SMALL_TILES;

// A factor in LDS: as in memory, or (SPREAD, X) with the halves of a block 544 bytes and blocks 1168 bytes apart, so that the two-byte
// writes of a turned tile, whose lanes meet in four banks otherwise, fall into all of them.
template <bool SPREAD>
struct LdsFactor {
  static constexpr int HALF = SPREAD ? 272 : 256, BLOCK = SPREAD ? 584 : 512;  // numbers
  _Float16* p;
  int kb;
  static size_t bytes(int rows, int k) { return (size_t)(rows / 32) * (k / 16) * 2 * BLOCK * 2; }
  __device__ __forceinline__ int low() const { return kb * BLOCK; }
  __device__ __forceinline__ _Float16* entry(int row, int k) const {
    return p + ((row >> 5) * 2 * kb + (k >> 4)) * BLOCK + ((k >> 3) & 1) * HALF + (row & 31) * 8 + (k & 7);
  }
  __device__ __forceinline__ const half8& fragment(int rb, int b, int lane) const {
    return *reinterpret_cast<const half8*>(p + (rb * 2 * kb + b) * BLOCK + (lane >> 5) * HALF + (lane & 31) * 8);
  }
  __device__ __forceinline__ const half8& low_fragment(int rb, int b, int lane) const {
    return *reinterpret_cast<const half8*>(p + low() + (rb * 2 * kb + b) * BLOCK + (lane >> 5) * HALF + (lane & 31) * 8);
  }
};
// one 32 x 32 tile of P Q^T, k blocks [k0, k1), an even number of them: two at a time, the next two's fragments on their way, and three
// sums apart, as a product waits for the one before it in its sum
template <class F, class G>
__device__ __forceinline__ void small_product(f32x16& acc, const F& P, int rb, const G& Q, int cb, int k0, int k1, int lane) {
  half8 f[2][2][4];
  auto read = [&](int to, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f[to][j][0] = P.fragment(rb, k + j, lane);
      f[to][j][1] = P.low_fragment(rb, k + j, lane);
      f[to][j][2] = Q.fragment(cb, k + j, lane);
      f[to][j][3] = Q.low_fragment(cb, k + j, lane);
    }
  };
  f32x16 low[2] = {};
  acc = f32x16{};
  auto multiply = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      low[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[c][j][1], f[c][j][2], low[0], 0, 0, 0);
      low[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[c][j][0], f[c][j][3], low[1], 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[c][j][0], f[c][j][2], acc, 0, 0, 0);
    }
  };
  if (k0 < k1) read(0, k0);
  for (int k = k0; k < k1; k += 4) {
    if (k + 2 < k1) read(1, k + 2);
    multiply(0);
    if (k + 4 < k1) read(0, k + 4);
    if (k + 2 < k1) multiply(1);
  }
  acc += low[0] + low[1];
}
// block (rows j, k i) from accumulators, as put_block leaves it
__device__ __forceinline__ void small_put(const LdsFactor<false>& f, int ib, int jb, const f32x16& v, int lane) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    half4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 h, l;
      split(v[4 * g + e], h, l);
      hi[e] = h; lo[e] = l;
    }
    _Float16* p = f.entry(jb * 32 + (lane & 31), ib * 32 + 8 * g + 4 * (lane >> 5));
    *reinterpret_cast<half4*>(p) = hi;
    *reinterpret_cast<half4*>(p + f.low()) = lo;
  }
}

template <typename T, typename OUT>
__global__ void __launch_bounds__(64 * SMALL_WAVES) ns_small_k(NsTable t, NsSteps a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ double red[SMALL_WAVES];
  const NsMatrix& q = t.m[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = q.n, m = q.m, nb = n / 32, mb = m / 32;
  _Float16* const at = reinterpret_cast<_Float16*>(smem);
  const LdsFactor<false> XT{at, n / 16}, AB{at + n * m * 2, n / 16};
  const LdsFactor<true> X{at + n * m * 2 + n * n * 2, m / 16};
  const int rows = (int)q.rows, cols = (int)q.cols, R = q.tall ? m : n, C = q.tall ? n : m;

  // Eight neighbours of a row a thread and round, lanes down the rows; all loads before the first wait.
  constexpr int ROUNDS = SMALL_TILES * 32 * 32 / 64 / 8;
  const int pieces = R * C / 8;
  const T* src = reinterpret_cast<const T*>(q.src);
  float u[ROUNDS][8], b[ROUNDS][8];
#pragma unroll
  for (int o = 0; o < ROUNDS; ++o) {
    const int p = threadIdx.x + o * 64 * SMALL_WAVES, r = p % R, c = p / R * 8, left = p < pieces && r < rows ? cols - c : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[o][e] = e < left ? to_f32(src[r * q.ld_src + c + e]) : 0.f;
      b[o][e] = e < left && q.momentum ? q.momentum[r * cols + c + e] : 0.f;
    }
  }
  double sum = 0.0;
#pragma unroll
  for (int o = 0; o < ROUNDS; ++o) {
    if (q.momentum) {
      const int p = threadIdx.x + o * 64 * SMALL_WAVES, r = p % R, c = p / R * 8, left = p < pieces && r < rows ? cols - c : 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        b[o][e] = fmaf(a.mu, b[o][e], u[o][e]);
        if (e < left) q.momentum[r * cols + c + e] = b[o][e];
        u[o][e] = fmaf(a.mu, b[o][e], u[o][e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += (double)u[o][e] * u[o][e];
  }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lane == 0) red[wave] = sum;
  __syncthreads();
  sum = red[0];
  for (int w = 1; w < SMALL_WAVES; ++w) sum += red[w];
  double by;
  const int small = start_scale(sum, a.eps, a.x[0], &by);
  // as a factor of rows r and k c, and as one of rows c and k r (whose neighbouring rows are 8 numbers apart)
#pragma unroll
  for (int o = 0; o < ROUNDS; ++o) {
    const int p = threadIdx.x + o * 64 * SMALL_WAVES, r = p % R, c = p / R * 8;
    if (p >= pieces) break;
    _Float16 *along = q.tall ? XT.entry(r, c) : X.entry(r, c), *turned = q.tall ? X.entry(c, r) : XT.entry(c, r);
    const int along_low = q.tall ? XT.low() : X.low(), turned_low = q.tall ? X.low() : XT.low();
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      _Float16 h, l;
      split((float)((double)u[o][e] * by), h, l);
      hi[e] = h; lo[e] = l;
      turned[e * 8] = h;
      turned[turned_low + e * 8] = l;
    }
    *reinterpret_cast<half8*>(along) = hi;
    *reinterpret_cast<half8*>(along + along_low) = lo;
  }
  __syncthreads();

  const int tiles = nb * nb;  // of A and B: one a wavefront, and two wavefronts each for A's sums
  const int middle = mb / 2 * 2, tile_a = wave >> 1, half = wave & 1;
  float* partial = reinterpret_cast<float*>(smem) + n * m;  // [tiles][16][64], where A goes afterwards
#pragma unroll 1
  for (int k = 0; k < a.steps; ++k) {
    const int up = max(0, small - k * a.growth), next_up = max(0, small - (k + 1) * a.growth);
    f32x16 acc[SMALL_TILES];
    // A = X X^T
    if (tile_a < tiles) {
      small_product(acc[0], X, tile_a / nb, X, tile_a % nb, half ? middle : 0, half ? X.kb : middle, lane);
      if (half)
#pragma unroll
        for (int e = 0; e < 16; ++e) partial[(tile_a * 16 + e) * 64 + lane] = acc[0][e];
    }
    __syncthreads();
    if (tile_a < tiles && !half)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[0][e] += partial[(tile_a * 16 + e) * 64 + lane];
    __syncthreads();
    if (tile_a < tiles && !half) {
      const float to_a = a.a[k] / (a.x[k] * a.x[k]);
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[0][e] = ldexpf(acc[0][e] * to_a, -2 * up);
      small_put(AB, tile_a / nb, tile_a % nb, acc[0], lane);
    }
    __syncthreads();
    // B = a I + b A + c A A, in A's place
    const int ib = wave / nb, jb = wave % nb;
    if (wave < tiles) {
      const float cb = a.cb / a.a[k], cc = a.cc / (a.a[k] * a.a[k]);
      small_product(acc[0], AB, ib, AB, jb, 0, AB.kb, lane);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const _Float16* p = AB.entry(jb * 32 + (lane & 31), ib * 32 + 8 * g + 4 * (lane >> 5));
        const half4 hi = *reinterpret_cast<const half4*>(p), lo = *reinterpret_cast<const half4*>(p + AB.low());
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool diagonal = ib == jb && acc_row(4 * g + e, lane) == (lane & 31);
          acc[0][4 * g + e] = (fmaf(cc, acc[0][4 * g + e], cb * ((float)hi[e] + (float)lo[e])) + (diagonal ? a.ca : 0.f)) * a.b[k];
        }
      }
    }
    __syncthreads();
    if (wave < tiles) small_put(AB, ib, jb, acc[0], lane);
    __syncthreads();
    // X <- B X; the last one with dst's columns along the lanes
    const bool last = k + 1 == a.steps, turn = last && q.tall;
    const int all = nb * mb, tiles_across = turn ? nb : mb;
    const LdsFactor<false> P = turn ? XT : AB, Q = turn ? AB : XT;
#pragma unroll
    for (int o = 0; o < SMALL_TILES; ++o) {
      const int tile = wave + o * SMALL_WAVES;
      if (tile < all) small_product(acc[o], P, tile / tiles_across, Q, tile % tiles_across, 0, AB.kb, lane);
    }
    const float unscale = (last ? 1.f : a.x[k + 1]) / (a.b[k] * a.x[k]);
    const int power = last ? -up : next_up - up;
    __syncthreads();  // every wavefront has read X^T
    float* result = reinterpret_cast<float*>(smem);  // the last X, as it lies in dst: where X^T was
#pragma unroll
    for (int o = 0; o < SMALL_TILES; ++o) {
      const int tile = wave + o * SMALL_WAVES;
      if (tile >= all) break;
      const int i = tile / tiles_across, j = tile % tiles_across;
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[o][e] = ldexpf(acc[o][e] * unscale, power);
      if (last) {
#pragma unroll
        for (int e = 0; e < 16; ++e) result[(i * 32 + acc_row(e, lane)) * C + j * 32 + (lane & 31)] = acc[o][e];
        continue;
      }
      small_put(XT, i, j, acc[o], lane);
      _Float16* p = X.entry(i * 32 + acc_row(0, lane), j * 32 + (lane & 31));
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        _Float16 h, l;
        split(acc[o][e], h, l);
        p[acc_row(e, 0) * 8] = h;
        p[X.low() + acc_row(e, 0) * 8] = l;
      }
    }
    __syncthreads();
  }
  const float* result = reinterpret_cast<const float*>(smem);
  for (int c = lane; c < cols; c += 64)
    for (int r = wave; r < rows; r += 4 * SMALL_WAVES) {
      float o[4], w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int rk = min(r + k * SMALL_WAVES, rows - 1);
        o[k] = result[rk * C + c];
        w[k] = q.master ? q.master[rk * cols + c] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) put_result<OUT>(q, r + k * SMALL_WAVES, c, o[k], a.decay, w[k]);
    }
}

// Gives every matrix of the table its workgroups; blocks(q): how many.
template <class F>
uint32_t spread(NsTable& t, F blocks) {
  int64_t at = 0;
  for (int i = 0; i < t.count; ++i) {
    t.first[i] = (int)at;
    at += blocks(t.m[i]);
  }
  for (int i = t.count; i < NS_TABLE; ++i) t.first[i] = INT_MAX;
  return (uint32_t)at;
}

template <int SIDE, int MODE, bool DEEP, typename OUT>
hipError_t launch_product(uint32_t blocks, const NsTable& t, const NsStep& p, hipStream_t st) {
  typedef NsTile<SIDE, DEEP> T;
  static bool attr_done = false;  // one flag per instantiation
  const auto kern = ns_product_k<SIDE, MODE, DEEP, OUT>;
  if (!attr_done) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
    if (e != hipSuccess) return e;
    attr_done = true;
  }
  kern<<<blocks, 64 * T::NW, T::LDS, st>>>(t, p);
  return hipGetLastError();
}
// Tiles of side `by` of matrix q's product, and their k.
template <int MODE>
int64_t tiles_of(const NsMatrix& q, int by) {
  const int64_t n = q.n / by;
  return MODE == NS_GRAM || MODE == NS_POLY ? n * (n + 1) / 2 : n * (q.m / by);
}
template <int MODE>
int64_t k_of(const NsMatrix& q) { return MODE == NS_GRAM ? q.m : q.n; }

// Equal tiles of 256 that leave a few for a round of their own: how many, and how many workgroups share the k range of each.  0: none that do.
template <int MODE>
int rest_of(const NsTable& t, int* parts) {
  const NsMatrix& z = t.m[t.count - 1];
  int64_t all = 0;
  for (int i = 0; i < t.count; ++i) {
    if (k_of<MODE>(t.m[i]) != k_of<MODE>(z)) return 0;
    all += tiles_of<MODE>(t.m[i], 256);
  }
  const int rest = (int)(all % 256);
  if (rest == 0 || rest > 128 || all < 256 || rest >= tiles_of<MODE>(z, 256) || k_of<MODE>(z) < NS_REST_K || t.count == NS_TABLE) return 0;
  *parts = std::min(NS_REST_PARTS, 256 / rest);
  return rest;
}

template <int SIDE, int MODE, typename OUT>
hipError_t product_of(NsTable& t, const NsStep& p, hipStream_t st) {
  constexpr int K = 16 * NsTile<SIDE, true>::KS;
  const auto parts_of = [&](const NsMatrix& q, int64_t most) { return (k_of<MODE>(q) / K + most - 1) / most; };
  int64_t most = 1 << 20;  // stages of a workgroup
  if constexpr (SIDE < 256) {
    // k ranges that the launch takes least time with, of those whose workgroups lie side by side; the longest of equal ones
    double least = 0.0;
    for (int64_t shared = 1 << 13; shared >= NS_SHARED_STAGES; shared /= 2) {
      NsTiles runs[NS_TABLE];
      int64_t units = 0, parts = 1;
      for (int i = 0; i < t.count; ++i) {
        const int64_t by = parts_of(t.m[i], shared), tiles = tiles_of<MODE>(t.m[i], SIDE);
        runs[i] = {tiles * by, (double)((k_of<MODE>(t.m[i]) / K + by - 1) / by)};
        units += (tiles * by + 7) / 8 * 8;
        parts = std::max(parts, by);
      }
      if (parts > 1 && units > NS_SHARED_UNITS) break;
      const double span = ns_span(runs, t.count);
      if (parts == 1 || span < least) {
        least = span;
        most = shared;
      }
    }
  }
  const uint32_t blocks = spread(t, [&](NsMatrix& q) {
    q.parts = (int)parts_of(q, most);
    q.tile0 = q.alone = 0;
    q.tiles = (int)tiles_of<MODE>(q, SIDE);
    return (int64_t)(q.tiles * q.parts + 7) / 8 * 8;
  });
  if constexpr (SIDE < 256) {
    if (blocks <= 256) return launch_product<SIDE, MODE, true, OUT>(blocks, t, p, st);
  } else {
    int parts;
    if (const int rest = rest_of<MODE>(t, &parts)) {
      NsTable u = t;
      u.m[u.count] = t.m[t.count - 1];
      NsMatrix &q = u.m[u.count - 1], &r = u.m[u.count];
      ++u.count;
      q.tiles -= rest;
      r.tile0 = q.tiles;
      r.tiles = rest;
      r.parts = parts;
      const uint32_t more = spread(u, [](const NsMatrix& x) { return (int64_t)(x.tiles * x.parts + 7) / 8 * 8; });
      r.alone = u.first[u.count - 1];
      return launch_product<SIDE, MODE, false, OUT>(more, u, p, st);
    }
  }
  return launch_product<SIDE, MODE, false, OUT>(blocks, t, p, st);
}
// Tiles of 256 or 128 by how long the launch takes with them, 64 where there would be few of 128.
template <int MODE, typename OUT = float>
hipError_t product(NsTable& t, int side, const NsStep& p, hipStream_t st) {
  NsTiles large[NS_TABLE + 1], middle[NS_TABLE];
  int64_t tiles = 0, k = 0;
  for (int i = 0; i < t.count; ++i) {
    large[i] = {tiles_of<MODE>(t.m[i], 256), (double)k_of<MODE>(t.m[i]) + (MODE == NS_POLY ? NS_COST_256_POLY : NS_COST_256)};
    middle[i] = {tiles_of<MODE>(t.m[i], 128), (double)k_of<MODE>(t.m[i]) * 0.25 * NS_COST_128};
    tiles += middle[i].count;
    k = std::max(k, k_of<MODE>(t.m[i]));
  }
  int runs = t.count, parts;
  if (const int rest = rest_of<MODE>(t, &parts)) {
    large[runs - 1].count -= rest;
    large[runs++] = {rest * parts, (double)k / parts + NS_COST_256_REST};
  }
  if (side >= 256 && ns_span(large, runs) < ns_span(middle, t.count)) return product_of<256, MODE, OUT>(t, p, st);
  if (side >= 128 && tiles >= (k < NS_LONG_K ? NS_TILES_128 : NS_TILES_128 / 2)) return product_of<128, MODE, OUT>(t, p, st);
  return product_of<64, MODE, OUT>(t, p, st);
}

// The products of one step.
hipError_t step_of(NsTable& t, int side, const NsStep& gram, const NsStep& poly, const NsStep& apply, bool last, int dt_dst, hipStream_t st) {
  hipError_t e = product<NS_GRAM>(t, side, gram, st);
  if (e == hipSuccess) e = product<NS_POLY>(t, side, poly, st);
  if (e != hipSuccess) return e;
  if (!last) return product<NS_APPLY>(t, side, apply, st);
  if (dt_dst == DT_BF16) return product<NS_LAST, bf16>(t, side, apply, st);
  return product<NS_LAST>(t, side, apply, st);
}

hipError_t steps_of(NsTable& t, int side, int dt_src, int dt_dst, const NsRun& run, unsigned char* shared, hipStream_t st) {
  const uint32_t parts = spread(t, [](const NsMatrix&) { return NS_NORM_PARTS; });
  if (dt_src == DT_BF16) ns_norm_k<bf16><<<parts, 256, 0, st>>>(t, run.mu, reinterpret_cast<unsigned*>(shared));
  else ns_norm_k<float><<<parts, 256, 0, st>>>(t, run.mu, reinterpret_cast<unsigned*>(shared));
  double r = 1.001;  // the norm is at least the largest singular value, but for rounding
  NsScales s;
  if (!ns_scales(run.co, r, &s)) return hipErrorInvalidValue;
  const int growth = ns_growth(run.co);
  const uint32_t squares = spread(t, [](const NsMatrix& q) { return (int64_t)(q.n / 64) * (q.m / 64); });
  if (dt_src == DT_BF16) ns_start_k<bf16><<<squares, 256, 0, st>>>(t, run.mu, run.eps, s.x);
  else ns_start_k<float><<<squares, 256, 0, st>>>(t, run.mu, run.eps, s.x);
  for (int k = 0; k < run.steps; ++k) {
    NsStep gram{}, poly{}, apply{};
    gram.shared = poly.shared = apply.shared = shared;
    gram.grown = apply.grown = k * growth;
    gram.growth = apply.growth = growth;
    gram.unscale = 1.f / (s.x * s.x);
    gram.out_scale = s.a;
    poly.ca = (float)run.co[0];
    poly.cb = (float)run.co[1] / s.a;
    poly.cc = (float)run.co[2] / (s.a * s.a);
    poly.out_scale = s.b;
    apply.unscale = 1.f / (s.b * s.x);
    apply.decay = run.decay;
    r = std::max(s.r_next, 1.0);  // (and what norms below eps are stored as)
    if (!ns_scales(run.co, r, &s)) return hipErrorInvalidValue;
    apply.out_scale = s.x;
    const bool last = k + 1 == run.steps;
    const hipError_t e = step_of(t, side, gram, poly, apply, last, dt_dst, st);
    if (e != hipSuccess) return e;
    if (!last)
      for (int i = 0; i < t.count; ++i) std::swap(t.m[i].xt, t.m[i].xt2);
  }
  return hipGetLastError();
}

hipError_t all_steps_of(const NsTable& t, int dt_src, int dt_dst, const NsRun& run, size_t lds, hipStream_t st) {
  NsSteps a{};
  a.steps = run.steps;
  a.growth = ns_growth(run.co);
  a.mu = run.mu; a.eps = run.eps; a.decay = run.decay;
  a.ca = (float)run.co[0]; a.cb = (float)run.co[1]; a.cc = (float)run.co[2];
  double r = 1.001;
  for (int k = 0; k <= run.steps; ++k) {
    NsScales s;
    if (!ns_scales(run.co, r, &s)) return hipErrorInvalidValue;
    a.x[k] = s.x;
    if (k < run.steps) { a.a[k] = s.a; a.b[k] = s.b; }
    r = std::max(s.r_next, 1.0);
  }
  const auto go = [&](auto kern) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, NS_SMALL_LDS);
    if (e != hipSuccess) return e;
    kern<<<t.count, 64 * SMALL_WAVES, lds, st>>>(t, a);
    return hipGetLastError();
  };
  if (dt_src == DT_BF16) return dt_dst == DT_BF16 ? go(ns_small_k<bf16, bf16>) : go(ns_small_k<bf16, float>);
  return dt_dst == DT_BF16 ? go(ns_small_k<float, bf16>) : go(ns_small_k<float, float>);
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
  hipError_t err = hipSuccess;
  ns_launches(count, false, [&](int i, int64_t* r, int64_t* c) { *r = items[i].rows; *c = items[i].cols; }, [&](const int* which, int n, int side, bool) {
    NsTable t{};
    unsigned char* ws = reinterpret_cast<unsigned char*>(workspace) + ns_shared_bytes(side);
    const int fill = side == NS_SMALL ? 32 : side;
    size_t lds = 0;
    for (int i = 0; i < n; ++i) {
      const NsItem& it = items[which[i]];
      NsMatrix& q = t.m[t.count++];
      q.rows = it.rows; q.cols = it.cols; q.ld_src = it.ld_src; q.ld_dst = it.ld_dst;
      q.src = it.src; q.momentum = it.momentum; q.dst = it.dst; q.master = it.master; q.copy = (bf16*)it.copy;
      q.factor = (float)(run.lr * 0.2 * sqrt((double)std::max(it.rows, it.cols)));
      q.tall = it.rows > it.cols;
      q.n = (int)ns_up(std::min(it.rows, it.cols), fill);
      q.m = (int)ns_up(std::max(it.rows, it.cols), fill);
      if (side == NS_SMALL) {
        lds = std::max(lds, ns_small_lds(it.rows, it.cols));
        static_assert(LdsFactor<true>::BLOCK * 2 == NS_SPREAD_BLOCK, "as ns_small_lds counts");
        continue;
      }
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
    if (err != hipSuccess) return;
    if (side == NS_SMALL) err = all_steps_of(t, dt_src, dt_dst, run, lds, st);
    else err = steps_of(t, side, dt_src, dt_dst, run, reinterpret_cast<unsigned char*>(workspace), st);
  });
  return err;
}

}  // namespace hift
