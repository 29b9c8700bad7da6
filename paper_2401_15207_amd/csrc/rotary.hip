// Rotary positions: the table of angles, the rotation of rows of heads by it, forward and backward, and the rotation of a batch's new
// queries and keys on their way into a paged cache.  And what else a model's new rows need by their place in such a cache: positions, angles, the wanted logits.
//
// Pair i of a head (of the first `rot` columns: (i, i + rot / 2) or (2 i, 2 i + 1)) turns by position * rate_i.  Rotated by (cos, sin) of the table:
//   y1 = x1 cos - x2 sin, y2 = x2 cos + x1 sin;   the adjoint has -sin for sin.
// Formed in fp32 from either type and rounded once.  All three kernels are bound by memory or, with few rows, by their launch (3 to 5 us on the device): heads of
// 2048 x 64 of 128 bf16 (67 MB) 12.7 us, 5.3 TB/s; a table of 65536 x 64 (34 MB written) 7.4 us, 4.5 TB/s; prompts of 4300 tokens appended, 32 / 32 heads (204 MB),
// 40 us, 5.1 TB/s.
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "common.h"
#include "kernels.h"
#include "paged_cache.h"

namespace hift {
namespace {

constexpr int BLK = 256;

// ---- table ----
struct TableArgs {
  int half;         // pairs
  int64_t first, count;
  double amplitude;
  float2* cs;
  double turns[ROTARY_ROT_MAX / 2];  // whole turns a position, by pair
  double step_cos[ROTARY_ROT_MAX / 2], step_sin[ROTARY_ROT_MAX / 2];  // and their cosine and sine
};

// cos and sin of 2 pi f, |f| <= 1/2: the multiple of a quarter nearest to f aside, what is left is an angle of at most pi / 4, of which the
// Taylor series' terms up to t^14 leave less than 1e-13, far below what rounding to fp32 does.
__device__ __forceinline__ void turn_of(double f, double& c, double& s) {
  const double q = rint(4.0 * f);
  const double t = 6.283185307179586476925 * fma(-0.25, q, f), u = t * t;
  double sn = 1.0 / 6227020800.0, cn = -1.0 / 87178291200.0;
  sn = fma(sn, u, -1.0 / 39916800.0); cn = fma(cn, u, 1.0 / 479001600.0);
  sn = fma(sn, u, 1.0 / 362880.0);    cn = fma(cn, u, -1.0 / 3628800.0);
  sn = fma(sn, u, -1.0 / 5040.0);     cn = fma(cn, u, 1.0 / 40320.0);
  sn = fma(sn, u, 1.0 / 120.0);       cn = fma(cn, u, -1.0 / 720.0);
  sn = fma(sn, u, -1.0 / 6.0);        cn = fma(cn, u, 1.0 / 24.0);
  sn = fma(sn, u, 1.0) * t;           cn = fma(cn, u, -0.5);
  cn = fma(cn, u, 1.0);
  const int k = (int)q & 3;  // quarters: -2 .. 2
  c = k & 1 ? sn : cn;
  s = k & 1 ? cn : sn;
  if (k == 1 || k == 2) c = -c;
  if (k >= 2) s = -s;
}

// A thread takes a pair at TABLE_ROWS positions, the first from its angle (in turns and 64 bits: at position 2^20 the error is below 2^-32 of a turn) and
// each next one by the rotation of one position, which takes a fifth of the operations (65536 x 64: 12 us with every angle by itself, 7.4 so) and adds less than
// 2^-50 a step.
constexpr int TABLE_ROWS = 8;
__global__ void __launch_bounds__(BLK) rotary_table_k(TableArgs p) {
  const int64_t first = (int64_t)blockIdx.x * BLK, group0 = first / p.half;
  const unsigned at = (unsigned)(first - group0 * p.half) + threadIdx.x, group = at / (unsigned)p.half, pair = at - group * (unsigned)p.half;
  const int64_t row = (group0 + group) * TABLE_ROWS;
  if (row >= p.count) return;
  const double a = (double)(p.first + row) * p.turns[pair], dc = p.step_cos[pair], ds = p.step_sin[pair];
  double c, s;
  turn_of(a - rint(a), c, s);
  c *= p.amplitude;
  s *= p.amplitude;
  float2* out = p.cs + row * p.half + pair;
  const int n = (int)min(p.count - row, (int64_t)TABLE_ROWS);
#pragma unroll
  for (int k = 0; k < TABLE_ROWS; ++k) {
    if (k < n) out[(int64_t)k * p.half] = make_float2((float)c, (float)s);
    const double next = fma(c, dc, -s * ds);
    s = fma(s, dc, c * ds);
    c = next;
  }
}

// ---- rotation ----
// V consecutive elements of a row
template <typename T, int V>
struct alignas(sizeof(T) * V) Elems {
  T v[V];
};
// The same of a row that nobody reads again: it leaves the caches first.
template <typename T, int V>
__device__ __forceinline__ Elems<T, V> last_read(const T* p) {
  typedef T Wide __attribute__((ext_vector_type(V)));
  return __builtin_bit_cast(Elems<T, V>, __builtin_nontemporal_load(reinterpret_cast<const Wide*>(p)));
}

// Written out, so that every variant gives the same bits.
__device__ __forceinline__ float first_of(float x1, float x2, float2 t) { return fmaf(-x2, t.y, x1 * t.x); }
__device__ __forceinline__ float second_of(float x1, float x2, float2 t) { return fmaf(x1, t.y, x2 * t.x); }

// Units of a head: 2 V columns of V pairs each for the first `half` / V of them, then V columns that are copied.
template <typename T, int V>
struct Unit {
  float2 cs[V];
  int a, b;  // columns of the two loads
  bool turns;
  __device__ __forceinline__ Unit(int u, int half, bool pairs, const float2* __restrict__ table_row, float sign) {
    turns = u * V < half;
    if (turns) {
      a = pairs ? 2 * u * V : u * V;
      b = pairs ? a + V : a + half;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        cs[e] = table_row[u * V + e];
        cs[e].y *= sign;
      }
    } else {
      a = b = 2 * half + (u - half / V) * V;
    }
  }
  template <bool PAIRS>
  __device__ __forceinline__ void turn(Elems<T, V>& x, Elems<T, V>& y) const {
    if constexpr (PAIRS && V > 1) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        T& p = 2 * e < V ? x.v[(2 * e) % V] : y.v[(2 * e) % V];
        T& q = 2 * e < V ? x.v[(2 * e + 1) % V] : y.v[(2 * e + 1) % V];
        const float x1 = to_f32(p), x2 = to_f32(q);
        p = from_f32<T>(first_of(x1, x2, cs[e]));
        q = from_f32<T>(second_of(x1, x2, cs[e]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float x1 = to_f32(x.v[e]), x2 = to_f32(y.v[e]);
        x.v[e] = from_f32<T>(first_of(x1, x2, cs[e]));
        y.v[e] = from_f32<T>(second_of(x1, x2, cs[e]));
      }
    }
  }
};

struct RotaryArgs {
  int heads, hd, half, units;  // units of a head
  int groups;                  // ceil(heads / heads of a thread)
  bool in_place;
  int64_t rows, ldx, ldy;
  const void* x;
  void* y;
  const int32_t* positions;
  int seq, table_rows;
  const float2* cs;
  float sign;
};

// A thread takes one unit of every groups-th head of a row, HPT heads in all: it reads its angles once for them, and neighbouring threads
// read neighbouring units.
template <typename T, int V, bool PAIRS, int HPT>
__global__ void __launch_bounds__(BLK) rotary_k(RotaryArgs p) {
  const int per_row = p.groups * p.units;
  const int64_t first = (int64_t)blockIdx.x * BLK;
  int64_t row = first / per_row;  // uniform
  const int in = (int)(first - row * per_row) + (int)threadIdx.x;
  row += in / per_row;
  if (row >= p.rows) return;
  const int item = in % per_row, h0 = item / p.units, u = item % p.units;
  const int pos = p.positions ? p.positions[row] : (int)(row % p.seq);
  const int at = min(max(pos, 0), p.table_rows - 1);
  const Unit<T, V> unit(u, p.half, PAIRS, p.cs + (int64_t)at * p.half, p.sign);
  if (!unit.turns && p.in_place) return;
  const T* x = (const T*)p.x + row * p.ldx;
  T* y = (T*)p.y + row * p.ldy;
  typedef Elems<T, V> E;
  E a[HPT], b[HPT];
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = h0 + j * p.groups;
    if (h < p.heads) {
      a[j] = *reinterpret_cast<const E*>(x + (int64_t)h * p.hd + unit.a);
      if (unit.turns) b[j] = *reinterpret_cast<const E*>(x + (int64_t)h * p.hd + unit.b);
    }
  }
#pragma unroll
  for (int j = 0; j < HPT; ++j) {
    const int h = h0 + j * p.groups;
    if (h < p.heads) {
      if (unit.turns) {
        unit.template turn<PAIRS>(a[j], b[j]);
        *reinterpret_cast<E*>(y + (int64_t)h * p.hd + unit.b) = b[j];
      }
      *reinterpret_cast<E*>(y + (int64_t)h * p.hd + unit.a) = a[j];
    }
  }
}

// Elements that one load takes: 16 bytes, or as many as divide every distance and address
int vector_of(int size, int64_t distances, uintptr_t addresses) {
  for (int v = 16 / size; v > 1; v /= 2)
    if (distances % v == 0 && addresses % (uintptr_t)(v * size) == 0) return v;
  return 1;
}
int64_t any_bits(std::initializer_list<int64_t> v) {
  int64_t b = 0;
  for (int64_t x : v) b |= x;
  return b;
}

template <typename T, int V>
hipError_t rotate_v(RotaryArgs p, bool pairs, hipStream_t st) {
  p.units = p.half / V + (p.hd - 2 * p.half) / V;
  // Few rows want every thread that there is; many want the angles read once for four heads.  bf16, 32 heads of 128, us, four heads a thread / one: 256 rows 5.0 / 3.6,
  // 1024 6.8 / 6.7, 2048 (2^19 units) 9.5 / 10.4, 4096 14.2 / 18.1.
  const bool many = p.rows * p.heads * p.units >= int64_t(1) << 19;
  const int hpt = many ? 4 : 1;
  p.groups = (p.heads + hpt - 1) / hpt;
  const int64_t n = p.rows * p.groups * p.units, blocks = (n + BLK - 1) / BLK;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  const dim3 grid((unsigned)blocks);
  if (pairs) {
    if (many) rotary_k<T, V, true, 4><<<grid, BLK, 0, st>>>(p);
    else rotary_k<T, V, true, 1><<<grid, BLK, 0, st>>>(p);
  } else {
    if (many) rotary_k<T, V, false, 4><<<grid, BLK, 0, st>>>(p);
    else rotary_k<T, V, false, 1><<<grid, BLK, 0, st>>>(p);
  }
  return hipGetLastError();
}

// ---- new tokens into a paged cache ----
struct AppendArgs {
  CacheView c;
  int heads, half, units;
  int64_t rows, ld, ldq;
  int max_new;
  const void* qkv;
  void* q;  // or null
  const float2* cs;
  int table_rows;
};

// One workgroup a new token; its row and page are uniform.  A thread keeps one unit's angles and walks over the heads of q, then of k.  The row is read past the
// caches (204 MB in all 47.5 -> 40 us); what is written is not, the attention reads it next (8192 tokens, 32 / 32 heads 67 us, written past them too 77).
template <typename T, int V, bool PAIRS>
__global__ void __launch_bounds__(BLK) append_k(AppendArgs p) {
  const int s = (int)(blockIdx.x / (unsigned)p.max_new), token = (int)(blockIdx.x % (unsigned)p.max_new);
  const CacheSeq of = cache_seq(p.c, s, p.rows, p.max_new);
  if (token >= of.fresh) return;
  const int64_t row = of.row0 + token;
  const int hd = p.c.head_dim, kv = p.c.kv_heads, pos = of.cached + token;
  const T* x = (const T*)p.qkv + row * p.ld;
  const int page = cache_page(p.c, s, pos);
  const int64_t slot = (int64_t)page * p.c.page_stride + (int64_t)(pos & (p.c.page - 1)) * hd;  // of head 0
  const int64_t head_at = (int64_t)p.c.page * hd;
  typedef Elems<T, V> E;
  const int per = BLK / p.units, lane_head = threadIdx.x / p.units, u = threadIdx.x % p.units;
  if (lane_head < per) {
    const Unit<T, V> unit(u, p.half, PAIRS, p.cs + (int64_t)min(pos, p.table_rows - 1) * p.half, 1.f);
    const int from = p.q ? 0 : p.heads, to = page < 0 ? p.heads : p.heads + kv;
    for (int h = from + lane_head; h < to; h += per) {
      E a = last_read<T, V>(x + (int64_t)h * hd + unit.a), b;
      if (unit.turns) {
        b = last_read<T, V>(x + (int64_t)h * hd + unit.b);
        unit.template turn<PAIRS>(a, b);
      }
      T* y = h < p.heads ? (T*)p.q + row * p.ldq + (int64_t)h * hd : (T*)p.c.k + slot + (h - p.heads) * head_at;
      *reinterpret_cast<E*>(y + unit.a) = a;
      if (unit.turns) *reinterpret_cast<E*>(y + unit.b) = b;
    }
  }
  if (page < 0) return;
  constexpr int VV = 16 / (int)sizeof(T);
  typedef Elems<T, VV> EV;
  const T* v = x + (int64_t)(p.heads + kv) * hd;
  const int pieces = hd / VV;
  for (int i = threadIdx.x; i < kv * pieces; i += BLK) {
    const int h = i / pieces, c = (i % pieces) * VV;
    *reinterpret_cast<EV*>((T*)p.c.v + slot + h * head_at + c) = last_read<T, VV>(v + (int64_t)h * hd + c);
  }
}

// Position of a new row, -1 for one that belongs to no sequence or lies beyond max_new: the sequence is looked for among the starts.
__device__ __forceinline__ int position_of(const CacheView& c, int64_t row, int64_t rows, int max_new) {
  if (c.sequences == 0) return -1;
  int lo = 0, hi = c.sequences;  // the last sequence that starts at the row or before
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (c.starts[mid] <= row) lo = mid;
    else hi = mid;
  }
  const CacheSeq of = cache_seq(c, lo, rows, max_new);
  const int64_t token = row - of.row0;
  return token >= 0 && token < of.fresh ? of.cached + (int)token : -1;
}

// One thread a row
__global__ void __launch_bounds__(BLK) cache_positions_k(CacheView c, int64_t rows, int max_new, int32_t* positions) {
  const int64_t row = (int64_t)blockIdx.x * BLK + threadIdx.x;
  if (row < rows) positions[row] = max(position_of(c, row, rows, max_new), 0);
}

// The table's entries of the rows' positions, one after the other: a thread one pair
__global__ void __launch_bounds__(BLK) cache_angles_k(CacheView c, int64_t rows, int max_new, int half, const float2* __restrict__ cs, int table_rows, float2* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * BLK + threadIdx.x, row = i / half;
  if (row >= rows) return;
  const int at = min(max(position_of(c, row, rows, max_new), 0), table_rows - 1);
  out[i] = cs[(int64_t)at * half + (i - row * half)];
}

// One workgroup a wanted row: its logits, or zeros where the row belongs to no sequence (nothing has computed its attention).
template <typename T, int V>
__global__ void __launch_bounds__(BLK) wanted_logits_k(CacheView c, int64_t rows, int max_new, const int32_t* __restrict__ pick, int vocab, const T* __restrict__ x, int64_t ldx,
                                                       T* __restrict__ y, int64_t ldy) {
  const int64_t i = blockIdx.x, row = pick ? min(max((int64_t)pick[i], (int64_t)0), rows - 1) : i;
  const bool none = position_of(c, row, rows, max_new) < 0;
  typedef Elems<T, V> E;
  for (int j = threadIdx.x * V; j < vocab; j += BLK * V) {
    E e = *reinterpret_cast<const E*>(x + i * ldx + j);
    if (none) {
#pragma unroll
      for (int k = 0; k < V; ++k) e.v[k] = from_f32<T>(0.f);
    }
    *reinterpret_cast<E*>(y + i * ldy + j) = e;
  }
}
template <typename T, int V>
void wanted_v(const CacheView& c, int64_t rows, int max_new, int64_t n, const int32_t* pick, int vocab, const void* x, int64_t ldx, void* y, int64_t ldy, hipStream_t st) {
  wanted_logits_k<T, V><<<(unsigned)n, BLK, 0, st>>>(c, rows, max_new, pick, vocab, (const T*)x, ldx, (T*)y, ldy);
}

template <typename T, int V>
hipError_t append_v(AppendArgs p, bool pairs, hipStream_t st) {
  p.units = p.half / V + (p.c.head_dim - 2 * p.half) / V;
  const int64_t blocks = (int64_t)p.c.sequences * p.max_new;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (pairs) append_k<T, V, true><<<(unsigned)blocks, BLK, 0, st>>>(p);
  else append_k<T, V, false><<<(unsigned)blocks, BLK, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t rotary_table(int rot, const double* turns, double amplitude, int64_t first, int64_t count, float* cos_sin, hipStream_t st) {
  if (count == 0) return hipSuccess;
  TableArgs p{};
  p.half = rot / 2; p.first = first; p.count = count; p.amplitude = amplitude; p.cs = (float2*)cos_sin;
  std::copy(turns, turns + rot / 2, p.turns);
  for (int i = 0; i < p.half; ++i) {
    p.step_cos[i] = cos(6.283185307179586476925 * turns[i]);
    p.step_sin[i] = sin(6.283185307179586476925 * turns[i]);
  }
  const int64_t blocks = ((count + TABLE_ROWS - 1) / TABLE_ROWS * p.half + BLK - 1) / BLK;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  rotary_table_k<<<(unsigned)blocks, BLK, 0, st>>>(p);
  return hipGetLastError();
}

hipError_t rotary(int dt, bool pairs, bool backward, int64_t rows, int heads, int hd, int rot, const void* x, int64_t ldx, void* y, int64_t ldy,
                  const int32_t* positions, int seq, const float* cos_sin, int table_rows, hipStream_t st) {
  if (rows == 0 || heads == 0) return hipSuccess;
  RotaryArgs p{};
  p.heads = heads; p.hd = hd; p.half = rot / 2; p.in_place = x == y;
  p.rows = rows; p.ldx = ldx; p.ldy = ldy; p.x = x; p.y = y;
  p.positions = positions; p.seq = seq; p.table_rows = table_rows; p.cs = (const float2*)cos_sin; p.sign = backward ? -1.f : 1.f;
  const int size = dt == DT_BF16 ? 2 : 4;
  const int v = vector_of(size, any_bits({hd, p.half, ldx, ldy}), reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y));
  if (dt == DT_BF16) {
    if (v == 8) return rotate_v<bf16, 8>(p, pairs, st);
    if (v == 4) return rotate_v<bf16, 4>(p, pairs, st);
    if (v == 2) return rotate_v<bf16, 2>(p, pairs, st);
    return rotate_v<bf16, 1>(p, pairs, st);
  }
  if (v == 4) return rotate_v<float, 4>(p, pairs, st);
  if (v == 2) return rotate_v<float, 2>(p, pairs, st);
  return rotate_v<float, 1>(p, pairs, st);
}

hipError_t cache_positions(const CacheView& c, int64_t rows, int max_new, int32_t* positions, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  cache_positions_k<<<(unsigned)((rows + BLK - 1) / BLK), BLK, 0, st>>>(c, rows, max_new, positions);
  return hipGetLastError();
}

hipError_t cache_angles(const CacheView& c, int64_t rows, int max_new, int rot, const float* cos_sin, int table_rows, float* out, hipStream_t st) {
  if (rows == 0) return hipSuccess;
  const int64_t blocks = (rows * (rot / 2) + BLK - 1) / BLK;
  if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
  cache_angles_k<<<(unsigned)blocks, BLK, 0, st>>>(c, rows, max_new, rot / 2, (const float2*)cos_sin, table_rows, (float2*)out);
  return hipGetLastError();
}

hipError_t wanted_logits(int dt, const CacheView& c, int64_t rows, int max_new, int64_t n, const int32_t* pick, int vocab, const void* x, int64_t ldx, void* y, int64_t ldy,
                         hipStream_t st) {
  if (n == 0) return hipSuccess;
  const int v = vector_of(dt == DT_BF16 ? 2 : 4, any_bits({vocab, ldx, ldy}), reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y));
  if (dt == DT_BF16) {
    if (v == 8) wanted_v<bf16, 8>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
    else if (v == 4) wanted_v<bf16, 4>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
    else if (v == 2) wanted_v<bf16, 2>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
    else wanted_v<bf16, 1>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
  } else {
    if (v == 4) wanted_v<float, 4>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
    else if (v == 2) wanted_v<float, 2>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
    else wanted_v<float, 1>(c, rows, max_new, n, pick, vocab, x, ldx, y, ldy, st);
  }
  return hipGetLastError();
}

hipError_t cache_append(int dt, const CacheView& c, int heads, bool pairs, int rot, const float* cos_sin, int table_rows, int64_t rows, int max_new,
                        const void* qkv, int64_t ld, void* q, int64_t ldq, hipStream_t st) {
  if (rows == 0 || c.sequences == 0 || max_new == 0) return hipSuccess;
  AppendArgs p{};
  p.c = c; p.heads = heads; p.half = rot / 2;
  p.rows = rows; p.ld = ld; p.ldq = ldq; p.max_new = max_new;
  p.qkv = qkv; p.q = q; p.cs = (const float2*)cos_sin; p.table_rows = table_rows;
  const int v = vector_of(dt == DT_BF16 ? 2 : 4, any_bits({c.head_dim, p.half}), 0);
  if (dt == DT_BF16) {
    if (v == 8) return append_v<bf16, 8>(p, pairs, st);
    if (v == 4) return append_v<bf16, 4>(p, pairs, st);
    if (v == 2) return append_v<bf16, 2>(p, pairs, st);
    return append_v<bf16, 1>(p, pairs, st);
  }
  if (v == 4) return append_v<float, 4>(p, pairs, st);
  if (v == 2) return append_v<float, 2>(p, pairs, st);
  return append_v<float, 1>(p, pairs, st);
}

}  // namespace hift
