// Host arithmetic of the Newton-Schulz orthogonalisation (muon.hip): scales of the fp16 factors, work space and launches of a list of
// matrices.  No HIP in here: the host compiler checks it.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace hift {

// One step maps a singular value t to t (a + b t^2 + c t^4).  With all of them in [0, r], the entries of X, of A = X X^T and of
// B = a I + b A + c A^2 are at most r, r^2 and q = max |a + b l + c l^2| over l in [0, r^2], since no entry of a matrix is larger than its
// largest singular value.  Each factor is stored times the largest power of two that keeps it at or below 2^15, where a sum of two fp16
// numbers holds 22 bits of whatever is not tiny against the largest entry there can be.
struct NsScales {
  float x, a, b;   // of X, A and B
  double r_next;   // bound on the singular values after the step
};
inline float ns_pow2(double bound) { return (float)ldexp(1.0, (int)floor(log2(32768.0 / bound))); }
// false: the coefficients let the singular values grow out of fp16's range
inline bool ns_scales(const double (&co)[3], double r, NsScales* s) {
  const double a = co[0], b = co[1], c = co[2], l_max = r * r;
  const auto q_of = [&](double l) { return fabs(a + b * l + c * l * l); };
  const auto t_of = [&](double l) { return sqrt(l) * q_of(l); };
  double q = std::max(q_of(0.0), q_of(l_max)), t = t_of(l_max);
  const auto inside = [&](double l) { return l > 0.0 && l < l_max; };
  if (c != 0.0 && inside(-b / (2.0 * c))) q = std::max(q, q_of(-b / (2.0 * c)));
  // extremes of t (a + b t^2 + c t^4): a + 3 b l + 5 c l^2 = 0
  const double disc = 9.0 * b * b - 20.0 * a * c;
  if (c != 0.0 && disc >= 0.0) {
    for (double sign : {-1.0, 1.0}) {
      const double l = (-3.0 * b + sign * sqrt(disc)) / (10.0 * c);
      if (inside(l)) t = std::max(t, t_of(l));
    }
  } else if (c == 0.0 && b != 0.0 && inside(-a / (3.0 * b))) {
    t = std::max(t, t_of(-a / (3.0 * b)));
  }
  // (the square of a large coefficient may not pass fp32 either)
  if (!(r > 0.0) || !(r < 1024.0) || !(q > 0.0) || !(q < 1024.0) || !(t < 1024.0)) return false;
  s->x = ns_pow2(r);
  s->a = ns_pow2(l_max);
  s->b = ns_pow2(q);
  s->r_next = std::max(t, 1e-3) * 1.001;  // (rounding; and a factor of zeros has a scale too)
  return true;
}

// While X is below 1 a step multiplies it by less than 2^ns_growth.
inline int ns_growth(const double (&co)[3]) { return (int)ceil(log2(fabs(co[0]) + fabs(co[1]) + fabs(co[2]) + 1.0)); }

constexpr int NS_STEPS_MAX = 16;   // steps of a call
constexpr int NS_TABLE = 16;       // matrices of a launch
constexpr int64_t NS_SIDE_MAX = 65536;
// Matrices share launches until together they have this many entries: a few large ones fill the last round of a launch's tiles over the
// 256 compute units, more would only need more work space.
constexpr int64_t NS_TOGETHER = int64_t(1) << 28;
// Both sides of a matrix are filled up with zeros to a multiple of this, the largest tile its products can have: 256 where at least 64
// such tiles cover it, else 128; 64 in launches that would have fewer than NS_FEW_TILES of 128 in the symmetric products, where filling up
// costs more than larger tiles give (four matrices of odd sizes up to 1000 take 163 us with 64, 174 with 128; eight of 512 x 2048 496 and
// 463).
constexpr int64_t NS_FEW_TILES = 64;
inline int ns_side(int64_t rows, int64_t cols) { return std::min(rows, cols) >= 1280 && rows * cols >= int64_t(64) * 256 * 256 ? 256 : 128; }
// From how many tiles of 128 on a launch takes them rather than tiles of 64, half as many where k is long.  Below, workgroups are too few and
// each one's chain of stages too long.  Layer 1024 wide: 877 us, 1091 with 64 throughout; two matrices of 512 x 512: 152 us, 247 with 128; four of
// 640 x 640: 197 and 293; 1536 x 6000: 876, with half as many never enough 1001; eight of 512 x 2048: 463, with half as many enough for any k
// 482.
constexpr int64_t NS_TILES_128 = 128, NS_LONG_K = 1536;
// Between tiles of 256 and 128 the shorter of the two launches, each tile taken to cost its k times its entries.  Tiles of 128 pass their
// operands through LDS twice as often: what that costs.  What a tile of 256 costs beside its k is its way in and out, which no second
// workgroup of the compute unit covers; in NS_POLY, which reads the tile's entries of A and writes B's twice, more; and a shared tile's
// (below) the way of its sums through memory.  A layer 4096 wide: 36.3 ms, with 128 throughout 39.1; three matrices of 2048 x 5632 and four of
// 2048 x 2048: 5.6 ms, with 256 for all launches of 192 such tiles or more 6.3.
constexpr double NS_COST_128 = 1.3, NS_COST_256 = 200.0, NS_COST_256_POLY = 800.0, NS_COST_256_REST = 1200.0;
// Tiles' k ranges are shared between workgroups where that shortens a launch and leaves it no more workgroups than NS_SHARED_UNITS; no range
// is shorter than so many stages.  Layer 1024 wide: 880 us, 973 without sharing, 972 with at most 256 workgroups, 912 with
// 512.  Stages: two matrices of 512 x 512 150 us, with 4 157; one of 256 x 1000 121, with 16 127.  The sums: 64 KB (128 x 128) each, and a
// counter.
constexpr int64_t NS_SHARED_UNITS = 304, NS_SHARED_STAGES = 8;
constexpr size_t NS_SHARED_BYTES = NS_SHARED_UNITS * (4 + 128 * 128 * 4);
// So are those of the tiles of 256 that would make a last round for at most half the compute units, by at most so many workgroups a tile and
// where k is at least so long.  With and without: a layer 4096 wide, whose X takes 12 rounds and 16 tiles, 36.8 and 37.3 ms; 4096 x 4200 4.20 and
// 4.29.
constexpr int NS_REST_PARTS = 4;
constexpr int64_t NS_REST_K = 2048;
constexpr size_t NS_REST_BYTES = NS_SHARED_UNITS * 4 + size_t(256) * 256 * 256 * 4;
inline size_t ns_shared_bytes(int side) { return side >= 256 ? NS_REST_BYTES : NS_SHARED_BYTES; }

// For lists whose large matrices go apart from the others (see ns_launches): which are large.
inline bool ns_large(int64_t rows, int64_t cols) { return std::min(rows, cols) >= 512; }
// Beside others they stay in those others' launches while their short sides' squares times the long ones are less than this together: launches of
// their own cost 100 us and more (1000 x 333, 129 x 257, 77 x 1300, 515 x 515: 161 us together, 294 apart).
constexpr int64_t NS_APART = int64_t(1) << 31;

// How long the 256 compute units take over tiles, run by run, each tile to the unit that is free first.  Runs of equal ones: how many and how long.
struct NsTiles {
  int64_t count;
  double length;
};
inline double ns_span(NsTiles* runs, int n) {
  std::sort(runs, runs + n, [](const NsTiles& p, const NsTiles& q) { return p.length > q.length; });
  struct { double free; int64_t units; } at[257];  // units by when they are free, the latest first
  int levels = 1;
  at[0] = {0.0, 256};
  double end = 0.0;
  for (int i = 0; i < n; ++i) {
    for (int64_t left = runs[i].count; left > 0;) {
      const auto first = at[--levels];
      const int64_t take = std::min(left, first.units);
      if (take < first.units) at[levels++] = {first.free, first.units - take};
      left -= take;
      const double done = first.free + runs[i].length;
      end = std::max(end, done);
      int to = levels;
      while (to > 0 && at[to - 1].free < done) --to;
      if (to > 0 && at[to - 1].free == done) {
        at[to - 1].units += take;
        continue;
      }
      for (int l = levels++; l > to; --l) at[l] = at[l - 1];
      at[to] = {done, take};
    }
  }
  return end;
}

inline int64_t ns_up(int64_t x, int side) { return (x + side - 1) / side * side; }
// Matrices whose factors X, X^T and A (two fp16 numbers to an entry) fit a compute unit's LDS with sides filled up to multiples of 32, and
// whose tiles of 32 x 32 two a wavefront at most: all steps in one launch, if a list holds no other (64 x 64: 28 us, 68 in launches for each
// product; four of those, 256 x 64 and 64 x 256: 55 and 82).  (Among others they ride along: their few tiles take no launches of their own.)
constexpr int NS_SMALL = 0, NS_SMALL_TILES = 2;
constexpr size_t NS_SMALL_LDS = 159 * 1024;
constexpr int NS_SPREAD_BLOCK = 1168;  // bytes of a 32 x 16 block of X there
inline size_t ns_small_lds(int64_t rows, int64_t cols) {
  const int64_t n = ns_up(std::min(rows, cols), 32), m = ns_up(std::max(rows, cols), 32);
  return (size_t)(n * m + n * n) * 4 + (size_t)(n / 32) * (m / 16) * 2 * NS_SPREAD_BLOCK;
}
inline bool ns_small(int64_t rows, int64_t cols) {
  const int64_t n = ns_up(std::min(rows, cols), 32) / 32, m = ns_up(std::max(rows, cols), 32) / 32;
  return ns_small_lds(rows, cols) <= NS_SMALL_LDS && n * m <= 8 * NS_SMALL_TILES && n <= 2;
}

// Work space of one matrix: X, X^T before and after a step, A and B, two fp16 numbers to an entry, the sums of its norm, and how far that is
// below eps.
constexpr int NS_NORM_PARTS = 256;
inline size_t ns_bytes(int64_t rows, int64_t cols) {
  const int side = ns_side(rows, cols);
  const int64_t n = ns_up(std::min(rows, cols), side), m = ns_up(std::max(rows, cols), side);
  return (size_t)(3 * n * m + 2 * n * n) * 4 + NS_NORM_PARTS * 8 + 16;
}
// The launches of a list: launch(indexes, how many, tile side, large) for matrices that share them, those with the most work first (their tiles
// then do not come last).  shape(i, &rows, &cols); matrices without entries are left out.
// few: large ones apart, for operators that treat them otherwise.  (All of this library's treat them alike and pass false.)
template <class S, class F>
inline void ns_launches(int count, bool few, S shape, F launch) {
  bool all_small = true, apart = true;
  for (int i = 0; i < count && all_small; ++i) {
    int64_t r, c;
    shape(i, &r, &c);
    all_small = r == 0 || c == 0 || ns_small(r, c);
  }
  if (all_small) {
    int which[NS_TABLE], n = 0;
    for (int i = 0; i < count; ++i) {
      int64_t r, c;
      shape(i, &r, &c);
      if (r > 0 && c > 0) which[n++] = i;
      if (n == NS_TABLE || (i + 1 == count && n > 0)) {
        launch((const int*)which, n, NS_SMALL, false);
        n = 0;
      }
    }
    return;
  }
  if (few) {
    int64_t work = 0;
    bool others = false;
    for (int i = 0; i < count; ++i) {
      int64_t r, c;
      shape(i, &r, &c);
      if (r == 0 || c == 0 || ns_side(r, c) == 256) continue;
      if (ns_large(r, c)) work += std::min(r, c) * r * c;
      else others = true;
    }
    apart = !others || work >= NS_APART;
  }
  for (int kind = 0; kind < (few ? 3 : 2); ++kind) {
    const int side = kind == 0 ? 256 : 128;
    const bool large = few && kind < 2;
    if (kind == 1 && large && !apart) continue;
    int which[NS_TABLE], n = 0;
    int64_t entries = 0, tiles = 0, longest[NS_TABLE];
    const auto flush = [&]() {
      if (n > 0) launch((const int*)which, n, side == 128 && !large && tiles < NS_FEW_TILES ? 64 : side, large);
      n = 0;
      entries = tiles = 0;
    };
    for (int i = 0; i < count; ++i) {
      int64_t r, c;
      shape(i, &r, &c);
      if (r == 0 || c == 0 || ns_side(r, c) != side || (few && kind > 0 && (apart && ns_large(r, c)) != large)) continue;
      if (n == NS_TABLE || (n > 0 && entries + r * c > NS_TOGETHER)) flush();
      int at = n++;
      for (; at > 0 && longest[at - 1] < std::max(r, c); --at) {
        which[at] = which[at - 1];
        longest[at] = longest[at - 1];
      }
      which[at] = i;
      longest[at] = std::max(r, c);
      entries += r * c;
      const int64_t t = ns_up(std::min(r, c), side) / side;
      tiles += t * (t + 1) / 2;
    }
    flush();
  }
}
template <class S>
inline size_t ns_workspace_bytes(int count, S shape) {
  size_t most = 0;
  ns_launches(count, false, shape, [&](const int* which, int n, int side, bool) {
    size_t sum = 0;
    if (side == NS_SMALL) return;
    for (int i = 0; i < n; ++i) {
      int64_t r, c;
      shape(which[i], &r, &c);
      sum += ns_bytes(r, c);
    }
    most = std::max(most, ns_shared_bytes(side) + sum);
  });
  return most;
}

}  // namespace hift
