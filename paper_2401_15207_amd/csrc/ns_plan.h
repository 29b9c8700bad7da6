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
// such tiles cover it, else 128; 64 in launches that would have fewer than NS_FEW_TILES of 128 in the symmetric products.
constexpr int64_t NS_FEW_TILES = 160;
inline int ns_side(int64_t rows, int64_t cols) { return std::min(rows, cols) >= 1280 && rows * cols >= int64_t(64) * 256 * 256 ? 256 : 128; }
// From how many tiles on a launch takes them that large.
constexpr int64_t NS_TILES_256 = 192, NS_TILES_128 = 128;
// Workgroups that share tiles' k ranges, in launches that have fewer workgroups than this otherwise; no range is shorter than so many
// stages.  Their sums: 64 KB (128 x 128) each, and a counter.
constexpr int64_t NS_SHARED_UNITS = 304, NS_SHARED_STAGES = 8;
constexpr size_t NS_SHARED_BYTES = NS_SHARED_UNITS * (4 + 128 * 128 * 4);

// Whose products are fewer for a bf16 result: smaller ones are bound by latency, and further off with them.
inline bool ns_large(int64_t rows, int64_t cols) { return std::min(rows, cols) >= 512; }

inline int64_t ns_up(int64_t x, int side) { return (x + side - 1) / side * side; }
// Matrices whose factors X, X^T and A (two fp16 numbers to an entry) fit a compute unit's LDS with sides filled up to multiples of 32, and
// whose tiles of 32 x 32 two a wavefront at most: all steps in one launch, if a list holds no other.  (Among others they ride along: their
// few tiles take no launches of their own.)
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

// Work space of one matrix: X, X^T before and after a step, A and B, two fp16 numbers to an entry, two diagonals, the sums
// of its norm, and how far that is below eps.
constexpr int NS_NORM_PARTS = 256;
inline size_t ns_bytes(int64_t rows, int64_t cols) {
  const int side = ns_side(rows, cols);
  const int64_t n = ns_up(std::min(rows, cols), side), m = ns_up(std::max(rows, cols), side);
  return (size_t)(3 * n * m + 2 * n * n) * 4 + (size_t)n * 8 + NS_NORM_PARTS * 8 + 16;
}
// The launches of a list: launch(indexes, how many, tile side, large) for matrices that share them, those with the most work first (their tiles
// then do not come last).  shape(i, &rows, &cols); matrices without entries are left out.
// few: large ones apart, as they take fewer products.
template <class S, class F>
inline void ns_launches(int count, bool few, S shape, F launch) {
  bool all_small = true;
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
  for (int kind = 0; kind < (few ? 3 : 2); ++kind) {
    const int side = kind == 0 ? 256 : 128;
    const bool large = few && kind < 2;
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
      if (r == 0 || c == 0 || ns_side(r, c) != side || (few && ns_large(r, c) != large)) continue;
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
  for (bool few : {false, true})
    ns_launches(count, few, shape, [&](const int* which, int n, int side, bool) {
      size_t sum = 0;
      if (side == NS_SMALL) return;
      for (int i = 0; i < n; ++i) {
        int64_t r, c;
        shape(which[i], &r, &c);
        sum += ns_bytes(r, c);
      }
      most = std::max(most, NS_SHARED_BYTES + sum);
    });
  return most;
}

}  // namespace hift
