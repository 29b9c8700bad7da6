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
constexpr int NS_PAD = 128;        // both sides of a matrix are filled up with zeros to a multiple of this
constexpr int64_t NS_SIDE_MAX = 65536;
// Matrices share launches until together they have this many entries: from there on a launch has several tiles for each of the 256
// compute units by itself, and more matrices would only need more work space.
constexpr int64_t NS_TOGETHER = int64_t(1) << 26;

inline int64_t ns_up(int64_t x) { return (x + NS_PAD - 1) / NS_PAD * NS_PAD; }
// Work space of one matrix: X, X^T before and after a step, A and B, two fp16 numbers to an entry, the sums of its norm, and
// how far that is below eps.
constexpr int NS_NORM_PARTS = 256;
inline size_t ns_bytes(int64_t rows, int64_t cols) {
  const int64_t n = ns_up(std::min(rows, cols)), m = ns_up(std::max(rows, cols));
  return (size_t)(3 * n * m + 2 * n * n) * 4 + NS_NORM_PARTS * 8 + 16;
}
// How many matrices from `first` on share launches.  shape(i, &rows, &cols)
template <class F>
inline int ns_together(int first, int count, F shape) {
  int64_t entries = 0;
  int n = 0;
  while (first + n < count && n < NS_TABLE) {
    int64_t r, c;
    shape(first + n, &r, &c);
    if (n > 0 && entries + r * c > NS_TOGETHER) break;
    entries += r * c;
    ++n;
  }
  return n;
}
template <class F>
inline size_t ns_workspace_bytes(int count, F shape) {
  size_t most = 0;
  for (int at = 0; at < count;) {
    const int n = ns_together(at, count, shape);
    size_t sum = 0;
    for (int i = at; i < at + n; ++i) {
      int64_t r, c;
      shape(i, &r, &c);
      sum += r > 0 && c > 0 ? ns_bytes(r, c) : 0;
    }
    most = std::max(most, sum);
    at += n;
  }
  return most;
}

}  // namespace hift
