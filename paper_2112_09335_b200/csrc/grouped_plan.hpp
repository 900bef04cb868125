// Host side of the products grouped by expert and of the orthogonalised updates: what a call asks for, what is refused, and the
// sizes of workspaces, and the scales of orthogonalised updates (computed on the device).  Nothing of CUDA in here, so that it can be tested on its own.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "grouped_words.hpp"

namespace gcn_admm_grouped {

enum Type { kF32 = 0, kBf16 = 1, kF16 = 2 };
inline int size_of(int type) { return type == kF32 ? 4 : 2; }
inline long long cdiv(long long a, long long b) { return (a + b - 1) / b; }

constexpr int kMaxGroups = 1024;            // their row ranges lie in shared memory
constexpr int kMaxWidth = 1 << 20;          // widths of operands
constexpr long long kMaxRows = 0x7fffff00;  // row numbers and those of a tile behind them are ints
constexpr int kMaxSide = 32768;             // rows and columns of a matrix to orthogonalise
constexpr int kMaxSteps = 64;
constexpr int kMaxBatch = 65535;
constexpr long long kMaxLd = 1LL << 38;     // strides: products with row numbers stay inside 64 bits

// y[i] = x[i] W_g (transposed: x[i] W_g^T) for the rows offsets[g] <= i < offsets[g+1].  Strides in elements.
struct Product {
  int type, out_type;
  const void* x;
  long long ldx;
  const void* w;
  long long ldw, stride_w;
  bool transposed;
  const int* offsets;
  int groups;
  long long rows;
  int k, n;
  void* y;
  long long ldy;
  bool unsplit = false;   // no room for images of fp32 weights: every tile splits them for itself
};
// dw_g = sum of x[i]^T y[i] over the rows of group g.
struct ProductTn {
  int type, out_type;
  const void* x;
  long long ldx;
  const void* y;
  long long ldy;
  const int* offsets;
  int groups;
  long long rows;
  int ka, nb;
  void* dw;
  long long lddw, stride_dw;
};
struct Orthogonal {
  int type, out_type;
  int batch, rows, cols;
  const void* g;
  long long ldg, stride_g;
  int steps;
  const float* coefficients;
  float eps, scale;
  void* out;
  long long ldo, stride_o;
};

inline bool aligned(const void* p, int type) { return reinterpret_cast<std::uintptr_t>(p) % (std::uintptr_t)size_of(type) == 0; }
inline bool good_types(int type, int out_type) { return type >= kF32 && type <= kF16 && (out_type == type || out_type == kF32); }
inline bool good_strides(long long a) { return a >= 0 && a <= kMaxLd; }

// Fills in the strides left at 0 and returns what is wrong with the call, or NULL.  Pointers are looked at, not followed.
inline const char* check(Product& p) {
  if (!good_types(p.type, p.out_type)) return "unknown type, or an out_type that is neither the type nor GCN_ADMM_F32";
  if (p.groups < 1 || p.groups > kMaxGroups) return "n_groups must be 1..1024";
  if (p.rows < 0 || p.rows > kMaxRows) return "rows must be 0..2147483392";
  if (p.k < 1 || p.n < 1 || p.k > kMaxWidth || p.n > kMaxWidth) return "k and n must be 1..1048576";
  if (!good_strides(p.ldx) || !good_strides(p.ldw) || !good_strides(p.stride_w) || !good_strides(p.ldy)) return "a stride is negative or too large";
  const int w_rows = p.transposed ? p.n : p.k, w_cols = p.transposed ? p.k : p.n;
  if (p.ldx == 0) p.ldx = p.k;
  if (p.ldw == 0) p.ldw = w_cols;
  if (p.stride_w == 0) p.stride_w = (long long)w_rows * p.ldw;
  if (p.ldy == 0) p.ldy = p.n;
  if (p.ldx < p.k || p.ldw < w_cols || p.ldy < p.n) return "a leading dimension is smaller than the width of its matrix";
  if (p.rows == 0) return nullptr;
  if (!p.x || !p.w || !p.y) return "NULL matrix";
  if (!aligned(p.x, p.type) || !aligned(p.w, p.type) || !aligned(p.y, p.out_type)) return "a matrix is not aligned to its elements";
  return nullptr;
}
inline const char* check(ProductTn& p) {
  if (!good_types(p.type, p.out_type)) return "unknown type, or an out_type that is neither the type nor GCN_ADMM_F32";
  if (p.groups < 1 || p.groups > kMaxGroups) return "n_groups must be 1..1024";
  if (p.rows < 0 || p.rows > kMaxRows) return "rows must be 0..2147483392";
  if (p.ka < 1 || p.nb < 1 || p.ka > kMaxWidth || p.nb > kMaxWidth) return "ka and nb must be 1..1048576";
  if (!good_strides(p.ldx) || !good_strides(p.ldy) || !good_strides(p.lddw) || !good_strides(p.stride_dw)) return "a stride is negative or too large";
  if (p.ldx == 0) p.ldx = p.ka;
  if (p.ldy == 0) p.ldy = p.nb;
  if (p.lddw == 0) p.lddw = p.nb;
  if (p.stride_dw == 0) p.stride_dw = (long long)p.ka * p.lddw;
  if (p.ldx < p.ka || p.ldy < p.nb || p.lddw < p.nb) return "a leading dimension is smaller than the width of its matrix";
  if (p.groups > 1 && p.stride_dw < (long long)(p.ka - 1) * p.lddw + p.nb) return "the results of two groups overlap";
  if (!p.dw || (p.rows > 0 && (!p.x || !p.y))) return "NULL matrix";
  if (!aligned(p.x, p.type) || !aligned(p.y, p.type) || !aligned(p.dw, p.out_type)) return "a matrix is not aligned to its elements";
  return nullptr;
}

// The iteration acts on every singular value s alone: s <- s (a + b s^2 + c s^4).  Largest |s| after a step that starts from 0..most,
// and the largest |a + b t + c t^2| on the way (the norm of the matrix that X is multiplied with).
struct Growth {
  double value, factor;
};
// Where these may have their maxima beside the ends of the interval: up to two s of a step's value, one t = s^2 of its factor; below 0: none.
struct Stationary {
  double s[2], value[2], t, factor;
};
GROUPED_BOTH double step_factor(double t, double a, double b, double c) { return fabs(a + t * (b + t * c)); }
GROUPED_BOTH Stationary stationary(double a, double b, double c) {
  Stationary at{{-1.0, -1.0}, {0.0, 0.0}, -1.0, 0.0};
  const auto consider = [&](int i, double t) {
    if (!(t > 0.0)) return;
    at.s[i] = sqrt(t);
    at.value[i] = at.s[i] * step_factor(t, a, b, c);
  };
  if (c == 0.0) {
    if (b != 0.0) consider(0, -a / (3.0 * b));
    return at;
  }
  if (-b / (2.0 * c) > 0.0) {
    at.t = -b / (2.0 * c);
    at.factor = step_factor(at.t, a, b, c);
  }
  const double d = 9.0 * b * b - 20.0 * a * c;   // of a + 3 b t + 5 c t^2
  if (d >= 0.0) {   // its roots, without the difference that loses one of them where c is small
    const double q = -0.5 * (3.0 * b + copysign(sqrt(d), b));
    consider(0, q / (5.0 * c));
    consider(1, a / q);
  }
  return at;
}
GROUPED_BOTH Growth grow(double most, double a, double b, double c, const Stationary& at) {
  const double end = step_factor(most * most, a, b, c);
  Growth g{most * end, fmax(fabs(a), end)};
  for (int i = 0; i < 2; ++i)
    if (at.s[i] > 0.0 && at.s[i] < most) g.value = fmax(g.value, at.value[i]);
  if (at.t > 0.0 && at.t < most * most) g.factor = fmax(g.factor, at.factor);
  return g;
}
GROUPED_BOTH Growth grow(double most, double a, double b, double c) { return grow(most, a, b, c, stationary(a, b, c)); }

// Scales of a matrix between its products: powers of two that bring what the bound of its singular values allows just below 2^15.  The bound starts from
// ||G|| / (||G|| + eps), which only the device knows, rounded up to a power of two, and follows the steps; it is kept above 2^-96, and that of P above
// 2^-400 (far below, fp32 results are zero for any `scale`), so that no factor leaves the range of fp32.
constexpr int kLeastBound = -96;
GROUPED_BOTH int scale_for(double most) { return 14 - ilogb(most); }   // the power of two
GROUPED_BOTH double first_bound(double ratio) {
  if (!(ratio > 0.0 && ratio < 1.0)) return 1.0;   // (a matrix of zeros or one that is not finite needs no scale)
  int e;
  if (frexp(ratio, &e) == 0.5) --e;
  return ldexp(1.0, e < kLeastBound ? kLeastBound : e);
}
// What the products of a step do beside multiplying: S = gram (X X^T), P = square (S S) + linear S + diagonal I, X' = scale (move (P X)); `scale` is
// the caller's in the last step, apart because move may be so small that with it fp32 would end.
struct StepFactors {
  float gram, square, linear, diagonal, move, scale;
};
GROUPED_BOTH double bound_behind(const Growth& g) { return fmax(g.value, 0x1p-96); }
// Of a step from a bound of `most` that grows by g.  `last`: the result leaves under `out_scale` instead of one of its own.
GROUPED_BOTH StepFactors step_factors(double most, const Growth& g, double a, double b, double c, bool last, float out_scale) {
  const int x = scale_for(most), s = scale_for(most * most), p = scale_for(fmax(g.factor, 0x1p-400));
  const int to = last ? 0 : scale_for(bound_behind(g));
  return StepFactors{(float)ldexp(1.0, s - 2 * x), (float)ldexp(c, p - 2 * s), (float)ldexp(b, p - s), (float)ldexp(a, p), (float)ldexp(1.0, to - p - x),
                     last ? out_scale : 1.f};
}
constexpr double kMostValue = 16.0, kMostFactor = 1024.0;

inline const char* check(Orthogonal& p) {
  if (!good_types(p.type, p.out_type)) return "unknown type, or an out_type that is neither the type nor GCN_ADMM_F32";
  if (p.batch < 1 || p.batch > kMaxBatch) return "batch must be 1..65535";
  if (p.rows < 1 || p.cols < 1 || p.rows > kMaxSide || p.cols > kMaxSide) return "rows and cols must be 1..32768";
  if (p.steps < 0 || p.steps > kMaxSteps) return "n_steps must be 0..64";
  if (p.steps > 0 && !p.coefficients) return "NULL coefficients";
  if (!(p.eps >= 0.f) || !std::isfinite(p.eps) || !std::isfinite(p.scale)) return "eps must be a finite number of at least 0, scale a finite number";
  if (!good_strides(p.ldg) || !good_strides(p.stride_g) || !good_strides(p.ldo) || !good_strides(p.stride_o)) return "a stride is negative or too large";
  if (p.ldg == 0) p.ldg = p.cols;
  if (p.stride_g == 0) p.stride_g = (long long)p.rows * p.ldg;
  if (p.ldo == 0) p.ldo = p.cols;
  if (p.stride_o == 0) p.stride_o = (long long)p.rows * p.ldo;
  if (p.ldg < p.cols || p.ldo < p.cols) return "a leading dimension is smaller than the width of its matrix";
  if (p.batch > 1 && p.stride_o < (long long)(p.rows - 1) * p.ldo + p.cols) return "two results overlap";
  if (!p.g || !p.out) return "NULL matrix";
  if (!aligned(p.g, p.type) || !aligned(p.out, p.out_type)) return "a matrix is not aligned to its elements";
  double most = 1.0;
  for (int i = 0; i < p.steps; ++i) {
    const float* const c = p.coefficients + 3 * i;
    if (!std::isfinite(c[0]) || !std::isfinite(c[1]) || !std::isfinite(c[2])) return "a coefficient is not finite";
    const Growth g = grow(most, c[0], c[1], c[2]);
    if (g.value > kMostValue || g.factor > kMostFactor) return "the coefficients let singular values grow above 16, or their factors above 1024";
    most = std::max(g.value, std::ldexp(1.0, kLeastBound));
  }
  return nullptr;
}

}  // namespace gcn_admm_grouped
