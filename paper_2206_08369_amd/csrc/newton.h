// The orthogonalised update of a pack's weight matrices (pmlp_orthogonalize,
// pmlp_muon_step).  Declarations shared by the host library and k_newton.hip.
#pragma once

#include <algorithm>
#include <cmath>

#include "pmlp_internal.h"

namespace pmlpk {

// The quintic whose iteration takes every singular value in (0, 1] towards 1 (Muon:
// Jordan and others, 2024): x <- x (a + b x^2 + c x^4).
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr int32_t kNsPiece = 4096; // entries of a piece of the momentum's pass, about
constexpr int32_t kNsGrid = 1 << 21;  // workgroups of a launch, at most (2^32 threads are too many)

// One model's matrix: rows x cols, with r = min(rows, cols) and c = max(rows, cols); the
// iteration's X is it, or its transpose where rows > cols.  rp, cp: r and c rounded up to
// 32, with zeros behind them.
struct NsMat {
  int64_t src;    // first entry in the caller's buffers, row stride ld
  int64_t wsrc;   // .. and in the handle's weights, row stride wld
  int32_t rows, cols, ld, wld;
  int32_t r, c, rp, cp;
  int64_t xo, ao; // first entry of its X (of rp cp) and A (of rp rp) in a slice's workspace
  int64_t ro, co; // .. of its rows' and columns' exponents in those of all
  int32_t piece0, pieces;  // its pieces
  int32_t m;
  int16_t root, grow;  // (ns_scales)
};
struct NsPiece {
  int32_t mat, row0, rows, pad;
};
// Tile (i, j) of a matrix, with all that a workgroup wants to know of it.
struct NsItem {
  int32_t mat, i, j, pad[5];
  NsMat t;
};
static_assert(sizeof(NsItem) == 128, "NsItem layout");

struct NsArgs {
  const NsMat* mats;
  const NsPiece* pieces;
  const float* G;
  const float* mom_in;  // null: no momentum
  float* mom_out;
  float mu;
  int32_t nesterov;
  double* sums;         // [pieces] sums of squares
  // exponents of X's rows and columns before and after a step, [2][nr] and [2][nc]; the rows'
  // largest |U| [nr], the columns' largest |X / rows' scales| in turn [3][nc], as float bits
  int8_t *rows, *cols;
  int64_t nr, nc;
  uint32_t *rmax, *cmax;
  int32_t* uneven;      // [M] whether a column has a scale
  // a slice of the matrices: planes of the high and the low half of every entry
  _Float16 *X[2], *XT[2];  // [2][nx] each: X and its transpose, before and after a step
  _Float16 *A, *P;         // [2][na]
  int64_t nx, na;
  int32_t tile;         // rows and columns of a workgroup's tile: 64 or 128
  // where the result goes: out, or the weights
  float* out;
  float* W;
  float lr, decay;
  const float* lrm;
  const uint32_t* fmask;
  int32_t fmw;
  int32_t* flag;
};

// mom_out = mu mom_in + G and the pieces' sums of squares of U (out null, W null), or,
// with W set, W -= lr (decay W + U).
hipError_t launch_ns_momentum(const NsArgs& a, int32_t piece0, int32_t pieces, bool apply, hipStream_t s);
// Before it, what the scales of turned matrices' rows come from.
hipError_t launch_ns_rows(const NsArgs& a, const NsItem* items, int32_t n, hipStream_t s);
// X = U / |U|_F, with the scales of its rows and columns
hipError_t launch_ns_load(const NsArgs& a, const NsItem* items, int32_t n, hipStream_t s);
enum NsProduct { NS_GRAM = 0, NS_POLY = 1, NS_STEP = 2, NS_LAST = 3 };
// Step `step`, from X[step % 2], XT[step % 2].  items: tiles of `tile` x `tile` (j <= i) of A and P, of `tile` x
// ns_step_columns(tile) of the steps.
inline int32_t ns_step_columns(int32_t tile) { return tile == 64 ? 64 : 256; }
hipError_t launch_ns_product(const NsArgs& a, int what, int step, const NsItem* items, int32_t n,
                             hipStream_t s);

// Exponents that the scales of an r x c X (newton_device.h) are derived with: of sqrt(c), which
// bounds a row's norm by its largest entry, and of 4 (3.45 + 5.64 sqrt(r)), which bounds what a
// step makes of a column's largest entry, but 2^10 at least: most matrices' columns then have scale
// 1, and the largest entry of a column still keeps 2^-24 of itself.
inline void ns_scales(NsMat* t) {
  auto up = [](double v) {
    int e = 0;
    while (std::ldexp(1.0, e) < v) ++e;
    return (int16_t)e;
  };
  t->root = up(std::sqrt((double)t->c));
  t->grow = std::max<int16_t>(10, up(4 * (3.45 + 5.64 * std::sqrt((double)t->r))));
}

// Matrices that fit LDS, a workgroup each: classes 0 .. 7 (r of 1 .. 8 tiles of 16, c up to
// 128), 8 (r up to 16 and c up to 512, or 32 and 256: output weights) and 9 .. 12 (wider, r up to
// 32, 64, 96, 128; their kernel takes every class).
constexpr int kNsClasses = 13, kNsLow = 8, kNsAny = 12;
inline bool ns_low(int32_t r, int32_t c) { return (r <= 16 && c <= 512) || (r <= 32 && c <= 256); }
constexpr size_t kNsSmallLds = 160 * 1024 - 128;  // dynamic LDS of a workgroup, at most
// Strips of two tiles in the lower triangle of tr x tr tiles.
__host__ __device__ constexpr int ns_strips(int tr) {
  int n = 0;
  for (int i = 0; i < tr; ++i) n += i / 2 + 1;
  return n;
}
// Parts that the columns are split in for A = X X^T, where its strips are fewer than the
// waves.
__host__ __device__ constexpr int ns_small_split(int tr, int waves) {
  const int n = waves / ns_strips(tr);
  return n < 1 ? 1 : n > 4 ? 4 : n;
}
// Waves of a workgroup of each class.
constexpr int kNsWaves[kNsClasses] = {4, 4, 4, 4, 8, 16, 16, 16, 4, 8, 8, 8, 8};
// For r up to 32, 64, 96, 128 in eight waves: units of work (32 columns and up to four tiles
// of rows) a wave, and entries a thread loads, at most.
constexpr int kNsUnits[4] = {5, 3, 3, 2}, kNsEntries[4] = {80, 64, 64, 48};
// LDS of an r x c matrix in so many waves.
inline size_t ns_small_lds(int32_t r, int32_t c, int waves) {
  const int cp = (c + 31) / 32 * 32, rp = (r + 31) / 32 * 32, tr = (r + 15) / 16;
  const int split = ns_small_split(tr, waves);
  return (size_t)32 * tr * ((2 * cp + 16) + (2 * rp + 16)) +
         (split > 1 ? (size_t)split * ns_strips(tr) * (tr == 1 ? 1024 : 2048) : 0) + 32 * tr + 2 * cp + 16;
}
// The class of an r x c matrix, or -1.
inline int ns_small_class(int32_t r, int32_t c) {
  if (r > 128 || c > 1280) return -1;
  if (c <= 128) return (r + 15) / 16 - 1;
  if (ns_low(r, c)) return kNsLow;
  const int k = (r - 1) / 32, units = (c + 31) / 32 * (k >= 2 ? 2 : 1);
  if (ns_small_lds(r, c, 8) > kNsSmallLds || units > 8 * kNsUnits[k] || r * c > 512 * kNsEntries[k])
    return -1;
  return kNsLow + 1 + k;
}
// Up to so many matrices go in one launch whatever their classes, and up to twice as many in two,
// the low ones and the others, if one of them has more than 64 rows: each launch ends with workgroups
// that wait for its longest.  Low ones alone are one launch of theirs.  (us, one / two / by class:
// 300 matrices of 1 to 100 rows, 100 columns 65 / 85 / 236, 1,000: 144 / 146 / 241, 2,000: 272 / 259 /
// 313, 6,000: 790 / 692 / 512; 300 of 1 to 64 rows, 64 columns 39 / 49 / 85, 1,000: 97 / 77 / 90, 2,040:
// 186 / 132 / 99.)
constexpr int kNsOneLaunch = 1024;
// From the gradient to the result, a workgroup for each matrix of the list; classes above
// kNsLow: any of the classes.
hipError_t launch_ns_small(const NsArgs& a, int cls, size_t lds, const int32_t* list, int32_t n,
                           int32_t steps, hipStream_t s);

}  // namespace pmlpk
