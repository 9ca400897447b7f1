// The orthogonalised update of a pack's weight matrices (pmlp_orthogonalize,
// pmlp_muon_step).  Declarations shared by the host library and k_newton.hip.
#pragma once

#include "pmlp_internal.h"

namespace pmlpk {

// The quintic whose iteration takes every singular value in (0, 1] towards 1 (Muon:
// Jordan and others, 2024): x <- x (a + b x^2 + c x^4).
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr int32_t kNsTile = 128;   // rows and columns of a workgroup's tile
constexpr int32_t kNsPiece = 8192; // entries of a piece of the momentum's pass, about

// One model's matrix: rows x cols, with r = min(rows, cols) and c = max(rows, cols); the
// iteration's X is it, or its transpose where rows > cols.  rp, cp: r and c rounded up to
// 32, with zeros behind them.
struct NsMat {
  int64_t src;    // first entry in the caller's buffers, row stride ld
  int64_t wsrc;   // .. and in the handle's weights, row stride wld
  int32_t rows, cols, ld, wld;
  int32_t r, c, rp, cp;
  int64_t xo, ao; // first entry of its X (of rp cp) and A (of rp rp) in a slice's workspace
  int32_t piece0, pieces;  // its pieces
  int32_t m, pad;
};
struct NsPiece {
  int32_t mat, row0, rows, pad;
};
struct NsItem {
  int32_t mat, i, j, pad;  // tile (i, j)
};

struct NsArgs {
  const NsMat* mats;
  const NsPiece* pieces;
  const float* G;
  const float* mom_in;  // null: no momentum
  float* mom_out;
  float mu;
  int32_t nesterov;
  double* sums;         // [pieces] sums of squares
  // a slice of the matrices: planes of the high and the low half of every entry
  _Float16 *X[2], *XT[2];  // [2][nx] each: X and its transpose, before and after a step
  _Float16 *A, *P;         // [2][na]
  int64_t nx, na;
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
// X = U / |U|_F
hipError_t launch_ns_load(const NsArgs& a, const NsItem* items, int32_t n, hipStream_t s);
enum NsProduct { NS_GRAM = 0, NS_POLY = 1, NS_STEP = 2, NS_LAST = 3 };
// from X[from], XT[from]
hipError_t launch_ns_product(const NsArgs& a, int what, int from, const NsItem* items, int32_t n,
                             hipStream_t s);

}  // namespace pmlpk
