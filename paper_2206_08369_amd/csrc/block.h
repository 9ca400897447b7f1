// Block packs (pmlp_create_block): a gated hidden layer, a layer norm over each
// model's hidden units, or both.  Declarations shared by the host library and
// the kernels of k_block*.hip.
#pragma once

#include "pmlp_internal.h"

namespace pmlpk {

constexpr float kNormEps = 1e-5f;

// Consecutive hidden units of one model: what one wave (workgroup) of the
// forward sums.  Models wider than the plan's cap have several pieces, which the
// output kernels merge in order.
struct BlkPiece {
  int64_t n0;
  int32_t len, m;
};
static_assert(sizeof(BlkPiece) == 16, "BlkPiece layout");

// The pack as the block kernels see it.
struct BlkPack {
  const float* W1;      // [Npad][F4]
  const float* V1;      // [Npad][F4], or null (no gate)
  float* W2;            // [O][ldw]
  float* gain;          // [Npad], or null (no norm)
  float* shift;         // [Npad]
  int64_t ldw;          // = Npad
  int64_t N;
  int32_t M, O, F, F4;
  const int64_t* seg_off;  // [M+1]
  const int32_t* mid;      // [Npad]
  const int32_t* actn;     // [Npad]
  const BlkPiece* pieces;  // in unit order
  const int32_t* poff;     // [M+1] first piece of each model
  int32_t npieces;
};

// The forward's tiles: up to 16 units of one model, in unit order.
struct BlkTile {
  int32_t n0, cnt, m, act;
};
static_assert(sizeof(BlkTile) == 16, "BlkTile layout");

// Outputs as the kernels pad them
__host__ __device__ inline int blk_om(int32_t O) { return O <= 2 ? 2 : O <= 4 ? 4 : 16; }

// Where the sums of model m lie: in the stored path its pieces poff[m] .. poff[m+1]-1;
// in the fused path (toff set) its runs.  A run is what one wave sums of a model: its
// tiles among `run` consecutive ones, r run .. (r + 1) run - 1; its record is m + r.
struct BlkMap {
  const int32_t* toff;  // [M+1] first tile of each model, or null
  int32_t run;
  const float* csum;    // with a norm: [pieces or records][blk_om] sums of gain W2 over their units
};
inline int64_t blk_records(const BlkPack& p, int32_t ntiles, int32_t run) {
  return (int64_t)p.M + (ntiles - 1) / run;
}

struct BlkFwdArgs {
  const float* X;  // [B][F]
  int32_t B, F;
  const BlkTile* tiles;
  int32_t ntiles;
  int32_t SC;      // samples of a workgroup, a multiple of 32
  int32_t wpc;     // workgroups for each SC samples
  int32_t waves;   // of a workgroup
  int32_t run;     // see BlkMap
  float* part;     // records of blk_planes planes of Br samples
  float* csum;     // see BlkMap
  int32_t Br;      // multiple of 32
};
#define PMLP_BLK_FWD_DECL(OM)                                               \
  int blk_fwd_slots_##OM(const BlkPack& p, int32_t SC, int32_t waves, bool runs); \
  hipError_t launch_blk_fused_fwd_##OM(const BlkPack& p, const BlkFwdArgs& a, hipStream_t s);
PMLP_BLK_FWD_DECL(2)
PMLP_BLK_FWD_DECL(16)
#undef PMLP_BLK_FWD_DECL

// C[p][q] = sum_k P[p][k] Q[q][k] of fp32 rows (16-byte aligned; K a multiple of 4):
// stored (EPI_STORE, EPI_GRAD: columns below ncols) or applied to C (EPI_SGD).
struct BlkGemm {
  const float *P, *Q;
  int64_t ldp, ldq, NP;
  int32_t NQ, K;
  float* out;
  int64_t ldo;
  int32_t ncols;
  float lr;
  const float* lrm;
  const int32_t* mid;
};
hipError_t launch_blk_gemm(const BlkGemm& a, int epi, hipStream_t s);

// Per piece and sample, planar: part[(piece * PQ + q) * Bp + b], q < O the sums
// S_o over the piece's units, and with a norm the mean and the sum of squared
// deviations of its hidden values after them; S_o are then sums of the deviations
// from that mean.
inline int32_t blk_planes(const BlkPack& p) { return p.O + (p.gain ? 2 : 0); }

// Z (and U) stored batch-minor: Zt [Npad][Bp], Ut [Npad][Bp] (null: no gate).
hipError_t launch_blk_fwd(const BlkPack& p, const float* Zt, const float* Ut, int32_t Bp,
                          float* part, float* csum, hipStream_t s);

// Logits out[b sb + m sm + o] of B samples from the pieces' sums.
hipError_t launch_blk_out(const BlkPack& p, const BlkMap& map, int64_t records, const float* part,
                          int32_t Bp, int32_t B, float* out, int64_t sm, int64_t sb, hipStream_t s);

// Losses and what the backward reads, from the pieces' sums:
//   G [M][Bp][blk_om]  dLoss/dlogits (0 past the batch and the outputs)
//   R [M][Bp][4]  with a norm: mu, r, a1, a2 (see k_blk_bwd)
//   Gs [M][O]     with a norm: sum_b G
// y: labels int32 [B], or Y float [B][O] for the regression head; flags as
// launch_ce.
struct BlkLoss {
  const int32_t* y;
  const float* Y;
  int32_t B;
  float* G;
  float* R;
  float* Gs;
  float* loss;
  int32_t* flag;
  const float* lrm;
};
// Br: the records' sample stride, Bp: G's and R's.
hipError_t launch_blk_loss(const BlkPack& p, const BlkMap& map, int64_t records, const float* part,
                           int32_t Br, int32_t Bp, const BlkLoss& l, hipStream_t s);

// Gradients of the output weights, gains and shifts (stored, or applied with
// the rate lr or lrm[m] where dW2 is null).
struct BlkGrads {
  float* dW2;     // [O][N]
  float* dgain;   // [N]
  float* dshift;  // [N]
  float lr;
  const float* lrm;
};
// dZ over Zt and dU over Ut, in place.
hipError_t launch_blk_bwd(const BlkPack& p, float* Zt, float* Ut, int32_t Bp, const float* G,
                          const float* R, const float* Gs, const BlkGrads& g, hipStream_t s);

// The whole backward, with Z computed again: dW1 and dV1 [N][F] stored, or applied
// to W1 and V1 where dW1 is null; the rest as launch_blk_bwd.  Bp: a multiple of 32.
struct BlkBwdArgs {
  const float* X;  // [B][F]
  int32_t B, F, Bp;
  int32_t SC;      // (set by the launcher) samples a chunk
  const BlkTile* tiles;
  int32_t ntiles;
  const float *G, *R, *Gs;
  float *dW1, *dV1;
  BlkGrads g;
};
constexpr int32_t kBlkFusedCols = 128;  // input columns (F4) of the fused kernels, at most
#define PMLP_BLK_BWD_DECL(OM) \
  hipError_t launch_blk_fused_bwd_##OM(const BlkPack& p, BlkBwdArgs a, hipStream_t s);
PMLP_BLK_BWD_DECL(2)
PMLP_BLK_BWD_DECL(4)
PMLP_BLK_BWD_DECL(16)
#undef PMLP_BLK_BWD_DECL

// Forward, loss and backward in one launch: workgroup w takes the models whose first
// tile is one of tiles w * group .. (w + 1) * group - 1, for all samples.  As
// launch_blk_fused_fwd with runs of one tile (f.SC .. f.run are not read), launch_blk_loss and
// launch_blk_fused_bwd (b.tiles: the forward's).
constexpr int32_t kBlkLocalBatch = 256;  // samples, at most
constexpr int32_t kBlkLocalGroup = 8;    // waves of a workgroup, and `group` at most
struct BlkLocal {
  int32_t group;
  const int32_t* toff;
};
// (slots: workgroups that the device holds at once, 0: it cannot run)
#define PMLP_BLK_LOCAL_DECL(OM)                                                           \
  int blk_local_slots_##OM(const BlkPack& p, int32_t Bp, int32_t group);                  \
  hipError_t launch_blk_local_##OM(const BlkPack& p, const BlkLocal& g, const BlkFwdArgs& f, \
                                   const BlkLoss& l, const BlkBwdArgs& b, hipStream_t s);
PMLP_BLK_LOCAL_DECL(2)
PMLP_BLK_LOCAL_DECL(4)
PMLP_BLK_LOCAL_DECL(16)
#undef PMLP_BLK_LOCAL_DECL

// V1 (tag 6, like W1), gain 1, shift 0 (either may be null).
hipError_t launch_blk_init(float* V1, int64_t N, int32_t F, int32_t F4, float bound, uint64_t key,
                           float* gain, float* shift, hipStream_t s);

}  // namespace pmlpk
