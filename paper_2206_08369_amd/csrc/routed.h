// Routed packs (pmlp_route and the calls after it): every sample is answered by a
// few models of the pack.  Declarations shared by the host library and the kernels
// of k_route.hip and k_routed.hip.
//
// A slot s = b K + k is the k-th choice of sample b; R = B K slots.  Slots are grouped
// by model, in slot order within a model (so that no sum depends on timing): model m's
// rows stand at places place[m] .. place[m] + count - 1 of the P places, and its range
// is padded to a multiple of kRtPad places that hold no slot.
#pragma once

#include "pmlp_internal.h"

namespace pmlpk {

constexpr int32_t kRtMaxK = 16;     // choices of a sample, at most
constexpr int32_t kRtMaxO = 16;     // outputs, at most
constexpr int32_t kRtPad = 32;      // places a model's range is padded to
constexpr int32_t kRtChunks = 256;  // runs of slots that are counted side by side, at most
constexpr int32_t kRtLdsModels = 16384;  // models whose counters lie in LDS
constexpr int32_t kRtOneSlots = 4096, kRtOneModels = 512;  // that one workgroup groups, at most

// Places of R slots on at most `groups` models, each padded: a multiple of kRtPad, so that rows of P
// values are aligned as one model's places are.
inline int64_t rt_places(int64_t R, int64_t groups) {
  return (R + (kRtPad - 1) * groups + kRtPad - 1) / kRtPad * kRtPad;
}
// Values of a hidden layer of N units, `widest` in the widest model, on those P places: each place,
// padding too, has the units of its own model.
inline int64_t rt_hidden(int64_t R, int64_t P, int64_t widest, int64_t N) {
  const int64_t own = widest * R + (kRtPad - 1) * N;
  return own < widest * P ? own : widest * P;
}

// A work unit: row block `a` and unit chunk `b` of model m, or unit tile `a`, column tile `b`
// and part `c` of its weight gradients; with what a workgroup wants to know of its model, so
// that it starts after one load.
struct RtItem {
  int32_t m, a, b, c;
  int64_t first;           // the model's first unit
  int64_t zoff;            // first of its hidden values, [places / 32][h][32]
  int32_t h, act;          // its units and activation
  int32_t rows, places;    // its rows, and its places
  int32_t place, pad[3];   // its first place
};
static_assert(sizeof(RtItem) == 64, "RtItem layout");

// What the items of a kind are counted in.
struct RtTiles {
  int32_t rt;  // places a row block
  int32_t uc;  // units a chunk, forward
  int32_t du;  // units a tile of the weight gradients
  int32_t df;  // columns a tile of them
  int32_t part;  // places a part of them (a multiple of kRtPad)
};

struct RtPlan {
  int32_t R, K, M, P;      // P: places, at most
  int32_t nchunk, chunk;   // runs of `chunk` slots (a multiple of 64)
  int32_t long_rows;       // rows from which on a model's weight gradients come first
  RtTiles t;
  int32_t F, O;
  const int64_t* seg_off;  // [M+1]
  const int32_t* act;      // [M]
  const int32_t* idx;      // [R]
  int32_t* hist;           // [nchunk][M]
  int32_t* count;          // [M]
  int32_t* place;          // [M+1]
  int64_t* zoff;           // [M+1] first value of model m's hidden rows [h_m][places of m]
  int32_t* ioff;           // [M+1] first forward item
  int32_t* joff;           // [M+1] first weight gradient item
  int32_t* slot;           // [P] slot of each place, or -1
  int32_t* row;            // [P] its sample, or -1
  // gradients: wdy[o][place] = weight dY_o of its slot, 0 where it holds none
  const float *weight, *dY;
  float* wdy;              // [O][P], or null
  RtItem* items;
  RtItem* jitems;          // null: forward only
  int32_t* flag;           // flag[3] is raised by an index outside [-1, M)
};

// Best K scores of each of B rows of M.
hipError_t launch_route(const float* scores, int32_t B, int32_t M, int32_t K, int32_t* idx,
                        float* weight, hipStream_t s);
// dscores [B][M] from the gradients of the weights.
hipError_t launch_route_bwd(const int32_t* idx, const float* weight, const float* dweight, int32_t B,
                            int32_t M, int32_t K, float* dscores, hipStream_t s);

// count, place, zoff, ioff, joff, slot and the items.
hipError_t launch_rt_plan(const RtPlan& p, hipStream_t s);

struct RtArgs {
  const float* X;   // [B][F]
  const float* W1;  // [Npad][F4]
  const float* V1;  // [Npad][F4], or null (no gate)
  const float* W2;  // [O][ldw]
  int64_t ldw;
  const int32_t* act;      // [M]
  const int64_t* seg_off;  // [M+1]
  int32_t F, F4, O, K, M, P;
  const int32_t *count, *place;
  const int64_t* zoff;
  const int32_t *slot, *row;
  const RtItem* items;
  const int32_t* nitems;
  int32_t most;      // items, at most
  float* part;       // [R][parts][O] sums over each wave's units (forward)
  int32_t parts;
  // gradients
  const float* weight;  // [R]
  const float* dY;      // [B][O]
  float *dZ, *dU, *H;   // [places of m / 32][h_m][32] at zoff[m]
  float* dwpart;        // [R][parts]
};

// Shapes of the tile kernel, by the pack and the slots.
struct RtShape {
  int32_t na, nb;  // 32-row operand tiles of a wave: projections' rows, samples
};
inline int32_t rt_units(const RtShape& s, bool gated) { return gated ? 64 : 64 * s.na; }
inline int32_t rt_rows(const RtShape& s) { return 64 * s.nb; }
hipError_t launch_rt_tile(const RtArgs& a, const RtShape& sh, bool train, hipStream_t s);

// Few slots: each on its own, straight from the indices.
constexpr int32_t kRtFewUnits = 64;  // units a workgroup
struct RtFew {
  const int32_t* idx;  // [R]
  int32_t R, chunks;   // chunks of kRtFewUnits units, of the widest model
  int32_t* flag;
};
hipError_t launch_rt_few(const RtArgs& a, const RtFew& f, hipStream_t s);
// The same and Y at once, a workgroup for each sample; chunks: of 16 units.
constexpr int32_t kRtSampleChunks = 16;  // K times chunks, at most
hipError_t launch_rt_sample(const RtArgs& a, const RtFew& f, const float* weight, float* Y, hipStream_t s);

// Y[b] = sum_k weight[b][k] sum of the parts of slot (b, k) that its model has.
struct RtJoin {
  const int32_t* idx;
  const float* weight;
  const int64_t* seg_off;
  int32_t B, K, M, O;
  int32_t parts;  // stride
  int32_t uc;     // units a part
  const float* part;
  float* Y;
};
hipError_t launch_rt_join(const RtJoin& a, hipStream_t s);

struct RtGrad {
  RtArgs a;
  RtTiles t;
  int32_t R;
  int64_t N;
  const RtItem* jitems;
  const int32_t* njitems;
  int32_t jmost;
  int32_t nparts;        // parts of a model with every slot
  float *dW1, *dV1, *dW2;
  const float* wdy;      // (RtPlan)
  float* wpart;          // [nparts][k][N][F] where nparts > 1
  float* w2part;         // [nparts][O][N] where nparts > 1
  const int32_t* mid;
  const uint32_t* fmask;
  int32_t fmw;
};
// Gradients of the weights and, from j (O = 1), of the slots' weights: Y[slot] = the sum of
// its parts.
hipError_t launch_rt_weights(const RtGrad& g, const RtShape& sh, const RtJoin& j, hipStream_t s);

}  // namespace pmlpk
