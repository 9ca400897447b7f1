// Block packs: forward, loss and backward of small packs in one launch.  Compiled once
// per class of outputs (PMLP_BLK_OM: 2, 4 or 16).
//
// A workgroup takes whole models (see BlkLocal), so that nothing it reads comes
// from another one: the tiles' sums, the output gradients and the norm's statistics
// pass from stage to stage through the same buffers as between the three kernels, with
// a barrier of the workgroup between them.  The samples' pieces are made once.
//
// What it saves is launches and the latency at the start of each kernel; what it costs
// is that a model's tiles stay on one CU.  It is taken where each wave has one tile and
// all workgroups run at once (block_local of the host).  Training steps, gated and
// normed, two outputs, in us, three launches -> one: 256 models of 8 units, 10
// columns, 32 samples 18 -> 13; of 48 units, 50 columns, 128 samples 37 -> 30; of 8
// units, 100 columns, 256 samples 67 -> 61.  In two rounds (1024 models of 48 units, one
// tile a wave of four) it lost, 38 -> 81 at 50 columns and 32 samples.

#include "block_loss.h"
#include "block_tiles.h"

#ifndef PMLP_BLK_OM
#error "compile with -DPMLP_BLK_OM=2|4|16"
#endif

namespace pmlpk {

namespace {

constexpr int OM = PMLP_BLK_OM;
constexpr int kRow = OM + 1;  // sums of 64 samples: the loss, and G_o

// The models [m0, m1) of group w.
__device__ __forceinline__ void group_models(const BlkLocal& g, const BlkFwdArgs& f, int w, int M,
                                             int& m0, int& m1) {
  auto first_from = [&](int t) {  // the first model whose first tile is t or later
    if (t >= f.ntiles) return M;
    const int m = f.tiles[t].m;
    return g.toff[m] < t ? m + 1 : m;
  };
  m0 = __builtin_amdgcn_readfirstlane(first_from(w * g.group));
  m1 = __builtin_amdgcn_readfirstlane(first_from((w + 1) * g.group));
}

// The losses and output gradients of models m0 .. m1 - 1, 64 samples of one a wave.
template <bool NORM>
__device__ __forceinline__ void local_loss(const BlkPack& p, const BlkMap& map,
                                           const BlkFwdArgs& f, const BlkLoss& l, int Bp, int m0, int m1, float* red) {
  const int tid = threadIdx.x, lane = tid & 63, nw = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nblk = (Bp + 63) >> 6;
  const float scale = l.Y ? 1.f / ((float)l.B * (float)p.O) : 1.f / (float)l.B;
  for (int i = wave; i < (m1 - m0) * nblk; i += nw) {
    const int m = m0 + i / nblk, b = 64 * (i % nblk) + lane;
    float C[OM], D[OM], gs[OM], loss = 0.f;
    if (NORM) norm_consts<OM>(p, m, lane, 0, 1, nullptr, C, D);
    const float rh = 1.f / (float)(p.seg_off[m + 1] - p.seg_off[m]);
#pragma unroll
    for (int o = 0; o < OM; ++o) gs[o] = 0.f;
    if (b < Bp) {
      Merged<OM> s;
      merge_pieces<OM, NORM>(p, map, f.part, f.csum, m, f.Br, b < l.B ? b : l.B - 1, 0, 1, s);
      sample_grads<OM, NORM>(p, l, m, b, Bp, s, C, D, rh, scale, loss, gs);
    }
    loss = group_sum_to_last(loss, 64);
    if (lane == 63) red[i * kRow + OM] = loss;
    if (NORM) {
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        gs[o] = group_sum_to_last(gs[o], 64);
        if (lane == 63) red[i * kRow + o] = gs[o];
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < (m1 - m0) * kRow; i += blockDim.x) {
    const int m = m0 + i / kRow, o = i % kRow;
    float s = 0.f;
    if (o == OM || (NORM && o < p.O))
      for (int k = 0; k < nblk; ++k) s += red[((m - m0) * nblk + k) * kRow + o];
    if (o == OM) {
      l.loss[m] = s * scale;
      if (!isfinite(s)) atomicAdd(l.flag + 2, 1);
      if (l.lrm && !isfinite(l.lrm[m])) l.flag[1] = 1;
    } else if (NORM && o < p.O) {
      l.Gs[(int64_t)m * p.O + o] = s;
    }
  }
}

template <int NC, int RM, bool GATED, bool NORM>
__global__ __launch_bounds__(64 * kBlkLocalGroup)
void k_blk_local(BlkPack p, BlkLocal g, BlkFwdArgs f, BlkLoss l, BlkBwdArgs b) {
  extern __shared__ __align__(16) char lds[];
  const int tid = threadIdx.x, nw = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int m0, m1;
  group_models(g, f, blockIdx.x, p.M, m0, m1);
  if (m0 == m1) return;
  const int t0 = g.toff[m0], t1 = g.toff[m1], Bp = b.Bp;
  fill_pieces<NC>(lds, Bp, f.X, 0, f.B, f.F, tid, blockDim.x);
  lds_barrier();
  fwd_tiles<NC, RM, (OM > 2), GATED, NORM, false>(p, f, lds, Bp, 0, Bp >> 5, t0 + wave, t1, nw, 1,
                                                  nullptr);
  __syncthreads();
  local_loss<NORM>(p, BlkMap{g.toff, 1, f.csum}, f, l, Bp, m0, m1, (float*)(lds + sums_at(NC, Bp)));
  __syncthreads();
  bwd_tiles<NC, RM, OM, GATED, NORM>(p, b, lds, Bp, 1, (t1 - t0 + nw - 1) / nw, t0 + wave, t1, nw);
}

typedef void (*BlkLocalFn)(BlkPack, BlkLocal, BlkFwdArgs, BlkLoss, BlkBwdArgs);
struct BlkLocalInst {
  BlkLocalFn fn;
  int NC;
};

template <int NC, int RM>
BlkLocalInst local_kind(bool gated, bool norm) {
  if (gated && norm) return {k_blk_local<NC, RM, true, true>, NC};
  if (gated) return {k_blk_local<NC, RM, true, false>, NC};
  return {k_blk_local<NC, RM, false, true>, NC};
}

BlkLocalInst local_of(const BlkPack& p) {
  const bool g = p.V1 != nullptr, n = p.gain != nullptr;
#define PMLP_CALL(NC, RM) local_kind<NC, RM>(g, n)
  PMLP_BLK_SHAPE(p.F4, PMLP_CALL)
#undef PMLP_CALL
  return {nullptr, 0};
}

// (a group has at most `group` models)
size_t local_lds(int NC, int32_t Bp, int32_t group) {
  return sums_at(NC, Bp) + (size_t)group * ((Bp + 63) / 64) * kRow * sizeof(float);
}

}  // namespace

#define PMLP_CAT_(a, b) a##b
#define PMLP_CAT(a, b) PMLP_CAT_(a, b)

int PMLP_CAT(blk_local_slots_, PMLP_BLK_OM)(const BlkPack& p, int32_t Bp, int32_t group) {
  const BlkLocalInst i = local_of(p);
  if (!i.fn || Bp > kBlkLocalBatch || group < 1 || group > kBlkLocalGroup) return 0;
  return resident_blocks((const void*)i.fn, 64 * kBlkLocalGroup, local_lds(i.NC, Bp, group));
}

hipError_t PMLP_CAT(launch_blk_local_, PMLP_BLK_OM)(const BlkPack& p, const BlkLocal& g,
                                                    const BlkFwdArgs& f, const BlkLoss& l,
                                                    const BlkBwdArgs& b, hipStream_t s) {
  const BlkLocalInst i = local_of(p);
  if (!i.fn || b.B < 1 || b.B != f.B || b.B != l.B || b.B > b.Bp || b.Bp % 32 || f.Br < b.Bp ||
      p.O > OM || f.ntiles < 1 || f.tiles != b.tiles || f.ntiles != b.ntiles || !g.toff ||
      PMLP_CAT(blk_local_slots_, PMLP_BLK_OM)(p, b.Bp, g.group) <= 0)
    return hipErrorInvalidValue;
  i.fn<<<(unsigned)((f.ntiles + g.group - 1) / g.group), 64 * kBlkLocalGroup,
         local_lds(i.NC, b.Bp, g.group), s>>>(p, g, f, l, b);
  return hipGetLastError();
}

}  // namespace pmlpk
