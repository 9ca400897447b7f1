// Block packs: products, gate, norm statistics and output sums in one kernel, for
// inputs of up to 128 columns.  Compiled once per class of outputs (PMLP_BLK_OM: 2 or
// 16).
//
// A wave takes 16 hidden units of one model (a tile) and the samples of its workgroup,
// whose pieces lie in LDS: it splits the units' W1 (and V1) rows once, into registers,
// and needs no other wave (an earlier form, with the samples in registers and the
// units passing through LDS in stages, spent as long at its barriers and on shared
// splitting as on its products).  A step takes 32 samples; lane (li, lk) ends with
// units 4 lk + r of sample li of both blocks of 16.  The sums over the tile's units
// (outputs, and with a norm the mean and the squared deviations) are stored per run
// and sample (BlkMap); the output and loss kernels merge a model's runs.  That costs
// blk_planes floats per 16 units and sample or fewer, against 16 (32 gated) for the
// pre-activations.
//
// Bound by its instructions, as the backward.  6000 models of 1 to 100 units, 100
// columns, 256 samples (in a trace of four passes): gated 207 us, 150 TFLOP/s of fp32
// products (0.90 PFLOP/s of bf16 ones), matrix and vector units busy 0.58 and 0.59; normed
// 152 us, 0.37 and 0.80.  With one sample it is bound by the weights: gated, 56 us
// for 245 MB (4.4 TB/s).  (A form with the tiles of whole models in one workgroup,
// which merged them itself, saved the output kernel's 7 us there and lost more by its
// uneven groups: 59 -> 66 us in all, at 10,000 samples 669 -> 692.)
//
// Two outputs are summed by vector FMAs and two lane swaps, more by fp32 matrix
// products whose second operand is the hidden values as they lie in the registers.
// A tile's mean is its first value plus the mean difference from it, and the squared
// deviations, as the outputs' sums, are taken from that mean: both stay exact for values
// that lie close together far from zero.  (One pass, deviations from the first value moved
// to the mean: as fast, and its errors up to 16 times those of the variance.)

#include "block_tiles.h"

#ifndef PMLP_BLK_OM
#error "compile with -DPMLP_BLK_OM=2|16"
#endif

namespace pmlpk {

namespace {

constexpr bool MF = PMLP_BLK_OM > 2;

// Threads of a workgroup, at most: as many waves as a SIMD's registers hold with few
// spilled, four, three or two (normed, 100 columns: 6000 models of 4 to 100 units, 256
// samples, 166 us with four, 170 with three; 16 outputs, 1000 samples of 40 models of 500 to
// 1000 units 90 with either).
template <int NC, bool GATED>
constexpr int max_threads() {
  return GATED ? (NC == 0 ? 1024 : NC <= 3 ? 768 : 512) : (NC <= 3 ? 1024 : 768);
}

template <int NC, int RM, bool GATED, bool NORM, bool RUNS>
__global__ __launch_bounds__((max_threads<NC, GATED>()))
void k_blk_fused_fwd(BlkPack p, BlkFwdArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int chunk = blockIdx.x / a.wpc, wg = blockIdx.x - chunk * a.wpc;
  const int SC = a.SC, b0 = chunk * SC;
  fill_pieces<NC>(lds, SC, a.X, b0, a.B, a.F, tid, blockDim.x);
  lds_barrier();
  const int steps = (std::min(SC, a.B - b0) + 31) >> 5;
  const int planes = p.O + (NORM ? 2 : 0);
  fwd_tiles<NC, RM, MF, GATED, NORM, RUNS>(
      p, a, lds, SC, b0, steps, RUNS ? wave * a.wpc + wg : wg * nw + wave, a.ntiles, a.wpc * nw, a.run,
      (float*)(lds + sums_at(NC, SC)) + wave * planes * acc_row(SC));
}

typedef void (*BlkFwdFn)(BlkPack, BlkFwdArgs);
struct BlkFwdInst {
  BlkFwdFn fn;
  int NC, threads;  // threads of a workgroup, at most (the occupancy query does not mind them)
};

template <int NC, int RM, bool RUNS>
BlkFwdInst fwd_kind(bool gated, bool norm) {
  if (gated && norm) return {k_blk_fused_fwd<NC, RM, true, true, RUNS>, NC, max_threads<NC, true>()};
  if (gated) return {k_blk_fused_fwd<NC, RM, true, false, RUNS>, NC, max_threads<NC, true>()};
  return {k_blk_fused_fwd<NC, RM, false, true, RUNS>, NC, max_threads<NC, false>()};
}

size_t fwd_lds(const BlkPack& p, int NC, int32_t SC, int32_t waves, bool runs) {
  if (!runs) return pieces_bytes(NC, SC);
  return sums_at(NC, SC) + (size_t)waves * blk_planes(p) * acc_row(SC) * sizeof(float);
}

BlkFwdInst fwd_of(const BlkPack& p, bool runs) {
  const bool g = p.V1 != nullptr, n = p.gain != nullptr;
#define PMLP_CALL(NC, RM) (runs ? fwd_kind<NC, RM, true>(g, n) : fwd_kind<NC, RM, false>(g, n))
  PMLP_BLK_SHAPE(p.F4, PMLP_CALL)
#undef PMLP_CALL
  return {nullptr, 0, 0};
}

}  // namespace

#define PMLP_CAT_(a, b) a##b
#define PMLP_CAT(a, b) PMLP_CAT_(a, b)

int PMLP_CAT(blk_fwd_slots_, PMLP_BLK_OM)(const BlkPack& p, int32_t SC, int32_t waves, bool runs) {
  const BlkFwdInst i = fwd_of(p, runs);
  return i.fn && 64 * waves <= i.threads ? resident_blocks((const void*)i.fn, 64 * waves, fwd_lds(p, i.NC, SC, waves, runs)) : 0;
}

hipError_t PMLP_CAT(launch_blk_fused_fwd_, PMLP_BLK_OM)(const BlkPack& p, const BlkFwdArgs& a,
                                                        hipStream_t s) {
  const BlkFwdInst i = fwd_of(p, a.run > 1);
  if (!i.fn || a.B < 1 || a.ntiles < 1 || a.wpc < 1 || a.waves < 1 ||
      a.run < 1 || 64 * a.waves > i.threads || a.SC < 32 ||
      a.SC % 32 || p.O > PMLP_BLK_OM)
    return hipErrorInvalidValue;
  const int nchunk = (a.B + a.SC - 1) / a.SC;
  if (a.Br < (a.B + 31) / 32 * 32 || (int64_t)nchunk * a.wpc > 0x7fffffff)
    return hipErrorInvalidValue;
  i.fn<<<(unsigned)(nchunk * a.wpc), 64 * a.waves, fwd_lds(p, i.NC, a.SC, a.waves, a.run > 1), s>>>(p, a);
  return hipGetLastError();
}

}  // namespace pmlpk
