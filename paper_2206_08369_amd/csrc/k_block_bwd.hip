// Block packs: the backward pass in one kernel, for inputs of up to 128 columns.
// Compiled once per class of outputs (PMLP_BLK_OM: 2, 4 or 16).
//
// A wave takes a tile, up to 16 consecutive hidden units of one activation (of whatever
// models), and all samples, so that its weights' gradients need no other wave; it holds
// the three bf16 pieces of its units' W1 (and V1) rows and their gradients'
// accumulators in registers.  The samples' pieces lie in LDS once, sample by sample (chunks of
// them in turn, where they do not fit), and serve both products: read as rows they
// are the operand of Z = X W1^T, which is computed again rather than stored by the
// forward and read back, and read through the transposing LDS load the operand of
// dW1 = dZ^T X.  A step takes 32 samples: after Z the lane (li, lk) holds unit li of
// the samples 4 lk + r of both blocks of 16, forms dZ there, and those eight values
// are, as they lie, a column of the second product's second operand (the sums over
// samples run in that order in both of its operands).  The lane ends with four
// consecutive columns of unit li's gradient, one store.
// The norm's gradient needs no sums over units (see k_block.hip).
//
// Bound by its instructions.  6000 models of 1 to 100 units, 100 columns, 256 samples (in
// a trace of four passes): gated 390 us, that is 159 TFLOP/s of fp32 products (0.95 PFLOP/s
// of bf16 ones), the matrix units busy 0.56 of the time and the vector units 0.45; normed
// 253 us, 0.40 and 0.52.  Wide models, ten outputs, 32 columns and samples, both: 181 us for
// 668 MB, 3.7 TB/s (a large copy 4.8).  Two waves a SIMD is what the registers allow;
// where the input has no block of 32 columns, three.
//
// The second product takes NF = 2 NC blocks of 16 columns, and one more for the fp32
// columns of the first; the last block may read past its columns into the next row,
// for columns that no one stores.

#include "block_tiles.h"

#ifndef PMLP_BLK_OM
#error "compile with -DPMLP_BLK_OM=2|4|16"
#endif

namespace pmlpk {

namespace {

constexpr int OM = PMLP_BLK_OM;

template <int NC, int RM, bool GATED, bool NORM>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(NC == 0 ? 3 : 2)))
void k_blk_fused_bwd(BlkPack p, BlkBwdArgs a) {
  extern __shared__ __align__(16) char lds[];
  const int nw = blockDim.x >> 6, nchunk = (a.Bp + a.SC - 1) / a.SC, stride = gridDim.x * nw;
  if (nchunk == 1) {
    fill_pieces<NC>(lds, a.SC, a.X, 0, a.B, a.F, threadIdx.x, blockDim.x);
    lds_barrier();
  }
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  bwd_tiles<NC, RM, OM, GATED, NORM>(p, a, lds, a.SC, nchunk, (a.ntiles + stride - 1) / stride,
                                     (int)blockIdx.x * nw + wave, a.ntiles, stride);
}

typedef void (*BlkBwdFn)(BlkPack, BlkBwdArgs);

struct BlkBwdInst {
  BlkBwdFn fn;
  int NC;
};

template <int NC, int RM>
BlkBwdInst bwd_kind(bool gated, bool norm) {
  if (gated && norm) return {k_blk_fused_bwd<NC, RM, true, true>, NC};
  if (gated) return {k_blk_fused_bwd<NC, RM, true, false>, NC};
  return {k_blk_fused_bwd<NC, RM, false, true>, NC};
}

BlkBwdInst bwd_of(const BlkPack& p) {
  const bool g = p.V1 != nullptr, n = p.gain != nullptr;
#define PMLP_CALL(NC, RM) bwd_kind<NC, RM>(g, n)
  PMLP_BLK_SHAPE(p.F4, PMLP_CALL)
#undef PMLP_CALL
  return {nullptr, 0};
}

// Samples a chunk: all of them where they fit in LDS, else the most equal parts.
int chunk_samples(int NC, int Bp, size_t lds_max) {
  for (int parts = 1;; ++parts) {
    const int SC = ((Bp + parts - 1) / parts + 31) & ~31;
    if (pieces_bytes(NC, SC) <= lds_max) return SC;
    if (SC == 32) return 0;
  }
}

}  // namespace

#define PMLP_CAT_(a, b) a##b
#define PMLP_CAT(a, b) PMLP_CAT_(a, b)

hipError_t PMLP_CAT(launch_blk_fused_bwd_, PMLP_BLK_OM)(const BlkPack& p, BlkBwdArgs a,
                                                        hipStream_t s) {
  const BlkBwdInst inst = bwd_of(p);
  const BlkBwdFn fn = inst.fn;
  int dev = 0, lmax = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess)
    e = hipDeviceGetAttribute(&lmax, hipDeviceAttributeMaxSharedMemoryPerBlock, dev);
  if (e != hipSuccess) return e;
  a.SC = fn ? chunk_samples(inst.NC, a.Bp, (size_t)lmax) : 0;
  if (a.SC <= 0 || a.Bp < 32 || a.Bp % 32 || a.B < 1 || a.B > a.Bp || p.O > OM || a.ntiles < 1)
    return hipErrorInvalidValue;
  const size_t lds = pieces_bytes(inst.NC, a.SC);
  // eight waves share the samples' pieces where those leave room for one workgroup
  // only (a gated paper pool: 418 us, with four 492), four where there is more (the
  // same time in large pools; small ones spread over twice the CUs)
  const int waves = 4 * lds > (size_t)lmax ? 8 : 4;
  const int slots = resident_blocks((const void*)fn, 64 * waves, lds);
  if (slots <= 0) return hipErrorInvalidValue;
  const int64_t grid = std::min<int64_t>(slots, (a.ntiles + waves - 1) / waves);
  fn<<<(unsigned)grid, 64 * waves, lds, s>>>(p, a);
  return hipGetLastError();
}

}  // namespace pmlpk
