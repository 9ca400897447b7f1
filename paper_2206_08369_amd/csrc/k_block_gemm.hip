// Block packs: the stored path's products where they are small.
//   C[p][q] = sum_k P[p][k] Q[q][k], fp32 as six bf16 products of three-piece splits.
//
// A workgroup of four waves takes 32 x 32 of C and every wave a quarter of the steps of
// 32 k; their sums are added in the order of the waves.  Operands come from the caches
// straight into registers and are split there, by each wave for itself: as many
// vector instructions as a 256 x 256 tile needs for 64 times the products, and 64 times
// as many workgroups, each with a quarter of the steps.  Taken where the large tiles are
// too few to fill the device (small_product of the host).
#include "block_device.h"

#include <algorithm>

namespace pmlpk {

namespace {

typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));

template <int EPI>
__global__ __launch_bounds__(256) void k_blk_gemm(BlkGemm a, int nqt) {
  __shared__ f32x4 red[4][4][64];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t p0 = (int64_t)(blockIdx.x / nqt) * 32;
  const int q0 = (int)(blockIdx.x % nqt) * 32;
  const float *pr[2], *qr[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {  // (past the last row: that one, not stored)
    pr[i] = a.P + std::min<int64_t>(p0 + 16 * i + li, a.NP - 1) * a.ldp;
    qr[i] = a.Q + (int64_t)std::min(q0 + 16 * i + li, a.NQ - 1) * a.ldq;
  }
  struct Step {
    f32x4 p[2][2], q[2][2];
  };
  auto load = [&](int s) {
    Step v;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int k = std::min(32 * s + 8 * lk + 4 * e, a.K - 4);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v.p[i][e] = *(const f32x4*)(pr[i] + k);
        v.q[i][e] = *(const f32x4*)(qr[i] + k);
      }
    }
    return v;
  };
  f32x4 acc[2][2];  // [p block][q block]
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (a.K + 31) >> 5;
  Step next = load(std::min(wave, steps - 1));
#pragma unroll 1
  for (int s = wave; s < steps; s += 4) {
    Step v = next;
    next = load(std::min(s + 4, steps - 1));
    bf16x8 p[2][3], q[2][3];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (32 * s + 8 * lk + 4 * e >= a.K) v.p[i][e] = v.q[i][e] = f32x4{0.f, 0.f, 0.f, 0.f};
      split3(v.p[i][0], v.p[i][1], p[i][0], p[i][1], p[i][2]);
      split3(v.q[i][0], v.q[i][1], q[i][0], q[i][1], q[i][2]);
    }
#define PMLP_PIECE(A, B)                                                                  \
_Pragma("unroll") for (int i = 0; i < 2; ++i)                                             \
_Pragma("unroll") for (int j = 0; j < 2; ++j) acc[i][j] =                                 \
    __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[j][B], p[i][A], acc[i][j], 0, 0, 0)
    PMLP_PIECE(2, 0);
    PMLP_PIECE(1, 1);
    PMLP_PIECE(0, 2);
    PMLP_PIECE(1, 0);
    PMLP_PIECE(0, 1);
    PMLP_PIECE(0, 0);
#undef PMLP_PIECE
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[wave][i][lane] = acc[i >> 1][i & 1];
  __syncthreads();
  // wave w has block w: row li of its rows of P, columns 4 lk ..
  f32x4 v = red[0][wave][lane];
#pragma unroll
  for (int w = 1; w < 4; ++w) v += red[w][wave][lane];
  const int64_t p = p0 + 16 * (wave >> 1) + li;
  const int q = q0 + 16 * (wave & 1) + 4 * lk;
  if (p >= a.NP || q >= a.ncols) return;
  float* const o = a.out + p * a.ldo + q;
  const float rate = EPI == EPI_SGD ? (a.lrm ? a.lrm[a.mid[p]] : a.lr) : 0.f;
  if (q + 4 <= a.ncols) {
    if (EPI == EPI_SGD) v = *(const f32x4_u*)o - rate * v;
    *(f32x4_u*)o = v;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (q + e < a.ncols) o[e] = EPI == EPI_SGD ? o[e] - rate * v[e] : v[e];
  }
}

}  // namespace

hipError_t launch_blk_gemm(const BlkGemm& a, int epi, hipStream_t s) {
  if (a.NP < 1 || a.NQ < 1 || a.K < 4 || a.K % 4 || a.ldp % 4 || a.ldq % 4 || a.ldp < a.K ||
      a.ldq < a.K || a.ncols < 1 || a.ncols > a.NQ || a.ldo < a.ncols)
    return hipErrorInvalidValue;
  note_variant("k_blk_gemm", kArithX3);
  const int nqt = (a.NQ + 31) / 32;
  const int64_t grid = (a.NP + 31) / 32 * nqt;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  switch (epi) {
    case EPI_STORE: k_blk_gemm<EPI_STORE><<<(unsigned)grid, 256, 0, s>>>(a, nqt); break;
    case EPI_SGD: k_blk_gemm<EPI_SGD><<<(unsigned)grid, 256, 0, s>>>(a, nqt); break;
    default: k_blk_gemm<EPI_GRAD><<<(unsigned)grid, 256, 0, s>>>(a, nqt); break;
  }
  return hipGetLastError();
}

}  // namespace pmlpk
