// Device code shared by the fused kernels of block packs.
#pragma once

#include "block.h"
#include "device_common.h"

namespace pmlpk {

// (n, mean, M2) of the union of two sets (Chan, Golub and LeVeque)
__device__ __forceinline__ void merge_stats(float& n, float& mean, float& m2, float nb, float meanb,
                                            float m2b) {
  const float t = n + nb;
  const float f = t > 0.f ? nb / t : 0.f;
  const float d = meanb - mean;
  mean = fmaf(d, f, mean);
  m2 += m2b + d * d * n * f;
  n = t;
}

// The same value, of which the compiler knows nothing: a load whose result passes
// through here is made where it stands, not in a branch on whether it is wanted
// (such branches made every load of a row wait for the one before).
template <class T>
__device__ __forceinline__ T opaque(T v) {
  asm volatile("" : "+v"(v));
  return v;
}

// A barrier for what lies in LDS.  (__syncthreads also waits for the loads from
// memory that are on their way into registers for the next stage.)
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

#define PMLP_EVERY_ACT                                                                      \
  PMLP_ACT(0) PMLP_ACT(1) PMLP_ACT(2) PMLP_ACT(3) PMLP_ACT(4) PMLP_ACT(5) PMLP_ACT(6)       \
  PMLP_ACT(7) PMLP_ACT(8) PMLP_ACT(9) PMLP_ACT(10) PMLP_ACT(11) PMLP_ACT(12)

// act_fwd with NaN for NaN also where its choice of a branch would drop it
__device__ __forceinline__ float blk_act(int a, float z) {
  if (a == 1) return z <= 0.f ? 0.f : z;
  if (a == 11) return fabsf(z) <= 0.5f ? 0.f : z;
  return act_fwd(a, z);
}

// Activation id a (uniform over the wave) of NV values.
template <int NV>
__device__ __forceinline__ void blk_acts(int a, const float (&z)[NV], float (&v)[NV]) {
  switch (a) {
#define PMLP_ACT(AA)                                                     \
  case AA: {                                                             \
    _Pragma("unroll") for (int j = 0; j < NV; ++j) v[j] = blk_act(AA, z[j]); \
    break;                                                               \
  }
    PMLP_EVERY_ACT
#undef PMLP_ACT
  }
}

// The gradients of unit n's output weights, gain and shift from T_o, stored or
// applied.  w: its output weights.
template <int OM, bool NORM>
__device__ __forceinline__ void blk_unit_grads(const BlkPack& p, const BlkGrads& out,
                                               const float* __restrict__ Gs, int64_t n, int m,
                                               float gn, const float (&w)[OM],
                                               const float (&T)[OM]) {
  const float sn = NORM ? p.shift[n] : 0.f;
  const float rate = out.lrm ? out.lrm[m] : out.lr;
  float dg = 0.f, ds = 0.f;
#pragma unroll
  for (int o = 0; o < OM; ++o)
    if (o < p.O) {
      float dw = T[o];
      if (NORM) {
        const float s = Gs[(int64_t)m * p.O + o];
        dg = fmaf(w[o], T[o], dg);
        ds = fmaf(w[o], s, ds);
        dw = fmaf(gn, T[o], sn * s);
      }
      if (out.dW2) out.dW2[(int64_t)o * p.N + n] = dw;
      else p.W2[(int64_t)o * p.ldw + n] = w[o] - rate * dw;
    }
  if (NORM) {
    if (out.dW2) {
      out.dgain[n] = dg;
      out.dshift[n] = ds;
    } else {
      p.gain[n] = gn - rate * dg;
      p.shift[n] = sn - rate * ds;
    }
  }
}

}  // namespace pmlpk
