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
  m2 += m2b + d * (n * f) * d;  // (d d alone may overflow where n is 0)
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

// Activations whose errors stay relative to their values where these are small: a norm
// divides by a deviation that may be as small, and the forms of act_fwd that subtract
// from 1 are off by 1e-7 however small the result.  (tanh units of pre-activations about
// 1e-3, normalised: outputs off by 5e-5 of their size with act_fwd.)  The polynomials are
// minimax ones of the relative error, below 0.25 units in the last place.  Both forms are
// computed and one taken: a branch for each value cost more than either.

// tanh z, given e = e^-2|z| and r = 1 / (1 + e): z + z^3 R(z^2) up to 1/2
__device__ __forceinline__ float blk_tanh(float z, float e, float r) {
  const float q = z * z;
  float p = fmaf(0.017256992f, q, -0.05305295f);
  p = fmaf(p, q, 0.13325988f);
  p = fmaf(p, q, -0.3333315f);
  const float small = fmaf(z * q, p, z), wide = copysignf((1.f - e) * r, z);
  return fabsf(z) < 0.5f ? small : wide;
}

// e^z - 1, given e^z, for z <= 0: z + z^2 R(z) down to -1/2
__device__ __forceinline__ float blk_expm1(float z, float ez) {
  float r = fmaf(0.0011282321f, z, 0.008196126f);
  r = fmaf(r, z, 0.041633245f);
  r = fmaf(r, z, 0.1666631f);
  r = fmaf(r, z, 0.49999988f);
  const float small = fmaf(z * z, r, z), wide = ez - 1.f;
  return z > -0.5f ? small : wide;
}

// log(1 + e), 0 <= e <= 1: 2 atanh s = 2 s + 2 s^3 R(s^2) of s = e / (2 + e)
__device__ __forceinline__ float blk_log1p(float e) {
  const float s = e * frcp(2.f + e), q = s * s;
  float r = fmaf(0.1401223f, q, 0.13999571f);
  r = fmaf(r, q, 0.2001085f);
  r = fmaf(r, q, 0.33333206f);
  return 2.f * fmaf(s * q, r, s);
}

// ELU (up, down 1) and SELU, given e^z
__device__ __forceinline__ float blk_elu(float z, float ez, float up, float down) {
  const float above = up * z, below = down * blk_expm1(z, ez);
  return z > 0.f ? above : below;
}

// softplus z, given e^-|z|
__device__ __forceinline__ float blk_softplus(float z, float e) {
  const float s = fmaxf(z, 0.f) + blk_log1p(e);
  return z > 20.f ? z : s;
}

// (NaN for NaN also where act_fwd's choice of a branch would drop it)
__device__ __forceinline__ float blk_act(int a, float z) {
  switch (a) {
    case 1: return z <= 0.f ? 0.f : z;
    case 2: {
      const float e = fexp(-2.f * fabsf(z));
      return blk_tanh(z, e, frcp(1.f + e));
    }
    case 4: return blk_elu(z, fexp(z), 1.f, 1.f);
    case 8: return blk_softplus(z, fexp(-fabsf(z)));
    case 10: return blk_elu(z, fexp(z), kSeluLambda, kSeluLambda * kSeluAlpha);
    case 11: return fabsf(z) <= 0.5f ? 0.f : z;
    default: return act_fwd(a, z);
  }
}

// Value and derivative together
__device__ __forceinline__ float blk_act_slope(int a, float z, float* d) {
  switch (a) {
    case 2: {
      const float e = fexp(-2.f * fabsf(z)), r = frcp(1.f + e);
      *d = 4.f * e * r * r;  // 1 / cosh^2: 1 - tanh^2 would leave nothing of a small one
      return blk_tanh(z, e, r);
    }
    case 4:
    case 10: {
      const float up = a == 10 ? kSeluLambda : 1.f, down = a == 10 ? kSeluLambda * kSeluAlpha : 1.f;
      const float e = fexp(z), below = down * e;
      *d = z > 0.f ? up : below;
      return blk_elu(z, e, up, down);
    }
    case 8: {
      const float e = fexp(-fabsf(z)), r = frcp(1.f + e);
      const float s = (z >= 0.f ? 1.f : e) * r;
      *d = z > 20.f ? 1.f : s;
      return blk_softplus(z, e);
    }
    default: return act_fwd_bwd(a, z, d);
  }
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

// ---------------------------------------------------------------------------
// The samples' three bf16 pieces in LDS, sample by sample, for both fused kernels.
// ---------------------------------------------------------------------------

// Row bytes of the pieces of 32 NC columns and up to eight more: 16 bytes times an
// odd number, which spreads 16 rows over all banks.
__host__ __device__ constexpr int row_bytes(int NC) { return 16 * (4 * NC + 1); }

// LDS of SC samples: three planes, and what a transposing load of the last row's
// columns may pass them by
inline size_t pieces_bytes(int NC, int SC) { return (size_t)3 * SC * row_bytes(NC) + 32; }

// Where sums of the workgroup may lie after them
__host__ __device__ constexpr size_t sums_at(int NC, int SC) {
  return ((size_t)3 * SC * row_bytes(NC) + 32 + 15) & ~(size_t)15;
}

// The pieces of the SC samples from b0 on (zero past the batch and the columns).
template <int NC>
__device__ __forceinline__ void fill_pieces(char* lds, int SC, const float* X, int b0, int B,
                                            int F, int tid, int threads) {
  constexpr int RB = row_bytes(NC), QR = RB / 8;  // quads of a row
  const int plane = SC * RB;
  for (int q = tid; q < SC * QR; q += threads) {
    const int s = q / QR, k = 4 * (q - s * QR), b = b0 + s;
    const float* xr = X + (int64_t)(b < B ? b : B - 1) * F;
    f32x2 x[2];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = xr[k + e < F ? k + e : F - 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float w = opaque(v[e]);
      x[e >> 1][e & 1] = k + e < F && b < B ? w : 0.f;
    }
    uint32_t p0[2], p1[2], p2[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      p0[e] = bf16_pair(x[e]);
      const f32x2 r1 = x[e] - bf16_pair_value(p0[e]);
      p1[e] = bf16_pair(r1);
      p2[e] = bf16_pair(r1 - bf16_pair_value(p1[e]));
    }
    char* d = lds + s * RB + 2 * k;
    *(uint2*)d = make_uint2(p0[0], p0[1]);
    *(uint2*)(d + plane) = make_uint2(p1[0], p1[1]);
    *(uint2*)(d + 2 * plane) = make_uint2(p2[0], p2[1]);
  }
}

// A unit's row of W1 and V1 as the lane (row li, columns 8 lk ..) holds it for a
// product's operand: 32 NC columns and RM fp32 steps of four, as loaded ..
template <int NC, int RM, int K>
struct UnitRaw {
  f32x4 w[K][NC > 0 ? 2 * NC : 1];
  float t[K][RM > 0 ? RM : 1];
  __device__ __forceinline__ void load(const BlkPack& pk, int64_t n, int lk) {
#pragma unroll
    for (int mt = 0; mt < K; ++mt) {
      const float* row = (mt ? pk.V1 : pk.W1) + n * pk.F4;
#pragma unroll
      for (int e = 0; e < 2 * NC; ++e) {
        const int k = 32 * (e >> 1) + 8 * lk + 4 * (e & 1);
        w[mt][e] = *(const f32x4*)(row + (k < pk.F4 ? k : pk.F4 - 4));
      }
#pragma unroll
      for (int q = 0; q < RM; ++q) t[mt][q] = row[32 * NC + 4 * q + lk];
    }
  }
};

// .. and in pieces.
template <int NC, int RM, int K>
struct UnitRows {
  bf16x8 p[K][NC > 0 ? NC : 1][3];
  float t[K][RM > 0 ? RM : 1];
  __device__ __forceinline__ void split(const UnitRaw<NC, RM, K>& r, int F4, int lk) {
#pragma unroll
    for (int mt = 0; mt < K; ++mt) {
#pragma unroll
      for (int q = 0; q < RM; ++q) t[mt][q] = opaque(r.t[mt][q]);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        f32x4 q[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          q[e] = opaque(r.w[mt][2 * c + e]);
          if (32 * c + 8 * lk + 4 * e >= F4) q[e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        split3(q[0], q[1], p[mt][c][0], p[mt][c][1], p[mt][c][2]);
      }
    }
  }
};

// Z and U of 16 units and the 32 samples whose pieces start at `at` (this lane's row):
// UNITS_FIRST: lane (li, lk) ends with units 4 lk + r of sample li, else with samples
// 4 lk + r of unit li; z[mt][i] of the samples' block i.  xat: its fp32 columns.
template <int NC, int RM, int K, bool UNITS_FIRST>
__device__ __forceinline__ void unit_products(const UnitRows<NC, RM, K>& w, const char* at,
                                              const char* xat, int plane,
                                              f32x4 (&z)[K][2]) {
  constexpr int RB = row_bytes(NC);
  unsigned short xp[RM > 0 ? RM : 1][2][3];
#pragma unroll
  for (int q = 0; q < RM; ++q)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 3; ++e)
        xp[q][i][e] = *(const unsigned short*)(xat + e * plane + (16 * i * RB + 8 * q));
#pragma unroll
  for (int mt = 0; mt < K; ++mt)
#pragma unroll
    for (int i = 0; i < 2; ++i) z[mt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    bf16x8 x[2][3];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 3; ++e) x[i][e] = *(const bf16x8*)(at + e * plane + (16 * i * RB + 64 * c));
    // the piece products smallest first, blocks and projections in turn
#define PMLP_PIECE(E, Q)                                                                   \
_Pragma("unroll") for (int mt = 0; mt < K; ++mt) _Pragma("unroll") for (int i = 0; i < 2; ++i) \
    z[mt][i] = UNITS_FIRST                                                                 \
                   ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[mt][c][Q], x[i][E], z[mt][i], 0, 0, 0) \
                   : __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i][E], w.p[mt][c][Q], z[mt][i], 0, 0, 0)
    PMLP_PIECE(2, 0);
    PMLP_PIECE(1, 1);
    PMLP_PIECE(0, 2);
    PMLP_PIECE(1, 0);
    PMLP_PIECE(0, 1);
    PMLP_PIECE(0, 0);
#undef PMLP_PIECE
  }
#pragma unroll
  for (int q = 0; q < RM; ++q)
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // the column again, exactly: the sum of its pieces
      const float x = (bf16_bits_to_f32(xp[q][i][2]) + bf16_bits_to_f32(xp[q][i][1])) +
                      bf16_bits_to_f32(xp[q][i][0]);
#pragma unroll
      for (int mt = 0; mt < K; ++mt)
        z[mt][i] = UNITS_FIRST
                       ? __builtin_amdgcn_mfma_f32_16x16x4f32(w.t[mt][q], x, z[mt][i], 0, 0, 0)
                       : __builtin_amdgcn_mfma_f32_16x16x4f32(x, w.t[mt][q], z[mt][i], 0, 0, 0);
    }
}

// The instance for F4 columns: NC chunks of 32 in three-piece products and RM fp32
// steps of four, or else a last chunk that is padded.  CALL(NC, RM) returns it.
#define PMLP_BLK_SHAPE(F4, CALL)                                       \
  switch ((F4) / 32 * 3 + ((F4) % 32 == 0 ? 0 : (F4) % 32 == 4 ? 1 : (F4) % 32 == 8 ? 2 : 3)) { \
    case 1: return CALL(0, 1);                                          \
    case 2: return CALL(0, 2);                                          \
    case 3: return CALL(1, 0);                                          \
    case 4: return CALL(1, 1);                                          \
    case 5: return CALL(1, 2);                                          \
    case 6: return CALL(2, 0);                                          \
    case 7: return CALL(2, 1);                                          \
    case 8: return CALL(2, 2);                                          \
    case 9: return CALL(3, 0);                                          \
    case 10: return CALL(3, 1);                                         \
    case 11: return CALL(3, 2);                                         \
    case 12: return CALL(4, 0);                                         \
    default: break;                                                     \
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
