// Device code shared by the kernels of k_newton.hip and k_newton_small.hip.
#pragma once

#include "device_common.h"
#include "newton.h"

namespace pmlpk {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// The steps in fp32's accuracy on the fp16 matrix cores.
//
// X (r x c) is held as X'_ij = X_ij / (d_i e_j) with powers of two d and e, and every value v as
// the fp16 numbers hi = v and lo = v - hi, both rounded, times a constant: 2^15 for X' and
// A' = D^-1 A D^-1, 2^14 for B = A' D, 2^12 for P'.  Two halves hold 23 bits of an X' from 2^-18 on
// and steps of 2^-39 below, so that a small row or column has the bits that the others have.
// The steps in these terms:
//   A' = X' E^2 X'^T,   P' = (b A' + c A' D^2 A') D^2,   X' <- (a X' + P' X') D E / (new D E).
//
// Rows: d_i is at least the norm of X's row i, at first by its largest entry times sqrt(c).  A'_ii
// is the norm's square beside d_i's, and a step makes a norm at most 3.4445 times as large: the next
// d_i is 4 times the least power of two above the norm, but 2 at most (no norm is above 1.21) and a
// quarter of the last at least.
// Columns: e_j is 1, which always does as no entry of X / d is above 1, or less where m, the
// largest one of column j, is below 2^-10 (more with many rows: ns_scales); X' there is then 2^-15
// at least, a step later.  What a step makes of m is bounded by the norm of P's row, at most 2.82
// |X_i| (the largest s |b + c s^2| for s up to 1.21), times the column's norm, at most
// m sqrt(sum d^2) <= 2 m sqrt(r): 4 m (3.4445 + 5.64 sqrt(r)), the 4 as d may fall to a quarter.  So
// |X'| <= 1 again.  Where all columns have 1 they keep it.
// No value passes what fp16 holds: |A'| <= 1, |B| <= 2, and |P'_ik| <= 4.775 |X_i| |X_k| d_k / d_i
// <= 11.6.
constexpr int kXBits = 15, kABits = 15, kBBits = 14, kPBits = 12;
template <int E>  // 2^-E
constexpr float kPow2Less = 1.f / (float)(1ull << E);

// The least e with v <= 2^e, for v > 0
__device__ __forceinline__ int up2(float v) {
  const uint32_t u = __float_as_uint(v);
  return (int)(u >> 23) - 127 + ((u & 0x7fffff) != 0);
}
// Exponents of d and e from the largest entries, and the next ones (sums of squares A'_ii; the
// largest entry of a column of X / d).  Rows and columns of zeros (or NaN) keep theirs.
__device__ __forceinline__ int held_exponent(int e, int most) { return e > most ? most : e < -126 ? -126 : e; }
__device__ __forceinline__ int row_exponent(const NsMat& t, float largest) {
  return largest > 0 ? held_exponent(up2(largest) + t.root, 0) : 0;
}
__device__ __forceinline__ int next_row_exponent(int d, float square) {
  if (!(square > 0)) return d;
  const int to = d + ((up2(square) + 1) >> 1) + 2;
  return held_exponent(to > d - 2 ? to : d - 2, 1);
}
__device__ __forceinline__ int column_exponent(const NsMat& t, float largest, int e) {
  return largest > 0 ? held_exponent(up2(largest) + t.grow, 0) : e;
}
// 2^e of eight exponents (0 below 2^-24, of whose squares nothing is left in a sum), and v 4^e
__device__ __forceinline__ f16x8 pow2_8(const uint2& b) {
  f16x8 s;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    s[j] = (_Float16)ldexpf(1.f, (int)(int8_t)((j < 4 ? b.x : b.y) >> (8 * (j & 3))));
  return s;
}
__device__ __forceinline__ f16x8 scaled_twice(const f16x8& v, const f16x8& s) { return (v * s) * s; }

__device__ __forceinline__ void halve(const f32x4& v, f16x4& hi, f16x4& lo) {
  hi = __builtin_convertvector(v, f16x4);
  lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), f16x4);
}
__device__ __forceinline__ void halve(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}
// f (hi + lo) + v
__device__ __forceinline__ f32x4 add_held(float f, const f16x4& hi, const f16x4& lo, f32x4 v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = fmaf(f, (float)lo[e], fmaf(f, (float)hi[e], v[e]));
  return v;
}

// A tile, by scalar loads: the list was written before any launch that reads it.
__device__ __forceinline__ NsItem ns_item(const NsItem* items, int at) {
  typedef int i32x16 __attribute__((ext_vector_type(16)));
  struct Two {
    i32x16 a, b;
  } v;
  const auto* p = (const __attribute__((address_space(4))) i32x16*)(items + at);
  v.a = p[0];
  v.b = p[1];
  return __builtin_bit_cast(NsItem, v);
}

// U at an entry whose momentum is up to date
__device__ __forceinline__ float direction(const NsArgs& a, int64_t at) {
  const float g = a.G[at];
  if (!a.mom_in) return g;
  const float m = a.mom_out[at];
  return a.nesterov ? fmaf(a.mu, m, g) : m;
}

// 1 / |U| from the sum of squares (a zero matrix stays zero; one that is not finite
// becomes NaN)
__device__ __forceinline__ double ns_scale(double total) {
  return !(total < INFINITY) ? (double)NAN : total > 0 ? 1 / sqrt(total) : 0;
}

__device__ __forceinline__ float ns_gain(const NsMat& t) {
  return sqrtf(fmaxf(1.f, (float)t.rows / (float)t.cols));
}

// W <- W - lr (decay W + u) of the matrix's entry (i, j) (column masks: W1 only)
__device__ __forceinline__ void apply(const NsArgs& a, const NsMat& t, int i, int j, float u) {
  const float lr = a.lrm ? a.lrm[t.m] : a.lr;
  const bool seen = !a.fmask || (a.fmask[(int64_t)t.m * a.fmw + (j >> 5)] >> (j & 31) & 1u);
  float* w = a.W + t.wsrc + (int64_t)i * t.wld + j;
  const float old = *w;
  *w = seen ? old - lr * fmaf(a.decay, old, u) : 0.f;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// Two transposing loads: of a group of 16 lanes, lane i gives the address of 8 bytes (four
// columns i % 4) of row i / 4 and receives column i of the four rows.
__device__ __forceinline__ f16x8 columns(const char* at, int then) {
  lds_char* p = (lds_char*)at;
  const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
  const s16x4 v =
      __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + then));
  return __builtin_bit_cast(f16x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

}  // namespace pmlpk
