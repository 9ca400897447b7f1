// Device code shared by the kernels of k_newton.hip and k_newton_small.hip.
#pragma once

#include "device_common.h"
#include "newton.h"

namespace pmlpk {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// X, A and P are held 2^13 times as large, every value v as the fp16 numbers hi = v and
// lo = v - hi, both rounded (see k_newton.hip); sums of products are then 2^26 times as
// large as theirs.
constexpr float kScale = 8192.f, kUnscale = 1.f / 8192.f;

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
