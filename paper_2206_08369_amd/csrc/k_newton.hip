// Newton-Schulz steps for many matrices of different shapes at once.
//
//   A = X X^T,  P = b A + c A A,  X <- a X + P X
//
// in fp32 accuracy on the fp16 matrix cores: every value v is held as the fp16 numbers
// hi = v 2^13 and lo = v 2^13 - hi (rounded; 23 bits of v, and no value is above 2.9: a
// singular value of X is at most 1.21 from the norm on, one of P at most 2.9), and a
// product takes hi hi + hi lo + lo hi, accumulated in fp32: what it leaves out is at most
// 2^-22 of each product, as fp32 sums of that length do.  (Six bf16 products would hold
// values of any size; these are normalised.)

#include "device_common.h"
#include "newton.h"

namespace pmlpk {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr float kScale = 8192.f, kUnscale = 1.f / (8192.f * 8192.f);

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
  const float t = v * kScale;
  hi = (_Float16)t;
  lo = (_Float16)(t - (float)hi);
}
__device__ __forceinline__ float join(_Float16 hi, _Float16 lo) {
  return ((float)hi + (float)lo) * (1.f / kScale);
}

__device__ __forceinline__ float direction(const NsArgs& a, int64_t at) {
  const float g = a.G[at];
  if (!a.mom_in) return g;
  const float m = a.mom_out[at];
  return a.nesterov ? fmaf(a.mu, m, g) : m;
}

// W <- W - lr (decay W + u) of model m's entry in column j (column masks: W1 only)
__device__ __forceinline__ void apply(const NsArgs& a, const NsMat& t, int i, int j, float u) {
  const float lr = a.lrm ? a.lrm[t.m] : a.lr;
  const bool seen = !a.fmask || (a.fmask[(int64_t)t.m * a.fmw + (j >> 5)] >> (j & 31) & 1u);
  float* w = a.W + t.wsrc + (int64_t)i * t.wld + j;
  const float old = *w;
  *w = seen ? old - lr * fmaf(a.decay, old, u) : 0.f;
}

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

}  // namespace

template <bool APPLY>
__global__ __launch_bounds__(256) void k_ns_momentum(NsArgs a, int piece0) {
  __shared__ double part[4];
  const NsPiece p = a.pieces[piece0 + blockIdx.x];
  const NsMat t = a.mats[p.mat];
  const int64_t n = (int64_t)p.rows * t.cols;
  double sum = 0;
  for (int64_t e = threadIdx.x; e < n; e += 256) {
    const int i = p.row0 + (int)(e / t.cols), j = (int)(e % t.cols);
    const int64_t at = t.src + (int64_t)i * t.ld + j;
    const float g = a.G[at];
    float u = g;
    if (a.mom_in) {
      const float m = fmaf(a.mu, a.mom_in[at], g);
      a.mom_out[at] = m;
      u = a.nesterov ? fmaf(a.mu, m, g) : m;
    }
    if (APPLY) apply(a, t, i, j, u);
    else sum += (double)u * (double)u;  // squares of any fp32 values fit
  }
  if (APPLY) {
    if (a.lrm && p.row0 == 0 && threadIdx.x == 0 && !(fabsf(a.lrm[t.m]) < INFINITY)) a.flag[1] = 1;
    return;
  }
  sum = wave_total(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) a.sums[piece0 + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

hipError_t launch_ns_momentum(const NsArgs& a, int32_t piece0, int32_t pieces, bool apply,
                              hipStream_t s) {
  note_variant("k_ns_momentum", kArithNone);
  if (apply) k_ns_momentum<true><<<(unsigned)pieces, 256, 0, s>>>(a, piece0);
  else k_ns_momentum<false><<<(unsigned)pieces, 256, 0, s>>>(a, piece0);
  return hipGetLastError();
}

// A 32 x 32 block at a time through LDS, for both orders of X.
__global__ __launch_bounds__(256) void k_ns_load(NsArgs a, const NsItem* items) {
  __shared__ float block[32][33];
  const NsItem it = items[blockIdx.x];
  const NsMat t = a.mats[it.mat];
  double total = 0;
  for (int q = 0; q < t.pieces; ++q) total += a.sums[t.piece0 + q];
  // (a zero matrix stays zero; one that is not finite becomes NaN)
  const double scale = !(total < INFINITY) ? (double)NAN : total > 0 ? 1 / sqrt(total) : 0;
  const bool turned = t.rows > t.cols;
  const int x = threadIdx.x & 31, y0 = threadIdx.x >> 5;
  _Float16 *X = a.X[0] + t.xo, *XT = a.XT[0] + t.xo;
  const int i1 = min(t.rp, (it.i + 1) * kNsTile), j1 = min(t.cp, (it.j + 1) * kNsTile);
  for (int i0 = it.i * kNsTile; i0 < i1; i0 += 32)
    for (int j0 = it.j * kNsTile; j0 < j1; j0 += 32) {
      __syncthreads();
      for (int y = y0; y < 32; y += 8) {
        // (along the matrix's rows: X's rows, or its columns)
        const int gi = (turned ? j0 : i0) + y, gj = (turned ? i0 : j0) + x;
        float v = 0.f;
        if (gi < t.rows && gj < t.cols)
          v = (float)(scale * (double)direction(a, t.src + (int64_t)gi * t.ld + gj));
        if (turned) block[x][y] = v;
        else block[y][x] = v;
      }
      __syncthreads();
      for (int y = y0; y < 32; y += 8) {
        _Float16 hi, lo;
        split(block[y][x], hi, lo);
        const int64_t at = (int64_t)(i0 + y) * t.cp + j0 + x;
        X[at] = hi;
        X[at + a.nx] = lo;
        split(block[x][y], hi, lo);
        const int64_t to = (int64_t)(j0 + y) * t.rp + i0 + x;
        XT[to] = hi;
        XT[to + a.nx] = lo;
      }
    }
}

hipError_t launch_ns_load(const NsArgs& a, const NsItem* items, int32_t n, hipStream_t s) {
  note_variant("k_ns_load", kArithNone);
  k_ns_load<<<(unsigned)n, 256, 0, s>>>(a, items);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The products, all of the form C[i][j] = sum_k L[i][k] Q[j][k] with k contiguous in both
// operands (the next X is stored in both orders for it).  Tiles of 128 x 128, four waves
// of 64 x 64.  A and P are symmetric: only tiles with j <= i are computed, and stored twice.
// ---------------------------------------------------------------------------

template <int WHAT>
__global__ __launch_bounds__(256, 2) void k_ns_product(NsArgs a, int from, const NsItem* items) {
  constexpr int KT = 32, ROW = 2 * KT, T = kNsTile;
  constexpr int PLANE = 2 * T * ROW;  // both operands' rows
  __shared__ __align__(16) char lds[2 * PLANE];
  const NsItem it = items[blockIdx.x];
  const NsMat t = a.mats[it.mat];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = wave & 1, wj = wave >> 1;
  const int i0 = it.i * T, j0 = it.j * T;
  const bool step = WHAT == NS_STEP || WHAT == NS_LAST;
  const _Float16* L = WHAT == NS_GRAM ? a.X[from] + t.xo : WHAT == NS_POLY ? a.A + t.ao : a.P + t.ao;
  const _Float16* Q = WHAT == NS_GRAM ? L : WHAT == NS_POLY ? L : a.XT[from] + t.xo;
  const int64_t lplane = WHAT == NS_GRAM ? a.nx : a.na, qplane = WHAT == NS_POLY ? a.na : a.nx;
  const int K = WHAT == NS_GRAM ? t.cp : t.rp;
  const int nj = step ? t.cp : t.rp;

  // 256 rows of four 16-byte chunks a plane: each thread takes one chunk of rows tid / 4 + 64 q
  const int c = tid & 3;
  const _Float16* row[4];
  char* put[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int r = 64 * q + (tid >> 2);
    if (r < T) {
      const int i = i0 + r < t.rp ? i0 + r : t.rp - 1;
      row[q] = L + (int64_t)i * K + 8 * c;
    } else {
      const int j = j0 + r - T < nj ? j0 + r - T : nj - 1;
      row[q] = Q + (int64_t)j * K + 8 * c;
    }
    put[q] = lds + r * ROW + ((c ^ ((r >> 1) & 3)) << 4);
  }
  f16x8 v[4][2];
  auto load = [&](int k) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q][0] = *(const f16x8*)(row[q] + k);
      v[q][1] = *(const f16x8*)(row[q] + (q < 2 ? lplane : qplane) + k);
    }
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  load(0);
  for (int k = 0; k < K; k += KT) {
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      *(f16x8*)put[q] = v[q][0];
      *(f16x8*)(put[q] + PLANE) = v[q][1];
    }
    if (k + KT < K) load(k + KT);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < KT / 16; ++ks) {
      const int cc = 2 * ks + (lane >> 5), r = lane & 31;
      f16x8 x[2][2], y[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int ri = wi * 64 + 32 * i + r, rj = T + wj * 64 + 32 * i + r;
          x[i][e] = *(const f16x8*)(lds + e * PLANE + ri * ROW + ((cc ^ ((ri >> 1) & 3)) << 4));
          y[i][e] = *(const f16x8*)(lds + e * PLANE + rj * ROW + ((cc ^ ((rj >> 1) & 3)) << 4));
        }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][1], y[j][0], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[j][1], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][0], y[j][0], acc[i][j], 0, 0, 0);
        }
    }
  }

  // lane: column j, rows 8 (e / 4) + 4 (lane / 32) + e % 4 of each 32
  const int half = 4 * (lane >> 5);
  const bool mirror = !step && it.i != it.j;
  const float gain = step ? sqrtf(fmaxf(1.f, (float)t.rows / (float)t.cols)) : 0.f;
#pragma unroll
  for (int bj = 0; bj < 2; ++bj) {
    const int j = j0 + wj * 64 + 32 * bj + (lane & 31);
    if (j >= nj) continue;
#pragma unroll
    for (int bi = 0; bi < 2; ++bi)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = i0 + wi * 64 + 32 * bi + 8 * q + half;  // .. i + 3
        if (i >= t.rp) continue;
        f16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x = acc[bi][bj][4 * q + e] * kUnscale;
          const int64_t at = (int64_t)(i + e) * nj + j;
          if (WHAT == NS_POLY) {
            const _Float16* old = a.A + t.ao + at;
            x = fmaf(kNsC, x, kNsB * join(old[0], old[a.na]));
          }
          if (step) {
            const _Float16* old = a.X[from] + t.xo + at;
            x = fmaf(kNsA, join(old[0], old[a.nx]), x);
          }
          if (WHAT == NS_LAST) {
            const bool turned = t.rows > t.cols;
            const int gi = turned ? j : i + e, gj = turned ? i + e : j;
            if (gi >= t.rows || gj >= t.cols) continue;
            if (a.W) apply(a, t, gi, gj, gain * x);
            else a.out[t.src + (int64_t)gi * t.ld + gj] = x;
            continue;
          }
          _Float16 h, l;
          split(x, h, l);
          hi[e] = h;
          lo[e] = l;
          _Float16* to = (WHAT == NS_GRAM ? a.A + t.ao : WHAT == NS_POLY ? a.P + t.ao
                                                                         : a.X[1 - from] + t.xo) + at;
          to[0] = h;
          to[WHAT == NS_STEP ? a.nx : a.na] = l;
        }
        if (WHAT == NS_LAST) continue;
        if (WHAT == NS_STEP || mirror) {
          _Float16* to = (WHAT == NS_GRAM ? a.A + t.ao : WHAT == NS_POLY ? a.P + t.ao
                                                                         : a.XT[1 - from] + t.xo) +
                         (int64_t)j * t.rp + i;
          *(f16x4*)to = hi;
          *(f16x4*)(to + (WHAT == NS_STEP ? a.nx : a.na)) = lo;
        }
      }
  }
  if (WHAT == NS_LAST && a.W && a.lrm && it.i == 0 && it.j == 0 && tid == 0 &&
      !(fabsf(a.lrm[t.m]) < INFINITY))
    a.flag[1] = 1;
}

hipError_t launch_ns_product(const NsArgs& a, int what, int from, const NsItem* items, int32_t n,
                             hipStream_t s) {
  note_variant("k_ns_product", kArithX3);
  switch (what) {
    case NS_GRAM: k_ns_product<NS_GRAM><<<(unsigned)n, 256, 0, s>>>(a, from, items); break;
    case NS_POLY: k_ns_product<NS_POLY><<<(unsigned)n, 256, 0, s>>>(a, from, items); break;
    case NS_STEP: k_ns_product<NS_STEP><<<(unsigned)n, 256, 0, s>>>(a, from, items); break;
    default: k_ns_product<NS_LAST><<<(unsigned)n, 256, 0, s>>>(a, from, items); break;
  }
  return hipGetLastError();
}

}  // namespace pmlpk
