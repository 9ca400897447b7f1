// Newton-Schulz steps for many matrices of different shapes at once.
//
//   A = X X^T,  P = b A + c A A,  X <- a X + P X
//
// in fp32 accuracy on the fp16 matrix cores: values are held as newton_device.h says, as fp16
// halves hi and lo beside powers of two for X's rows and columns, and a product takes hi hi + hi lo
// + lo hi, accumulated in fp32: what it leaves out is at most 2^-22 of each product, as fp32 sums
// of that length do, and 2^-38 of what a row and column may hold.  (Six bf16 products would hold
// values of any size without scales.)

#include <algorithm>

#include "newton_device.h"

namespace pmlpk {

// (Without APPLY, also what the scales of X's rows come from where they are the matrix's rows.)
template <bool APPLY>
__global__ __launch_bounds__(256) void k_ns_momentum(NsArgs a, int piece0) {
  __shared__ double part[4];
  __shared__ uint32_t largest[32];  // a wide matrix of more than 128 columns: 31 rows a piece, at most
  const NsPiece p = a.pieces[piece0 + blockIdx.x];
  const NsMat t = a.mats[p.mat];
  // (a piece of several rows has at most kNsPiece entries; one of a row may have any number)
  const int n = p.rows * t.cols;
  const bool turned = t.rows > t.cols;
  if (!APPLY) {
    if (threadIdx.x < 32) largest[threadIdx.x] = 0;
    __syncthreads();
  }
  double sum = 0;
  float m = 0.f;  // of this thread's entries of a row
  int i = threadIdx.x / t.cols, j = threadIdx.x - i * t.cols;
  const int di = 256 / t.cols, dj = 256 - di * t.cols;
#pragma unroll 4
  for (int e = threadIdx.x; e < n; e += 256) {
    const int64_t at = t.src + (int64_t)(p.row0 + i) * t.ld + j;
    const float g = a.G[at];
    float u = g;
    if (a.mom_in) {
      const float m = fmaf(a.mu, a.mom_in[at], g);
      a.mom_out[at] = m;
      u = a.nesterov ? fmaf(a.mu, m, g) : m;
    }
    if (APPLY) apply(a, t, p.row0 + i, j, u);
    else sum += (double)u * (double)u;  // squares of any fp32 values fit
    const int row = i;
    i += di;
    j += dj;
    if (j >= t.cols) {
      j -= t.cols;
      ++i;
    }
    if (!APPLY && !turned) {
      m = fmaxf(m, fabsf(u));
      if (i == row && e + 256 < n) continue;
      atomicMax(largest + row, __float_as_uint(m));
      m = 0.f;
    }
  }
  if (!APPLY) {  // what k_ns_rows and k_ns_load raise
    const int q = piece0 + (int)blockIdx.x - t.piece0;
    if (turned) {
      for (int e = q * 256 + threadIdx.x; e < t.rp; e += t.pieces * 256) a.rmax[t.ro + e] = 0;
    } else if (q == 0 && t.rows + threadIdx.x < t.rp) {
      a.rmax[t.ro + t.rows + threadIdx.x] = 0;
    }
    for (int e = q * 256 + threadIdx.x; e < t.cp; e += t.pieces * 256)
      for (int c = 0; c < 3; ++c) a.cmax[c * a.nc + t.co + e] = 0;
    if (q == 0 && threadIdx.x == 0) a.uneven[t.m] = 0;
  }
  if (APPLY) {
    if (a.lrm && p.row0 == 0 && threadIdx.x == 0 && !(fabsf(a.lrm[t.m]) < INFINITY)) a.flag[1] = 1;
    return;
  }
  sum = wave_total(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (!turned && threadIdx.x < p.rows) a.rmax[t.ro + p.row0 + threadIdx.x] = largest[threadIdx.x];
  if (threadIdx.x == 0) a.sums[piece0 + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

hipError_t launch_ns_momentum(const NsArgs& a, int32_t piece0, int32_t pieces, bool apply,
                              hipStream_t s) {
  note_variant("k_ns_momentum", kArithNone);
  for (int32_t at = 0; at < pieces; at += kNsGrid) {
    const unsigned grid = (unsigned)std::min(kNsGrid, pieces - at);
    if (apply) k_ns_momentum<true><<<grid, 256, 0, s>>>(a, piece0 + at);
    else k_ns_momentum<false><<<grid, 256, 0, s>>>(a, piece0 + at);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

namespace {
// 1 / |U|_F, by a workgroup of 256
__device__ __forceinline__ double norm_scale(const NsArgs& a, const NsMat& t, double* part) {
  const int tid = threadIdx.x;
  double total = 0;
  for (int q = tid; q < t.pieces; q += 256) total += a.sums[t.piece0 + q];
  total = wave_total(total);
  if ((tid & 63) == 0) part[tid >> 6] = total;
  __syncthreads();
  return ns_scale((part[0] + part[1]) + (part[2] + part[3]));
}
}  // namespace

// The largest |U| of every row of a turned X, which is a column of the matrix.  (A maximum does
// not depend on the order.)
__global__ __launch_bounds__(256) void k_ns_rows(NsArgs a, const NsItem* items) {
  const NsItem it = ns_item(items, blockIdx.x);
  const NsMat& t = it.t;
  const int x = threadIdx.x & 31, y0 = threadIdx.x >> 5;
  const int j1 = min(t.rows, (it.j + 1) * a.tile);
  for (int i = it.i * a.tile + x; i < min(t.cols, (it.i + 1) * a.tile); i += 32) {
    float m = 0.f;
    for (int j = it.j * a.tile + y0; j < j1; j += 8) m = fmaxf(m, fabsf(direction(a, t.src + (int64_t)j * t.ld + i)));
    if (m > 0) atomicMax(a.rmax + t.ro + i, __float_as_uint(m));
  }
}

hipError_t launch_ns_rows(const NsArgs& a, const NsItem* items, int32_t n, hipStream_t s) {
  note_variant("k_ns_rows", kArithNone);
  k_ns_rows<<<(unsigned)n, 256, 0, s>>>(a, items);
  return hipGetLastError();
}

// A 32 x 32 block at a time through LDS, for both orders of X.  The columns' scales need the largest
// |X / d| of each first: X is loaded without them, with those maxima, and once more (AGAIN) where a
// column is small enough to need one, which few matrices have.  (40 of 500 to 1,000 x 1,000: 68 us
// for the maxima alone in a pass of their own.)
template <bool AGAIN>
__global__ __launch_bounds__(256) void k_ns_load(NsArgs a, const NsItem* items) {
  __shared__ float block[32][33];
  __shared__ double part[4];
  __shared__ int rows[128], cols[128];
  const NsItem it = ns_item(items, blockIdx.x);
  const NsMat& t = it.t;
  const int tid = threadIdx.x;
  if (AGAIN) {
    bool any = false;
    for (int j = tid; j < t.c; j += 256) any |= column_exponent(t, __uint_as_float(a.cmax[t.co + j]), 0) != 0;
    if (!__syncthreads_or(any)) return;
    if (it.i == 0 && it.j == 0 && tid == 0) a.uneven[t.m] = 1;
  }
  const double scale = norm_scale(a, t, part);
  if (tid < a.tile) {
    const int i = it.i * a.tile + tid, j = it.j * a.tile + tid;
    if (i < t.rp) {
      const int d = row_exponent(t, (float)(scale * (double)__uint_as_float(a.rmax[t.ro + i])));
      rows[tid] = d;
      if (!AGAIN && it.j == 0) a.rows[t.ro + i] = (int8_t)d;
    }
    if (AGAIN && j < t.cp) {
      cols[tid] = column_exponent(t, __uint_as_float(a.cmax[t.co + j]), 0);
      if (it.i == 0) a.cols[t.co + j] = (int8_t)cols[tid];
    }
  }
  __syncthreads();
  const bool turned = t.rows > t.cols;
  const int x = tid & 31, y0 = tid >> 5;        // reading: four rows, one column
  const int y = tid >> 3, x4 = 4 * (tid & 7);   // storing: one row, four columns
  _Float16 *X = a.X[0] + t.xo, *XT = a.XT[0] + t.xo;
  const int i1 = min(t.rp, (it.i + 1) * a.tile), j1 = min(t.cp, (it.j + 1) * a.tile);
  for (int j0 = it.j * a.tile; j0 < j1; j0 += 32) {
    float m[4] = {};  // the largest entries of its column or columns
    for (int i0 = it.i * a.tile; i0 < i1; i0 += 32) {
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // (along the matrix's rows: X's rows, or its columns)
        const int gi = (turned ? j0 : i0) + y0 + 8 * q, gj = (turned ? i0 : j0) + x;
        v[q] = 0.f;
        if (gi < t.rows && gj < t.cols)
          v[q] = ldexpf((float)(scale * (double)direction(a, t.src + (int64_t)gi * t.ld + gj)),
                        kXBits - rows[(turned ? gj : gi) - it.i * a.tile] -
                            (AGAIN ? cols[(turned ? gi : gj) - it.j * a.tile] : 0));
        if (!AGAIN) m[q] = fmaxf(m[q], fabsf(v[q]));
      }
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (turned) block[x][y0 + 8 * q] = v[q];
        else block[y0 + 8 * q][x] = v[q];
      }
      __syncthreads();
      f16x4 hi, lo;
      halve(f32x4{block[y][x4], block[y][x4 + 1], block[y][x4 + 2], block[y][x4 + 3]}, hi, lo);
      _Float16* at = X + (int64_t)(i0 + y) * t.cp + j0 + x4;
      *(f16x4*)at = hi;
      *(f16x4*)(at + a.nx) = lo;
      halve(f32x4{block[x4][y], block[x4 + 1][y], block[x4 + 2][y], block[x4 + 3][y]}, hi, lo);
      at = XT + (int64_t)(j0 + y) * t.rp + i0 + x4;
      *(f16x4*)at = hi;
      *(f16x4*)(at + a.nx) = lo;
    }
    if (AGAIN) continue;
    if (!turned) {  // a lane's four are of one column of X
      const float v = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
      if (v > 0) atomicMax(a.cmax + t.co + j0 + x, __float_as_uint(v * kPow2Less<kXBits>));
      continue;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float v = m[q];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
      if (x == 0 && v > 0) atomicMax(a.cmax + t.co + j0 + y0 + 8 * q, __float_as_uint(v * kPow2Less<kXBits>));
    }
  }
}

hipError_t launch_ns_load(const NsArgs& a, const NsItem* items, int32_t n, hipStream_t s) {
  note_variant("k_ns_load", kArithNone);
  k_ns_load<false><<<(unsigned)n, 256, 0, s>>>(a, items);
  k_ns_load<true><<<(unsigned)n, 256, 0, s>>>(a, items);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The products, all of the form C[i][j] = sum_k L[i][k] Q[j][k] with k contiguous in both
// operands (the next X is stored in both orders for it).  Tiles of T x TJ, four waves of
// T / 2 x TJ / 2.  A and P are symmetric: only tiles with j <= i are computed, and stored
// twice.  A lane ends with four consecutive rows of a column; a wave's block goes through
// LDS, where it is read by rows of either order, 16 bytes a lane.
//
// Bound by the matrix cores behind LDS and two barriers a stage, and by the stores of both
// orders: 40 matrices of 500 to 1,000 x 1,000 120 us for A, 108 for P, 247 for a step (191, 169
// and 186 TFLOP/s of the 355 that three fp16 products at a large library product's rate make;
// MFMA busy 0.38, 0.35, 0.31), 119, 101 and 237 without the scales.  Steps of 128 x 128 tiles
// took 254 us where these took 240.
// ---------------------------------------------------------------------------

template <int WHAT, int T, int TJ>
__global__ __launch_bounds__(256, 2) void k_ns_product(NsArgs a, int number, const NsItem* items, int n) {
  constexpr int KT = 32, ROW = 2 * KT, W = T / 2, WJ = TJ / 2, NT = W / 32, NJ = WJ / 32;
  constexpr int NQ = (T + TJ) / 64, NQL = T / 64;
  constexpr int PLANE = (T + TJ) * ROW;   // both operands' rows
  constexpr int CB = WJ < 64 ? WJ : 64;   // columns of a wave's block that go through LDS at a time
  constexpr int BR = 2 * W + 16;          // bytes of a column of it there
  constexpr int BLOCK = CB * BR;
  constexpr int LDS = 2 * PLANE > 4 * BLOCK ? 2 * PLANE : 4 * BLOCK;
  __shared__ __align__(16) char lds[LDS];
  __shared__ __align__(16) float by_row[T];  // factors of the tile's rows
  // Workgroups go to the eight dies in turn; each die takes a run of the list, and with it
  // whole matrices, whose tiles share rows in its cache.
  const int at = (blockIdx.x & 7) * ((n + 7) / 8) + (blockIdx.x >> 3);
  if (at >= n) return;
  const NsItem it = ns_item(items, at);
  const NsMat& t = it.t;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = wave & 1, wj = wave >> 1;
  const int i0 = it.i * T, j0 = it.j * TJ;
  constexpr bool step = WHAT == NS_STEP || WHAT == NS_LAST;
  const int from = number & 1;
  const int8_t *rows = a.rows + from * a.nr + t.ro, *cols = a.cols + from * a.nc + t.co;
  const bool uneven = WHAT != NS_POLY && a.uneven[t.m];
  if (WHAT != NS_GRAM && tid < T) {
    const int i = i0 + tid < t.rp ? i0 + tid : t.rp - 1;
    int e = rows[i];
    if (WHAT == NS_POLY) e *= 2;
    if (WHAT == NS_STEP) {
      const _Float16* q = a.A + t.ao + (int64_t)i * t.rp + i;
      const int next = next_row_exponent(e, ((float)q[0] + (float)q[a.na]) * kPow2Less<kABits>);
      if (it.j == 0) a.rows[(1 - from) * a.nr + t.ro + i] = (int8_t)next;
      e -= next;
    }
    by_row[tid] = ldexpf(1.f, e);
  }
  const _Float16* L = WHAT == NS_GRAM ? a.X[from] + t.xo : WHAT == NS_POLY ? a.A + t.ao : a.P + t.ao;
  const _Float16* Q = WHAT == NS_GRAM ? L : WHAT == NS_POLY ? L : a.XT[from] + t.xo;
  const int64_t lplane = WHAT == NS_GRAM ? a.nx : a.na, qplane = WHAT == NS_POLY ? a.na : a.nx;
  const int K = WHAT == NS_GRAM ? t.cp : t.rp;
  const int nj = step ? t.cp : t.rp;

  // T + TJ rows of four 16-byte chunks a plane: each thread takes one chunk of rows tid / 4 + 64 q
  const int c = tid & 3;
  const _Float16* row[NQ];
  char* put[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int r = 64 * q + (tid >> 2);
    if (q < NQL) {
      const int i = i0 + r < t.rp ? i0 + r : t.rp - 1;
      row[q] = L + (int64_t)i * K + 8 * c;
    } else {
      const int j = j0 + r - T < nj ? j0 + r - T : nj - 1;
      row[q] = Q + (int64_t)j * K + 8 * c;
    }
    put[q] = lds + r * ROW + ((c ^ ((r >> 2) & 3)) << 4);
  }
  // DEPTH stages are on their way from memory: a small tile's stage is multiplied long before
  // the next one arrives.
  constexpr int DEPTH = T == 64 ? 4 : TJ == 128 ? 2 : 1;
  f16x8 v[DEPTH][NQ][2];
  // (A' is multiplied with A' D^2, X' with X' E^2 where E is not 1.)
  constexpr bool scales = !step;
  const int8_t* by = (WHAT == NS_GRAM ? cols : rows) + 8 * c;
  uint2 ex[scales ? DEPTH : 1];
  auto load = [&](int d, int k) {
    if (scales) ex[d] = *(const uint2*)(by + k);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      v[d][q][0] = *(const f16x8*)(row[q] + k);
      v[d][q][1] = *(const f16x8*)(row[q] + (q < NQL ? lplane : qplane) + k);
    }
  };
  f32x16 acc[NT][NJ];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (d * KT < K) load(d, d * KT);
  // What the product is added to, [j][i]; a small tile has it before its last product.
  constexpr int LPR = W / 8;         // lanes of 16 bytes to a row of the wave's block
  constexpr bool AHEAD = T == 64 && WHAT != NS_GRAM && WHAT != NS_LAST;
  const int bi0 = i0 + wi * W, bw0 = j0 + wj * WJ;  // this wave's block
  const _Float16* old = WHAT == NS_POLY ? a.A + t.ao : a.XT[from] + t.xo;
  const int64_t plane = step ? a.nx : a.na;
  auto old_at = [&](int h, int q, int bj0) {
    const int r = q * (64 / LPR) + lane / LPR, ch = lane % LPR;
    const int j = min(bj0 + r, nj - 1), i = min(bi0 + 8 * ch, t.rp - 8);
    return *(const f16x8*)(old + h * plane + (int64_t)j * t.rp + i);
  };
  f16x8 held[2][AHEAD ? CB * LPR / 64 : 1];
  if (AHEAD)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < CB * LPR / 64; ++q) held[h][q] = old_at(h, q, bw0);
  for (int k0 = 0; k0 < K; k0 += DEPTH * KT) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int k = k0 + d * KT;
      if (k >= K) break;
      if (WHAT == NS_POLY || (WHAT == NS_GRAM && uneven)) {
        const f16x8 s = pow2_8(ex[scales ? d : 0]);
#pragma unroll
        for (int q = NQL; q < NQ; ++q)
#pragma unroll
          for (int h = 0; h < 2; ++h) v[d][q][h] = scaled_twice(v[d][q][h], s);
      }
      lds_barrier();
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        *(f16x8*)put[q] = v[d][q][0];
        *(f16x8*)(put[q] + PLANE) = v[d][q][1];
      }
      if (k + DEPTH * KT < K) load(d, k + DEPTH * KT);
      lds_barrier();
#pragma unroll
    for (int ks = 0; ks < KT / 16; ++ks) {
      const int cc = 2 * ks + (lane >> 5), r = lane & 31;
      f16x8 x[NT][2], y[NJ][2];
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int ri = wi * W + 32 * i + r;
          x[i][e] = *(const f16x8*)(lds + e * PLANE + ri * ROW + ((cc ^ ((ri >> 2) & 3)) << 4));
        }
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int rj = T + wj * WJ + 32 * j + r;
          y[j][e] = *(const f16x8*)(lds + e * PLANE + rj * ROW + ((cc ^ ((rj >> 2) & 3)) << 4));
        }
      // (small products first, the tiles in turn)
#pragma unroll
      for (int h = 0; h < 3; ++h)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i][h == 0], y[j][h == 1], acc[i][j], 0, 0, 0);
    }
    }
  }

  const int half = 4 * (lane >> 5);
  if (WHAT == NS_LAST) {
    const bool turned = t.rows > t.cols;
    const float gain = ns_gain(t);
#pragma unroll
    for (int bj = 0; bj < NJ; ++bj) {
      const int j = bw0 + 32 * bj + (lane & 31);
      if (j >= nj) continue;
      const float by_column = ldexpf(kPow2Less<kXBits>, uneven ? (int)cols[j] : 0);
#pragma unroll
      for (int bi = 0; bi < NT; ++bi)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int i = bi0 + 32 * bi + 8 * q + half;  // .. i + 3
          if (i >= t.rp) continue;
          const _Float16* old = a.XT[from] + t.xo + (int64_t)j * t.rp + i;
          const f16x4 hi = *(const f16x4*)old, lo = *(const f16x4*)(old + a.nx);
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[bi][bj][4 * q + e] * kPow2Less<kPBits>;
          v = add_held(kNsA, hi, lo, v) * by_column;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = v[e] * by_row[i + e - i0];
            const int gi = turned ? j : i + e, gj = turned ? i + e : j;
            if (gi >= t.rows || gj >= t.cols) continue;
            if (a.W) apply(a, t, gi, gj, gain * x);
            else a.out[t.src + (int64_t)gi * t.ld + gj] = x;
          }
        }
    }
    if (a.W && a.lrm && it.i == 0 && it.j == 0 && tid == 0 && !(fabsf(a.lrm[t.m]) < INFINITY))
      a.flag[1] = 1;
    return;
  }
  if (bi0 >= t.rp || bw0 >= nj) {  // (no wave waits below)
    __syncthreads();
    return;
  }
  __syncthreads();  // the operands have been read: LDS is the waves' own from here on
  char* block = lds + wave * BLOCK;  // [column][row]
  _Float16* to = WHAT == NS_GRAM ? a.A + t.ao : WHAT == NS_POLY ? a.P + t.ao : a.X[1 - from] + t.xo;
  _Float16* tt = WHAT == NS_STEP ? a.XT[1 - from] + t.xo : to;  // [j][i]: stride rp
  constexpr float unscale = WHAT == NS_GRAM   ? kPow2Less<2 * kXBits - kABits>
                            : WHAT == NS_POLY ? kNsC * kPow2Less<2 * kABits - kPBits>
                                              : kPow2Less<kPBits>;
  constexpr float add = WHAT == NS_POLY ? kNsB * kPow2Less<kABits - kPBits> : kNsA;
#pragma unroll
  for (int bi = 0; bi < NT; ++bi)
#pragma unroll
    for (int bj = 0; bj < NJ; ++bj) acc[bi][bj] *= unscale;
  const bool other = WHAT == NS_STEP || it.i != it.j;  // the order [i][j] too
#pragma unroll
  for (int cb = 0; cb < WJ / CB; ++cb) {
    const int bj0 = bw0 + cb * CB;
    if (bj0 >= nj) continue;
    if (WHAT != NS_GRAM) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int q = 0; q < CB * LPR / 64; ++q) {
          const int r = q * (64 / LPR) + lane / LPR, ch = lane % LPR;
          *(f16x8*)(block + r * BR + 16 * ch) = AHEAD ? held[h][q] : old_at(h, q, bj0);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int bi = 0; bi < NT; ++bi)
#pragma unroll
          for (int bj = 0; bj < CB / 32; ++bj)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              f32x16& c = acc[bi][cb * (CB / 32) + bj];
              const f16x4 o = *(const f16x4*)(block + (32 * bj + (lane & 31)) * BR + 2 * (32 * bi + 8 * q + half));
#pragma unroll
              for (int e = 0; e < 4; ++e)
                c[4 * q + e] = fmaf(add, (float)o[e], c[4 * q + e]);
            }
        __builtin_amdgcn_wave_barrier();
      }
    }
    if (WHAT == NS_STEP) {
#pragma unroll
      for (int bj = 0; bj < CB / 32; ++bj) {
        const int j = bj0 + 32 * bj + (lane & 31);
        const bool there = j < nj;
        int e = 0, next = 0;
        if (uneven && there) {
          e = cols[j];
          next = column_exponent(t, __uint_as_float(a.cmax[number % 3 * a.nc + t.co + j]), e);
        }
        const float by_column = ldexpf(1.f, e - next);
        float m = 0.f;
#pragma unroll
        for (int bi = 0; bi < NT; ++bi) {
          f32x16& c = acc[bi][cb * (CB / 32) + bj];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 f = *(const f32x4*)(by_row + wi * W + 32 * bi + 8 * q + half);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              c[4 * q + k] *= f[k] * by_column;
              if (bi0 + 32 * bi < t.rp) m = fmaxf(m, fabsf(c[4 * q + k]));
            }
          }
        }
        if (!uneven) continue;
        m = fmaxf(m, __shfl_xor(m, 32));
        if (there && lane < 32) {
          atomicMax(a.cmax + (number + 1) % 3 * a.nc + t.co + j, __float_as_uint(ldexpf(m, next - kXBits)));
          if (it.i == 0 && wi == 0) {
            a.cols[(1 - from) * a.nc + t.co + j] = (int8_t)next;
            a.cmax[(number + 2) % 3 * a.nc + t.co + j] = 0;
          }
        }
      }
    }
    // the wave's block, a plane of it, times its rows' or its columns' factors (P')
    auto put_block = [&](int h, bool by_rows) __attribute__((always_inline)) {
#pragma unroll
      for (int bj = 0; bj < CB / 32; ++bj) {
        const int j = bj0 + 32 * bj + (lane & 31);
        const float by_column = WHAT == NS_POLY && !by_rows ? ldexpf(1.f, 2 * (int)rows[j < nj ? j : 0]) : 1.f;
#pragma unroll
        for (int bi = 0; bi < NT; ++bi)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x16& c = acc[bi][cb * (CB / 32) + bj];
            f32x4 v{c[4 * q], c[4 * q + 1], c[4 * q + 2], c[4 * q + 3]};
            if (WHAT == NS_POLY)
              v *= by_rows ? *(const f32x4*)(by_row + wi * W + 32 * bi + 8 * q + half)
                           : f32x4{by_column, by_column, by_column, by_column};
            f16x4 hi, lo;
            halve(v, hi, lo);
            *(f16x4*)(block + (32 * bj + (lane & 31)) * BR + 2 * (32 * bi + 8 * q + half)) = h ? lo : hi;
          }
      }
      __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      put_block(h, true);
#pragma unroll
      for (int q = 0; q < CB * LPR / 64; ++q) {
        const int r = q * (64 / LPR) + lane / LPR, ch = lane % LPR;
        const int j = bj0 + r, i = bi0 + 8 * ch;
        if (j < nj && i < t.rp)
          *(f16x8*)(tt + h * plane + (int64_t)j * t.rp + i) = *(const f16x8*)(block + r * BR + 16 * ch);
      }
      if (other) {
        if (WHAT == NS_POLY) {
          __builtin_amdgcn_wave_barrier();
          put_block(h, false);
        }
        // transposing loads: lane (li, lk) gets row li of the block's 16, columns 8 lk .. + 7
        const int li = lane & 15, lk = lane >> 4;
#pragma unroll
        for (int r = 0; r < W; r += 16)
#pragma unroll
          for (int cc = 0; cc < CB; cc += 32) {
            const char* at = block + (cc + 8 * lk + (li >> 2)) * BR + 2 * r + 8 * (li & 3);
            const f16x8 o = columns(at, 4 * BR);
            const int i = bi0 + r + li, j = bj0 + cc + 8 * lk;
            if (i < t.rp && j < nj) *(f16x8*)(to + h * plane + (int64_t)i * nj + j) = o;
          }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

namespace {
// (TS: columns of a tile of the steps)
template <int T, int TS>
void product(const NsArgs& a, int what, int step, const NsItem* items, int n, hipStream_t s) {
  const unsigned grid = (unsigned)((n + 7) / 8 * 8);
  switch (what) {
    case NS_GRAM: k_ns_product<NS_GRAM, T, T><<<grid, 256, 0, s>>>(a, step, items, n); break;
    case NS_POLY: k_ns_product<NS_POLY, T, T><<<grid, 256, 0, s>>>(a, step, items, n); break;
    case NS_STEP: k_ns_product<NS_STEP, T, TS><<<grid, 256, 0, s>>>(a, step, items, n); break;
    default: k_ns_product<NS_LAST, T, TS><<<grid, 256, 0, s>>>(a, step, items, n); break;
  }
}
}  // namespace

hipError_t launch_ns_product(const NsArgs& a, int what, int step, const NsItem* items, int32_t n,
                             hipStream_t s) {
  note_variant("k_ns_product", kArithF16x2);
  if (a.tile == 64) product<64, 64>(a, what, step, items, n, s);
  else product<128, 256>(a, what, step, items, n, s);
  return hipGetLastError();
}

}  // namespace pmlpk
