// Newton-Schulz steps of matrices that fit a workgroup's LDS: one launch from the gradient
// to the result.  Values are held as newton_device.h says: fp16 halves beside powers of two for
// the rows and columns of X.
//
// LDS: X' [RP][C], a plane of each half, and one such pair for B = A' D, which P' replaces, and the
// exponents of D and E, [2] each in turn.  All operands come from there:
//   A' = X' E^2 X'^T    rows of X' for both operands, one of them times E^2 where E is not 1;
//   P' = (b A' + c B B^T) D^2   rows of B; A' is still in the registers of the wave that made it;
//   X' <- a X' + X'^T-columns x P':  D[col][row] = sum_k X[k][col] P[row][k], the first operand
//       by transposing loads, so that a lane ends with four consecutive columns of a row and
//       stores 8 bytes a plane.  The k of a fragment are then rows 4 lk + j and 16 + 4 lk + j;
//       the columns of A and P lie in that order.
// Rows are 16 bytes times an odd number apart: the 16-byte reads of 16 rows are spread over all
// banks.  The transposing loads read 32 bytes of each of eight rows, and a mirrored tile is stored
// 2 bytes a lane and four rows apart: two ways on a bank.
//
// Bound by LDS, vector work and latency: a 2 x 4 block of tiles reads 12 fragments for its 24
// matrix instructions, what one LDS feeds four SIMDs with.  10,000 matrices of 1 to 100 x 100: 581
// us; LDS busy 0.37 to 0.48 of the time and 0.42 of that with bank conflicts, VALU 0.43 to 0.57 with
// halving and scaling, one to three workgroups a compute unit.  (507 us without the scales.)

#include <algorithm>
#include <type_traits>

#include "newton_device.h"

namespace pmlpk {

namespace {

// Bytes from the start of a row of A or P to its column 16 t + 4 k: each 32 columns lie in
// the order in which the transposing loads bring 32 rows of X, 4 k + (0 .. 3) and
// 16 + 4 k + (0 .. 3) for k = 0 .. 3.
__device__ __forceinline__ int held_column(int t, int k) { return 64 * (t >> 1) + 8 * (t & 1) + 16 * k; }

// Four consecutive values of a row, in both planes
__device__ __forceinline__ void put4(char* at, int plane, const f32x4& v) {
  f16x4 hi, lo;
  halve(v, hi, lo);
  *(f16x4*)at = hi;
  *(f16x4*)(at + plane) = lo;
}
__device__ __forceinline__ f32x4 add4(float f, const char* at, int plane, const f32x4& v) {
  return add_held(f, *(const f16x4*)at, *(const f16x4*)(at + plane), v);
}

// The lower triangle of a symmetric matrix in strips of two tiles: strip q is tiles
// (ti, tj) and (ti, tj + 1), of which the second may lie above the diagonal.
__device__ __forceinline__ void strip_of(int q, int& ti, int& tj) {
  ti = 0;
  while (q >= (ti >> 1) + 1) q -= (ti++ >> 1) + 1;
  tj = 2 * q;
}

// A value of which the compiler knows nothing (or it keeps the entries' places from one walk to
// the next, in memory)
__device__ __forceinline__ int afresh(int v) {
  asm("" : "+v"(v));
  return v;
}

// This thread's entries of a matrix: row i, column j, `at` entries from its first one.
template <int NT>
struct Walk {
  int i, j, di, dj, cols;
  int64_t at, dat, wrap;
  __device__ __forceinline__ Walk(int tid, const NsMat& t) : cols(t.cols) {
    i = tid / cols;
    j = tid - i * cols;
    di = NT / cols;
    dj = NT - di * cols;
    at = (int64_t)i * t.ld + j;
    dat = (int64_t)di * t.ld + dj;
    wrap = t.ld - cols;
  }
  __device__ __forceinline__ void next() {
    i += di;
    j += dj;
    at += dat;
    if (j >= cols) {
      j -= cols;
      ++i;
      at += wrap;
    }
  }
};
constexpr int kAhead = 8;  // entries that a thread loads at a time

// The largest of 16 lanes' values, or of every 16th lane's
__device__ __forceinline__ float row16_max(float v) {
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float column4_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// 2^(times d + add) for four rows' exponents
__device__ __forceinline__ f32x4 pow2_4(int b, int times, int add) {
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = ldexpf(1.f, times * (int)(int8_t)(b >> (8 * e)) + add);
  return v;
}

// EPT: entries a thread; QPT: groups of four columns of X, with its padding
template <int TR, int NW, int UMAX, int EPT, int QPT>
__device__ __forceinline__ void small_matrix(const NsArgs& a, const NsMat& t, int steps, char* lds,
                                             double* total) {
  constexpr int NT = 64 * NW, RP = (TR + 1) / 2 * 32, TRB = RP / 32, NB = ns_strips(TR);
  constexpr int NG = NW == 16 ? (TR + 1) / 2 : TR <= 4 ? 1 : 2, RG = (TR + NG - 1) / NG;  // row tiles of a unit
  constexpr int KS = ns_small_split(TR, NW), PER = (NB + NW - 1) / NW;
  constexpr int RS = TR == 1 ? 1 : 2;  // tiles of a strip
  constexpr int SP = 2 * RP + 16;
  const int C = t.cp, SX = 2 * C + 16, pairs = C / 32;
  const int xplane = 16 * TR * SX, pplane = 16 * TR * SP;
  char *X = lds, *A = lds + 2 * xplane;
  f32x4* part = (f32x4*)(A + 2 * pplane);  // [KS][NB][RS][64]
  int8_t* const rows_at = (int8_t*)(part + (KS > 1 ? KS * NB * RS * 64 : 0));  // exponents of D [2][16 TR],
  int8_t* const cols_at = rows_at + 32 * TR;                               // .. of E [2][C]
  int* const uneven = (int*)(cols_at + 2 * C);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lk = lane >> 4;
  const bool turned = t.rows > t.cols;
  const int n = t.rows * t.cols;

  // ---- momentum, norm, X ------------------------------------------------------------
  if (tid == 0) *uneven = 0;
  for (int e = tid; e < 2 * pplane / 16; e += NT) ((f32x4*)A)[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float* G = a.G + t.src;
  const float* mom_in = a.mom_in ? a.mom_in + t.src : nullptr;
  float* mom_out = a.mom_in ? a.mom_out + t.src : nullptr;
  static_assert(EPT % kAhead == 0, "entries are loaded so many at a time");
  float u[EPT];  // entries tid, tid + NT, .. (of the first one again past the last)
  double sum = 0;
  {
    Walk<NT> w(tid, t);
#pragma unroll
    for (int b = 0; b < EPT; b += kAhead) {
      if (NT * b >= n) continue;
      float m[kAhead];
      int64_t at[kAhead];
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        at[q] = tid + NT * (b + q) < n ? w.at : 0;
        w.next();
        u[b + q] = G[at[q]];
      }
      if (mom_in) {
#pragma unroll
        for (int q = 0; q < kAhead; ++q) m[q] = mom_in[at[q]];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          const float v = fmaf(a.mu, m[q], u[b + q]);
          if (tid + NT * (b + q) < n) mom_out[at[q]] = v;
          u[b + q] = a.nesterov ? fmaf(a.mu, v, u[b + q]) : v;
        }
      }
#pragma unroll
      for (int q = 0; q < kAhead; ++q)
        if (tid + NT * (b + q) < n) sum += (double)u[b + q] * (double)u[b + q];
    }
  }
  sum = wave_total(sum);
  if (lane == 0) total[wave] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < NW; ++w) sum += total[w];
  const double scale = ns_scale(sum);
  const float scale32 = (float)scale;
  const bool plain = scale > 1e-30 && scale < 1e30;  // (a factor of float32 is all they need)
  const int XF = 4 * C + 16;  // bytes of a row of X as fp32, over both planes
  {
    Walk<NT> w(afresh(tid), t);
#pragma unroll
    for (int b = 0; b < EPT; ++b) {
      if (tid + NT * b < n) {
        u[b] = plain ? scale32 * u[b] : (float)(scale * (double)u[b]);
        *(float*)(X + (turned ? w.j * XF + 4 * w.i : w.i * XF + 4 * w.j)) = u[b];
      }
      w.next();
    }
  }
  __syncthreads();
  // the scales: rows by 16 lanes, columns by 16 of a wave
  for (int i = tid >> 4; i < 16 * TR; i += NT / 16) {
    float m = 0.f;
    if (i < t.r)
      for (int j = 4 * li; j < t.c; j += 64) {
        const f32x4 v = *(const f32x4*)(X + i * XF + 4 * j);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < t.c) m = fmaxf(m, fabsf(v[k]));
      }
    m = row16_max(m);
    if (li == 0) rows_at[i] = (int8_t)row_exponent(t, m);
  }
  __syncthreads();
  // (Eight rows show of most matrices that no column is small.)
  auto scale_columns = [&](auto count) __attribute__((always_inline)) {
    for (int g = wave; g < C / 16; g += NW) {
      const int j = 16 * g + li;
      float m = 0.f;
#pragma unroll
      for (int q = 0; q < decltype(count)::value; ++q) {
        const int i = 4 * q + lk;
        const float v = ldexpf(fabsf(*(const float*)(X + i * XF + 4 * j)), -(int)rows_at[i]);
        m = fmaxf(m, i < t.r && j < t.c ? v : 0.f);
      }
      m = column4_max(m);
      const int e = j < t.c ? column_exponent(t, m, decltype(count)::value < 4 * TR ? -1 : 0) : 0;
      if (lane < 16) cols_at[j] = (int8_t)e;
      if (e) *uneven = 1;
    }
    __syncthreads();
  };
  scale_columns(std::integral_constant<int, 2>());
  bool even = *uneven == 0;
  if (!even) {
    __syncthreads();
    if (tid == 0) *uneven = 0;
    __syncthreads();
    scale_columns(std::integral_constant<int, 4 * TR>());
    even = *uneven == 0;
  }
  {
    f32x4 v[QPT];
    const int i0 = 4 * tid / C, j0 = 4 * tid - i0 * C, di = 4 * NT / C, dj = 4 * NT - di * C;
    int i = i0, j = j0;
    auto next = [&] {
      i += di;
      j += dj;
      if (j >= C) {
        j -= C;
        ++i;
      }
    };
#pragma unroll
    for (int b = 0; b < QPT; ++b, next()) {
      v[b] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i >= t.r || j >= t.c) continue;
      v[b] = *(const f32x4*)(X + i * XF + 4 * j);
      const int d = kXBits - (int)rows_at[i], at = even ? 0 : *(const int*)(cols_at + j);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[b][k] = j + k < t.c ? ldexpf(v[b][k], d - (int)(int8_t)(at >> (8 * k))) : 0.f;
    }
    __syncthreads();
    i = i0;
    j = j0;
#pragma unroll
    for (int b = 0; b < QPT; ++b, next())
      if (i < 16 * TR) put4(X + i * SX + 2 * j, xplane, v[b]);
  }
  __syncthreads();

  // (Both ways compiled on their own: the scales of columns take registers.)
  auto iterate = [&](auto all_even) __attribute__((always_inline)) {
    constexpr bool even = decltype(all_even)::value;
    f32x4 held[PER][RS];  // this wave's strips of A'
    for (int step = 0; step < steps; ++step) {
      // (Places in LDS anew in each step: kept from the first one they would go to memory.)
      const int lane = afresh(tid & 63), li = lane & 15, lk = lane >> 4;
      // A tile of a symmetric matrix, rows 16 ti + 4 lk + e of column 16 tj + li, and mirrored: each
      // value times the scale of the column of B or P' that it goes to
      auto put_symmetric = [&](int ti, int tj, const f32x4& v, const f32x4& by_row, float by_column) __attribute__((always_inline)) {
        f16x4 hi, lo;
        halve(v * by_row, hi, lo);
        char* to = A + (16 * tj + li) * SP + held_column(ti, lk);
        *(f16x4*)to = hi;
        *(f16x4*)(to + pplane) = lo;
        if (ti == tj) return;
        halve(v * by_column, hi, lo);
        char* at = A + (16 * ti + 4 * lk) * SP + held_column(tj, li >> 2) + 2 * (li & 3);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          *(_Float16*)(at + e * SP) = hi[e];
          *(_Float16*)(at + e * SP + pplane) = lo[e];
        }
      };
      // Tiles (ti, tj) and (ti, tj + 1) of S S^T over the 32-column steps k0 <= k < k1, with columns
      // times 4^e where `scaled`.
      auto strip_product = [&](const char* S, int stride, int plane, int ti, int tj, int k0, int k1,
                               auto scaled, const int8_t* e, f32x4 (&acc)[RS]) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < RS; ++q) acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
        const char* x0 = S + (16 * ti + li) * stride + 16 * lk;
        const char* y0 = S + (16 * tj + li) * stride + 16 * lk;
        const int second = tj < ti ? 16 * stride : 0;
        f16x8 x[2][2], y[2][RS][2];  // [stage]
        auto fetch = [&](int b, int k) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            x[b][h] = *(const f16x8*)(x0 + h * plane + 64 * k);
            y[b][0][h] = *(const f16x8*)(y0 + h * plane + 64 * k);
            if (RS > 1) y[b][RS - 1][h] = *(const f16x8*)(y0 + second + h * plane + 64 * k);
          }
          if constexpr (decltype(scaled)::value) {
            const f16x8 by = pow2_8(*(const uint2*)(e + 32 * k + 8 * lk));
#pragma unroll
            for (int h = 0; h < 2; ++h) x[b][h] = scaled_twice(x[b][h], by);
          }
        };
        auto multiply = [&](int b) {
#pragma unroll
          for (int h = 0; h < 3; ++h)  // (small products first, the tiles in turn)
#pragma unroll
            for (int q = 0; q < RS; ++q)
              acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[b][h == 0], y[b][q][h == 1], acc[q], 0, 0, 0);
        };
        // (past the last step that again: a branch around the loads would wait for all)
        if (k0 < k1) fetch(0, k0);
        for (int k = k0; k < k1; k += 2) {
          fetch(1, k + 1 < k1 ? k + 1 : k1 - 1);
          multiply(0);
          if (k + 1 >= k1) break;
          fetch(0, k + 2 < k1 ? k + 2 : k1 - 1);
          multiply(1);
        }
      };
      const int8_t* const rows = rows_at + (step & 1) * 16 * TR;
      const int8_t* const cols = cols_at + (step & 1) * C;
      int8_t* const next_rows = rows_at + (~step & 1) * 16 * TR;
      int8_t* const next_cols = cols_at + (~step & 1) * C;
      // exponents of the rows of a strip's tiles that a lane has, and of its columns
      int of_rows[PER], of_column[PER][RS];
      // ---- A' -------------------------------------------------------------------------
      if (!even)
        for (int q = wave; q < C / 16; q += NW) {
          const int j = 16 * q + li;
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < 4 * TR; ++i)
            m = fmaxf(m, fabsf((float)*(const _Float16*)(X + (4 * i + lk) * SX + 2 * j)));
          m = ldexpf(column4_max(m), (int)cols[j] - kXBits);
          if (lane < 16) next_cols[j] = (int8_t)column_exponent(t, m, cols[j]);
        }
      auto gram = [&](int b, int k0, int k1, f32x4 (&acc)[RS]) __attribute__((always_inline)) {
        int ti, tj;
        strip_of(b, ti, tj);
        if (even) strip_product(X, SX, xplane, ti, tj, k0, k1, std::false_type(), cols, acc);
        else strip_product(X, SX, xplane, ti, tj, k0, k1, std::true_type(), cols, acc);
      };
      if (KS > 1) {
        for (int q = wave; q < NB * KS; q += NW) {
          const int b = q % NB, ks = q / NB;
          f32x4 acc[RS];
          gram(b, ks * pairs / KS, (ks + 1) * pairs / KS, acc);
#pragma unroll
          for (int r = 0; r < RS; ++r) part[((ks * NB + b) * RS + r) * 64 + lane] = acc[r];
        }
        __syncthreads();
      }
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        const int b = wave + u * NW;
        if (b >= NB) continue;
        int ti, tj;
        strip_of(b, ti, tj);
        of_rows[u] = *(const int*)(rows + 16 * ti + 4 * lk);
#pragma unroll
        for (int r = 0; r < RS; ++r) of_column[u][r] = rows[16 * (tj + r < ti ? tj + r : ti) + li];
        if (KS == 1) gram(b, 0, pairs, held[u]);
#pragma unroll
        for (int r = 0; r < RS; ++r) {
          if (tj + r > ti) continue;
          if (KS > 1) {
            held[u][r] = part[(RS * b + r) * 64 + lane];
#pragma unroll
            for (int k = 1; k < KS; ++k) held[u][r] += part[((k * NB + b) * RS + r) * 64 + lane];
          }
          held[u][r] *= kPow2Less<2 * kXBits>;
          put_symmetric(ti, tj + r, held[u][r], pow2_4(of_rows[u], 1, kBBits),
                        ldexpf(1.f, of_column[u][r] + kBBits));
        }
      }
      __syncthreads();
      // ---- P', over B -------------------------------------------------------------------
      f32x4 poly[PER][RS];
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        if (wave + u * NW >= NB) continue;
        int ti, tj;
        strip_of(wave + u * NW, ti, tj);
#pragma unroll
        for (int r = 0; r < RS; ++r)
          if (tj + r == ti && lk == li >> 2) {
            const f32x4& v = held[u][r];
            const int q = li & 3;
            const float square = q == 0 ? v[0] : q == 1 ? v[1] : q == 2 ? v[2] : v[3];
            next_rows[16 * ti + li] = (int8_t)next_row_exponent(of_column[u][r], square);
          }
        strip_product(A, SP, pplane, ti, tj, 0, TRB, std::false_type(), nullptr, poly[u]);
#pragma unroll
        for (int r = 0; r < RS; ++r)
          if (tj + r <= ti) poly[u][r] = kNsB * held[u][r] + (kNsC * kPow2Less<2 * kBBits>) * poly[u][r];
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        if (wave + u * NW >= NB) continue;
        int ti, tj;
        strip_of(wave + u * NW, ti, tj);
#pragma unroll
        for (int r = 0; r < RS; ++r)
          if (tj + r <= ti)
            put_symmetric(ti, tj + r, poly[u][r], pow2_4(of_rows[u], 2, kPBits),
                          ldexpf(1.f, 2 * of_column[u][r] + kPBits));
      }
      __syncthreads();
      // ---- X' --------------------------------------------------------------------------
      f32x4 next[UMAX][2][RG];
#pragma unroll
      for (int u = 0; u < UMAX; ++u) {
        const int unit = wave + u * NW;
        if (unit >= pairs * NG) continue;
        const int pair = unit % pairs, r0 = unit / pairs * RG;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int r = 0; r < RG; ++r) next[u][p][r] = f32x4{0.f, 0.f, 0.f, 0.f};
        int by_row[RG];
#pragma unroll
        for (int r = 0; r < RG; ++r) {
          const int row = 16 * (NG * RG > TR && r0 + r >= TR ? TR - 1 : r0 + r) + li;
          by_row[r] = (int)rows[row] - (int)next_rows[row];
        }
        const char* x0 = X + (4 * lk + (li >> 2)) * SX + 64 * pair + 8 * (li & 3);
        const char* p0 = A + (16 * r0 + li) * SP + 16 * lk;
#pragma unroll
        for (int k = 0; k < TRB; ++k) {
          f16x8 x[2][2];
#pragma unroll
          for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              // (16 rows are left of an odd number of tiles: their second reading meets the zeros
              // in P's last 16 columns)
              x[p][h] = columns(x0 + h * xplane + 32 * k * SX + 32 * p, 2 * k + 1 < TR ? 16 * SX : 0);
          f16x8 y[RG][2];
#pragma unroll
          for (int r = 0; r < RG; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              // (a tile past the last one reads the last one again, and is not stored)
              const int tile = NG * RG > TR && r0 + r >= TR ? r - 1 : r;
              y[r][h] = *(const f16x8*)(p0 + h * pplane + 16 * tile * SP + 64 * k);
            }
#pragma unroll
          for (int h = 0; h < 3; ++h)
#pragma unroll
            for (int r = 0; r < RG; ++r)
#pragma unroll
              for (int p = 0; p < 2; ++p)
                next[u][p][r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[p][h == 0], y[r][h == 1], next[u][p][r], 0, 0, 0);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int r = 0; r < RG; ++r) {
            if (NG * RG > TR && r0 + r >= TR) continue;
            next[u][p][r] = add4(kNsA, X + (16 * (r0 + r) + li) * SX + 2 * (32 * pair + 16 * p + 4 * lk),
                                 xplane, kPow2Less<kPBits> * next[u][p][r]);
          }
#pragma unroll
        for (int r = 0; r < RG; ++r) {
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            next[u][p][r] *= ldexpf(1.f, by_row[r]);
            if (even) continue;
            const int col = 32 * pair + 16 * p + 4 * lk;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              next[u][p][r][e] = ldexpf(next[u][p][r][e], (int)cols[col + e] - (int)next_cols[col + e]);
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < UMAX; ++u) {
        const int unit = wave + u * NW;
        if (unit >= pairs * NG) continue;
        const int pair = unit % pairs, r0 = unit / pairs * RG;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int r = 0; r < RG; ++r) {
            if (NG * RG > TR && r0 + r >= TR) continue;
            const int row = 16 * (r0 + r) + li, col = 32 * pair + 16 * p + 4 * lk;
            if (step + 1 < steps) put4(X + row * SX + 2 * col, xplane, next[u][p][r]);
            else *(f32x4*)(X + row * XF + 4 * col) = next[u][p][r];
          }
      }
      __syncthreads();
    }

    // ---- the result ---------------------------------------------------------------------
    const float gain = ns_gain(t);
    const int8_t* const rows = rows_at + (steps & 1) * 16 * TR;
    const int8_t* const cols = cols_at + (steps & 1) * C;
    Walk<NT> w(tid, t);
#pragma unroll 4
    for (int e = tid; e < n; e += NT) {
      const int i = turned ? w.j : w.i, j = turned ? w.i : w.j;
      const float x = ldexpf(*(const float*)(X + i * XF + 4 * j), (int)rows[i] + (even ? 0 : (int)cols[j]) - kXBits);
      if (a.W) apply(a, t, w.i, w.j, gain * x);
      else a.out[t.src + w.at] = x;
      w.next();
    }
    if (a.W && a.lrm && tid == 0 && !(fabsf(a.lrm[t.m]) < INFINITY)) a.flag[1] = 1;
  };
  if (even) iterate(std::true_type());
  else iterate(std::false_type());
}

}  // namespace

// TR tiles of rows, up to 128 columns.  (OCC: waves of a SIMD that LDS leaves room for.)
template <int TR, int OCC>
__global__ __launch_bounds__(64 * kNsWaves[TR - 1], OCC) void k_ns_small(NsArgs a, const int32_t* list,
                                                                        int steps) {
  constexpr int NW = kNsWaves[TR - 1];
  extern __shared__ __align__(16) char lds[];
  __shared__ double total[NW];
  const NsMat t = a.mats[list[blockIdx.x]];
  constexpr int all = 16 * TR * 128 / (64 * NW);  // entries a thread
  small_matrix<TR, NW, 1, (all + kAhead - 1) / kAhead * kAhead, (all + 3) / 4>(a, t, steps, lds, total);
}

// Few rows and many columns, at four waves a SIMD (k_ns_small_any takes the registers of two, and
// one workgroup a compute unit: 600 matrices of 10 x 1 to 100 in one launch 48 us, 17 so).
__global__ __launch_bounds__(64 * kNsWaves[kNsLow], 4) void k_ns_low(NsArgs a, const int32_t* list, int steps) {
  constexpr int NW = kNsWaves[kNsLow];
  extern __shared__ __align__(16) char lds[];
  __shared__ double total[NW];
  const NsMat t = a.mats[list[blockIdx.x]];
  if (t.r <= 16) small_matrix<1, NW, 512 / 32 / NW, 16 * 512 / (64 * NW), 8>(a, t, steps, lds, total);
  else small_matrix<2, NW, 256 / 32 / NW, 32 * 256 / (64 * NW), 8>(a, t, steps, lds, total);
}

// Any of them, and wider ones.  (X in LDS has at most 40,960 entries: 20 groups of four a thread.)
__global__ __launch_bounds__(512, 2) void k_ns_small_any(NsArgs a, const int32_t* list, int steps) {
  extern __shared__ __align__(16) char lds[];
  __shared__ double total[8];
  const NsMat t = a.mats[list[blockIdx.x]];
  switch ((t.r + 15) / 16) {
#define PMLP_NS(TR)                                                                        \
  case TR:                                                                                 \
    small_matrix<TR, 8, kNsUnits[(TR - 1) / 2], kNsEntries[(TR - 1) / 2], 20>(a, t, steps, lds, total); \
    break;
    PMLP_NS(1) PMLP_NS(2) PMLP_NS(3) PMLP_NS(4) PMLP_NS(5) PMLP_NS(6) PMLP_NS(7) PMLP_NS(8)
#undef PMLP_NS
    default: break;
  }
}

hipError_t launch_ns_small(const NsArgs& a, int cls, size_t lds, const int32_t* list, int32_t n,
                           int32_t steps, hipStream_t s) {
  auto go = [&](auto fn) {
    note_variant(cls < kNsLow ? "k_ns_small" : cls == kNsLow ? "k_ns_low" : "k_ns_small_any", kArithF16x2);
    if (const hipError_t e = hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)kNsSmallLds))
      return e;
    for (int32_t at = 0; at < n; at += kNsGrid) {
      fn<<<(unsigned)std::min(kNsGrid, n - at), 64 * kNsWaves[cls], lds, s>>>(a, list + at, steps);
      if (const hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
  };
  switch (cls) {
    case 0: return go(k_ns_small<1, 6>);
    case 1: return go(k_ns_small<2, 4>);
    case 2: return go(k_ns_small<3, 4>);
    case 3: return go(k_ns_small<4, 3>);
    case 4: return go(k_ns_small<5, 4>);
    case 5: return go(k_ns_small<6, 4>);
    case 6: return go(k_ns_small<7, 4>);
    case 7: return go(k_ns_small<8, 4>);
    case kNsLow: return go(k_ns_low);
    default: return go(k_ns_small_any);
  }
}

}  // namespace pmlpk
