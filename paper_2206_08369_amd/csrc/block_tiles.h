// Block packs: the tiles of the fused kernels, forward and backward.
#pragma once

#include "block_device.h"

#include <algorithm>

namespace pmlpk {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// a summed over lanes l and l ^ 32 in the lower half of the wave, b in the upper
__device__ __forceinline__ float sum32(float a, float b) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false,
                                                   false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// a summed over lanes l and l ^ 16 in the even rows of 16, b in the odd
__device__ __forceinline__ float sum16(float a, float b) {
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false,
                                                   false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// a of the lower half of the wave in both, of the upper half in both
__device__ __forceinline__ void halves(float a, float& lower, float& upper) {
  const uint32_t u = __float_as_uint(a);
  const u32x2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  lower = __uint_as_float(r[0]);
  upper = __uint_as_float(r[1]);
}

// a, the same in every lane, in a scalar register
__device__ __forceinline__ float uniform(float a) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(a)));
}

// The forward of runs of `run` tiles r, r + step, .. (below tile `end`) by one wave:
// their sums over the `steps` blocks of 32 samples from b0 on whose pieces lie in LDS
// (SC of them).  RUNS: the sums of a run's tiles are added up in `acc`, planes of
// acc_row(SC) samples, each value by one lane; else a run is one tile.
__host__ __device__ constexpr int acc_row(int SC) { return SC + 4; }

template <int NC, int RM, bool MF, bool GATED, bool NORM, bool RUNS>
__device__ __forceinline__ void fwd_tiles(const BlkPack& p, const BlkFwdArgs& a, const char* lds,
                                          int SC, int b0, int steps, int r, int end, int step,
                                          int run, float* acc) {
  constexpr int K = GATED ? 2 : 1, RB = row_bytes(NC);
  const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4, plane = SC * RB;
  const char* const zrow = lds + li * RB + 16 * lk;
  const char* const xrow = lds + li * RB + 64 * NC + 2 * lk;
  const int PQ = p.O + (NORM ? 2 : 0), om = blk_om(p.O);
  // Where a tile's rows leave registers free the next tile's are loaded while this one
  // is at work (a tile of few steps is as long as its wait for them).
  constexpr bool AHEAD = NC <= 1;
  struct Next {  // a tile's rows, and gain and W2 of the outputs (MF: of output li)
    UnitRaw<NC, RM, K> w;
    float w2[MF ? 1 : 2][4], g[4];
  } nx;
  auto fetch = [&](int n0, int cnt) {
    nx.w.load(p, n0 + std::min(li, cnt - 1), lk);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t n = n0 + std::min(4 * lk + r, cnt - 1);
      nx.g[r] = NORM ? p.gain[n] : 1.f;
#pragma unroll
      for (int o = 0; o < (MF ? 1 : 2); ++o) {
        const int ow = MF ? li : o;
        nx.w2[o][r] = p.W2[(int64_t)(ow < p.O ? ow : 0) * p.ldw + n];
      }
    }
  };
  auto tile_at = [&](int t) { return a.tiles[std::min(t, end - 1)]; };
  auto after = [&](int t, int& of) {  // the tile that follows t of run `of`
    if (RUNS && t + 1 < std::min((of + 1) * run, end)) return t + 1;
    of += step;
    return of * run;
  };
  int rn = r, tn = after(r * run, rn), have = 0;  // the next tile; units of the run before this
  f32x4 cr = f32x4{0.f, 0.f, 0.f, 0.f};           // and their C_o
  BlkTile q = tile_at(r * run), qn = tile_at(tn);
  if (AHEAD) fetch(q.n0, q.cnt);
#pragma unroll 1
  for (int t = r * run; t < end;) {
    const int n0 = __builtin_amdgcn_readfirstlane(q.n0);
    const int cnt = __builtin_amdgcn_readfirstlane(q.cnt), act = __builtin_amdgcn_readfirstlane(q.act);
    int rnn = rn;
    const int tnn = after(tn, rnn);
    const BlkTile qnn = tile_at(tnn);
    const int m = __builtin_amdgcn_readfirstlane(q.m);
    const bool last = !RUNS || rn != r || __builtin_amdgcn_readfirstlane(qn.m) != m;
    if (!AHEAD) fetch(n0, cnt);
    UnitRows<NC, RM, K> w;
    w.split(nx.w, p.F4, lk);
    f32x4 w2[MF ? 1 : 2];  // gain * W2 of this lane's units
    const int mine = cnt - 4 * lk;  // units of this lane: min(4, mine), if positive
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int o = 0; o < (MF ? 1 : 2); ++o) {
        const float v = opaque(nx.w2[o][r]) * opaque(nx.g[r]);
        w2[o][r] = (MF ? li : o) < p.O && r < mine ? v : 0.f;
      }
    // C_o of the tile, as the lane's sums below have their outputs
    f32x4 ct = f32x4{0.f, 0.f, 0.f, 0.f};
    if (NORM && MF) {
      const f32x4 u = w2[0];
      ct = __builtin_amdgcn_mfma_f32_16x16x4f32((u[0] + u[1]) + (u[2] + u[3]), 1.f, ct, 0, 0, 0);
    } else if (NORM) {
      const f32x4 u = w2[0], v = w2[MF ? 0 : 1];
      const float c = (u[0] + u[1]) + (u[2] + u[3]), d = (v[0] + v[1]) + (v[2] + v[3]);
      ct[0] = sum16(sum32(c, c), sum32(d, d));
    }
    if (AHEAD) fetch(qn.n0, qn.cnt);
    float* const rec = a.part + (int64_t)(m + r) * PQ * a.Br + b0;  // (at 32-bit offsets)
    const float rc = uniform(1.f / (float)cnt);
    // merging with the `have` units before (see merge_stats)
    const float share = uniform((float)cnt / (float)(have + cnt)), both = uniform(share * (float)have);
#pragma unroll 1
    for (int st = 0; st < steps; ++st) {
      const int at = 32 * st * RB;
      f32x4 z[K][2];
      unit_products<NC, RM, K, true>(w, zrow + at, xrow + at, plane, z);
      float zv[8], h[8];
#pragma unroll
      for (int v = 0; v < 8; ++v) zv[v] = z[0][v >> 2][v & 3];
      blk_acts<8>(act, zv, h);
      if (GATED) {
#pragma unroll
        for (int v = 0; v < 8; ++v) h[v] *= z[K - 1][v >> 2][v & 3];
      }
      if (cnt < 16) {
#pragma unroll
        for (int v = 0; v < 8; ++v) h[v] = (v & 3) < mine ? h[v] : 0.f;
      }
      const int row = acc_row(SC), at0 = 32 * st + li;
      // Means of the blocks that this lane's sums are of (both, or its half's, lk >> 1):
      // the tile's, and the run's before it and after it.
      constexpr int NB = MF ? 2 : 1;
      float mean[2], m2, me[NB], ma[NB], mb[NB];
      auto own = [&](float a, float b) { return lk >> 1 ? b : a; };
      if (NORM) {
        float piv[2], d[2] = {0.f, 0.f}, e[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          piv[i] = __shfl(h[4 * i], li);  // the first unit's value
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float& v = h[4 * i + r];
            v = (cnt == 16 || r < mine) ? v - piv[i] : 0.f;
            d[i] += v;
          }
        }
        m2 = sum32(d[0], d[1]);
        halves(sum16(m2, m2), d[0], d[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mean[i] = fmaf(d[i], rc, piv[i]);
          const float off = piv[i] - mean[i];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float& v = h[4 * i + r];
            v = (cnt == 16 || r < mine) ? v + off : 0.f;
            e[i] = fmaf(v, v, e[i]);
          }
        }
        m2 = sum32(e[0], e[1]);
        m2 = sum16(m2, m2);
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          ma[j] = mb[j] = me[j] = MF ? mean[j] : own(mean[0], mean[1]);
          if (RUNS && have) {
            ma[j] = acc[p.O * row + at0 + 16 * (MF ? j : lk >> 1)];
            mb[j] = fmaf(me[j] - ma[j], share, ma[j]);
          }
        }
      }
      if (MF) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(w2[0][r], h[4 * i + r], s, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * lk + r < p.O) {
              const int o = 4 * lk + r;
              float v = s[r];
              if (RUNS && have) v += acc[o * row + at0 + 16 * i];
              if (RUNS && NORM && have) {
                const int j = MF ? i : 0;
                v = fmaf(me[j] - mb[j], ct[r], v);
                v = fmaf(ma[j] - mb[j], cr[r], v);
              }
              if (last) rec[(uint32_t)(o * a.Br + at0 + 16 * i)] = v;
              else acc[o * row + at0 + 16 * i] = v;
            }
        }
      } else {
        float s[2][2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int o = 0; o < 2; ++o) {
            s[i][o] = h[4 * i] * w2[MF ? 0 : o][0];
#pragma unroll
            for (int r = 1; r < 4; ++r) s[i][o] = fmaf(h[4 * i + r], w2[MF ? 0 : o][r], s[i][o]);
          }
        // row lk ends with block lk >> 1 of output lk & 1
        float v = sum16(sum32(s[0][0], s[1][0]), sum32(s[0][1], s[1][1]));
        const int at = (lk & 1) * row + at0 + 16 * (lk >> 1);
        if (RUNS && have) v += acc[at];
        if (RUNS && NORM && have) {
          v = fmaf(me[0] - mb[0], ct[0], v);
          v = fmaf(ma[0] - mb[0], cr[0], v);
        }
        if (last) rec[(uint32_t)((lk & 1) * a.Br + at0 + 16 * (lk >> 1))] = v;
        else acc[at] = v;
      }
      if (NORM) {
        float* const sum = acc + p.O * row + at0 + 16 * (lk >> 1);
        if (RUNS && have) {
          const float d = own(me[0] - ma[0], me[NB - 1] - ma[NB - 1]);
          m2 += sum[row] + d * both * d;
        }
        const float v = lk & 1 ? m2 : own(mb[0], mb[NB - 1]);
        if (last) rec[(uint32_t)((p.O + (lk & 1)) * a.Br + at0 + 16 * (lk >> 1))] = v;
        else sum[(lk & 1) * row] = v;
      }
    }
    if (NORM) {
      if (RUNS && have) ct += cr;
      if (RUNS) cr = ct;
      if (last && b0 == 0 && li == 0) {
        float* const c = a.csum + (int64_t)(m + r) * om;
        if (MF && 4 * lk < om) *(f32x4*)(c + 4 * lk) = ct;
        if (!MF && lk < 2) c[lk] = ct[0];
      }
    }
    have = last ? 0 : have + cnt;
    t = tn;
    r = rn;
    tn = tnn;
    rn = rnn;
    q = qn;
    qn = qnn;
  }
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_u __attribute__((ext_vector_type(4), aligned(4)));  // rows of any F
typedef __attribute__((address_space(3))) char lds_char;

// The backward of tiles first, first + stride, .. below `end` by one wave (as many
// rounds for each wave of the workgroup); nchunk > 1: over chunks of SC samples, whose
// pieces the workgroup makes in turn (else they lie in LDS).
template <int NC, int RM, int OM, bool GATED, bool NORM>
__device__ __forceinline__ void bwd_tiles(const BlkPack& p, const BlkBwdArgs& a, char* lds, int SC,
                                          int nchunk, int rounds, int first, int end, int stride) {
  constexpr int NF = 2 * NC + (RM ? 1 : 0), K = GATED ? 2 : 1, RB = row_bytes(NC);
  constexpr bool MF = OM > 4;  // the output layer's products by matrix instructions
  constexpr int NO = MF ? 4 : OM;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int F = a.F, F4 = p.F4, plane = SC * RB;
  // this lane's places in the pieces: a row of the first product, and of the second
  const int zrow = li * RB + 16 * lk, xrow = li * RB + 64 * NC + 2 * lk;
  const int trow = (4 * lk + (li >> 2)) * RB + 8 * (li & 3);

  // Up to four outputs: each lane its unit's weights and sums T_o.  More go through
  // fp32 matrix products, a model at a time: w2[0..3] are then outputs 4 lk + q of
  // unit li, and T[0..3] their sums.
  //
  // Loads run ahead of their use and of the stores of the tile before (they return in
  // order): a block's output gradients and statistics by a block, over the ends of
  // tiles, and where a tile's rows leave registers free those by a tile.
  constexpr bool AHEAD = NC <= 1;
  struct Next {
    UnitRaw<NC, RM, K> w;
    float w2[NO], g, s;
  } nx;
  auto fetch = [&](int64_t n) {
    nx.w.load(p, n, lk);
    nx.g = NORM ? p.gain[n] : 1.f;
    nx.s = NORM ? p.shift[n] : 0.f;
#pragma unroll
    for (int o = 0; o < NO; ++o) {
      const int ow = MF ? 4 * lk + o : o, oc = ow < p.O ? ow : 0;
      nx.w2[o] = p.W2[(int64_t)oc * p.ldw + n];
    }
  };
  UnitRows<NC, RM, K> w;
  float w2[NO], gn = 1.f, sn = 0.f;
  auto take = [&] {
    w.split(nx.w, F4, lk);
    gn = opaque(nx.g);
    sn = opaque(nx.s);
#pragma unroll
    for (int o = 0; o < NO; ++o) {
      const float v = opaque(nx.w2[o]);
      w2[o] = (MF ? 4 * lk + o : o) < p.O ? v : 0.f;
    }
  };
  struct Up {
    f32x4 g[MF ? 2 : OM], r[NORM ? 4 : 1];
  };
  // block b (its first sample) of the lanes' models m
  auto load_up = [&](int m, int b) {
    Up u;
    const int ml = __builtin_amdgcn_readfirstlane(m);
    const uint32_t at = (uint32_t)(b + 4 * lk);  // first of four samples
    if (MF) {
      const float* const g = a.G + (int64_t)ml * a.Bp * OM;
      u.g[0] = *(const f32x4*)(g + (uint32_t)(b + li) * OM + 4 * lk);
#pragma unroll
      for (int r = 0; r < 4; ++r) u.g[MF ? 1 : 0][r] = g[(at + r) * OM + li];
    } else {
      const float* const g = a.G + ((int64_t)m * a.Bp + at) * OM;
#pragma unroll
      for (int v = 0; v < NO; ++v) u.g[MF ? 0 : v] = *(const f32x4*)(g + 4 * v);
    }
    if (NORM) {
      // (with many outputs at a 32-bit offset: two registers fewer keep the loads ahead
      // from waiting for a spilled one; with few it was slower)
      const float* const R = MF ? a.R + (int64_t)ml * a.Bp * 4 +
                                      ((uint32_t)(m - ml) * (uint32_t)a.Bp + at) * 4u
                                : a.R + ((int64_t)m * a.Bp + at) * 4;
#pragma unroll
      for (int r = 0; r < 4; ++r) u.r[NORM ? r : 0] = *(const f32x4*)(R + 4 * r);
    }
    return u;
  };
  auto pin = [&](Up& u) {  // (the loads stay where they are)
#pragma unroll
    for (int v = 0; v < (MF ? 2 : OM); ++v) u.g[v] = opaque(u.g[v]);
#pragma unroll
    for (int r = 0; r < (NORM ? 4 : 0); ++r) u.r[NORM ? r : 0] = opaque(u.r[NORM ? r : 0]);
  };
  auto tile_at = [&](int t) { return a.tiles[std::min(t, end - 1)]; };
  auto unit_of = [&](const BlkTile& q) { return (int64_t)q.n0 + std::min(li, q.cnt - 1); };
  int tile = first;
  BlkTile q = tile_at(tile), qn = tile_at(tile + stride);
  int m = p.mid[unit_of(q)];
  Up up = load_up(m, 0);
  if (AHEAD) {
    fetch(unit_of(q));
    take();
  }
#pragma unroll 1
  for (int round = 0; round < rounds; ++round, tile += stride) {
    const bool live = tile < end;
    const int n0 = __builtin_amdgcn_readfirstlane(q.n0);
    const int cnt = __builtin_amdgcn_readfirstlane(q.cnt), act = __builtin_amdgcn_readfirstlane(q.act);
    const int64_t n = n0 + std::min(li, cnt - 1);
    const int m_lo = __builtin_amdgcn_readfirstlane(m), m_hi = __builtin_amdgcn_readlane(m, 15);
    const BlkTile qnn = tile_at(tile + 2 * stride);
    const int mn = p.mid[unit_of(qn)];
    if (AHEAD) {
      fetch(unit_of(qn));
    } else {
      fetch(n);
      take();
    }
    float T[NO];
#pragma unroll
    for (int o = 0; o < NO; ++o) T[o] = 0.f;
    f32x4 acc[K][NF];
#pragma unroll
    for (int mt = 0; mt < K; ++mt)
#pragma unroll
      for (int j = 0; j < NF; ++j) acc[mt][j] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll 1
    for (int b0 = 0; b0 < a.Bp; b0 += SC) {
      if (nchunk > 1) {
        lds_barrier();
        fill_pieces<NC>(lds, SC, a.X, b0, a.B, F, tid, blockDim.x);
        lds_barrier();
      }
      if (!live) continue;
      const int steps = (a.Bp - b0 < SC ? a.Bp - b0 : SC) >> 5;
#pragma unroll 1
      for (int st = 0; st < steps; ++st) {
        const int s = 32 * st;
        // ---- Z (and U) of 32 samples ------------------------------------------
        f32x4 z[K][2];
        unit_products<NC, RM, K, false>(w, lds + s * RB + zrow, lds + s * RB + xrow, plane, z);
        pin(up);
        // ---- dZ (and dU) ------------------------------------------------------
        f32x4 dz[K][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool last = i == 1 && b0 + s + 32 >= a.Bp;
          Up next = load_up(last ? mn : m, last ? 0 : b0 + s + 16 * (i + 1));
          float zv[4], av[4], dv[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) zv[r] = z[0][i][r];
          act_and_slope<4>(act, zv, av, dv);
          f32x4 h, dn = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            h[r] = GATED ? av[r] * z[K - 1][i][r] : av[r];
            if (NORM) h[r] = (h[r] - up.r[NORM ? r : 0][0]) * up.r[NORM ? r : 0][1];
          }
          if (MF) {
            // dN = G W2 and T += G^T h, the sums in the order of the registers.  Both
            // products run for each model of the tile over all its units, and a unit takes
            // its own model's: multiplying the others by zero instead would let a model
            // whose G is not finite into their sums.
            f32x4 ga = up.g[0], gt = up.g[MF ? 1 : 0];
#pragma unroll 1
            for (int mm = m_lo;;) {
              f32x4 d = f32x4{0.f, 0.f, 0.f, 0.f}, t = d;
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                d = __builtin_amdgcn_mfma_f32_16x16x4f32(ga[r], w2[r % NO], d, 0, 0, 0);
                t = __builtin_amdgcn_mfma_f32_16x16x4f32(gt[r], h[r], t, 0, 0, 0);
              }
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                dn[r] = m == mm ? d[r] : dn[r];
                T[r % NO] += m == mm ? t[r] : 0.f;
              }
              if (++mm > m_hi) break;
              const uint32_t b = (uint32_t)(b0 + s + 16 * i + 4 * lk);
              const float* const g = a.G + (int64_t)mm * a.Bp * OM;
              ga = *(const f32x4*)(g + (uint32_t)(b0 + s + 16 * i + li) * OM + 4 * lk);
#pragma unroll
              for (int r = 0; r < 4; ++r) gt[r] = g[(b + r) * OM + li];
            }
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int o = 0; o < NO; ++o) {
                const float G = up.g[MF ? 0 : (r * OM + o) >> 2][(r * OM + o) & 3];
                dn[r] = fmaf(G, w2[o], dn[r]);
                T[o] = fmaf(G, h[r], T[o]);
              }
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (NORM) {
              const f32x4 q = up.r[NORM ? r : 0];
              dn[r] = q[1] * (fmaf(gn, dn[r], -q[2]) - h[r] * q[3]);
            }
            dz[0][i][r] = GATED ? dn[r] * z[K - 1][i][r] * dv[r] : dn[r] * dv[r];
            if (GATED) dz[K - 1][i][r] = dn[r] * av[r];
          }
          if (i == 0) pin(next);
          up = next;
        }
        // ---- dW1 (and dV1) += dZ^T X ------------------------------------------
        bf16x8 dp[K][3];
#pragma unroll
        for (int mt = 0; mt < K; ++mt)
          split3(dz[mt][0], dz[mt][1], dp[mt][0], dp[mt][1], dp[mt][2]);
#pragma unroll
        for (int j = 0; j < NF; ++j) {
          bf16x8 x[3];
#pragma unroll
          for (int e = 0; e < 3; ++e) {
            const lds_char* at = (const lds_char*)lds + (e * plane + s * RB + trow + 32 * j);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4*)(at + 16 * RB));
            x[e] = __builtin_bit_cast(
                bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          }
#define PMLP_PIECE(Q, E)                                             \
_Pragma("unroll") for (int mt = 0; mt < K; ++mt) acc[mt][j] =        \
    __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[E], dp[mt][Q], acc[mt][j], 0, 0, 0)
          PMLP_PIECE(2, 0);
          PMLP_PIECE(1, 1);
          PMLP_PIECE(0, 2);
          PMLP_PIECE(1, 0);
          PMLP_PIECE(0, 1);
          PMLP_PIECE(0, 0);
#undef PMLP_PIECE
        }
      }
    }
    // ---- the gradients, stored or applied ---------------------------------------
    const float rate = a.g.lrm ? a.g.lrm[m] : a.g.lr;
    float gs[NORM ? NO : 1];  // sum_b G of the unit's model
#pragma unroll
    for (int o = 0; o < (NORM ? NO : 0); ++o) {
      const int ow = MF ? 4 * lk + o : o;
      gs[NORM ? o : 0] = a.Gs[(int64_t)m * p.O + (ow < p.O ? ow : 0)];
    }
    float dw[NO], dg = 0.f, ds = 0.f, old[NO];
#pragma unroll
    for (int o = 0; o < NO; ++o) {
      if (!MF) {
        T[o] += __shfl_xor(T[o], 16);
        T[o] += __shfl_xor(T[o], 32);
      }
      dw[o] = T[o];
      old[o] = w2[o];
      if (NORM) {
        const float sg = gs[NORM ? o : 0];
        dg = fmaf(w2[o], T[o], dg);
        ds = fmaf(w2[o], sg, ds);
        dw[o] = fmaf(gn, T[o], sn * sg);
      }
    }
    if (NORM && MF) {
      dg += __shfl_xor(dg, 16);
      ds += __shfl_xor(ds, 16);
      dg += __shfl_xor(dg, 32);
      ds += __shfl_xor(ds, 32);
    }
    const float og = gn, os = sn;
    if (AHEAD) take();
    if (live) {
      // (a lane has unit li's columns 16 j + 4 lk ..)
#pragma unroll
      for (int mt = 0; mt < K; ++mt) {
        const bool to = a.dW1 != nullptr;
        float* const row = to ? (mt ? a.dV1 : a.dW1) + n * F
                              : const_cast<float*>(mt ? p.V1 : p.W1) + n * F4;
#pragma unroll
        for (int j = 0; j < NF; ++j) {
          const int f = 16 * j + 4 * lk;
          if (li >= cnt || f >= F) continue;
          const f32x4 g = acc[mt][j];
          if (f + 4 <= F) {
            if (to) *(f32x4_u*)(row + f) = g;
            else *(f32x4*)(row + f) -= rate * g;
          } else {
#pragma unroll
            for (int r = 0; r < 3; ++r) {
              if (f + r >= F) continue;
              if (to) row[f + r] = g[r];
              else row[f + r] -= rate * g[r];
            }
          }
        }
      }
      if (li < cnt && (MF || lk == 0)) {
#pragma unroll
        for (int q = 0; q < NO; ++q) {
          const int o = MF ? 4 * lk + q : q;
          if (o >= p.O) continue;
          if (a.g.dW2) a.g.dW2[(int64_t)o * p.N + n] = dw[q];
          else p.W2[(int64_t)o * p.ldw + n] = old[q] - rate * dw[q];
        }
        if (NORM && lk == 0) {
          if (a.g.dW2) {
            a.g.dgain[n] = dg;
            a.g.dshift[n] = ds;
          } else {
            p.gain[n] = og - rate * dg;
            p.shift[n] = os - rate * ds;
          }
        }
      }
    }
    q = qn;
    qn = qnn;
    m = mn;
  }
}

}  // namespace pmlpk
