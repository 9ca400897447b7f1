// Block packs: the backward pass in one kernel, for inputs of up to 128 columns.
// Compiled once per class of outputs (PMLP_BLK_OM: 2, 4 or 16).
//
// A wave takes a tile, up to 16 consecutive hidden units of one activation (of whatever
// models), and all samples, so that its weights' gradients need no other wave; it holds the three
// bf16 pieces of its units' W1 (and V1) rows and their gradients' accumulators in
// registers.  The samples' pieces lie in LDS once, sample by sample (chunks of
// them in turn, where they do not fit), and serve both products: read as rows they
// are the operand of Z = X W1^T, which is computed again rather than stored by the
// forward and read back, and read through the transposing LDS load the operand of
// dW1 = dZ^T X.  A step takes 32 samples: after Z the lane (li, lk) holds unit li of
// the samples 4 lk + r of both blocks of 16, forms dZ there, and those eight values
// are, as they lie, a row of the second product's first operand (the sums over
// samples run in that order in both of its operands).
// The norm's gradient needs no sums over units (see k_block.hip).
//
// The second product takes NF = 2 NC blocks of 16 columns, and one more for the fp32
// columns of the first; the last block may read past its columns into the next row,
// for columns that no one stores.

#include "block_device.h"

#include <algorithm>

#ifndef PMLP_BLK_OM
#error "compile with -DPMLP_BLK_OM=2|4|16"
#endif

namespace pmlpk {

namespace {

constexpr int OM = PMLP_BLK_OM;
constexpr bool MF = OM > 4;  // the output layer's products by matrix instructions
constexpr int NO = MF ? 4 : OM;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// Values and slopes of activation id A.
template <int NV>
__device__ __forceinline__ void act_and_slope(int A, const float (&z)[NV], float (&v)[NV],
                                              float (&d)[NV]) {
  switch (A) {
#define PMLP_ACT(AA)                                                                     \
  case AA: {                                                                             \
    _Pragma("unroll") for (int j = 0; j < NV; ++j) v[j] = act_fwd_bwd(AA, z[j], &d[j]); \
    break;                                                                               \
  }
    PMLP_EVERY_ACT
#undef PMLP_ACT
  }
}

template <int NC, int RM, bool GATED, bool NORM>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(NC <= 1 && !MF && !(GATED && NORM) ? 3 : 2)))
void k_blk_fused_bwd(BlkPack p, BlkBwdArgs a) {
  constexpr int NF = 2 * NC + (RM ? 1 : 0), K = GATED ? 2 : 1, RB = row_bytes(NC);

  extern __shared__ __align__(16) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int F = a.F, F4 = p.F4, SC = a.SC, plane = SC * RB;
  const int rounds = (a.ntiles + gridDim.x * nw - 1) / (gridDim.x * nw);

  const int nchunk = (a.Bp + SC - 1) / SC;
  if (nchunk == 1) {
    fill_pieces<NC>(lds, SC, a.X, 0, a.B, F, tid, blockDim.x);
    lds_barrier();
  }
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
    float w2[NO], gs[NORM ? NO : 1], g, s;
  } nx;
  auto fetch = [&](int64_t n, int m) {
    nx.w.load(p, n, lk);
    nx.g = NORM ? p.gain[n] : 1.f;
    nx.s = NORM ? p.shift[n] : 0.f;
#pragma unroll
    for (int o = 0; o < NO; ++o) {
      const int ow = MF ? 4 * lk + o : o, oc = ow < p.O ? ow : 0;
      nx.w2[o] = p.W2[(int64_t)oc * p.ldw + n];
      if (NORM) nx.gs[NORM ? o : 0] = a.Gs[(int64_t)m * p.O + oc];
    }
  };
  UnitRows<NC, RM, K> w;
  float w2[NO], gs[NORM ? NO : 1], gn = 1.f, sn = 0.f;  // (gs: sum_b G of the unit's model)
  auto take = [&] {
    w.split(nx.w, F4, lk);
    gn = opaque(nx.g);
    sn = opaque(nx.s);
#pragma unroll
    for (int o = 0; o < NO; ++o) {
      const float v = opaque(nx.w2[o]);
      w2[o] = (MF ? 4 * lk + o : o) < p.O ? v : 0.f;
      if (NORM) gs[NORM ? o : 0] = opaque(nx.gs[NORM ? o : 0]);
    }
  };
  struct Up {
    f32x4 g[MF ? 2 : OM], r[NORM ? 4 : 1];
  };
  // block b (its first sample) of the lanes' models m
  auto load_up = [&](int m, int b) {
    Up u;
    const uint32_t at = (uint32_t)(b + 4 * lk);  // first of four samples
    if (MF) {
      const float* const g =
          a.G + (int64_t)__builtin_amdgcn_readfirstlane(m) * a.Bp * OM;
      u.g[0] = *(const f32x4*)(g + (uint32_t)(b + li) * OM + 4 * lk);
#pragma unroll
      for (int r = 0; r < 4; ++r) u.g[MF ? 1 : 0][r] = g[(at + r) * OM + li];
    } else {
      const float* const g = a.G + ((int64_t)m * a.Bp + at) * OM;
#pragma unroll
      for (int v = 0; v < NO; ++v) u.g[MF ? 0 : v] = *(const f32x4*)(g + 4 * v);
    }
    if (NORM) {
      const float* const R = a.R + ((int64_t)m * a.Bp + at) * 4;
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
  const int stride = gridDim.x * nw;
  auto tile_at = [&](int t) { return a.tiles[std::min(t, a.ntiles - 1)]; };
  auto unit_of = [&](const BlkTile& q) { return (int64_t)q.n0 + std::min(li, q.cnt - 1); };
  int tile = (int)blockIdx.x * nw + wave;
  BlkTile q = tile_at(tile), qn = tile_at(tile + stride);
  int m = p.mid[unit_of(q)];
  Up up = load_up(m, 0);
  if (AHEAD) {
    fetch(unit_of(q), m);
    take();
  }
#pragma unroll 1
  for (int round = 0; round < rounds; ++round, tile += stride) {
    const bool live = tile < a.ntiles;
    const int n0 = __builtin_amdgcn_readfirstlane(q.n0);
    const int cnt = __builtin_amdgcn_readfirstlane(q.cnt), act = __builtin_amdgcn_readfirstlane(q.act);
    const int64_t n = n0 + std::min(li, cnt - 1);
    const int m_lo = __builtin_amdgcn_readfirstlane(m), m_hi = __builtin_amdgcn_readlane(m, 15);
    const BlkTile qnn = tile_at(tile + 2 * stride);
    const int mn = p.mid[unit_of(qn)];
    if (AHEAD) {
      fetch(unit_of(qn), mn);
    } else {
      fetch(n, m);
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
            // dN = G W2 and T += G^T h, the sums in the order of the registers
            f32x4 t = f32x4{T[0], T[1], T[2 % NO], T[3 % NO]};
            f32x4 ga = up.g[0], gt = up.g[MF ? 1 : 0];
#pragma unroll 1
            for (int mm = m_lo;;) {
              f32x4 d = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                d = __builtin_amdgcn_mfma_f32_16x16x4f32(ga[r], w2[r % NO], d, 0, 0, 0);
                t = __builtin_amdgcn_mfma_f32_16x16x4f32(gt[r], m == mm ? h[r] : 0.f, t, 0, 0, 0);
              }
#pragma unroll
              for (int r = 0; r < 4; ++r) dn[r] = m == mm ? d[r] : dn[r];
              if (++mm > m_hi) break;
              const uint32_t b = (uint32_t)(b0 + s + 16 * i + 4 * lk);
              const float* const g = a.G + (int64_t)mm * a.Bp * OM;
              ga = *(const f32x4*)(g + (uint32_t)(b0 + s + 16 * i + li) * OM + 4 * lk);
#pragma unroll
              for (int r = 0; r < 4; ++r) gt[r] = g[(b + r) * OM + li];
            }
#pragma unroll
            for (int o = 0; o < 4; ++o) T[o % NO] = t[o];
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
    __builtin_amdgcn_mfma_f32_16x16x32_bf16(dp[mt][Q], x[E], acc[mt][j], 0, 0, 0)
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
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float row_rate = __shfl(rate, 4 * lk + r);
        if (4 * lk + r >= cnt) continue;
        const int64_t nr = n0 + 4 * lk + r;
#pragma unroll
        for (int mt = 0; mt < K; ++mt) {
          float* const dW = mt ? a.dV1 : a.dW1;
          float* const W = const_cast<float*>(mt ? p.V1 : p.W1);
#pragma unroll
          for (int j = 0; j < NF; ++j) {
            const int f = 16 * j + li;
            if (f >= F) continue;
            if (dW) dW[nr * F + f] = acc[mt][j][r];
            else W[nr * F4 + f] -= row_rate * acc[mt][j][r];
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
  // only, four where there is more
  const int waves = 4 * lds > (size_t)lmax ? 8 : 4;
  const int slots = resident_blocks((const void*)fn, 64 * waves, lds);
  if (slots <= 0) return hipErrorInvalidValue;
  const int64_t grid = std::min<int64_t>(slots, (a.ntiles + waves - 1) / waves);
  fn<<<(unsigned)grid, 64 * waves, lds, s>>>(p, a);
  return hipGetLastError();
}

}  // namespace pmlpk
