// Block packs: products, gate, norm statistics and output sums in one kernel, for
// inputs of up to 128 columns.  Compiled once per number of waves (PMLP_BLK_NW:
// 1, 2, 4 or 8 waves of 32 samples; 0: one wave of 16).
//
// A workgroup takes a batch of 16 NI NW samples and a run of 16-unit tiles, none of
// which crosses a model.  Wave w holds the three bf16 pieces of its own 16 NI
// samples in registers.  Stages of ST tiles pass through LDS, double buffered: the
// waves share the loads and splits of the tiles' W1 (and V1) rows, in operand
// order, and the rows of gain * W2; the loads are a stage ahead.  With the weights
// as the first operand lane (li, lk) ends with units 4 lk + r of sample li, so that
// the sums over a model's units stay in the lane and meet over the four lk once per
// model.  Up to four outputs are summed by vector FMAs, more by fp32 matrix
// products, whose second operand is the hidden values as they lie in the registers.
// The pre-activations are never stored.
//
// Products: K = 32 NC columns in three-piece products and up to RM fp32 steps of
// four columns after them.

#include "block_device.h"

#include <algorithm>

#ifndef PMLP_BLK_NW
#error "compile with -DPMLP_BLK_NW=0|1|2|4|8"
#endif

namespace pmlpk {

namespace {

constexpr int kNI = PMLP_BLK_NW == 0 ? 1 : 2;
constexpr int kNW = PMLP_BLK_NW == 0 ? 1 : PMLP_BLK_NW;
constexpr int kBS = 16 * kNI * kNW;  // samples of a workgroup

// tiles a stage: two or four waves' worth of strips
template <bool GATED>
struct Stage {
  static constexpr int ST = kNW == 8 ? (GATED ? 2 : 4) : (kNW == 4 && !GATED ? 2 : 1);
};

// LDS of one tile: the pieces of its strips, their fp32 remainders, the output rows
template <int NC, int RM, int OM, bool GATED>
struct TileLds {
  static constexpr int K = GATED ? 2 : 1;
  static constexpr int kW2 = K * (NC * 3072 + RM * 256);
  static constexpr int bytes = kW2 + OM * 64 + 16;  // (and the tile's info and model)
};

template <int NC, int RM, int OM, bool GATED, bool NORM>
__global__ __launch_bounds__(64 * kNW) __attribute__((amdgpu_waves_per_eu(2)))
void k_blk_fused_fwd(BlkPack p, BlkFwdArgs a) {
  constexpr int NI = kNI, NW = kNW, ST = Stage<GATED>::ST, K = GATED ? 2 : 1;
  using L = TileLds<NC, RM, OM, GATED>;
  constexpr int UNITS = K * NC * ST;                 // chunk strips of a stage
  constexpr int UPW = NC ? (UNITS + NW - 1) / NW : 1;  // of one wave
  constexpr int REMS = K * ST;                       // remainder strips, a wave each in turn
  constexpr int RPW = (REMS + NW - 1) / NW;
  constexpr int W2E = OM * 16 / 64 ? OM * 16 / 64 : 1;  // output weights per lane
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int chunk = blockIdx.x / a.wpc, w = blockIdx.x - chunk * a.wpc;
  const int F = a.F, F4 = p.F4, rem = RM ? (F4 - 32 * NC) >> 2 : 0;
  const int t0 = (int)((int64_t)w * a.ntiles / a.wpc);
  const int t1 = (int)((int64_t)(w + 1) * a.ntiles / a.wpc);
  if (t0 >= t1) return;

  // this wave's samples
  bf16x8 x0[NI][NC > 0 ? NC : 1], x1[NI][NC > 0 ? NC : 1], x2[NI][NC > 0 ? NC : 1];
  float xt[NI][RM > 0 ? RM : 1];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int b = chunk * kBS + 16 * (wave * NI + i) + li;
    const float* xr = a.X + (int64_t)(b < a.B ? b : a.B - 1) * F;
    float v[NC > 0 ? 8 * NC : 1], t[RM > 0 ? RM : 1];  // all loads first
#pragma unroll
    for (int e = 0; e < 8 * NC; ++e) {
      const int k = 32 * (e >> 3) + 8 * lk + (e & 7);
      v[e] = xr[k < F ? k : F - 1];
    }
#pragma unroll
    for (int q = 0; q < RM; ++q) {
      const int k = 32 * NC + 4 * q + lk;
      t[q] = xr[k < F ? k : F - 1];
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      f32x4 q[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = opaque(v[8 * c + e]);
        q[e >> 2][e & 3] = 32 * c + 8 * lk + e < F && b < a.B ? w : 0.f;
      }
      split3(q[0], q[1], x0[i][c], x1[i][c], x2[i][c]);
    }
#pragma unroll
    for (int q = 0; q < RM; ++q) {
      const float w = opaque(t[q]);
      xt[i][q] = q < rem && 32 * NC + 4 * q + lk < F && b < a.B ? w : 0.f;
    }
  }

  // This wave's part of a stage: up to UPW chunk strips, RPW remainder strips and
  // one tile's output rows.  Every load is made, of the last strip or tile again
  // where there is none, so that waits count what is in flight; descriptors come by
  // scalar loads a stage ahead of the loads that need them.
  constexpr int NPART = UPW + RPW + 1;
  const auto* const tiles = (const __attribute__((address_space(4))) BlkTile*)(uintptr_t)a.tiles;
  auto part_tile = [&](int i) {  // tile within the stage of part i
    if (i < UPW) return NC ? std::min(wave + i * NW, UNITS - 1) / (K * (NC ? NC : 1)) : 0;
    if (i < UPW + RPW) return std::min(wave + (i - UPW) * NW, REMS - 1) / K;
    return std::min(wave, ST - 1);
  };
  struct Desc {
    int n0[NPART], info[NPART], m;  // (m: of tile `wave`)
  };
  auto load_desc = [&](int ts) {
    Desc d;
#pragma unroll
    for (int i = 0; i < NPART; ++i) {
      const int t = std::min(ts + part_tile(i), t1 - 1);
      d.n0[i] = tiles[t].n0;
      d.info[i] = tiles[t].info;
      if (i == NPART - 1) d.m = tiles[t].m;
    }
    return d;
  };
  struct Raw {
    f32x4 c[2 * UPW];
    float t[RPW][RM > 0 ? RM : 1];
    float w2[W2E], g[W2E];
    int cnt[NPART];
    int word, m;  // of tile `wave`
  } raw;
  // row li of a tile, or the tile's last unit (put() makes such rows zero)
  const float *W1 = p.W1, *V1 = p.V1;
  asm volatile("" : "+s"(W1), "+s"(V1));  // (or each choice of one is a load of its address)
  auto fetch = [&](const Desc& ds) {
#pragma unroll
    for (int i = 0; i < NPART; ++i) raw.cnt[i] = ds.info[i] & 255;
#pragma unroll
    for (int i = 0; i < (NC ? UPW : 0); ++i) {
      const int u = std::min(wave + i * NW, UNITS - 1), v = u % (K * (NC ? NC : 1));
      const int mat = v / (NC ? NC : 1), c = v - mat * NC;
      const float* row =
          (mat ? V1 : W1) + (int64_t)(ds.n0[i] + std::min(li, raw.cnt[i] - 1)) * F4;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = 32 * c + 8 * lk + 4 * e;
        raw.c[2 * i + e] = *(const f32x4*)(row + (k < F4 ? k : F4 - 4));
      }
    }
#pragma unroll
    for (int i = 0; i < (RM ? RPW : 0); ++i) {
      const float* row = (std::min(wave + i * NW, REMS - 1) % K ? V1 : W1) +
                         (int64_t)(ds.n0[UPW + i] + std::min(li, raw.cnt[UPW + i] - 1)) * F4;
#pragma unroll
      for (int s = 0; s < RM; ++s) raw.t[i][s] = row[s < rem ? 32 * NC + 4 * s + lk : 0];
    }
    const int n0 = ds.n0[NPART - 1], cnt = raw.cnt[NPART - 1];
#pragma unroll
    for (int e = 0; e < W2E; ++e) {
      const int v = lane + 64 * e, o = v >> 4, u = v & 15;
      const int64_t n = n0 + (u < cnt ? u : 0);
      raw.w2[e] = p.W2[(int64_t)(o < p.O ? o : 0) * p.ldw + n];
      raw.g[e] = NORM ? p.gain[n] : 1.f;
    }
    raw.word = ds.info[NPART - 1];
    raw.m = ds.m;
  };
  auto put = [&](int buf) {
    char* const base = lds + buf * ST * L::bytes;
#pragma unroll
    for (int i = 0; i < (NC ? UPW : 0); ++i) {
      const int u = wave + i * NW;
      const int j = u / (K * (NC ? NC : 1)), v = u - j * (K * NC), c = v % (NC ? NC : 1);
      const bool in = li < raw.cnt[i];
      f32x4 r[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const f32x4 w = opaque(raw.c[2 * i + e]);
        const bool ok = in && 32 * c + 8 * lk + 4 * e < F4;
#pragma unroll
        for (int q = 0; q < 4; ++q) r[e][q] = ok ? w[q] : 0.f;
      }
      bf16x8 p0, p1, p2;
      split3(r[0], r[1], p0, p1, p2);
      if (u < UNITS) {
        bf16x8* d = (bf16x8*)(base + j * L::bytes + v * 3072) + lane;
        d[0] = p0;
        d[64] = p1;
        d[128] = p2;
      }
    }
#pragma unroll
    for (int i = 0; i < (RM ? RPW : 0); ++i) {
      const int u = wave + i * NW;
      const bool in = li < raw.cnt[UPW + i];
      float* d = (float*)(base + (u / K) * L::bytes + K * NC * 3072 + (u % K) * (RM * 256)) + lane;
#pragma unroll
      for (int s = 0; s < RM; ++s) {
        const float w = opaque(raw.t[i][s]);
        if (u < REMS) d[64 * s] = in && s < rem ? w : 0.f;
      }
    }
    float* d = (float*)(base + wave * L::bytes + L::kW2) + lane;
#pragma unroll
    for (int e = 0; e < W2E; ++e) {
      const int v = lane + 64 * e;
      const float w = opaque(raw.w2[e]) * opaque(raw.g[e]);
      if (wave < ST && v < 16 * OM)
        d[64 * e] = (v >> 4) < p.O && (v & 15) < raw.cnt[NPART - 1] ? w : 0.f;
    }
    if (wave < ST && lane < 2) ((int*)d)[16 * OM] = lane ? raw.m : raw.word;
  };

  // running sums of the open model: outputs (lane's own units; with matrix products
  // outputs 4 lk + r over all units) and statistics
  constexpr bool MF = OM > 4;
  constexpr int NS = MF ? 4 : OM;
  f32x4 accS[NI];
  float S[NI][NS], mean[NI], m2[NI], cnt = 0.f;
  auto reset = [&] {
    cnt = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      mean[i] = m2[i] = 0.f;
      accS[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int o = 0; o < NS; ++o) S[i][o] = 0.f;
    }
  };
  reset();
  // model m ends (or this workgroup's part of it)
  auto emit = [&](int m) {
    const int PQ = p.O + (NORM ? 2 : 0);
    float* const rec = a.part + (int64_t)(m + w) * PQ * a.Bp + chunk * kBS + 16 * wave * NI + li;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (MF) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * lk + r < p.O) rec[(int64_t)(4 * lk + r) * a.Bp + 16 * i] = accS[i][r];
      } else {
#pragma unroll
        for (int o = 0; o < NS; ++o) {
          S[i][o] += __shfl_xor(S[i][o], 16);
          S[i][o] += __shfl_xor(S[i][o], 32);
        }
#pragma unroll
        for (int o = 0; o < NS; ++o)
          if (lk == o && o < p.O) rec[(int64_t)o * a.Bp + 16 * i] = S[i][o];
      }
    }
    if (NORM) {
#pragma unroll
      for (int s = 16; s < 64; s <<= 1) {
        const float nb = __shfl_xor(cnt, s);
        float n = cnt;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const float mb = __shfl_xor(mean[i], s), qb = __shfl_xor(m2[i], s);
          n = cnt;
          merge_stats(n, mean[i], m2[i], nb, mb, qb);
        }
        cnt = n;
      }
      if (lk < 2) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          rec[(int64_t)(p.O + lk) * a.Bp + 16 * i] = lk ? m2[i] : mean[i];
      }
    }
    reset();
  };

  Desc next = load_desc(t0);
  fetch(next);
  next = load_desc(t0 + ST);
  put(0);
  fetch(next);
  next = load_desc(t0 + 2 * ST);
  lds_barrier();
  int buf = 0;
#pragma unroll 1
  for (int ts = t0; ts < t1; ts += ST, buf ^= 1) {
#pragma unroll 1
    for (int j = 0; j < ST && ts + j < t1; ++j) {
      const char* const base = lds + (buf * ST + j) * L::bytes;
      const int2 word = *(const int2*)(base + L::kW2 + 64 * OM);
      float wt[K][RM > 0 ? RM : 1];
#pragma unroll
      for (int mt = 0; mt < K; ++mt)
#pragma unroll
        for (int s = 0; s < RM; ++s)
          wt[mt][s] = ((const float*)(base + K * NC * 3072 + mt * (RM * 256)))[64 * s + lane];
      f32x4 acc[K][NI];
#pragma unroll
      for (int mt = 0; mt < K; ++mt)
#pragma unroll
        for (int i = 0; i < NI; ++i) acc[mt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        bf16x8 wc[K][3];
#pragma unroll
        for (int mt = 0; mt < K; ++mt)
#pragma unroll
          for (int e = 0; e < 3; ++e)
            wc[mt][e] = ((const bf16x8*)(base + (mt * NC + c) * 3072))[64 * e + lane];
        // the piece products smallest first, the blocks and projections in turn
#define PMLP_PIECE(E, XP)                                     \
_Pragma("unroll") for (int mt = 0; mt < K; ++mt)              \
_Pragma("unroll") for (int i = 0; i < NI; ++i) acc[mt][i] = \
    __builtin_amdgcn_mfma_f32_16x16x32_bf16(wc[mt][E], XP[i][c], acc[mt][i], 0, 0, 0)
        PMLP_PIECE(0, x2);
        PMLP_PIECE(1, x1);
        PMLP_PIECE(2, x0);
        PMLP_PIECE(0, x1);
        PMLP_PIECE(1, x0);
        PMLP_PIECE(0, x0);
#undef PMLP_PIECE
      }
#pragma unroll
      for (int s = 0; s < RM; ++s)
        if (s < rem) {
#pragma unroll
          for (int mt = 0; mt < K; ++mt)
#pragma unroll
            for (int i = 0; i < NI; ++i)
              acc[mt][i] =
                  __builtin_amdgcn_mfma_f32_16x16x4f32(wt[mt][s], xt[i][s], acc[mt][i], 0, 0, 0);
        }
      const int info = __builtin_amdgcn_readfirstlane(word.x), tcnt = info & 255;
      float z[4 * NI], h[4 * NI];
#pragma unroll
      for (int v = 0; v < 4 * NI; ++v) z[v] = acc[0][v >> 2][v & 3];
      blk_acts<4 * NI>((info >> 8) & 255, z, h);
      if (GATED) {
#pragma unroll
        for (int v = 0; v < 4 * NI; ++v) h[v] *= acc[K - 1][v >> 2][v & 3];
      }
      const int mine = tcnt - 4 * lk;  // units of this lane: min(4, mine), if positive
      if (tcnt < 16) {
#pragma unroll
        for (int v = 0; v < 4 * NI; ++v) h[v] = (v & 3) < mine ? h[v] : 0.f;
      }
      const float* const w2 = (const float*)(base + L::kW2);
      if (MF) {
        const f32x4 wv = *(const f32x4*)(w2 + 16 * li + 4 * lk);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < NI; ++i)
            accS[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[r], h[4 * i + r], accS[i], 0, 0, 0);
      } else {
#pragma unroll
        for (int o = 0; o < NS; ++o) {
          const f32x4 wv = *(const f32x4*)(w2 + 16 * o + 4 * lk);
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[i][o] = fmaf(h[4 * i + r], wv[r], S[i][o]);
        }
      }
      if (NORM) {
        if (tcnt == 16) {
          const float n = cnt + 4.f, f = 4.f * frcp(n), nf = cnt * f;
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const float* v = h + 4 * i;
            const float mu = 0.25f * ((v[0] + v[1]) + (v[2] + v[3]));
            float qs = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) qs = fmaf(v[r] - mu, v[r] - mu, qs);
            const float d = mu - mean[i];
            mean[i] = fmaf(d, f, mean[i]);
            m2[i] += fmaf(d * d, nf, qs);
          }
          cnt = n;
        } else if (mine > 0) {
          const float nt = (float)(mine < 4 ? mine : 4);
          float n = cnt;
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const float* v = h + 4 * i;
            const float mu = ((v[0] + v[1]) + (v[2] + v[3])) / nt;
            float qs = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) qs += r < mine ? (v[r] - mu) * (v[r] - mu) : 0.f;
            n = cnt;
            merge_stats(n, mean[i], m2[i], nt, mu, qs);
          }
          cnt = n;
        }
      }
      if (ts + j + 1 == t1 || (info & kBlkLast)) emit(__builtin_amdgcn_readfirstlane(word.y));
    }
    put(buf ^ 1);
    fetch(next);
    next = load_desc(ts + 3 * ST);
    lds_barrier();
  }
}

typedef void (*BlkFwdFn)(BlkPack, BlkFwdArgs);
struct BlkFwdInst {
  BlkFwdFn fn;
  int lds;
};

template <int NC, int RM, int OM>
BlkFwdInst inst_kind(bool gated, bool norm) {
#define PMLP_INST(G, N) \
  BlkFwdInst { k_blk_fused_fwd<NC, RM, OM, G, N>, 2 * Stage<G>::ST * TileLds<NC, RM, OM, G>::bytes }
  if (gated && norm) return PMLP_INST(true, true);
  if (gated) return PMLP_INST(true, false);
  return PMLP_INST(false, true);
#undef PMLP_INST
}

template <int NC, int RM>
BlkFwdInst inst_out(int O, bool gated, bool norm) {
  if (O <= 2) return inst_kind<NC, RM, 2>(gated, norm);
  if (O <= 4) return inst_kind<NC, RM, 4>(gated, norm);
  return inst_kind<NC, RM, 16>(gated, norm);
}

// The instance for F4 columns: 32 NC of them in three-piece products, then up to
// three fp32 steps of four, or else a last chunk that is padded.
BlkFwdInst inst_of(const BlkPack& p) {
  const bool g = p.V1 != nullptr, n = p.gain != nullptr;
  const int c = p.F4 / 32, r = p.F4 % 32 / 4;
  switch (r == 0 ? 2 * c : r <= 3 ? 2 * c + 1 : 2 * c + 2) {
    case 1: return inst_out<0, 3>(p.O, g, n);
    case 2: return inst_out<1, 0>(p.O, g, n);
    case 3: return inst_out<1, 3>(p.O, g, n);
    case 4: return inst_out<2, 0>(p.O, g, n);
    case 5: return inst_out<2, 3>(p.O, g, n);
    case 6: return inst_out<3, 0>(p.O, g, n);
    case 7: return inst_out<3, 3>(p.O, g, n);
    case 8: return inst_out<4, 0>(p.O, g, n);
    default: return BlkFwdInst{nullptr, 0};
  }
}

}  // namespace

#define PMLP_CAT_(a, b) a##b
#define PMLP_CAT(a, b) PMLP_CAT_(a, b)

int PMLP_CAT(blk_fwd_slots_, PMLP_BLK_NW)(const BlkPack& p) {
  const BlkFwdInst i = inst_of(p);
  return i.fn ? resident_blocks((const void*)i.fn, 64 * kNW, i.lds) : 0;
}

hipError_t PMLP_CAT(launch_blk_fused_fwd_, PMLP_BLK_NW)(const BlkPack& p, const BlkFwdArgs& a,
                                                        hipStream_t s) {
  const BlkFwdInst i = inst_of(p);
  const int nchunk = (a.B + kBS - 1) / kBS;
  if (!i.fn || a.B < 1 || a.ntiles < 1 || a.wpc < 1 || a.Bp < nchunk * kBS ||
      (int64_t)nchunk * a.wpc > 0x7fffffff)
    return hipErrorInvalidValue;
  i.fn<<<(unsigned)(nchunk * a.wpc), 64 * kNW, i.lds, s>>>(p, a);
  return hipGetLastError();
}

}  // namespace pmlpk
