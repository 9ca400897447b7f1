// Block packs: products, gate, norm statistics and output sums in one kernel, for
// inputs of up to 128 columns.  Compiled once per class of outputs (PMLP_BLK_OM: 2 or
// 16).
//
// A wave takes 16 hidden units of one model (a tile) and the samples of its workgroup,
// whose pieces lie in LDS: it splits the units' W1 (and V1) rows once, into registers,
// and needs no other wave (an earlier form, with the samples in registers and the
// units passing through LDS in stages, spent as long at its barriers and on shared
// splitting as on its products).  A step takes 32 samples; lane (li, lk) ends with
// units 4 lk + r of sample li of both blocks of 16.  The sums over the tile's units
// (outputs, and with a norm the mean and the squared deviations) are stored per tile
// and sample; the output and loss kernels merge a model's tiles.  That costs blk_planes
// floats per 16 units and sample, against 16 (32 gated) for the pre-activations.
//
// Two outputs are summed by vector FMAs and two lane swaps, more by fp32 matrix
// products whose second operand is the hidden values as they lie in the registers.
// The squared deviations are taken from one of the tile's own values, then moved to
// the mean: (h - K)^2 exceeds the variance at most 15 times over 16 values, so that
// loses four bits at worst, wherever the mean is.

#include "block_device.h"

#include <algorithm>

#ifndef PMLP_BLK_OM
#error "compile with -DPMLP_BLK_OM=2|16"
#endif

namespace pmlpk {

namespace {

constexpr bool MF = PMLP_BLK_OM > 2;

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

// Threads of a workgroup, at most: as many waves as a SIMD's registers hold without
// spilling, four, three or two.
template <int NC, bool GATED>
constexpr int max_threads() {
  return GATED ? (NC == 0 ? 1024 : NC <= 3 ? 768 : 512) : (NC <= 3 ? 1024 : 768);
}

template <int NC, int RM, bool GATED, bool NORM>
__global__ __launch_bounds__((max_threads<NC, GATED>()))
void k_blk_fused_fwd(BlkPack p, BlkFwdArgs a) {
  constexpr int K = GATED ? 2 : 1, RB = row_bytes(NC);
  extern __shared__ __align__(16) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int chunk = blockIdx.x / a.wpc, wg = blockIdx.x - chunk * a.wpc;
  const int SC = a.SC, plane = SC * RB, b0 = chunk * SC;
  fill_pieces<NC>(lds, SC, a.X, b0, a.B, a.F, tid, blockDim.x);
  lds_barrier();
  const int steps = (std::min(SC, a.B - b0) + 31) >> 5;
  const char* const zrow = lds + li * RB + 16 * lk;
  const char* const xrow = lds + li * RB + 64 * NC + 2 * lk;
  const int PQ = p.O + (NORM ? 2 : 0);

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
  const int step = a.wpc * nw;
  auto tile_at = [&](int t) { return a.tiles[std::min(t, a.ntiles - 1)]; };
  BlkTile q = tile_at(wg * nw + wave), qn = tile_at(wg * nw + wave + step);
  if (AHEAD) fetch(q.n0, q.cnt);
#pragma unroll 1
  for (int t = wg * nw + wave; t < a.ntiles; t += step) {
    const int n0 = __builtin_amdgcn_readfirstlane(q.n0);
    const int cnt = __builtin_amdgcn_readfirstlane(q.cnt), act = __builtin_amdgcn_readfirstlane(q.act);
    const BlkTile qnn = tile_at(t + 2 * step);
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
    if (AHEAD) fetch(qn.n0, qn.cnt);
    float* const rec = a.part + (int64_t)t * PQ * a.Br + b0 + li;
    const float rn = 1.f / (float)cnt;
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
      float* const dst = rec + 32 * st;
      if (MF) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s = __builtin_amdgcn_mfma_f32_16x16x4f32(w2[0][r], h[4 * i + r], s, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * lk + r < p.O) dst[(int64_t)(4 * lk + r) * a.Br + 16 * i] = s[r];
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
        // row lk ends with block lk & 1 of output lk >> 1
        const float v = sum16(sum32(s[0][0], s[0][1]), sum32(s[1][0], s[1][1]));
        dst[(int64_t)(lk >> 1) * a.Br + 16 * (lk & 1)] = v;
      }
      if (NORM) {
        float mean[2], m2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float piv = __shfl(h[4 * i], li);  // the first unit's value
          float d = 0.f, e = 0.f;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float v = (cnt == 16 || r < mine) ? h[4 * i + r] - piv : 0.f;
            d += v;
            e = fmaf(v, v, e);
          }
          d = sum32(d, d);
          e = sum32(e, e);
          d = sum16(d, d);
          e = sum16(e, e);
          mean[i] = fmaf(d, rn, piv);
          m2[i] = fmaxf(fmaf(-d * rn, d, e), e != e ? e : 0.f);
        }
        const float v = lk & 2 ? (lk & 1 ? m2[1] : m2[0]) : (lk & 1 ? mean[1] : mean[0]);
        dst[(int64_t)(p.O + (lk >> 1)) * a.Br + 16 * (lk & 1)] = v;
      }
    }
    q = qn;
    qn = qnn;
  }
}

typedef void (*BlkFwdFn)(BlkPack, BlkFwdArgs);
struct BlkFwdInst {
  BlkFwdFn fn;
  int NC, threads;  // threads of a workgroup, at most (the occupancy query does not mind them)
};

template <int NC, int RM>
BlkFwdInst fwd_kind(bool gated, bool norm) {
  if (gated && norm) return {k_blk_fused_fwd<NC, RM, true, true>, NC, max_threads<NC, true>()};
  if (gated) return {k_blk_fused_fwd<NC, RM, true, false>, NC, max_threads<NC, true>()};
  return {k_blk_fused_fwd<NC, RM, false, true>, NC, max_threads<NC, false>()};
}

BlkFwdInst fwd_of(const BlkPack& p) {
  const bool g = p.V1 != nullptr, n = p.gain != nullptr;
#define PMLP_CALL(NC, RM) fwd_kind<NC, RM>(g, n)
  PMLP_BLK_SHAPE(p.F4, PMLP_CALL)
#undef PMLP_CALL
  return {nullptr, 0, 0};
}

}  // namespace

#define PMLP_CAT_(a, b) a##b
#define PMLP_CAT(a, b) PMLP_CAT_(a, b)

int PMLP_CAT(blk_fwd_slots_, PMLP_BLK_OM)(const BlkPack& p, int32_t SC, int32_t waves) {
  const BlkFwdInst i = fwd_of(p);
  return i.fn && 64 * waves <= i.threads ? resident_blocks((const void*)i.fn, 64 * waves, pieces_bytes(i.NC, SC)) : 0;
}

hipError_t PMLP_CAT(launch_blk_fused_fwd_, PMLP_BLK_OM)(const BlkPack& p, const BlkFwdArgs& a,
                                                        hipStream_t s) {
  const BlkFwdInst i = fwd_of(p);
  if (!i.fn || a.B < 1 || a.ntiles < 1 || a.wpc < 1 || a.waves < 1 || 64 * a.waves > i.threads || a.SC < 32 ||
      a.SC % 32 || p.O > PMLP_BLK_OM)
    return hipErrorInvalidValue;
  const int nchunk = (a.B + a.SC - 1) / a.SC;
  if (a.Br < (a.B + 31) / 32 * 32 || (int64_t)nchunk * a.wpc > 0x7fffffff)
    return hipErrorInvalidValue;
  i.fn<<<(unsigned)(nchunk * a.wpc), 64 * a.waves, pieces_bytes(i.NC, a.SC), s>>>(p, a);
  return hipGetLastError();
}

}  // namespace pmlpk
