// Block packs: the gated hidden layer and the layer norm of packed MLPs, on
// pre-activations that are stored (any shape), and the output and loss kernels
// that every path shares.
//
// Model m's hidden values are H = act_m(X W1^T), or, gated, act_m(X W1^T) *
// (X V1^T).  With a norm the output weights see g Hh + s, Hh = (H - mu) r over
// the model's own h units, r = (var + eps)^-1/2.  As the output product is
// linear, its sums and the norm's statistics come from one pass over the units: with
// k a piece of the model's units, m_k the mean over it and c that of the first piece,
//   S_k,o = sum_n in k (H_n - m_k) g_n W2[o,n],  C_k,o = sum_n in k g_n W2[o,n]
//   P_o = r (sum_k (S_k,o + (m_k - c) C_k,o) - (mu - c) C_o),  C_o = sum_n g_n W2[o,n]
//   logits_o = P_o + D_o,                                      D_o = sum_n s_n W2[o,n]
// and the two means over the units that the norm's gradient needs come from the
// outputs' gradients G, with no pass of their own:
//   dN_n = sum_o G_o W2[o,n]                      (gradient of g Hh + s)
//   dH_n = r (g_n dN_n - a1 - Hh_n a2)
//   a1 = 1/h sum_n g_n dN_n = 1/h sum_o G_o C_o,  a2 = 1/h sum_n g_n dN_n Hh_n = 1/h sum_o G_o P_o.
// With T_o = sum_b G_o Hh_n the parameters' gradients are
//   dW2[o,n] = g_n T_o + s_n sum_b G_o,  dg_n = sum_o W2[o,n] T_o,  ds_n = sum_o W2[o,n] sum_b G_o.
// The statistics are running means and sums of squared deviations (Welford's
// update; two sets merge by Chan, Golub and LeVeque's formula), all in fp32: a sum
// of squares minus a squared mean would lose the variance of a layer whose mean is
// large, as the difference of sum_n H_n g_n W2[o,n] and mu C_o would its outputs.  No sum
// here has terms larger than a few of the model's largest deviations times its weights.
// A piece's mean is rounded once more to be stored, by as much as its hidden values are
// (storing it as one of them and the difference kept sums and variance free of that, and
// took up to 14 % longer: a fifth number a piece, and its room in LDS).
//
// The stored path (more than 128 input columns) spends its time in its three large
// products; 1200 models of 1 to 200 units, 1000 columns, 1024 samples, gated, in a trace of
// four passes: 5680 us of them at 174 TFLOP/s (a library fp32 product reached 152; a pass
// among a hundred takes 5600 us in all, them at about 200), k_blk_fwd 222 us and k_blk_bwd
// 372 us for 1.0 and 2.0 GB.

#include "block_loss.h"

namespace pmlpk {

namespace {

constexpr int kFU = 4;  // units per lane group whose loads are in flight

// One wave per (piece, block of 4 LG samples).  Lane l takes four samples and
// every NG-th unit (LG = lanes per unit, NG = 64 / LG), as k_m3_fwd.  Bound by
// reading Z and U once with two outputs, by its vector instructions with many (1114
// models, 151 columns, ten outputs, 60 samples: 0.9 TB/s).
template <int OM, bool GATED, bool NORM>
__global__ __launch_bounds__(kBlock) void k_blk_fwd(BlkPack p, const float* __restrict__ Zt,
                                                    const float* __restrict__ Ut, int Bp, int LG,
                                                    int nbblk, float* __restrict__ part,
                                                    float* __restrict__ csum) {
  const int lane = threadIdx.x & 63;
  const int64_t wv = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int pc = (int)(wv / nbblk), blk = (int)(wv - (int64_t)pc * nbblk);
  if (pc >= p.npieces) return;
  const BlkPiece q = p.pieces[pc];
  const int NG = 64 / LG, g = lane / LG;
  const int b = 4 * (blk * LG + lane - g * LG);
  const bool valid = b < Bp;
  const int bl = valid ? b : Bp - 4;
  const int a = p.actn[q.n0];
  float S[4][OM], C[OM];
  float mean[4] = {0.f, 0.f, 0.f, 0.f}, m2[4] = {0.f, 0.f, 0.f, 0.f}, cnt = 0.f;
  float piv[4] = {0.f, 0.f, 0.f, 0.f};  // the lane's first unit's values, from which it counts
#pragma unroll
  for (int o = 0; o < OM; ++o) {
    C[o] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) S[i][o] = 0.f;
  }
  for (int u0 = g; u0 < q.len; u0 += kFU * NG) {
    f32x4 z[kFU], v[kFU];
    float w[kFU][OM];
#pragma unroll
    for (int u = 0; u < kFU; ++u) {  // (past the piece: its last unit, not used)
      const int k = u0 + u * NG < q.len ? u0 + u * NG : q.len - 1;
      const int64_t n = q.n0 + k;
      z[u] = *(const f32x4*)(Zt + n * Bp + bl);
      if (GATED) v[u] = *(const f32x4*)(Ut + n * Bp + bl);
      const float gn = NORM ? p.gain[n] : 1.f;
#pragma unroll
      for (int o = 0; o < OM; ++o) w[u][o] = o < p.O ? p.W2[(int64_t)o * p.ldw + n] * gn : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kFU; ++u) {
      if (u0 + u * NG >= q.len) break;
      cnt += 1.f;
      const float rc = NORM ? 1.f / cnt : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float h = blk_act(a, z[u][i]);
        if (GATED) h *= v[u][i];
        if (NORM) {
          if (cnt == 1.f) piv[i] = h;
          h -= piv[i];
          const float d = h - mean[i];
          mean[i] = fmaf(d, rc, mean[i]);
          m2[i] = fmaf(d, h - mean[i], m2[i]);
        }
#pragma unroll
        for (int o = 0; o < OM; ++o) S[i][o] = fmaf(h, w[u][o], S[i][o]);
      }
      if (NORM)
#pragma unroll
        for (int o = 0; o < OM; ++o) C[o] += w[u][o];
    }
  }
  if (NORM) {  // from the first unit's values to the mean as it is rounded
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mean[i] += piv[i];
#pragma unroll
      for (int o = 0; o < OM; ++o) S[i][o] = fmaf(piv[i] - mean[i], C[o], S[i][o]);
    }
  }
  for (int s = LG; s < 64; s <<= 1) {
    if (NORM) {
      const float nb = __shfl_xor(cnt, s);
      float n = cnt, Cb[OM];
#pragma unroll
      for (int o = 0; o < OM; ++o) Cb[o] = __shfl_xor(C[o], s);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ma = mean[i], mb = __shfl_xor(ma, s), qb = __shfl_xor(m2[i], s);
        n = cnt;
        merge_stats(n, mean[i], m2[i], nb, mb, qb);
        const float da = ma - mean[i], db = mb - mean[i];
#pragma unroll
        for (int o = 0; o < OM; ++o) {
          const float Sb = __shfl_xor(S[i][o], s);
          S[i][o] = fmaf(da, C[o], fmaf(db, Cb[o], S[i][o] + Sb));
        }
      }
#pragma unroll
      for (int o = 0; o < OM; ++o) C[o] += Cb[o];
      cnt = n;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int o = 0; o < OM; ++o) S[i][o] += __shfl_xor(S[i][o], s);
    }
  }
  if (NORM && blk == 0 && lane == 0) {
#pragma unroll
    for (int o = 0; o < OM; ++o)
      csum[(int64_t)pc * OM + o] = C[o];
  }
  if (g != 0 || !valid) return;
  float* dst = part + (int64_t)pc * (p.O + (NORM ? 2 : 0)) * Bp + b;
#pragma unroll
  for (int o = 0; o < OM; ++o)
    if (o < p.O) *(f32x4*)(dst + (int64_t)o * Bp) = f32x4{S[0][o], S[1][o], S[2][o], S[3][o]};
  if (NORM) {
    *(f32x4*)(dst + (int64_t)p.O * Bp) = f32x4{mean[0], mean[1], mean[2], mean[3]};
    *(f32x4*)(dst + (int64_t)(p.O + 1) * Bp) = f32x4{m2[0], m2[1], m2[2], m2[3]};
  }
}

// One workgroup for nb samples of a model, G groups of threads over its pieces, or
// (nb = 64, G = 1, alone) one wave.
template <int OM, bool NORM>
__global__ __launch_bounds__(1024) void k_blk_out(BlkPack p, BlkMap map,
                                                  const float* __restrict__ part,
                                                  const float* __restrict__ csum, int Br, int B,
                                                  int per, int nblk, int G, int alone,
                                                  float* __restrict__ out, int64_t sm, int64_t sb) {
  extern __shared__ float lds[];
  __shared__ float red[16 * 2 * OM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int64_t wk = alone ? (int64_t)blockIdx.x * nw + wave : blockIdx.x;
  const int m = (int)(wk / nblk);
  if (m >= p.M) return;
  const int b0 = (int)(wk - (int64_t)m * nblk) * per;
  const int nb = alone ? 64 : blockDim.x / G, g = alone ? 0 : tid / nb, l = alone ? lane : tid - g * nb;
  float C[OM], D[OM];
  if (NORM) norm_consts<OM>(p, m, lane, alone ? 0 : wave, alone ? 1 : nw, red, C, D);
  for (int s0 = b0; s0 < B && s0 < b0 + per; s0 += nb) {
    const int b = s0 + l < B ? s0 + l : B - 1;
    Merged<OM> s;
    merge_pieces<OM, NORM>(p, map, part, csum, m, Br, b, g, G, s);
    merge_groups<OM, NORM>(s, g, G, nb, l, lds);
    if (g > 0 || s0 + l >= B) continue;
    float r;
    if (NORM) apply_norm<OM>(s, C, &r);
#pragma unroll
    for (int o = 0; o < OM; ++o)
      if (o < p.O) out[(int64_t)b * sb + (int64_t)m * sm + o] = NORM ? s.P[o] + D[o] : s.P[o];
  }
}

// One workgroup per model, its threads over the samples and (G groups) its pieces.
template <int OM, bool NORM>
__global__ __launch_bounds__(1024) void k_blk_loss(BlkPack p, BlkMap map,
                                                   const float* __restrict__ part,
                                                   const float* __restrict__ csum, int Br, int Bp,
                                                   int G, BlkLoss l, float scale) {
  extern __shared__ float lds[];
  __shared__ float red[16 * (2 * OM + 1)];
  const int m = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
  const int nb = blockDim.x / G, g = tid / nb, at = tid - g * nb;
  const int B = l.B;
  float C[OM], D[OM];
  if (NORM) norm_consts<OM>(p, m, lane, wave, nw, red, C, D);
  const float rh = 1.f / (float)(p.seg_off[m + 1] - p.seg_off[m]);
  if (l.lrm && tid == 0 && !isfinite(l.lrm[m])) l.flag[1] = 1;
  float loss = 0.f, gs[OM];
#pragma unroll
  for (int o = 0; o < OM; ++o) gs[o] = 0.f;
  for (int s0 = 0; s0 < Bp; s0 += nb) {
    const int b = s0 + at;
    Merged<OM> s;
    merge_pieces<OM, NORM>(p, map, part, csum, m, Br, b < B ? b : B - 1, g, G, s);
    merge_groups<OM, NORM>(s, g, G, nb, at, lds);
    if (g > 0 || b >= Bp) continue;
    sample_grads<OM, NORM>(p, l, m, b, Bp, s, C, D, rh, scale, loss, gs);
  }
  loss = group_sum_to_last(loss, 64);
  if (NORM)
#pragma unroll
    for (int o = 0; o < OM; ++o) gs[o] = group_sum_to_last(gs[o], 64);
  __syncthreads();
  if (lane == 63) {
    red[16 * 2 * OM + wave] = loss;
#pragma unroll
    for (int o = 0; o < OM; ++o) red[wave * 2 * OM + o] = gs[o];
  }
  __syncthreads();
  if (tid == 0) {
    float s = 0.f;
    for (int w = 0; w < nw; ++w) s += red[16 * 2 * OM + w];
    l.loss[m] = s * scale;
    if (!isfinite(s)) atomicAdd(l.flag + 2, 1);
  }
  if (NORM && tid < p.O) {
    float s = 0.f;
    for (int w = 0; w < nw; ++w) s += red[w * 2 * OM + tid];
    l.Gs[(int64_t)m * p.O + tid] = s;
  }
}

// dZ over Z and dU over U; the gradients of W2, gain and shift.  LG lanes take a
// unit's samples, four each and 4 LG a pass.  Bound by reading and writing Z and U
// once, with many outputs by its vector instructions.
template <int OM, bool GATED, bool NORM>
__global__ __launch_bounds__(kBlock) void k_blk_bwd(BlkPack p, float* __restrict__ Zt,
                                                    float* __restrict__ Ut, int Bp, int LG,
                                                    const float* __restrict__ G,
                                                    const float* __restrict__ R,
                                                    const float* __restrict__ Gs, BlkGrads out) {
  const int lane = threadIdx.x & 63;
  const int64_t wv = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int NG = 64 / LG, g = lane / LG, l = lane - g * LG;
  const int64_t n = wv * NG + g;
  if (n >= p.N) return;
  const int m = p.mid[n], a = p.actn[n];
  const float gn = NORM ? p.gain[n] : 1.f;
  float w[OM], T[OM];
#pragma unroll
  for (int o = 0; o < OM; ++o) {
    w[o] = o < p.O ? p.W2[(int64_t)o * p.ldw + n] : 0.f;
    T[o] = 0.f;
  }
  for (int b = 4 * l; b < Bp; b += 4 * LG) {
    f32x4 z = *(const f32x4*)(Zt + n * Bp + b), u = f32x4{1.f, 1.f, 1.f, 1.f};
    if (GATED) u = *(const f32x4*)(Ut + n * Bp + b);
    const float* gr = G + ((int64_t)m * Bp + b) * OM;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float d;
      const float av = blk_act_slope(a, z[i], &d);
      float hv = GATED ? av * u[i] : av;
      f32x4 st;
      if (NORM) {
        st = *(const f32x4*)(R + ((int64_t)m * Bp + b + i) * 4);
        hv = (hv - st[0]) * st[1];
      }
      float dn = 0.f;
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        const float go = gr[i * OM + o];
        dn = fmaf(go, w[o], dn);
        T[o] = fmaf(go, hv, T[o]);
      }
      if (NORM) dn = st[1] * (gn * dn - st[2] - hv * st[3]);
      z[i] = dn * u[i] * d;
      u[i] = dn * av;
    }
    *(f32x4*)(Zt + n * Bp + b) = z;
    if (GATED) *(f32x4*)(Ut + n * Bp + b) = u;
  }
#pragma unroll
  for (int o = 0; o < OM; ++o) T[o] = group_sum_to_last(T[o], LG);
  if (l != LG - 1) return;
  blk_unit_grads<OM, NORM>(p, out, Gs, n, m, gn, w, T);
}

__global__ __launch_bounds__(kBlock) void k_blk_init(float* V1, int64_t N, int F, int F4, float bound,
                                                     uint64_t key, float* gain, float* shift) {
  const int64_t step = (int64_t)gridDim.x * kBlock, i0 = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (V1)
    for (int64_t i = i0; i < N * F; i += step) {
      const int64_t n = i / F;
      V1[n * F4 + (i - n * F)] = uniform_weight(key, 6, (uint64_t)i, bound);
    }
  if (gain)
    for (int64_t i = i0; i < N; i += step) {
      gain[i] = 1.f;
      shift[i] = 0.f;
    }
}

// lanes per unit: four samples each, at most a wave
int lanes_per_unit(int32_t Bp) {
  int lg = 4;
  while (lg < 64 && 4 * lg < Bp) lg <<= 1;
  return lg;
}

}  // namespace

#define PMLP_BLK_OM(O, CALL) \
  do {                       \
    if ((O) <= 2) CALL(2);   \
    else if ((O) <= 4) CALL(4); \
    else CALL(16);           \
  } while (0)

hipError_t launch_blk_fwd(const BlkPack& p, const float* Zt, const float* Ut, int32_t Bp,
                          float* part, float* csum, hipStream_t s) {
  note_variant("k_blk_fwd", kArithNone);
  const int LG = lanes_per_unit(Bp), nb = ceil_div_i(Bp, 4 * LG);
  const int64_t waves = (int64_t)p.npieces * nb;
  if (waves > (int64_t)0x3fffffff) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)ceil_div_i(waves, 4);
#define PMLP_CALL(OM)                                                                        \
  do {                                                                                       \
    if (Ut && p.gain) k_blk_fwd<OM, true, true><<<grid, kBlock, 0, s>>>(p, Zt, Ut, Bp, LG, nb, part, csum); \
    else if (Ut) k_blk_fwd<OM, true, false><<<grid, kBlock, 0, s>>>(p, Zt, Ut, Bp, LG, nb, part, csum);     \
    else k_blk_fwd<OM, false, true><<<grid, kBlock, 0, s>>>(p, Zt, Ut, Bp, LG, nb, part, csum);     \
  } while (0)
  PMLP_BLK_OM(p.O, PMLP_CALL);
#undef PMLP_CALL
  return hipGetLastError();
}

// Groups of threads over a model's pieces: by the pieces of an average model, one where
// the models alone fill the device.  Wide models, both, two outputs, 32 samples, the
// loss kernel in us with 1, 2, 4 and 8 groups: one model of 20,000 units 237, 129, 72,
// 44; 64 of 2000 19, 14, 11, 10; 1000 of 1000 16, 13, 12, 18; ten outputs and 256
// samples, 1000 of 1000: 58, 69, 123, 123.
static int piece_groups(const BlkPack& p, int64_t records, int most) {
  const int64_t pieces = records / p.M;
  int G = 1;
  while (G < most && pieces >= 8 * G && (int64_t)p.M * G < 512) G <<= 1;
  return G;
}

static size_t groups_lds(const BlkPack& p, int G, int nb) {
  return (size_t)(G - 1) * nb * (blk_om(p.O) + 3) * sizeof(float);
}

hipError_t launch_blk_out(const BlkPack& p, const BlkMap& map, int64_t records, const float* part,
                          int32_t Br, int32_t B, float* out, int64_t sm, int64_t sb, hipStream_t s) {
  note_variant("k_blk_out", kArithNone);
  const int G = piece_groups(p, records, 16), alone = G == 1, nb = 64;
  int per = 1024;  // samples of a model at once: fewer where that leaves the device idle
  while (per > nb && (int64_t)p.M * ceil_div_i(B, per) < (alone ? 8192 : 1024)) per >>= 1;
  const int nblk = ceil_div_i(B, per), threads = alone ? 256 : nb * G;
  const int64_t grid = alone ? ((int64_t)p.M * nblk + 3) / 4 : (int64_t)p.M * nblk;
  if (grid > (int64_t)0x7fffffff) return hipErrorInvalidValue;
  const size_t lds = groups_lds(p, G, nb);
#define PMLP_CALL(OM)                                                                          \
  do {                                                                                         \
    if (p.gain)                                                                                \
      k_blk_out<OM, true><<<(unsigned)grid, threads, lds, s>>>(p, map, part, map.csum, Br, B, per, nblk, G, \
                                                               alone, out, sm, sb);             \
    else                                                                                       \
      k_blk_out<OM, false><<<(unsigned)grid, threads, lds, s>>>(p, map, part, map.csum, Br, B, per, nblk, \
                                                                G, alone, out, sm, sb);         \
  } while (0)
  PMLP_BLK_OM(p.O, PMLP_CALL);
#undef PMLP_CALL
  return hipGetLastError();
}

hipError_t launch_blk_loss(const BlkPack& p, const BlkMap& map, int64_t records, const float* part,
                           int32_t Br, int32_t Bp, const BlkLoss& l, hipStream_t s) {
  note_variant("k_blk_loss", kArithNone);
  const int nb = Bp >= 256 ? 256 : (Bp + 63) & ~63;
  const int most = 1024 / nb, G = piece_groups(p, records, most >= 8 ? 8 : most >= 4 ? 4 : most >= 2 ? 2 : 1);
  const int threads = G == 1 && Bp >= 1024 ? 1024 : nb * G;
  const size_t lds = groups_lds(p, G, threads / G);
  const float scale = l.Y ? 1.f / ((float)l.B * (float)p.O) : 1.f / (float)l.B;
#define PMLP_CALL(OM)                                                                              \
  do {                                                                                             \
    if (p.gain)                                                                                    \
      k_blk_loss<OM, true><<<(unsigned)p.M, threads, lds, s>>>(p, map, part, map.csum, Br, Bp, G, l, scale);  \
    else                                                                                           \
      k_blk_loss<OM, false><<<(unsigned)p.M, threads, lds, s>>>(p, map, part, map.csum, Br, Bp, G, l, scale); \
  } while (0)
  PMLP_BLK_OM(p.O, PMLP_CALL);
#undef PMLP_CALL
  return hipGetLastError();
}

hipError_t launch_blk_bwd(const BlkPack& p, float* Zt, float* Ut, int32_t Bp, const float* G,
                          const float* R, const float* Gs, const BlkGrads& g, hipStream_t s) {
  note_variant("k_blk_bwd", kArithNone);
  const int LG = lanes_per_unit(Bp);
  const int64_t waves = (p.N + 64 / LG - 1) / (64 / LG);
  if (waves > (int64_t)0x7ffffff0) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)ceil_div_i(waves, 4);
#define PMLP_CALL(OM)                                                                           \
  do {                                                                                          \
    if (Ut && p.gain)                                                                           \
      k_blk_bwd<OM, true, true><<<grid, kBlock, 0, s>>>(p, Zt, Ut, Bp, LG, G, R, Gs, g);         \
    else if (Ut)                                                                                \
      k_blk_bwd<OM, true, false><<<grid, kBlock, 0, s>>>(p, Zt, Ut, Bp, LG, G, R, Gs, g);        \
    else                                                                                        \
      k_blk_bwd<OM, false, true><<<grid, kBlock, 0, s>>>(p, Zt, Ut, Bp, LG, G, R, Gs, g);        \
  } while (0)
  PMLP_BLK_OM(p.O, PMLP_CALL);
#undef PMLP_CALL
  return hipGetLastError();
}

hipError_t launch_blk_init(float* V1, int64_t N, int32_t F, int32_t F4, float bound, uint64_t key,
                           float* gain, float* shift, hipStream_t s) {
  const int64_t n = V1 ? N * F : N;
  k_blk_init<<<grid_for(n), kBlock, 0, s>>>(V1, N, F, F4, bound, key, gain, shift);
  return hipGetLastError();
}

}  // namespace pmlpk
