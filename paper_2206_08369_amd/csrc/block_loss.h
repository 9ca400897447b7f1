// Block packs: a model's outputs, losses and output gradients from the sums over its
// pieces (see k_block.hip).
#pragma once

#include "block_device.h"

namespace pmlpk {

// C_o and D_o of model m, summed by the waves of a workgroup (wave of nw) through
// `red`, or by one wave for itself (nw = 1).
template <int OM>
__device__ __forceinline__ void norm_consts(const BlkPack& p, int m, int lane, int wave, int nw,
                                            float* red, float (&C)[OM], float (&D)[OM]) {
#pragma unroll
  for (int o = 0; o < OM; ++o) C[o] = D[o] = 0.f;
  const int64_t e = p.seg_off[m + 1];
  for (int64_t n0 = p.seg_off[m] + 64 * wave; n0 < e; n0 += 128 * nw) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // (two units' loads in flight)
      const int64_t k = n0 + 64 * nw * u + lane, n = k < e ? k : e - 1;
      const float gn = p.gain[n], sn = p.shift[n];
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        const float w = p.W2[(int64_t)(o < p.O ? o : 0) * p.ldw + n];
        C[o] = fmaf(k < e ? gn : 0.f, w, C[o]);
        D[o] = fmaf(k < e ? sn : 0.f, w, D[o]);
      }
    }
  }
#pragma unroll
  for (int o = 0; o < OM; ++o) {
    C[o] = group_sum_to_last(C[o], 64);
    D[o] = group_sum_to_last(D[o], 64);
  }
  if (nw == 1) {
#pragma unroll
    for (int o = 0; o < OM; ++o) {
      C[o] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(C[o]), 63));
      D[o] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(D[o]), 63));
    }
    return;
  }
  if (lane == 63) {
#pragma unroll
    for (int o = 0; o < OM; ++o) {
      red[wave * 2 * OM + o] = C[o];
      red[wave * 2 * OM + OM + o] = D[o];
    }
  }
  __syncthreads();
#pragma unroll
  for (int o = 0; o < OM; ++o) {
    C[o] = D[o] = 0.f;
    for (int w = 0; w < nw; ++w) {
      C[o] += red[w * 2 * OM + o];
      D[o] += red[w * 2 * OM + OM + o];
    }
  }
  __syncthreads();
}

// A model's sums for one sample over some of its pieces.
template <int OM>
struct Merged {
  float P[OM], n, mean, m2;
  float piv;  // with a norm: the first piece's mean, from which `mean` and P count
};

// Those of pieces k0 + g, k0 + g + G, .. of model m (uniform over a wave), four pieces'
// loads in flight.  A piece's deviations from its own mean m_k become deviations from
// the first piece's by (m_k - piv) C_k: the hidden values' mean itself, which may be
// large beside their deviations, is in none of the sums.
template <int OM, bool NORM>
__device__ __forceinline__ void merge_pieces(const BlkPack& p, const BlkMap& map,
                                             const float* part, const float* csum, int m, int Br,
                                             int b, int g, int G, Merged<OM>& s) {
  s.n = s.mean = s.m2 = 0.f;
#pragma unroll
  for (int o = 0; o < OM; ++o) s.P[o] = 0.f;
  int k0, k1, t0 = 0;  // its pieces or records
  if (map.toff) {
    t0 = map.toff[m];
    k0 = m + t0 / map.run;
    k1 = m + (map.toff[m + 1] - 1) / map.run + 1;
  } else {
    k0 = p.poff[m];
    k1 = p.poff[m + 1];
  }
  const int width = (int)(p.seg_off[m + 1] - p.seg_off[m]);
  s.piv = NORM ? part[((int64_t)k0 * (p.O + 2) + p.O) * Br + b] : 0.f;
  constexpr int U = OM <= 4 ? 4 : 2;
  for (int k = k0 + g; k < k1; k += U * G) {
    float v[U][OM], c[NORM ? U : 1][OM], mb[U], qb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (past the last: it again, not used)
      const int ku = k + u * G < k1 ? k + u * G : k1 - 1;
      const float* src = part + (int64_t)ku * (p.O + (NORM ? 2 : 0)) * Br + b;
#pragma unroll
      for (int o = 0; o < OM; ++o) v[u][o] = src[(int64_t)(o < p.O ? o : 0) * Br];
      if (NORM) {
        mb[u] = src[(int64_t)p.O * Br] - s.piv;
        qb[u] = src[(int64_t)(p.O + 1) * Br];
        const float* const cs = csum + (int64_t)(OM > 4 ? __builtin_amdgcn_readfirstlane(ku) : ku) * OM;
#pragma unroll
        for (int o = 0; o < OM; ++o) c[NORM ? u : 0][o] = cs[o];
      }
    }
    if (NORM && OM <= 4)  // (made with the other loads, not each where it is used)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int o = 0; o < OM; ++o) c[NORM ? u : 0][o] = opaque(c[NORM ? u : 0][o]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k + u * G >= k1) break;
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        s.P[o] += v[u][o];
        if (NORM) s.P[o] = fmaf(mb[u], c[NORM ? u : 0][o], s.P[o]);
      }
      if (NORM) {
        const int ku = k + u * G;
        int units;
        if (map.toff) {  // (from the run's first tile, or the model's, to its last)
          const int at = max((ku - m) * map.run - t0, 0);
          units = (int)min((uint32_t)width, 16u * ((ku - m + 1) * map.run - t0)) - 16 * at;
        } else {
          units = p.pieces[ku].len;
        }
        merge_stats(s.n, s.mean, s.m2, (float)units, mb[u], qb[u]);
      }
    }
  }
}

// The groups g of a workgroup (G of them, nb threads each) merge what each has for
// the same sample, in the order of g; group 0 ends with the whole.
template <int OM, bool NORM>
__device__ __forceinline__ void merge_groups(Merged<OM>& s, int g, int G, int nb, int l,
                                             float* lds) {
  if (G == 1) return;
  constexpr int W = OM + 3;
  if (g > 0) {
    float* d = lds + (size_t)(g - 1) * W * nb + l;
#pragma unroll
    for (int o = 0; o < OM; ++o) d[o * nb] = s.P[o];
    d[OM * nb] = s.n;
    d[(OM + 1) * nb] = s.mean;
    d[(OM + 2) * nb] = s.m2;
  }
  __syncthreads();
  if (g == 0) {
    for (int k = 0; k < G - 1; ++k) {
      const float* d = lds + (size_t)k * W * nb + l;
#pragma unroll
      for (int o = 0; o < OM; ++o) s.P[o] += d[o * nb];
      if (NORM) merge_stats(s.n, s.mean, s.m2, d[OM * nb], d[(OM + 1) * nb], d[(OM + 2) * nb]);
    }
  }
  __syncthreads();
}

// With a norm: the statistics (mean: the hidden values' own), and P_o.  r = 0 for a model of one unit, whose norm is
// constant, so that its gradient is exactly zero.
template <int OM>
__device__ __forceinline__ void apply_norm(Merged<OM>& s, const float (&C)[OM], float* r) {
  *r = s.n > 1.f ? 1.f / sqrtf(s.m2 / s.n + kNormEps) : 0.f;
#pragma unroll
  for (int o = 0; o < OM; ++o) s.P[o] = *r * (s.P[o] - s.mean * C[o]);
  s.mean += s.piv;
}

// One sample's logits (s: its merged sums), share of the loss, dLoss/dlogits G and
// what the backward needs of the norm (R), stored; past the batch zeros.
template <int OM, bool NORM>
__device__ __forceinline__ void sample_grads(const BlkPack& p, const BlkLoss& l, int m, int b, int Bp,
                                             Merged<OM>& s, const float (&C)[OM],
                                             const float (&D)[OM], float rh, float scale, float& loss,
                                             float (&gs)[OM]) {
  float Gr[OM], r = 0.f, a1 = 0.f, a2 = 0.f;
  if (b < l.B) {
    if (NORM) apply_norm<OM>(s, C, &r);
    float L[OM];
#pragma unroll
    for (int o = 0; o < OM; ++o) L[o] = NORM ? s.P[o] + D[o] : s.P[o];
    if (l.Y) {
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        const float d = o < p.O ? L[o] - l.Y[(int64_t)b * p.O + (o < p.O ? o : 0)] : 0.f;
        loss = fmaf(d, d, loss);
        Gr[o] = 2.f * d * scale;
      }
    } else {
      // e_o / sum e, and for the label minus the others' share of it, so that a
      // sample's gradients add up to zero (shift's are sums of them over the batch)
      float mx = -INFINITY, se = 0.f, rest = 0.f, ly = 0.f;
#pragma unroll
      for (int o = 0; o < OM; ++o) mx = o < p.O ? fmaxf(mx, L[o]) : mx;
      const int yb = l.y[b];
      if (yb < 0 || yb >= p.O) l.flag[0] = 1;
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        Gr[o] = o < p.O ? expf(L[o] - mx) : 0.f;
        se += Gr[o];
        rest += o == yb ? 0.f : Gr[o];
        if (o == yb) ly = L[o];
      }
      const float lse = mx + logf(se), share = scale / se;
#pragma unroll
      for (int o = 0; o < OM; ++o) Gr[o] = (o == yb ? -rest : Gr[o]) * share;
      loss += lse - ly;
    }
    if (NORM) {
#pragma unroll
      for (int o = 0; o < OM; ++o) {
        gs[o] += Gr[o];
        a1 = fmaf(Gr[o], C[o], a1);
        a2 = fmaf(Gr[o], s.P[o], a2);
      }
    }
  } else {
    s.mean = 0.f;
#pragma unroll
    for (int o = 0; o < OM; ++o) Gr[o] = 0.f;
  }
  float* row = l.G + ((int64_t)m * Bp + b) * OM;
#pragma unroll
  for (int o = 0; o < OM; o += 2) *(f32x2*)(row + o) = f32x2{Gr[o], Gr[o + 1]};
  if (NORM) *(f32x4*)(l.R + ((int64_t)m * Bp + b) * 4) = f32x4{s.mean, r, a1 * rh, a2 * rh};
}

}  // namespace pmlpk
