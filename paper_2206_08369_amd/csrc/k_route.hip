// Routing: the K best models of each sample, and the slots grouped by model.

#include "device_common.h"
#include "routed.h"

namespace pmlpk {

namespace {

// Scores in the order of choice as unsigned numbers: a higher score first, of equal
// ones the lower index (-0 equals +0).  0 stands for -inf and NaN, which are never chosen.
__device__ __forceinline__ uint64_t score_key(float s, int m) {
  if (!(s > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(s == 0.f ? 0.f : s);
  const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return ((uint64_t)o << 32) | (uint32_t)~m;
}
__device__ __forceinline__ float key_score(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)v, d);
    v = o > v ? o : v;
  }
  return v;
}

}  // namespace

// One round per choice: the best key below the last one.  The row is read once a round,
// from cache after the first.  T threads a row.
template <int T>
__global__ __launch_bounds__(256) void k_route(const float* __restrict__ scores, int B, int M, int K,
                                               int32_t* __restrict__ idx, float* __restrict__ weight) {
  __shared__ uint64_t best[4];
  const int t = threadIdx.x % T, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = (int64_t)blockIdx.x * (256 / T) + threadIdx.x / T;
  if (T == 64 && b >= B) return;  // (a row is one wave: no barrier below)
  const float* row = scores + b * M;
  uint64_t last = ~0ull, mine = 0;
  for (int k = 0; k < K; ++k) {
    uint64_t top = 0;
    for (int m = t; m < M; m += T) {
      const uint64_t key = score_key(row[m], m);
      top = key < last && key > top ? key : top;
    }
    top = wave_max(top);
    if (T > 64) {
      __syncthreads();
      if (lane == 0) best[wave] = top;
      __syncthreads();
      for (int w = 0; w < T / 64; ++w) top = best[w] > top ? best[w] : top;
    }
    if (lane == k) mine = top;
    last = top;  // 0: none left, and none below it
  }
  if (t >= 64) return;
  const float top = __shfl(key_score(mine), 0);
  const float e = lane < K && mine ? expf(key_score(mine) - top) : 0.f;
  float sum = 0.f;
  for (int k = 0; k < K; ++k) sum += __shfl(e, k);
  if (lane >= K) return;
  idx[b * K + lane] = mine ? (int32_t)~(uint32_t)mine : -1;
  weight[b * K + lane] = mine ? e / sum : 0.f;
}

hipError_t launch_route(const float* scores, int32_t B, int32_t M, int32_t K, int32_t* idx,
                        float* weight, hipStream_t s) {
  note_variant("k_route", kArithNone);
  if (M <= 1024) k_route<64><<<(unsigned)((B + 3) / 4), 256, 0, s>>>(scores, B, M, K, idx, weight);
  else k_route<256><<<(unsigned)B, 256, 0, s>>>(scores, B, M, K, idx, weight);
  return hipGetLastError();
}

// ds_k = w_k (dw_k - sum_j w_j dw_j), the gradient of a softmax, at the chosen scores.
__global__ __launch_bounds__(256) void k_route_bwd(const int32_t* __restrict__ idx,
                                                   const float* __restrict__ weight,
                                                   const float* __restrict__ dweight, int B, int M,
                                                   int K, float* __restrict__ dscores) {
  const int lane = threadIdx.x & 63;
  const int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b >= B) return;
  const bool on = lane < K;
  const int i = on ? idx[b * K + lane] : -1;
  const bool live = on && i >= 0 && i < M;
  const float w = live ? weight[b * K + lane] : 0.f, d = live ? dweight[b * K + lane] : 0.f;
  float mean = 0.f;
  for (int k = 0; k < K; ++k) mean = fmaf(__shfl(w, k), __shfl(d, k), mean);
  const float ds = w * (d - mean);
  for (int m0 = 0; m0 < M; m0 += 64) {
    const int m = m0 + lane;
    float v = 0.f;
    for (int k = 0; k < K; ++k) {
      const float s = __shfl(ds, k);
      if (__shfl(i, k) == m) v += s;
    }
    if (m < M) dscores[b * M + m] = v;
  }
}

hipError_t launch_route_bwd(const int32_t* idx, const float* weight, const float* dweight, int32_t B,
                            int32_t M, int32_t K, float* dscores, hipStream_t s) {
  note_variant("k_route_bwd", kArithNone);
  k_route_bwd<<<(unsigned)((B + 3) / 4), 256, 0, s>>>(idx, weight, dweight, B, M, K, dscores);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Grouping: a counting sort that keeps the order of slots.  Each of up to 256 waves
// walks a run of slots, 64 at a time; a column of `hist` says where each run's rows of a
// model start.  A wave's counters are its own, and it waits for each of its additions.
// ---------------------------------------------------------------------------

namespace {

__device__ __forceinline__ int slot_model(const RtPlan& p, int64_t s, int64_t end, bool report) {
  if (s >= end) return -1;
  const int m = p.idx[s];
  if (m >= 0 && m < p.M) return m;
  if (report && m != -1) p.flag[3] = 1;
  return -1;
}

// The lanes with this lane's model.
__device__ __forceinline__ uint64_t peers_of(int m) {
  uint64_t todo = __ballot(m >= 0), peers = 0;
  while (todo) {
    const int key = __shfl(m, __ffsll((unsigned long long)todo) - 1);
    const uint64_t same = __ballot(m == key);
    if (m == key) peers = same;
    todo &= ~same;
  }
  return peers;
}

// Walks run c: `take(slot, model, rank in counter)` for each slot with a model.
template <class Take>
__device__ __forceinline__ void walk(const RtPlan& p, int c, int32_t* counter, bool report, Take take) {
  const int lane = threadIdx.x & 63;
  const int64_t first = (int64_t)c * p.chunk;
  const int64_t end = first + p.chunk < p.R ? first + p.chunk : p.R;
  for (int64_t s0 = first; s0 < end; s0 += 64) {
    const int m = slot_model(p, s0 + lane, end, report);
    const uint64_t peers = peers_of(m);
    const int leader = peers ? __ffsll((unsigned long long)peers) - 1 : lane;
    int base = 0;
    if (peers && lane == leader) base = atomicAdd(counter + m, __popcll(peers));
    base = __shfl(base, leader);
    if (m >= 0) take(s0 + lane, m, base + __popcll(peers & ((1ull << lane) - 1)));
  }
}

}  // namespace

__global__ __launch_bounds__(64) void k_rt_count(RtPlan p) {
  extern __shared__ int32_t lds[];
  const int c = blockIdx.x;
  int32_t* row = p.hist + (int64_t)c * p.M;
  const bool in_lds = p.M <= kRtLdsModels;
  int32_t* counter = in_lds ? lds : row;
  for (int m = threadIdx.x; m < p.M; m += 64) counter[m] = 0;
  __threadfence_block();
  __syncthreads();
  walk(p, c, counter, true, [](int64_t, int, int) {});
  __syncthreads();
  if (in_lds)
    for (int m = threadIdx.x; m < p.M; m += 64) row[m] = lds[m];
  // no slot yet
  for (int64_t i = (int64_t)c * 64 + threadIdx.x; i < p.P; i += (int64_t)gridDim.x * 64) p.slot[i] = -1;
}

__global__ __launch_bounds__(256) void k_rt_columns(RtPlan p) {
  const int m = blockIdx.x * 256 + threadIdx.x;
  if (m >= p.M) return;
  int sum = 0;
  for (int c = 0; c < p.nchunk; ++c) {
    int32_t* at = p.hist + (int64_t)c * p.M + m;
    const int n = *at;
    *at = sum;
    sum += n;
  }
  p.count[m] = sum;
}

namespace {

__device__ __forceinline__ int up(int a, int b) { return (a + b - 1) / b; }

// Exclusive sums over the 1,024 threads of a workgroup of four numbers each.
struct Sums {
  int32_t place, item, jitem;
  int64_t z;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return Sums{a.place + b.place, a.item + b.item, a.jitem + b.jitem, a.z + b.z};
}

__device__ __forceinline__ Sums model_sums(const RtPlan& p, int m) {
  const int n = p.count[m], rows = up(n, kRtPad) * kRtPad;
  const int h = (int)(p.seg_off[m + 1] - p.seg_off[m]);
  Sums s;
  s.place = rows;
  s.item = up(n, p.t.rt) * up(h, p.t.uc);
  s.jitem = p.jitems ? (n ? up(rows, p.t.part) : 1) * up(h, p.t.du) * up(p.F, p.t.df) : 0;
  s.z = (int64_t)rows * h;
  return s;
}

}  // namespace

__global__ __launch_bounds__(1024) void k_rt_scan(RtPlan p) {
  __shared__ Sums lds[1024];
  const int t = threadIdx.x, each = up(p.M, 1024);
  const int m0 = t * each < p.M ? t * each : p.M, m1 = m0 + each < p.M ? m0 + each : p.M;
  Sums mine{0, 0, 0, 0};
  for (int m = m0; m < m1; ++m) mine = mine + model_sums(p, m);
  lds[t] = mine;
  __syncthreads();
  for (int d = 1; d < 1024; d <<= 1) {
    Sums v = lds[t];
    if (t >= d) v = v + lds[t - d];
    __syncthreads();
    lds[t] = v;
    __syncthreads();
  }
  Sums at = t ? lds[t - 1] : Sums{0, 0, 0, 0};
  for (int m = m0; m < m1; ++m) {
    p.place[m] = at.place;
    p.zoff[m] = at.z;
    p.ioff[m] = at.item;
    p.joff[m] = at.jitem;
    at = at + model_sums(p, m);
  }
  if (t == 1023) {
    p.place[p.M] = at.place;
    p.zoff[p.M] = at.z;
    p.ioff[p.M] = at.item;
    p.joff[p.M] = at.jitem;
  }
}

// The first nchunk workgroups put the slots into their places, the others list items, a
// model each.
__global__ __launch_bounds__(64) void k_rt_place(RtPlan p) {
  extern __shared__ int32_t lds[];
  const int lane = threadIdx.x;
  if ((int)blockIdx.x < p.nchunk) {
    const int c = blockIdx.x;
    int32_t* row = p.hist + (int64_t)c * p.M;
    const bool in_lds = p.M <= kRtLdsModels;
    if (in_lds)
      for (int m = lane; m < p.M; m += 64) lds[m] = row[m];
    __syncthreads();
    walk(p, c, in_lds ? lds : row, false,
         [&](int64_t s, int m, int r) { p.slot[p.place[m] + r] = (int32_t)s; });
    return;
  }
  const int m = blockIdx.x - p.nchunk;
  const int h = (int)(p.seg_off[m + 1] - p.seg_off[m]);
  const int nu = up(h, p.t.uc), i0 = p.ioff[m], n = p.ioff[m + 1] - i0;
  for (int i = lane; i < n; i += 64) p.items[i0 + i] = RtItem{m, i / nu, i % nu, 0};
  if (!p.jitems) return;
  const int nt = up(h, p.t.du), nf = up(p.F, p.t.df), j0 = p.joff[m], k = p.joff[m + 1] - j0;
  for (int i = lane; i < k; i += 64) p.jitems[j0 + i] = RtItem{m, i / nf % nt, i % nf, i / nf / nt};
}

hipError_t launch_rt_plan(const RtPlan& p, hipStream_t s) {
  note_variant("k_rt_place", kArithNone);
  const size_t lds = p.M <= kRtLdsModels ? (size_t)p.M * sizeof(int32_t) : 0;
  k_rt_count<<<p.nchunk, 64, lds, s>>>(p);
  k_rt_columns<<<(unsigned)ceil_div_i(p.M, 256), 256, 0, s>>>(p);
  k_rt_scan<<<1, 1024, 0, s>>>(p);
  k_rt_place<<<(unsigned)(p.nchunk + p.M), 64, lds, s>>>(p);
  return hipGetLastError();
}

}  // namespace pmlpk
