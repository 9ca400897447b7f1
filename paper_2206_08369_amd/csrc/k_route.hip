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

// The largest of the wave's values, in every lane (zeros come in from outside a row)
template <int CTRL, int ROWMASK>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  const uint32_t o = __builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWMASK, 0xf, true);
  return o > v ? o : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = dpp_max<0x111, 0xf>(v);  // row_shr:1, 2, 4, 8
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);  // row_bcast:15 into rows 1 and 3
  v = dpp_max<0x143, 0xc>(v);  // row_bcast:31 into rows 2 and 3
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  const uint32_t hi = wave_max((uint32_t)(v >> 32));
  const uint32_t lo = wave_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return ((uint64_t)hi << 32) | lo;
}

}  // namespace

// One round per choice: the best key below the last one.  T threads a row, E scores a
// thread in registers (0: more than fit, read again from cache in every round); only the
// thread that held the last choice looks for its next best.  6,000 scores of 32 samples,
// four choices: 19 us where every round read them again, 8 so.  (E as small as the row allows:
// 1,824 scores of 5,377 samples 47 us with 32, 18 with 8.)
template <int T, int E>
__global__ __launch_bounds__(256) void k_route(const float* __restrict__ scores, int B, int M, int K,
                                               int32_t* __restrict__ idx, float* __restrict__ weight) {
  __shared__ uint64_t best[2][4];
  const int t = threadIdx.x % T, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t b = (int64_t)blockIdx.x * (256 / T) + threadIdx.x / T;
  if (T == 64 && b >= B) return;  // (a row is one wave: no barrier below)
  const float* row = scores + b * M;
  float v[E > 0 ? E : 1];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = t + T * e < M ? row[t + T * e] : -INFINITY;
  auto own_best = [&](uint64_t last) {
    uint64_t top = 0;
    if (E > 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint64_t key = score_key(v[e], t + T * e);
        top = key < last && key > top ? key : top;
      }
    } else {
      for (int m = t; m < M; m += T) {
        const uint64_t key = score_key(row[m], m);
        top = key < last && key > top ? key : top;
      }
    }
    return top;
  };
  uint64_t own = own_best(~0ull), mine = 0;
  for (int k = 0; k < K; ++k) {
    uint64_t top = wave_max(own);
    if (T > 64) {
      if (lane == 0) best[k & 1][wave] = top;
      __syncthreads();
      for (int w = 0; w < T / 64; ++w) top = best[k & 1][w] > top ? best[k & 1][w] : top;
    }
    if (lane == k) mine = top;
    if (top == 0) break;  // none left
    if (own == top) own = own_best(top);
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
  const unsigned waves = (unsigned)((B + 3) / 4);
  if (M <= 256) k_route<64, 4><<<waves, 256, 0, s>>>(scores, B, M, K, idx, weight);
  else if (M <= 1024) k_route<64, 16><<<waves, 256, 0, s>>>(scores, B, M, K, idx, weight);
  else if (M <= 2048) k_route<256, 8><<<(unsigned)B, 256, 0, s>>>(scores, B, M, K, idx, weight);
  else if (M <= 4096) k_route<256, 16><<<(unsigned)B, 256, 0, s>>>(scores, B, M, K, idx, weight);
  else if (M <= 8192) k_route<256, 32><<<(unsigned)B, 256, 0, s>>>(scores, B, M, K, idx, weight);
  else k_route<256, 0><<<(unsigned)B, 256, 0, s>>>(scores, B, M, K, idx, weight);
  return hipGetLastError();
}

// ds_k = w_k (dw_k - sum_j w_j dw_j), the gradient of a softmax, at the chosen scores.  K is
// KM at most.
template <int KM>
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
  // (the choices as scalars: a comparison and an addition each for 64 scores)
  int ck[KM];
  float cs[KM];
#pragma unroll
  for (int k = 0; k < KM; ++k) {
    ck[k] = k < K ? __builtin_amdgcn_readlane(i, k) : -1;
    cs[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ds), k));
  }
#pragma unroll 4
  for (int m = lane; m < M; m += 64) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < KM; ++k) v += ck[k] == m ? cs[k] : 0.f;
    dscores[b * M + m] = v;
  }
}

hipError_t launch_route_bwd(const int32_t* idx, const float* weight, const float* dweight, int32_t B,
                            int32_t M, int32_t K, float* dscores, hipStream_t s) {
  note_variant("k_route_bwd", kArithNone);
  const unsigned grid = (unsigned)((B + 3) / 4);
  if (K <= 2) k_route_bwd<2><<<grid, 256, 0, s>>>(idx, weight, dweight, B, M, K, dscores);
  else if (K <= 4) k_route_bwd<4><<<grid, 256, 0, s>>>(idx, weight, dweight, B, M, K, dscores);
  else if (K <= 8) k_route_bwd<8><<<grid, 256, 0, s>>>(idx, weight, dweight, B, M, K, dscores);
  else k_route_bwd<kRtMaxK><<<grid, 256, 0, s>>>(idx, weight, dweight, B, M, K, dscores);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Grouping: a counting sort that keeps the order of slots.  Each of up to 256 waves
// walks a run of slots, 64 at a time; a column of `hist` says where each run's rows of a
// model start.  A wave's counters are its own, and it waits for each of its additions.  Bound
// by latency: 32,768 slots, 600 models 5.4 us to count, 3.7 for the columns, 4.4 for the
// scan and 8.7 to place and list.
// ---------------------------------------------------------------------------

namespace {

__device__ __forceinline__ int slot_model(const RtPlan& p, int64_t s, int64_t end, bool report) {
  if (s >= end) return -1;
  const int m = p.idx[s];
  if (m >= 0 && m < p.M) return m;
  if (report && m != -1) p.flag[3] = 1;
  return -1;
}

// The lanes with this lane's model, of M: bit by bit, those that agree.
__device__ __forceinline__ uint64_t peers_of(int m, int M) {
  uint64_t peers = __ballot(m >= 0);
  for (int bit = 0; (M - 1) >> bit; ++bit) {
    const bool on = m >> bit & 1;
    const uint64_t ones = __ballot(on);
    peers &= on ? ones : ~ones;
  }
  return m >= 0 ? peers : 0;
}

// Walks run c: `take(slot, model, rank in counter)` for each slot with a model.
template <class Take>
__device__ __forceinline__ void walk(const RtPlan& p, int c, int32_t* counter, bool report, Take take) {
  const int lane = threadIdx.x & 63;
  const int64_t first = (int64_t)c * p.chunk;
  const int64_t end = first + p.chunk < p.R ? first + p.chunk : p.R;
  for (int64_t s0 = first; s0 < end; s0 += 64) {
    const int m = slot_model(p, s0 + lane, end, report);
    const uint64_t peers = peers_of(m, p.M);
    const int leader = peers ? __ffsll((unsigned long long)peers) - 1 : lane;
    int base = 0;
    if (peers && lane == leader) base = atomicAdd(counter + m, __popcll(peers));
    base = __shfl(base, leader);
    if (m >= 0) take(s0 + lane, m, base + __popcll(peers & ((1ull << lane) - 1)));
  }
}

// Places hold no slot yet.
__device__ __forceinline__ void clear_places(const RtPlan& p, int64_t first, int64_t stride) {
  for (int64_t i = first; i < p.P; i += stride) {
    p.slot[i] = -1;
    p.row[i] = -1;
    if (p.wdy)
      for (int o = 0; o < p.O; ++o) p.wdy[(int64_t)o * p.P + i] = 0.f;
  }
}

__device__ __forceinline__ void put_slot(const RtPlan& p, int64_t s, int at) {
  const int64_t b = s / p.K;
  p.slot[at] = (int32_t)s;
  p.row[at] = (int32_t)b;
  if (!p.wdy) return;
  const float w = p.weight[s];
  for (int o = 0; o < p.O; ++o) p.wdy[(int64_t)o * p.P + at] = w * p.dY[b * p.O + o];
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
  clear_places(p, (int64_t)c * 64 + threadIdx.x, (int64_t)gridDim.x * 64);
}

// Where each run's rows of a model start: 16 models a workgroup, 16 threads to each.
__global__ __launch_bounds__(256) void k_rt_columns(RtPlan p) {
  __shared__ int32_t sums[16][17];
  constexpr int EACH = kRtChunks / 16;
  const int q = threadIdx.x >> 4, m = blockIdx.x * 16 + (threadIdx.x & 15);
  int v[EACH], sum = 0;
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int c = q * EACH + e;
    v[e] = m < p.M && c < p.nchunk ? p.hist[(int64_t)c * p.M + m] : 0;
  }
#pragma unroll
  for (int e = 0; e < EACH; ++e) sum += v[e];
  sums[q][threadIdx.x & 15] = sum;
  __syncthreads();
  if (m >= p.M) return;
  int at = 0;
  for (int r = 0; r < q; ++r) at += sums[r][threadIdx.x & 15];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int c = q * EACH + e;
    if (c < p.nchunk) p.hist[(int64_t)c * p.M + m] = at;
    at += v[e];
  }
  if (q == 15) p.count[m] = at;
}

namespace {

__device__ __forceinline__ int up(int a, int b) { return (a + b - 1) / b; }

struct Sums {
  int32_t place, item, jitem, long_jitem;
  int64_t z;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return Sums{a.place + b.place, a.item + b.item, a.jitem + b.jitem,
              a.long_jitem + b.long_jitem, a.z + b.z};
}

__device__ __forceinline__ Sums model_sums(const RtPlan& p, int n, int h) {
  const int rows = up(n, kRtPad) * kRtPad;
  Sums s;
  s.place = rows;
  s.item = up(n, p.t.rt) * up(h, p.t.uc);
  s.jitem = p.jitems ? (n ? up(rows, p.t.part) : 1) * up(h, p.t.du) * up(p.F, p.t.df) : 0;
  s.long_jitem = n > p.long_rows ? s.jitem : 0;
  s.z = (int64_t)rows * h;
  return s;
}

__device__ __forceinline__ Sums from_lane(const Sums& v, int lane) {
  return Sums{__shfl(v.place, lane), __shfl(v.item, lane), __shfl(v.jitem, lane), __shfl(v.long_jitem, lane),
              (int64_t)__shfl((long long)v.z, lane)};
}

// The sums over models before each, by a workgroup of 1,024 threads: count(m) slots and
// units(m), which `take(m, sums, total)` receives for every m up to M.  p.ioff[M] and
// p.joff[M], the numbers of items, are written.
template <class Count, class Units, class Take>
__device__ __forceinline__ void scan_models(const RtPlan& p, Sums* lds, int M, Count count, Units units,
                                            Take take) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, each = up(M, 1024);
  const int m0 = t * each < M ? t * each : M, m1 = m0 + each < M ? m0 + each : M;
  Sums mine{};
  for (int m = m0; m < m1; ++m) mine = mine + model_sums(p, count(m), units(m));
  Sums upto = mine;  // over the lanes up to this one
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums v = from_lane(upto, lane - d);
    if (lane >= d) upto = upto + v;
  }
  if (lane == 63) lds[wave] = upto;
  __syncthreads();
  Sums at{}, total{};
  for (int w = 0; w < 16; ++w) {
    if (w < wave) at = at + lds[w];
    total = total + lds[w];
  }
  at = at + upto;
  at = Sums{at.place - mine.place, at.item - mine.item, at.jitem - mine.jitem,
            at.long_jitem - mine.long_jitem, at.z - mine.z};
  for (int m = m0; m < m1; ++m) {
    take(m, at, total);
    at = at + model_sums(p, count(m), units(m));
  }
  if (t == 1023) {
    take(M, at, total);
    p.ioff[M] = at.item;
    p.joff[M] = at.jitem;
  }
}

// Model m's items, by a wave.
__device__ __forceinline__ void list_items(const RtPlan& p, int m) {
  const int lane = threadIdx.x & 63;
  RtItem it;
  it.m = m;
  it.c = 0;
  it.first = p.seg_off[m];
  it.zoff = p.zoff[m];
  it.h = (int)(p.seg_off[m + 1] - it.first);
  it.act = p.act[m];
  it.rows = p.count[m];
  it.place = p.place[m];
  it.places = p.place[m + 1] - it.place;
  it.pad[0] = it.pad[1] = it.pad[2] = 0;
  const int nu = up(it.h, p.t.uc), i0 = p.ioff[m], n = p.ioff[m + 1] - i0;
  for (int i = lane; i < n; i += 64) {
    it.a = i / nu;
    it.b = i % nu;
    p.items[i0 + i] = it;
  }
  if (!p.jitems) return;
  const int nt = up(it.h, p.t.du), nf = up(p.F, p.t.df), j0 = p.joff[m];
  const int k = model_sums(p, it.rows, it.h).jitem;
  for (int i = lane; i < k; i += 64) {
    it.a = i / nf % nt;
    it.b = i % nf;
    it.c = i / nf / nt;
    p.jitems[j0 + i] = it;
  }
}

}  // namespace

// (The weight gradients of models with more than p.long_rows rows, twice the mean, come first:
// their chains of stages are the longest.  32 models of 500 to 1,000 units, 1,000 columns, 16,384
// slots 524 -> 479 us; 489 where those of 1.25 times the mean do.)
__global__ __launch_bounds__(1024) void k_rt_scan(RtPlan p) {
  __shared__ Sums lds[16];
  scan_models(p, lds, p.M, [&](int m) { return p.count[m]; },
              [&](int m) { return (int)(p.seg_off[m + 1] - p.seg_off[m]); },
              [&](int m, const Sums& at, const Sums& total) {
                p.place[m] = at.place;
                p.zoff[m] = at.z;
                p.ioff[m] = at.item;
                const bool first = m < p.M && p.count[m] > p.long_rows;
                p.joff[m] = first ? at.long_jitem : total.long_jitem + (at.jitem - at.long_jitem);
              });
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
         [&](int64_t s, int m, int r) { put_slot(p, s, p.place[m] + r); });
    return;
  }
  list_items(p, blockIdx.x - p.nchunk);
}

// All of it by one workgroup, a run of slots for each of its 16 waves: few slots and models
// are sooner counted in one than started in four (64 slots, 60 models: 8 us).
__global__ __launch_bounds__(1024) void k_rt_plan_one(RtPlan p) {
  constexpr int STEPS = kRtOneSlots / 1024;
  __shared__ int32_t counter[16 * kRtOneModels];
  __shared__ RtItem model[kRtOneModels];
  __shared__ int32_t ioff[kRtOneModels + 1], joff[kRtOneModels + 1];
  __shared__ Sums total[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, M = p.M;
  const int first = wave * 64 * STEPS;
  for (int i = tid; i < 16 * M; i += 1024) counter[i] = 0;
  int key[STEPS], rank[STEPS];
#pragma unroll
  for (int q = 0; q < STEPS; ++q) key[q] = slot_model(p, first + 64 * q + lane, p.R, true);
  clear_places(p, tid, 1024);
  __syncthreads();
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {  // (see walk)
    if (first + 64 * q >= p.R) continue;
    const uint64_t peers = peers_of(key[q], M);
    const int leader = peers ? __ffsll((unsigned long long)peers) - 1 : lane;
    int base = 0;
    if (peers && lane == leader) base = atomicAdd(&counter[wave * M + key[q]], __popcll(peers));
    rank[q] = __shfl(base, leader) + __popcll(peers & ((1ull << lane) - 1));
  }
  __syncthreads();
  if (tid < M) {
    RtItem& t = model[tid];
    int n = 0;
    for (int w = 0; w < 16; ++w) {
      const int c = counter[w * M + tid];
      counter[w * M + tid] = n;
      n += c;
    }
    t.m = tid;
    t.c = 0;
    t.first = p.seg_off[tid];
    t.h = (int)(p.seg_off[tid + 1] - t.first);
    t.act = p.act[tid];
    t.rows = n;
    p.count[tid] = n;
  }
  __syncthreads();
  scan_models(p, total, M, [&](int m) { return model[m].rows; },
              [&](int m) { return model[m].h; },
              [&](int m, const Sums& at, const Sums&) {
                if (m < M) {
                  model[m].place = at.place;
                  model[m].zoff = at.z;
                  model[m].places = up(model[m].rows, kRtPad) * kRtPad;
                }
                ioff[m] = at.item;
                joff[m] = at.jitem;
                p.place[m] = at.place;
              });
  __syncthreads();
#pragma unroll
  for (int q = 0; q < STEPS; ++q)
    if (key[q] >= 0)
      put_slot(p, first + 64 * q + lane, model[key[q]].place + counter[wave * M + key[q]] + rank[q]);
  auto model_of = [&](const int32_t* off, int i) {  // the last one that starts at or before i
    int lo = 0, hi = M;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (off[mid] <= i) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  for (int i = tid; i < ioff[M]; i += 1024) {
    const int m = model_of(ioff, i);
    RtItem t = model[m];
    const int nu = up(t.h, p.t.uc);
    t.a = (i - ioff[m]) / nu;
    t.b = (i - ioff[m]) % nu;
    p.items[i] = t;
  }
  if (!p.jitems) return;
  for (int i = tid; i < joff[M]; i += 1024) {
    const int m = model_of(joff, i), j = i - joff[m];
    RtItem t = model[m];
    const int nt = up(t.h, p.t.du), nf = up(p.F, p.t.df);
    t.a = j / nf % nt;
    t.b = j % nf;
    t.c = j / nf / nt;
    p.jitems[i] = t;
  }
}

hipError_t launch_rt_plan(const RtPlan& p, hipStream_t s) {
  if (p.R <= kRtOneSlots && p.M <= kRtOneModels) {
    note_variant("k_rt_plan_one", kArithNone);
    k_rt_plan_one<<<1, 1024, 0, s>>>(p);
    return hipGetLastError();
  }
  note_variant("k_rt_place", kArithNone);
  const size_t lds = p.M <= kRtLdsModels ? (size_t)p.M * sizeof(int32_t) : 0;
  k_rt_count<<<p.nchunk, 64, lds, s>>>(p);
  k_rt_columns<<<(unsigned)ceil_div_i(p.M, 16), 256, 0, s>>>(p);
  k_rt_scan<<<1, 1024, 0, s>>>(p);
  k_rt_place<<<(unsigned)(p.nchunk + p.M), 64, lds, s>>>(p);
  return hipGetLastError();
}

}  // namespace pmlpk
