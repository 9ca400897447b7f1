// Products of routed packs: each model's rows of the batch with its own weights.

#include <algorithm>

#include "block_device.h"
#include "routed.h"

namespace pmlpk {

typedef float f32x16 __attribute__((ext_vector_type(16)));

namespace {

// Four floats at any float's address
struct __attribute__((packed, aligned(4))) Quad {
  float v[4];
};
__device__ __forceinline__ f32x4 load_any4(const float* p) {
  const Quad q = *(const Quad*)p;
  return f32x4{q.v[0], q.v[1], q.v[2], q.v[3]};
}

// The three pieces of four values
__device__ __forceinline__ void split3_4(const f32x4& v, uint2 (&p)[3]) {
  f32x2 r[2] = {f32x2{v[0], v[1]}, f32x2{v[2], v[3]}};
#pragma unroll
  for (int e = 0; e < 3; ++e) {
    const uint32_t lo = bf16_pair(r[0]), hi = bf16_pair(r[1]);
    p[e] = make_uint2(lo, hi);
    if (e == 2) break;
    r[0] -= bf16_pair_value(lo);
    r[1] -= bf16_pair_value(hi);
  }
}

// Two transposing loads: of a group of 16 lanes, lane i gives the address of 8 bytes (four
// columns i % 4) of row i / 4 and receives column i of the four rows; then of the rows
// `then` bytes further.
__device__ __forceinline__ bf16x8 transposed(const char* at, int then) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) char lds_char;
  lds_char* p = (lds_char*)at;
  const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
  const s16x4 v =
      __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + then));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
}

constexpr int kKT = 32;           // columns of a stage
constexpr int kRow = 2 * kKT;     // bytes of a row of one piece in LDS
// Chunk c (8 columns) of a row: rows four apart share banks, so their chunks change places.
__device__ __forceinline__ int lds_chunk(int row, int c) {
  return row * kRow + ((c ^ ((row >> 2) & 3)) << 4);
}

// acc += a b over 16 columns, the piece products smallest first
__device__ __forceinline__ f32x16 mfma_x3_32(const bf16x8 (&a)[3], const bf16x8 (&b)[3], f32x16 acc) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2], b[0], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[1], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[2], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[0], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[1], acc, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[0], acc, 0, 0, 0);
}

// One 32-column stage of a workgroup's tile: RA rows of the first operand, RB of the
// second, in three planes each.
template <int RA, int RB>
struct Stage {
  static constexpr int kA = RA * kRow, kB = RB * kRow;
  static constexpr int kBytes = 3 * (kA + kB);
  __device__ static __forceinline__ void put(char* lds, bool second, int row, int c, const f32x4& u,
                                             const f32x4& v) {
    bf16x8 p[3];
    split3(u, v, p[0], p[1], p[2]);
    char* at = lds + (second ? 3 * kA : 0) + lds_chunk(row, c);
#pragma unroll
    for (int e = 0; e < 3; ++e) *(bf16x8*)(at + e * (second ? kB : kA)) = p[e];
  }
  // row a0 + 32 i + lane % 32 of the first operand, b0 + .. of the second
  template <int NA, int NB>
  __device__ static __forceinline__ void multiply(const char* lds, int a0, int b0, int lane,
                                                  f32x16 (&acc)[NA][NB]) {
#pragma unroll
    for (int ks = 0; ks < kKT / 16; ++ks) {
      const int c = 2 * ks + (lane >> 5), r = lane & 31;
      bf16x8 a[NA][3], b[NB][3];
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int e = 0; e < 3; ++e)
          a[i][e] = *(const bf16x8*)(lds + e * kA + lds_chunk(a0 + 32 * i + r, c));
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 3; ++e)
          b[j][e] = *(const bf16x8*)(lds + 3 * kA + e * kB + lds_chunk(b0 + 32 * j + r, c));
#pragma unroll
      for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = mfma_x3_32(a[i], b[j], acc[i][j]);
    }
  }
};

// The unit (of the chunk) and the projection that row `r` of the first operand is: a
// gated chunk interleaves 32 rows of W1 and 32 of V1, so that a wave has both of a unit.
template <bool GATED>
__device__ __forceinline__ int operand_unit(int r) {
  return GATED ? ((r >> 6) << 5) + (r & 31) : r;
}
template <bool GATED>
__device__ __forceinline__ bool operand_gate(int r) {
  return GATED && (r & 32);
}

// A work unit, by scalar loads: the list was written by an earlier launch.
__device__ __forceinline__ RtItem item_at(const RtItem* items, int at) {
  typedef int i32x16 __attribute__((ext_vector_type(16)));
  const auto* p = (const __attribute__((address_space(4))) i32x16*)(items + at);
  return __builtin_bit_cast(RtItem, *p);
}

// Workgroups go to the eight dies in turn; each die takes a run of the items, so that
// its cache holds the rows and weights that its workgroups share.
__device__ __forceinline__ int die_order(int i, int n) {
  const int each = (n + 7) / 8;
  return (i & 7) * each + (i >> 3);
}

}  // namespace

// Z (and U) of a chunk of units and a block of rows of one model, then the activation and
// either the sums over the units with W2 (forward) or the hidden gradients (TRAIN).
// Units are the first operand's rows and samples the second's: a lane has one sample and
// 16 units of every tile.  (So a sample's sums over units are within a lane but for one swap,
// and its hidden values are stored in lines of 32 places.)
//
// Bound by the matrix cores and the vector work of splitting beside them: an operand's value is
// cut into pieces once a stage (some 11 instructions for two) and meets 64 or 128 rows of the
// other.  48 gated models of 500 to 1,000 units, 1,000 columns, 16,384 samples of four choices:
// 1,330 us, 145 TFLOP/s of the 187 that six bf16 products at a large library product's rate
// make; MFMA busy 0.49 and VALU 0.40.  Two workgroups a compute unit take turns: one that has
// two stages in LDS and cuts the next between the products of the last took 2,000 us.
template <int NA, int NB, bool GATED, bool TRAIN>
__global__ __launch_bounds__(256, 2) void k_rt_tile(RtArgs a) {
  constexpr int RA = 64 * NA, RB = 64 * NB, UC = GATED ? 64 : RA, NU = GATED ? 1 : NA;
  typedef Stage<RA, RB> St;
  __shared__ __align__(16) char lds[St::kBytes];
  __shared__ __align__(16) float w2s[kRtMaxO * UC];  // [O][UC]
  // the rows' slots, weights and output gradients
  __shared__ int32_t slot_of[RB];
  __shared__ float weight_of[TRAIN ? RB : 1], dys[TRAIN ? kRtMaxO * RB : 1];  // dys [O][RB]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wu = wave & 1, wr = wave >> 1;
  const int n = *a.nitems, each = (n + 7) / 8;
  for (int it = blockIdx.x; it < 8 * each; it += gridDim.x) {
    const int at = die_order(it, n);
    if (at >= n) continue;
    const RtItem item = item_at(a.items, at);
    const int64_t n0 = item.first + (int64_t)item.b * UC;
    const int left = item.h - item.b * UC;  // units from here on
    const int units = left < UC ? left : UC;
    const int rows = item.rows, places = item.places;  // without, with the padding
    const int p0 = item.a * RB;
    const int32_t* slots = a.slot + item.place;
    const float* ra[NA];
    const float* rb[NB];
    bool live[NB];
#pragma unroll
    for (int q = 0; q < NA; ++q) {
      const int r = 64 * q + (tid >> 2);
      int u = operand_unit<GATED>(r);
      u = u < units ? u : units - 1;  // (a row that is there; its results are dropped)
      ra[q] = (operand_gate<GATED>(r) ? a.V1 : a.W1) + (n0 + u) * a.F4;
    }
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      const int p = p0 + 64 * q + (tid >> 2);
      const int b = p < rows ? a.row[item.place + p] : -1;
      live[q] = b >= 0;
      rb[q] = a.X + (int64_t)(live[q] ? b : 0) * a.F;
    }
    const int c = tid & 3;
    // (two stages on their way: few columns arrive at once)
    f32x4 va[2][NA][2], vb[2][NB][2];
    auto load = [&](int d, int k0) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = k0 + 8 * c + 4 * e;
#pragma unroll
        for (int q = 0; q < NA; ++q)
          va[d][q][e] = k < a.F4 ? *(const f32x4*)(ra[q] + k) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < NB; ++q) {
          f32x4 v{0.f, 0.f, 0.f, 0.f};
          if (live[q]) {
            if (k + 4 <= a.F) v = load_any4(rb[q] + k);
            else
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (k + j < a.F) v[j] = rb[q][k + j];
          }
          vb[d][q][e] = v;
        }
      }
    };
    f32x16 acc[NA][NB];
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    __syncthreads();  // the item before has read its LDS
    for (int i = tid; i < a.O * UC; i += 256) {
      const int o = i / UC, u = i % UC;
      w2s[i] = u < units ? a.W2[(int64_t)o * a.ldw + n0 + u] : 0.f;
    }
    if (tid < RB) {
      const int s = p0 + tid < rows ? slots[p0 + tid] : -1;
      slot_of[tid] = s;
      if (TRAIN) weight_of[tid] = s >= 0 ? a.weight[s] : 0.f;
    }
    if (TRAIN)
      for (int i = tid; i < a.O * RB; i += 256) {
        const int o = i / RB, p = p0 + i % RB;
        dys[i] = p < rows ? a.dY[(int64_t)a.row[item.place + p] * a.O + o] : 0.f;
      }
    load(0, 0);
    if (kKT < a.F) load(1, kKT);
    for (int k0 = 0; k0 < a.F; k0 += 2 * kKT) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int k = k0 + d * kKT;
        if (k >= a.F) break;
#pragma unroll
        for (int q = 0; q < NA; ++q) St::put(lds, false, 64 * q + (tid >> 2), c, va[d][q][0], va[d][q][1]);
#pragma unroll
        for (int q = 0; q < NB; ++q) St::put(lds, true, 64 * q + (tid >> 2), c, vb[d][q][0], vb[d][q][1]);
        if (k + 2 * kKT < a.F) load(d, k + 2 * kKT);
        lds_barrier();
        St::template multiply<NA, NB>(lds, wu * 32 * NA, wr * 32 * NB, lane, acc);
        lds_barrier();
      }
    }

    const int act = item.act;
    const int half = 4 * (lane >> 5);
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int r = (wr * NB + j) * 32 + (lane & 31), p = p0 + r;
      const int s = slot_of[r];
      const float w = TRAIN ? weight_of[r] : 0.f;
      float dw = 0.f;
      float hid[NU][16];
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int u0 = (wu * NU + i) * 32;  // units u0 + 8 (e / 4) + half + e % 4
        float z[16], v[16], d[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = acc[i][j][e];
        if (!TRAIN) {
          blk_acts<16>(act, z, v);
        } else {
          act_and_slope<16>(act, z, v, d);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const bool there = u0 + 8 * (e >> 2) + half + (e & 3) < units;
          hid[i][e] = there ? (GATED ? v[e] * acc[NA - 1][j][e] : v[e]) : 0.f;
        }
        if (!TRAIN) continue;
        float g[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) g[e] = 0.f;
        for (int o = 0; o < a.O; ++o) {
          const float y = dys[o * RB + r];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 w2 = *(const f32x4*)(w2s + o * UC + u0 + 8 * q + half);
#pragma unroll
            for (int e = 0; e < 4; ++e) g[4 * q + e] = fmaf(y, w2[e], g[4 * q + e]);
          }
        }
        // (Places that hold no slot have zero samples, weights and gradients: what is
        // stored there adds nothing.)
        const int64_t z0 = item.zoff + (int64_t)(p >> 5) * item.h * 32 +
                           (int64_t)(item.b * UC + u0 + half) * 32 + (lane & 31);
        float *const hz = a.H + z0, *const dz = a.dZ + z0, *const du = GATED ? a.dU + z0 : nullptr;
        if (p0 + (wr * NB + j) * 32 >= places) continue;  // (the same for all lanes)
        auto store = [&](int e) {
          const int u = (8 * (e >> 2) + (e & 3)) * 32;
          const float dh = w * g[e];
          hz[u] = hid[i][e];
          dz[u] = GATED ? dh * d[e] * acc[NA - 1][j][e] : dh * d[e];
          if (GATED) du[u] = dh * v[e];
        };
#pragma unroll
        for (int e = 0; e < 16; ++e) dw = fmaf(hid[i][e], g[e], dw);
        if (u0 + 32 <= units) {
#pragma unroll
          for (int e = 0; e < 16; ++e) store(e);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (u0 + 8 * (e >> 2) + half + (e & 3) < units) store(e);
        }
      }
      const int part = 2 * item.b + wu;
      if (TRAIN) {
        dw += __shfl_xor(dw, 32);
        if (s >= 0 && lane < 32) a.dwpart[(int64_t)s * a.parts + part] = dw;
        continue;
      }
      for (int o = 0; o < a.O; ++o) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 w2 = *(const f32x4*)(w2s + o * UC + (wu * NU + i) * 32 + 8 * q + half);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf(hid[i][4 * q + e], w2[e], sum);
          }
        sum += __shfl_xor(sum, 32);
        if (s >= 0 && lane < 32) a.part[((int64_t)s * a.parts + part) * a.O + o] = sum;
      }
    }
  }
}

namespace {

// Workgroups for at most `most` items, whose number only the device knows: a multiple of
// eight (die_order), and no more than some rounds of what the device holds at once.
unsigned groups_for(int64_t most) {
  const int64_t g = (most + 7) / 8 * 8;
  return (unsigned)(g < 8 ? 8 : g > 8192 ? 8192 : g);
}

template <bool TRAIN>
hipError_t tile(const RtArgs& a, const RtShape& sh, hipStream_t s) {
#define PMLP_RT_TILE(NA, NB, G)                                                                   \
  k_rt_tile<NA, NB, G, TRAIN><<<groups_for(a.most), 256, 0, s>>>(a)
  if (a.V1) {
    if (sh.nb == 2) PMLP_RT_TILE(2, 2, true);
    else PMLP_RT_TILE(2, 1, true);
  } else if (sh.na == 2) {
    if (sh.nb == 2) PMLP_RT_TILE(2, 2, false);
    else PMLP_RT_TILE(2, 1, false);
  } else {
    if (sh.nb == 2) PMLP_RT_TILE(1, 2, false);
    else PMLP_RT_TILE(1, 1, false);
  }
#undef PMLP_RT_TILE
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rt_tile(const RtArgs& a, const RtShape& sh, bool train, hipStream_t s) {
  note_variant("k_rt_tile", kArithX3);
  return train ? tile<true>(a, sh, s) : tile<false>(a, sh, s);
}

// ---------------------------------------------------------------------------
// Few slots, each straight from its index.  A wave takes 16 units of the slot's model, four at
// a time, 16 lanes along the columns of each: bound by the weights' read, or by launches (32
// requests to 6,000 gated models of 1 to 100 units, four each: 4.6 us, and 3.3 for the join).
// A unit's sum ends in one of its lanes, which takes the activation and the product with W2
// (where all 16 lanes took both, 2,331 slots of 1 to 250 units, 37 columns took 17.5 us, 10.2
// so).
// ---------------------------------------------------------------------------

namespace {

template <int CTRL>
__device__ __forceinline__ float dpp_move(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sums over 16 lanes of each of NI = 4 or 16 values, value li % NI to lane li: a lane keeps the
// half with its bit and gives the other to the lane that keeps that.
template <int CTRL, int N>
__device__ __forceinline__ void give_half(bool upper, const float (&v)[N], float (&to)[N / 2]) {
#pragma unroll
  for (int j = 0; j < N / 2; ++j)
    to[j] = (upper ? v[j + N / 2] : v[j]) + dpp_move<CTRL>(upper ? v[j] : v[j + N / 2]);
}
__device__ __forceinline__ float scatter_sums(const float (&v)[4]) {
  const int li = threadIdx.x & 15;
  float b[2], c[1];
  give_half<0x4e>(li & 2, v, b);  // lane ^ 2
  give_half<0xb1>(li & 1, b, c);  // lane ^ 1
  const float t = dpp_add<0x128, 0xf>(c[0]);  // row_ror:8
  return dpp_add<0x124, 0xf>(t);              // row_ror:4
}
__device__ __forceinline__ float scatter_sums(const float (&v)[16]) {
  const int li = threadIdx.x & 15;
  float a[8], b[4], c[2], d[1];
  give_half<0x128>(li & 8, v, a);  // row_ror:8, lane ^ 8
  give_half<0x141>(li & 4, a, b);  // row_half_mirror, lane ^ 7
  give_half<0x4e>(li & 2, b, c);
  give_half<0xb1>(li & 1, c, d);
  return d[0];
}

// Unit few_unit(n0) of the NI * 4 from n0 on for the sample x, 0 from `end` on.
template <int NI>
__device__ __forceinline__ int64_t few_unit(int64_t n0) {
  const int lane = threadIdx.x & 63;
  return n0 + 4 * (lane & (NI - 1)) + (lane >> 4);
}
template <bool GATED, int NI>
__device__ __forceinline__ float few_units(const RtArgs& a, const float* x, int64_t n0, int64_t end, int act) {
  const int lane = threadIdx.x & 63, li = lane & 15, lu = lane >> 4;
  float z[NI] = {}, u[NI] = {};
  int64_t w[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) w[i] = (n0 + 4 * i + lu < end ? n0 + 4 * i + lu : end - 1) * a.F4;
  for (int k = 4 * li; k < a.F4; k += 64) {
    f32x4 xv{0.f, 0.f, 0.f, 0.f};
    if (k + 4 <= a.F) xv = load_any4(x + k);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k + j < a.F) xv[j] = x[k + j];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const f32x4 wv = *(const f32x4*)(a.W1 + w[i] + k);
#pragma unroll
      for (int j = 0; j < 4; ++j) z[i] = fmaf(wv[j], xv[j], z[i]);
      if (GATED) {
        const f32x4 vv = *(const f32x4*)(a.V1 + w[i] + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[i] = fmaf(vv[j], xv[j], u[i]);
      }
    }
  }
  const float zs[1] = {scatter_sums(z)};
  float h[1];
  blk_acts<1>(act, zs, h);
  if (GATED) h[0] *= scatter_sums(u);
  return few_unit<NI>(n0) < end ? h[0] : 0.f;
}

// W2 at the lane's unit, of outputs o0 .. o0 + 3 (NI = 16), or of li / 4, 4 + li / 4 .. (NI = 4)
template <int NI>
__device__ __forceinline__ void few_w2(const RtArgs& a, int64_t n0, int64_t end, int o0, float (&w)[4]) {
  const int64_t n = few_unit<NI>(n0) < end ? few_unit<NI>(n0) : end - 1;
  const int o = NI == 16 ? o0 : (threadIdx.x & 15) >> 2;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int oq = o + (NI == 16 ? 1 : 4) * q;
    w[q] = a.W2[(int64_t)(oq < a.O ? oq : a.O - 1) * a.ldw + n];
  }
}

// The units' sums with W2, lane o's output o's; w: what few_w2 gives for o0 = 0.
template <int NI>
__device__ __forceinline__ float few_output(const RtArgs& a, int64_t n0, int64_t end, float h, float (&w)[4]) {
  const int lane = threadIdx.x & 63;
  const bool there = few_unit<NI>(n0) < end;
  float y = 0.f;
  if (NI == 16) {
    for (int o0 = 0; o0 < a.O; o0 += 4) {
      if (o0) few_w2<NI>(a, n0, end, o0, w);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float t = group_sum_to_last(there ? h * w[q] : 0.f, 64);
        const float all = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(t), 63));
        if (lane == o0 + q) y = all;
      }
    }
    return y;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (4 * q >= a.O) break;
    float t = there ? h * w[q] : 0.f;
    t += dpp_move<0xb1>(t);
    t += dpp_move<0x4e>(t);
    t += __shfl_xor(t, 16);
    t += __shfl_xor(t, 32);
    if ((lane & 3) == q) y = t;
  }
  return __shfl(y, 4 * (lane & 3) + ((lane >> 2) & 3));
}

}  // namespace

// 64 units of a slot a workgroup.  A die takes a run of the slots: dies in turn, the workgroups with
// something to do could all come to one, as every eighth does where one model is wide and the others
// are not.  (600 models of 1 to 50 units and one of 1,000, 100 columns, 4,096 slots 102 us, 45 so.)
template <bool GATED>
__global__ __launch_bounds__(256) void k_rt_few(RtArgs a, RtFew f) {
  const int at = die_order(blockIdx.x, f.R * f.chunks);
  if (at >= f.R * f.chunks) return;
  const int s = at / f.chunks, chunk = at % f.chunks;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m = f.idx[s];
  if (m < 0 || m >= a.M) {
    if (m != -1 && tid == 0 && chunk == 0) f.flag[3] = 1;
    return;
  }
  const int64_t first = a.seg_off[m], end = a.seg_off[m + 1];
  const int64_t n0 = first + (int64_t)chunk * kRtFewUnits + 16 * wave;
  if (first + (int64_t)chunk * kRtFewUnits >= end) return;
  __shared__ float sums[4][kRtMaxO];
  float w2[4];
  few_w2<4>(a, n0, end, 0, w2);
  const float h = few_units<GATED, 4>(a, a.X + (int64_t)(s / a.K) * a.F, n0, end, a.act[m]);
  const float t = few_output<4>(a, n0, end, h, w2);
  if (lane < kRtMaxO) sums[wave][lane] = t;
  __syncthreads();
  if (tid < a.O)
    a.part[((int64_t)s * a.parts + chunk) * a.O + tid] =
        (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]);
}

// .. and a wave, for up to 64 columns and 1,024 such chunks or more.  (130 models of 1 to 250
// units, 2,048 slots with the join, 37 columns 14.5 us either way, 64 columns 14.0 against 14.4, 65
// columns 17.7 either way, 100 columns 18.8 against 19.1; 256 slots of 37 columns 7.9 against 7.3.)
template <bool GATED>
__global__ __launch_bounds__(256) void k_rt_few_waves(RtArgs a, RtFew f) {
  const int lane = threadIdx.x & 63;
  const int groups = (f.R * f.chunks + 3) / 4;
  const int64_t q = (int64_t)die_order(blockIdx.x, groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (q >= (int64_t)f.R * f.chunks) return;
  const int s = (int)(q / f.chunks), chunk = (int)(q % f.chunks);
  const int m = f.idx[s];
  if (m < 0 || m >= a.M) {
    if (m != -1 && lane == 0 && chunk == 0) f.flag[3] = 1;
    return;
  }
  const int64_t end = a.seg_off[m + 1], n0 = a.seg_off[m] + (int64_t)chunk * kRtFewUnits;
  if (n0 >= end) return;
  float w2[4];
  few_w2<16>(a, n0, end, 0, w2);
  const float h = few_units<GATED, 16>(a, a.X + (int64_t)(s / a.K) * a.F, n0, end, a.act[m]);
  const float t = few_output<16>(a, n0, end, h, w2);
  if (lane < a.O) a.part[q * a.O + lane] = t;
}

// A sample a workgroup, its models' units in turn over the waves: Y without a second launch.
template <bool GATED>
__global__ __launch_bounds__(256) void k_rt_sample(RtArgs a, RtFew f, const float* weight, float* Y) {
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ float sums[4][kRtMaxO];
  float y = 0.f;  // lane o < 16: output o
  for (int q = wave; q < a.K * f.chunks; q += 4) {
    const int k = q / f.chunks, m = f.idx[b * a.K + k];
    if (m < 0 || m >= a.M) {
      if (m != -1 && lane == 0) f.flag[3] = 1;
      continue;
    }
    const int64_t end = a.seg_off[m + 1], n0 = a.seg_off[m] + 16 * (q % f.chunks);
    if (n0 >= end) continue;
    float w2[4];
    few_w2<4>(a, n0, end, 0, w2);
    const float w = weight[b * a.K + k];
    const float h = few_units<GATED, 4>(a, a.X + b * a.F, n0, end, a.act[m]);
    y = fmaf(w, few_output<4>(a, n0, end, h, w2), y);
  }
  if (lane < kRtMaxO) sums[wave][lane] = y;
  __syncthreads();
  if (tid < a.O) Y[b * a.O + tid] = (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]);
}

hipError_t launch_rt_sample(const RtArgs& a, const RtFew& f, const float* weight, float* Y, hipStream_t s) {
  note_variant("k_rt_sample", kArithNone);
  const unsigned grid = (unsigned)(f.R / a.K);
  if (a.V1) k_rt_sample<true><<<grid, 256, 0, s>>>(a, f, weight, Y);
  else k_rt_sample<false><<<grid, 256, 0, s>>>(a, f, weight, Y);
  return hipGetLastError();
}

hipError_t launch_rt_few(const RtArgs& a, const RtFew& f, hipStream_t s) {
  const unsigned grid = (unsigned)(f.R * f.chunks);
  const bool waves = grid >= 1024 && a.F4 <= 64;
  note_variant(waves ? "k_rt_few_waves" : "k_rt_few", kArithNone);
  if (waves) {
    const unsigned groups = ((grid + 3) / 4 + 7) / 8 * 8;  // (die_order)
    if (a.V1) k_rt_few_waves<true><<<groups, 256, 0, s>>>(a, f);
    else k_rt_few_waves<false><<<groups, 256, 0, s>>>(a, f);
  } else if (a.V1) k_rt_few<true><<<(grid + 7) / 8 * 8, 256, 0, s>>>(a, f);
  else k_rt_few<false><<<(grid + 7) / 8 * 8, 256, 0, s>>>(a, f);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Sums over a model's parts, in order.  (32 requests of four choices 3 us, 65,536 slots of up
// to 32 parts of ten sums 50: a chain of loads a thread.)
// ---------------------------------------------------------------------------

namespace {
__device__ __forceinline__ float slot_sum(const RtJoin& a, int64_t s, int m, int o) {
  const int n = (int)((a.seg_off[m + 1] - a.seg_off[m] + a.uc - 1) / a.uc);
  const float* at = a.part + s * a.parts * a.O + o;
  float sum = 0.f;
  for (int q = 0; q < n; ++q) sum += at[(int64_t)q * a.O];
  return sum;
}
}  // namespace

__global__ __launch_bounds__(256) void k_rt_join(RtJoin a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.B * a.O) return;
  const int64_t b = i / a.O;
  const int o = (int)(i - b * a.O);
  float y = 0.f;
  for (int k = 0; k < a.K; ++k) {
    const int m = a.idx[b * a.K + k];
    if (m < 0 || m >= a.M) continue;
    y = fmaf(a.weight[b * a.K + k], slot_sum(a, b * a.K + k, m, o), y);
  }
  a.Y[i] = y;
}

hipError_t launch_rt_join(const RtJoin& a, hipStream_t s) {
  note_variant("k_rt_join", kArithNone);
  k_rt_join<<<(unsigned)ceil_div_i((int64_t)a.B * a.O, 256), 256, 0, s>>>(a);
  return hipGetLastError();
}
// ---------------------------------------------------------------------------
// Weight gradients: dW1_m = dZ_m X_m (and dV1_m = dU_m X_m) over the places of model m,
// units the first operand's rows and columns of X the second's.
// ---------------------------------------------------------------------------

namespace {

template <int NA, int NB, bool GATED>
struct DwTile {
  static constexpr int RA = 64 * NA, RB = 64 * NB, UC = GATED ? 64 : RA;
  // X lies in LDS as it comes, [place][column], and goes to the products through transposing
  // loads, 64 bytes of four rows at a time: rows are 64 bytes past (or short of) all banks apart.
  static constexpr int kA = RA * kRow, XROW = 2 * RB + 64, kX = kKT * XROW;
  static constexpr int kBytes = 3 * (kA + kX);
};

// Workgroup `block` of `blocks`
template <int NA, int NB, bool GATED>
__device__ __forceinline__ void weight_tiles(const RtGrad& g, char* lds, int block, int blocks) {
  typedef DwTile<NA, NB, GATED> T;
  constexpr int RB = T::RB, UC = T::UC, kA = T::kA, XROW = T::XROW, kX = T::kX;
  const RtArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wu = wave & 1, wf = wave >> 1;
  const int n = *g.njitems;
  // (In the list's order, dies in turn: the tiles of a model with many rows, which take
  // longest, are spread over all of them.  32 models of 500 to 1,000 units on 16,384 rows: 415
  // us where each die took a run of the list, 278 so.)
  for (int at = block; at < n; at += blocks) {
    const RtItem item = item_at(g.jitems, at);
    const int m = item.m;
    const int64_t first = item.first;
    const int h = item.h, places = item.places;
    const int u0 = item.a * UC, f0 = item.b * RB;
    const int units = h - u0 < UC ? h - u0 : UC;
    const int b0 = item.c * g.t.part, b1 = b0 + g.t.part < places ? b0 + g.t.part : places;
    const bool split = places > g.t.part;
    const int32_t* brow = a.row + item.place;
    const int c = tid & 3;
    const float* ra[NA];
#pragma unroll
    for (int q = 0; q < NA; ++q) {
      const int r = 64 * q + (tid >> 2);
      int u = operand_unit<GATED>(r);
      u = u < units ? u : units - 1;
      ra[q] = (operand_gate<GATED>(r) ? a.dU : a.dZ) + item.zoff + (int64_t)(u0 + u) * 32 + 8 * c;
    }
    // Four columns of X from column f on, of places tid / TX + NY q of a stage.  The samples
    // of the places come a stage before their values.  (A place without one takes sample 0,
    // and zeros; columns past the last are not stored.)
    constexpr int TX = RB / 4, NY = 256 / TX, NQ = kKT / NY;
    const int f = f0 + 4 * (tid % TX), y = tid / TX;
    f32x4 va[NA][2], vx[NQ];
    int br[NQ];
    auto fetch_rows = [&](int k0) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) br[q] = brow[k0 + y + NY * q];
    };
    auto load = [&](int k0) {
#pragma unroll
      for (int q = 0; q < NA; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) va[q][e] = *(const f32x4*)(ra[q] + (int64_t)k0 * h + 4 * e);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float* x = a.X + (int64_t)(br[q] >= 0 ? br[q] : 0) * a.F;
        f32x4 v;
        if (f + 4 <= a.F) v = load_any4(x + f);
        else
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = x[f + j < a.F ? f + j : a.F - 1];
        vx[q] = v;
        if (br[q] < 0) vx[q] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    f32x16 acc[NA][NB];
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    __syncthreads();
    if (b0 < b1) {
      fetch_rows(b0);
      load(b0);
      if (b0 + kKT < b1) fetch_rows(b0 + kKT);
    }
    for (int k0 = b0; k0 < b1; k0 += kKT) {
#pragma unroll
      for (int q = 0; q < NA; ++q) {
        bf16x8 p[3];
        split3(va[q][0], va[q][1], p[0], p[1], p[2]);
#pragma unroll
        for (int e = 0; e < 3; ++e) *(bf16x8*)(lds + e * kA + lds_chunk(64 * q + (tid >> 2), c)) = p[e];
      }
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        uint2 p[3];
        split3_4(vx[q], p);
#pragma unroll
        for (int e = 0; e < 3; ++e)
          *(uint2*)(lds + 3 * kA + e * kX + (y + NY * q) * XROW + 8 * (tid % TX)) = p[e];
      }
      if (k0 + kKT < b1) {
        load(k0 + kKT);
        if (k0 + 2 * kKT < b1) fetch_rows(k0 + 2 * kKT);
      }
      lds_barrier();
#pragma unroll
      for (int ks = 0; ks < kKT / 16; ++ks) {
        const int cc = 2 * ks + (lane >> 5), r = lane & 31;
        bf16x8 av[NA][3], bv[NB][3];
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int e = 0; e < 3; ++e)
            av[i][e] = *(const bf16x8*)(lds + e * kA + lds_chunk(wu * 32 * NA + 32 * i + r, cc));
        // 16 lanes: columns 16 (lane / 16 % 2) .., places 8 (lane / 32) ..
        const char* x0 = lds + 3 * kA + (16 * ks + 8 * (lane >> 5) + ((lane & 15) >> 2)) * XROW +
                         2 * (wf * 32 * NB + (lane & 16) + 4 * (lane & 3));
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int e = 0; e < 3; ++e) bv[j][e] = transposed(x0 + e * kX + 64 * j, 4 * XROW);
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[i][j] = mfma_x3_32(av[i], bv[j], acc[i][j]);
      }
      lds_barrier();
    }
    const int half = 4 * (lane >> 5);
    const int64_t size = g.N * a.F;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int col = f0 + (wf * NB + j) * 32 + (lane & 31);
      if (col >= a.F) continue;
      const bool seen = !g.fmask || (g.fmask[(int64_t)m * g.fmw + (col >> 5)] >> (col & 31) & 1u);
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        float* out = GATED && i ? g.dV1 : g.dW1;
        if (split) out = g.wpart + ((int64_t)item.c * (GATED ? 2 : 1) + (GATED ? i : 0)) * size;
        const int base = GATED ? wu * 32 : (wu * NA + i) * 32;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int u = base + 8 * (e >> 2) + half + (e & 3);
          if (u < units) out[(first + u0 + u) * a.F + col] = seen ? acc[i][j][e] : 0.f;
        }
      }
    }
  }
}

// dW2[o][unit] = sum over the places of wdy[o] H[unit], by fp32 matrix products: a workgroup
// takes 16 units of a tile of the weight gradients and a part of their model's places, 64 of
// every 256 a wave, and all outputs.  A lane loads four consecutive places of its row and
// feeds them to four products, in the same order for both operands.
// sums: [4][64] of the workgroup
__device__ __forceinline__ void output_weights(const RtGrad& g, f32x4* sums, int block, int blocks) {
  const RtArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = *g.njitems, nf = (a.F + g.t.df - 1) / g.t.df;
  const int each = (g.t.du / 16 + nf - 1) / nf;  // runs of 16 units to an item, at most
  for (int64_t it = block; it < (int64_t)n * each; it += blocks) {
    const RtItem item = item_at(g.jitems, (int)(it / each));
    const int64_t first = item.first;
    const int h = item.h, end = (item.a + 1) * g.t.du < h ? (item.a + 1) * g.t.du : h;
    const int places = item.places;
    const int b0 = item.c * g.t.part, b1 = b0 + g.t.part < places ? b0 + g.t.part : places;
    float* out = places > g.t.part ? g.w2part + (int64_t)item.c * a.O * g.N : g.dW2;
    const float* wd = g.wdy + (int64_t)(li < a.O ? li : a.O - 1) * a.P + item.place + 4 * lk;
    // the tile's units in turn over its column tiles (not always on the same die)
    const int u0 = item.a * g.t.du + 16 * ((item.b + item.a + item.c) % nf + nf * (int)(it % each));
    if (u0 < end) {
      const int u = u0 + li < h ? u0 + li : h - 1;
      const float* hrow = a.H + item.zoff + (int64_t)u * 32 + 4 * lk;
      f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
      // 64 places at a time, the next ones on their way (past the end: the last again, unused)
      f32x4 hv[2][4], y[2][4];
      auto load = [&](int b, int p) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int k = p + 16 * q < b1 ? p + 16 * q : b1 - 16;
          hv[b][q] = *(const f32x4*)(hrow + (int64_t)(k >> 5) * 32 * h + (k & 16));
          y[b][q] = *(const f32x4*)(wd + k);
        }
      };
      auto multiply = [&](int b, int p) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (p + 16 * q >= b1) break;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[b][q][e], hv[b][q][e], acc[e & 1], 0, 0, 0);
        }
      };
      const int p0 = b0 + 64 * wave;
      if (p0 < b1) load(0, p0);
      for (int p = p0; p < b1; p += 512) {
        if (p + 256 < b1) load(1, p + 256);
        multiply(0, p);
        if (p + 256 >= b1) break;
        if (p + 512 < b1) load(0, p + 512);
        multiply(1, p + 256);
      }
      sums[64 * wave + lane] = acc[0] + acc[1];
      __syncthreads();
      if (wave == 0) {
        // lane: unit u0 + li, outputs 4 lk + e
        const f32x4 t = (sums[lane] + sums[64 + lane]) + (sums[128 + lane] + sums[192 + lane]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (u0 + li < h && 4 * lk + e < a.O) out[(int64_t)(4 * lk + e) * g.N + first + u0 + li] = t[e];
      }
      __syncthreads();
    }
  }
}

}  // namespace

// All that the hidden gradients lead to, side by side: the first `tiles` workgroups take tiles
// of the input weights' gradients, the next `outs` the output weights', the rest the slots'.
// (Three launches before: 600 models of 1 to 100 units, 32,768 slots 139 us a call, 127 so.)
//
// Bound as k_rt_tile, by the matrix cores and the cutting beside them, with the tails of models
// of unlike numbers of rows: 32 models of 500 to 1,000 units, 1,000 columns, 16,384 slots 250
// us, of which the products need 131 at the rate of k_rt_tile's comment; MFMA busy 0.39.  The
// 600 small ones take 55 us, by how long a tile's chain of loads, cuts and products is.
template <int NA, int NB, bool GATED>
__global__ __launch_bounds__(256, 2) void k_rt_dw(RtGrad g, RtJoin j, int tiles, int outs) {
  __shared__ __align__(16) char lds[DwTile<NA, NB, GATED>::kBytes];
  const int block = blockIdx.x;
  if (block < tiles) {
    weight_tiles<NA, NB, GATED>(g, lds, block, tiles);
  } else if (block < tiles + outs) {
    output_weights(g, (f32x4*)lds, block - tiles, outs);
  } else {
    const int64_t s = (int64_t)(block - tiles - outs) * 256 + threadIdx.x;
    if (s >= (int64_t)j.B * j.K) return;
    const int m = j.idx[s];
    j.Y[s] = m < 0 || m >= j.M ? 0.f : slot_sum(j, s, m, 0);
  }
}

// The sums of the parts of models that have several, in order.
__global__ __launch_bounds__(256) void k_rt_sum_parts(RtGrad g) {
  const RtArgs& a = g.a;
  const int64_t n = blockIdx.x;
  const int m = g.mid[n];
  const int places = a.place[m + 1] - a.place[m];
  if (places <= g.t.part) return;
  const int parts = (places + g.t.part - 1) / g.t.part;
  const int k = a.V1 ? 2 : 1;
  const int64_t size = g.N * a.F;
  for (int f = threadIdx.x; f < k * a.F; f += 256) {
    const int v = f >= a.F;
    const int64_t at = n * a.F + f - (v ? a.F : 0);
    float t = 0.f;
#pragma unroll 8
    for (int q = 0; q < parts; ++q) t += g.wpart[((int64_t)q * k + v) * size + at];
    (v ? g.dV1 : g.dW1)[at] = t;
  }
  if (threadIdx.x < (unsigned)a.O) {
    const int64_t at = threadIdx.x * g.N + n;
    float t = 0.f;
#pragma unroll 8
    for (int q = 0; q < parts; ++q) t += g.w2part[(int64_t)q * a.O * g.N + at];
    g.dW2[at] = t;
  }
}

hipError_t launch_rt_weights(const RtGrad& g, const RtShape& sh, const RtJoin& j, hipStream_t s) {
  note_variant("k_rt_dw", kArithX3);
  const int tiles = (int)groups_for(g.jmost);
  const int outs = (int)groups_for((int64_t)g.jmost * std::max(1, g.t.du / 16 * g.t.df / g.a.F));
  const unsigned grid = tiles + outs + (unsigned)ceil_div_i((int64_t)j.B * j.K, 256);
#define PMLP_RT_DW(NA, NB, G) k_rt_dw<NA, NB, G><<<grid, 256, 0, s>>>(g, j, tiles, outs)
  if (g.a.V1) {
    if (sh.nb == 2) PMLP_RT_DW(2, 2, true);
    else PMLP_RT_DW(2, 1, true);
  } else if (sh.na == 2) {
    if (sh.nb == 2) PMLP_RT_DW(2, 2, false);
    else PMLP_RT_DW(2, 1, false);
  } else {
    if (sh.nb == 2) PMLP_RT_DW(1, 2, false);
    else PMLP_RT_DW(1, 1, false);
  }
#undef PMLP_RT_DW
  if (const hipError_t e = hipGetLastError()) return e;
  if (g.nparts > 1) k_rt_sum_parts<<<(unsigned)g.N, 256, 0, s>>>(g);
  return hipGetLastError();
}

}  // namespace pmlpk
