// What the gate's kernels and the forward of a few tokens share: a token's logits
// in float64, and the top-k of its logits by one wave in rounds of an arg-max
// (larger value first, ties to the lower id).
#pragma once

#include <type_traits>

#include "tg_device.h"

namespace tg {

__device__ __forceinline__ bool better(float v, int id, float bv, int bid) {
  return v > bv || (v == bv && id < bid);
}

// Arg-max of (v, id) over the 16 lanes of each DPP row: xor 1, xor 2
// (quad permutes), then half-row and row mirrors; afterwards every lane of a
// row holds the row's best.
__device__ __forceinline__ void row_best(float& bv, int& bid) {
#define TG_DPP_STEP(ctrl)                                                                 \
  do {                                                                                    \
    const float ov = __int_as_float(                                                      \
        __builtin_amdgcn_update_dpp(0, __float_as_int(bv), ctrl, 0xF, 0xF, false));       \
    const int oid = __builtin_amdgcn_update_dpp(0, bid, ctrl, 0xF, 0xF, false);           \
    if (better(ov, oid, bv, bid)) {                                                       \
      bv = ov;                                                                            \
      bid = oid;                                                                          \
    }                                                                                     \
  } while (0)
  TG_DPP_STEP(0xB1);   // quad_perm [1,0,3,2]
  TG_DPP_STEP(0x4E);   // quad_perm [2,3,0,1]
  TG_DPP_STEP(0x141);  // row_half_mirror
  TG_DPP_STEP(0x140);  // row_mirror
#undef TG_DPP_STEP
}

// The same over the wave: the four rows are compared with lane reads.
__device__ __forceinline__ void wave_best(float& bv, int& bid) {
  row_best(bv, bid);
  float gv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(bv), 0));
  int gid = __builtin_amdgcn_readlane(bid, 0);
#pragma unroll
  for (int r = 1; r < 4; ++r) {
    const float rv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(bv), 16 * r));
    const int rid = __builtin_amdgcn_readlane(bid, 16 * r);
    if (better(rv, rid, gv, gid)) {
      gv = rv;
      gid = rid;
    }
  }
  bv = gv;
  bid = gid;
}

// Lane j < k holds the token's j-th choice: its id and its weight
// exp(l_j - l_0) / sum_{j'<k} exp(l_j' - l_0), the sum in rank order.
__device__ __forceinline__ void store_topk(float my_v, int my_id, int k, int t,
                                           int32_t* __restrict__ ids, float* __restrict__ w) {
  const int lane = lane_id();
  const float v0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_v), 0));
  const float ex = (lane < k) ? expf(my_v - v0) : 0.0f;
  float z = 0.0f;
  for (int j = 0; j < k; ++j) z += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ex), j));
  if (lane < k) {
    ids[(size_t)t * k + lane] = my_id;
    w[(size_t)t * k + lane] = ex / z;
  }
}

// Top-k over the logits held in `lg` (LDS, E <= 64 * NQ floats) by one
// wave; writes ids and weights of token t. Each round takes the best
// remaining candidate of every lane, reduces the rows with DPP and the four
// rows with lane reads, so no round goes through LDS.
template <int NQ>
__device__ void wave_topk(const float* lg, int E, int k, int t, int32_t* __restrict__ ids,
                          float* __restrict__ w) {
  const int lane = lane_id();
  float v[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int e = lane + q * kWave;
    v[q] = (e < E) ? lg[e] : 0.0f;
  }
  uint32_t taken = 0;
  float my_v = 0.0f;
  int my_id = 0;
  for (int j = 0; j < k; ++j) {
    float bv = -__builtin_inff();
    int bid = 0x7fffffff;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int e = lane + q * kWave;
      if (e < E && !(taken & (1u << q)) && better(v[q], e, bv, bid)) {
        bv = v[q];
        bid = e;
      }
    }
    wave_best(bv, bid);
    if ((bid & (kWave - 1)) == lane) taken |= 1u << (bid / kWave);
    if (lane == j) {
      my_v = bv;
      my_id = bid;
    }
  }
  store_topk(my_v, my_id, k, t, ids, w);
}

// wave_topk for the smallest NQ that covers E.
__device__ __forceinline__ void wave_topk_any(const float* lg, int E, int k, int t,
                                              int32_t* __restrict__ ids, float* __restrict__ w) {
  if (E <= 64) wave_topk<1>(lg, E, k, t, ids, w);
  else if (E <= 128) wave_topk<2>(lg, E, k, t, ids, w);
  else if (E <= 256) wave_topk<4>(lg, E, k, t, ids, w);
  else if (E <= 512) wave_topk<8>(lg, E, k, t, ids, w);
  else wave_topk<16>(lg, E, k, t, ids, w);
}

// Sum over the wave of a float64 held per lane, the same on every lane, in
// a fixed order: DPP row steps (xor 1, xor 2, half-row mirror, row mirror)
// give each 16-lane row its sum, then the four row sums are added.
__device__ __forceinline__ double wave_sum_f64(double v) {
#define TG_DPP_ADD(ctrl)                                                                     \
  do {                                                                                       \
    const int lo = __builtin_amdgcn_update_dpp(0, (int)__double2loint(v), ctrl, 0xF, 0xF,     \
                                               false);                                       \
    const int hi = __builtin_amdgcn_update_dpp(0, (int)__double2hiint(v), ctrl, 0xF, 0xF,     \
                                               false);                                       \
    v += __hiloint2double(hi, lo);                                                           \
  } while (0)
  TG_DPP_ADD(0xB1);
  TG_DPP_ADD(0x4E);
  TG_DPP_ADD(0x141);
  TG_DPP_ADD(0x140);
#undef TG_DPP_ADD
  double total = 0.0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int lo = __builtin_amdgcn_readlane((int)__double2loint(v), 16 * r);
    const int hi = __builtin_amdgcn_readlane((int)__double2hiint(v), 16 * r);
    total += __hiloint2double(hi, lo);
  }
  return total;
}

// float64 logits of one token for the NC experts e[0..NC-1] (wave-uniform).
// Lane l sums 8-element chunks l, l + 64, ... of the row, then the lanes are
// added. The vector unit bounds it: per product and wave an unpack, a
// widening (8 cycles, measured) and an FMA, 16 cycles; the next chunk's loads
// are in flight meanwhile.
template <int NC>
__device__ __forceinline__ void logits_of(const uint4* __restrict__ xr,
                                          const uint16_t* __restrict__ wg, int d, const int* e,
                                          float* out) {
  const int nchunk = d / 8;
  double acc[NC];
  uint4 xn, wn[NC];
  auto load = [&](int c) {
    xn = xr[c];
#pragma unroll
    for (int q = 0; q < NC; ++q) wn[q] = reinterpret_cast<const uint4*>(wg + (size_t)e[q] * d)[c];
  };
#pragma unroll
  for (int q = 0; q < NC; ++q) acc[q] = 0.0;
  load(min(lane_id(), nchunk - 1));
  for (int c = lane_id(); c < nchunk; c += kWave) {
    const uint32_t xs[4] = {xn.x, xn.y, xn.z, xn.w};
    uint4 wv[NC];
#pragma unroll
    for (int q = 0; q < NC; ++q) wv[q] = wn[q];
    load(min(c + kWave, nchunk - 1));  // one chunk ahead
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double x0 = (double)__uint_as_float(xs[i] << 16);
      const double x1 = (double)__uint_as_float(xs[i] & 0xffff0000u);
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        const uint32_t ws[4] = {wv[q].x, wv[q].y, wv[q].z, wv[q].w};
        acc[q] = fma(x0, (double)__uint_as_float(ws[i] << 16), acc[q]);
        acc[q] = fma(x1, (double)__uint_as_float(ws[i] & 0xffff0000u), acc[q]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < NC; ++q) out[q] = (float)wave_sum_f64(acc[q]);
}

// logits_of for the first 8, 4, 2 or 1 of n experts: id(j) gives the j-th,
// out(j, logit) takes its logit on every lane. Returns how many.
template <typename Id, typename Out>
__device__ __forceinline__ int run_of_logits(const uint4* __restrict__ xr,
                                             const uint16_t* __restrict__ wg, int d, int n, Id id,
                                             Out out) {
  auto take = [&](auto nc) {
    constexpr int NC = decltype(nc)::value;
    int e[NC];
    float v[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) e[j] = id(j);
    logits_of<NC>(xr, wg, d, e, v);
#pragma unroll
    for (int j = 0; j < NC; ++j) out(j, v[j]);
    return NC;
  };
  if (n >= 8) return take(std::integral_constant<int, 8>{});
  if (n >= 4) return take(std::integral_constant<int, 4>{});
  if (n >= 2) return take(std::integral_constant<int, 2>{});
  return take(std::integral_constant<int, 1>{});
}

}  // namespace tg
