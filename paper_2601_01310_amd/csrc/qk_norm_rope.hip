// Per-head norms of queries and keys, their rotation by position, and the new
// K and V rows written into their cache pages, in one pass over qkv.
//
// y = x * rsqrt(sum(x^2) / D + eps) * w per head, then (a, b) -> (a cos -
// b sin, b cos + a sin) over the first rot elements, float32, one rounding.
// Every element is read and written once; the kernel is bound by HBM for many
// rows (16383 rows of 48 heads of 128: 80 us, 5.1 TB/s, the rate of a plain
// copy) and by the latency of one dependent load chain for few (one row: 4 us).
//
// A lane holds 8 neighbouring elements (16 bytes) of a head, so D / 8 lanes
// hold a head and a wave 64 / (D / 8) of them: the sum of squares takes log2
// shuffles inside the group, and the partner of a pair (i, i + rot/2) lies in
// another lane of the group at the same place. A wave stays with one row and
// takes its heads in turn: the weights and the row's cos and sin are loaded
// once per wave.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 256;
constexpr int kU = 4;  // heads per lane group in flight

template <class T, int D, bool kNext>
__global__ __launch_bounds__(kBlock) void qk_norm_rope_kernel(
    const uint16_t* qkv, int64_t qkv_stride, const uint16_t* __restrict__ qw,
    const uint16_t* __restrict__ kw, const float* __restrict__ cos_sin,
    const int32_t* __restrict__ positions, const int32_t* __restrict__ slots, uint16_t* q_out,
    int64_t q_out_stride, uint16_t* __restrict__ kc, uint16_t* __restrict__ vc, int64_t page_stride,
    int page_shift, int n_slots, int rows, int Hq, int Hkv, int rot, int max_pos, float eps,
    int heads_per_wave) {
  constexpr int kLanes = D / 8, kHeads = kWave / kLanes;
  const int row = blockIdx.x * (kBlock / kWave) + threadIdx.x / kWave;
  if (row >= rows) return;
  const int lane = threadIdx.x % kWave, c = lane % kLanes, sub = lane / kLanes;
  const int heads = Hq + 2 * Hkv;
  const int h_end = min(heads, (int)(blockIdx.y + 1) * heads_per_wave);
  const int slot = slots[row];
  const bool cached = slot >= 0 && slot < n_slots;
  const int64_t at = (int64_t)(slot >> page_shift) * page_stride +
                     (int64_t)(slot & ((1 << page_shift) - 1)) * Hkv * D + c * 8;
  const uint16_t* src = qkv + (int64_t)row * qkv_stride + c * 8;
  uint16_t* dst = q_out + (int64_t)row * q_out_stride + c * 8;

  // cos and sin of this lane's elements: the pairs (i, i + rot/2) have one
  // angle per element, the pairs (2i, 2i + 1) one per two.
  float cs[8], sn[8];
  const int half = rot / 2, rl = rot / 16;  // lanes of one half
  const bool turns = c * 8 < rot;
  if (turns) {
    const int pos = max(0, min(positions[row], max_pos - 1));
    const float* t = cos_sin + (int64_t)pos * rot;
    if (kNext) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cs[i] = t[c * 4 + i];
        sn[i] = t[half + c * 4 + i];
      }
    } else {
      const int i0 = (c < rl ? c : c - rl) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        cs[i] = t[i0 + i];
        sn[i] = c < rl ? -t[half + i0 + i] : t[half + i0 + i];
      }
    }
  }
  const int partner = lane - c + (c < rl ? c + rl : c - rl);

  float w[2][8];
  if (qw) {
    unpack8<T>(*reinterpret_cast<const uint4*>(qw + c * 8), w[0]);
    unpack8<T>(*reinterpret_cast<const uint4*>(kw + c * 8), w[1]);
  }

  for (int h0 = blockIdx.y * heads_per_wave + sub; h0 < h_end; h0 += kU * kHeads) {
    uint4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int h = h0 + u * kHeads;
      x[u] = h < h_end ? *reinterpret_cast<const uint4*>(src + (int64_t)h * D) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int h = h0 + u * kHeads;
      float f[8];
      unpack8<T>(x[u], f);
      const bool key = h >= Hq;
      if (qw) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(f[i], f[i], s);
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) s += __shfl_xor(s, m);
        const float r = rsqrtf(s * (1.0f / D) + eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * r * (key ? w[1][i] : w[0][i]);
      }
      if (kNext) {
        if (turns) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = f[2 * i], b = f[2 * i + 1];
            f[2 * i] = a * cs[i] - b * sn[i];
            f[2 * i + 1] = b * cs[i] + a * sn[i];
          }
        }
      } else if (rot > 0) {
        float g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = __shfl(f[i], partner);
        if (turns) {
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = f[i] * cs[i] + g[i] * sn[i];
        }
      }
      if (h < Hq) {
        if (h < h_end) *reinterpret_cast<uint4*>(dst + (int64_t)h * D) = pack8<T>(f);
      } else if (h < h_end && cached) {
        if (h < Hq + Hkv)
          *reinterpret_cast<uint4*>(kc + at + (int64_t)(h - Hq) * D) = pack8<T>(f);
        else
          *reinterpret_cast<uint4*>(vc + at + (int64_t)(h - Hq - Hkv) * D) = x[u];
      }
    }
  }
}

template <class T, int D>
hipError_t launch(const tg_qk_args* a, hipStream_t s) {
  const tg_kv_cache& c = a->cache;
  const int heads = a->Hq + 2 * c.Hkv, per = kWave / (D / 8);
  // Few rows: one pass of a wave's lane groups over kU heads each, so that all
  // heads are in flight at once. Many rows fill the device without, and a wave
  // takes a whole row, loading its angles once. A wave per row against a pass
  // per wave, in us: 48 heads of 128, 1024 rows 9.9 / 7.2, 2048 rows 13.0 /
  // 12.3, 3000 rows 15.3 / 16.2, 8192 rows 34.6 / 34.9; 12 heads of 256, 1024
  // rows 7.5 / 5.6, 2048 rows 8.8 / 8.0, 3000 rows 10.7 / 11.5, 8192 rows
  // 21.3 / 22.7. (32 heads of 64 are one pass either way.)
  const int heads_per_wave = a->T >= 2560 ? heads : per * kU;
  const dim3 grid((a->T + kBlock / kWave - 1) / (kBlock / kWave),
                  (heads + heads_per_wave - 1) / heads_per_wave);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, static_cast<const uint16_t*>(a->qkv),
                       a->qkv_stride, static_cast<const uint16_t*>(a->q_weight),
                       static_cast<const uint16_t*>(a->k_weight), a->cos_sin, a->positions, a->slots,
                       static_cast<uint16_t*>(a->q_out), a->q_out_stride,
                       static_cast<uint16_t*>(c.k) + a->layer * c.layer_stride,
                       static_cast<uint16_t*>(c.v) + a->layer * c.layer_stride, c.page_stride,
                       __builtin_ctz(c.page_size), c.n_pages * c.page_size, a->T, a->Hq, c.Hkv,
                       a->rot, a->max_pos, a->eps, heads_per_wave);
  };
  if (a->interleaved) go(qk_norm_rope_kernel<T, D, true>);
  else go(qk_norm_rope_kernel<T, D, false>);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(const tg_qk_args* a, hipStream_t s) {
  if (a->T == 0) return hipSuccess;
  const bool bf = a->cache.dtype == TG_BF16;
  switch (a->cache.D) {
    case 64: return bf ? launch<Bf16, 64>(a, s) : launch<F16, 64>(a, s);
    case 128: return bf ? launch<Bf16, 128>(a, s) : launch<F16, 128>(a, s);
    default: return bf ? launch<Bf16, 256>(a, s) : launch<F16, 256>(a, s);
  }
}

}  // namespace tg
