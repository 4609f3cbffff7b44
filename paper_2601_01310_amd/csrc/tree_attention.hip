// Attention of a tree of rows over a paged cache: the plain kernel, one wave
// per row and head, one pass over the positions with a running maximum and
// sum.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 256;

template <class T, int D>
__global__ __launch_bounds__(kBlock) void tree_attention_kernel(
    const uint16_t* __restrict__ q, int64_t q_stride, const uint16_t* __restrict__ kc,
    const uint16_t* __restrict__ vc, int64_t page_stride, int page_shift, int n_pages,
    int max_pages, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask, int words, int B, int T_,
    int max_nodes, int Hq, int Hkv, float scale, uint16_t* __restrict__ out, int64_t out_stride) {
  constexpr int kPer = D / kWave;  // elements of a head per lane
  const int lane = threadIdx.x % kWave, b = blockIdx.z;
  const int h = blockIdx.y * (kBlock / kWave) + threadIdx.x / kWave;
  int first, n;
  request_rows(off, b, T_, max_nodes, &first, &n);
  if (h >= Hq) return;
  const int L = max(0, lengths[b]), width = Hkv * D;
  const int64_t cap = (int64_t)max_pages << page_shift;
  for (int node = blockIdx.x; node < n; node += gridDim.x) {
    const uint16_t* qr = q + (int64_t)(first + node) * q_stride + (int64_t)h * D;
    float x[kPer], o[kPer];
    for (int i = 0; i < kPer; ++i) {
      const uint32_t u = qr[lane + i * kWave];
      x[i] = T::lo(u) * scale;
      o[i] = 0.0f;
    }
    float m = -INFINITY, sum = 0.0f;
    const int64_t end = min((int64_t)L + n, cap);
    for (int64_t p = 0; p < end; ++p) {
      const int j = (int)(p - L);
      if (j >= 0 && !(mask ? mask[(int64_t)(first + node) * words + j / 64] >> (j % 64) & 1
                           : j <= node))
        continue;
      const int page = table[(int64_t)b * max_pages + (p >> page_shift)];
      if (page < 0 || page >= n_pages) continue;
      const int64_t at = page * page_stride + (p & ((1 << page_shift) - 1)) * width +
                         (int64_t)(h / (Hq / Hkv)) * D + lane;
      float s = 0.0f;
      for (int i = 0; i < kPer; ++i) s = fmaf(x[i], T::lo((uint32_t)kc[at + i * kWave]), s);
      for (int d = 1; d < kWave; d *= 2) s += __shfl_xor(s, d);
      const float m2 = fmaxf(m, s), a = __expf(m - m2), e = __expf(s - m2);
      m = m2;
      sum = sum * a + e;
      for (int i = 0; i < kPer; ++i) o[i] = fmaf(e, T::lo((uint32_t)vc[at + i * kWave]), o[i] * a);
    }
    const float r = sum > 0.0f ? 1.0f / sum : 0.0f;
    for (int i = 0; i < kPer; ++i)
      out[(int64_t)(first + node) * out_stride + (int64_t)h * D + lane + i * kWave] =
          (uint16_t)T::pack(o[i] * r, 0.0f);
  }
}

template <class T, int D>
hipError_t launch(const tg_tree_attn_args* a, hipStream_t s) {
  const tg_kv_cache& c = a->cache;
  hipLaunchKernelGGL((tree_attention_kernel<T, D>), dim3(a->max_nodes, (a->Hq + 3) / 4, c.B),
                     dim3(kBlock), 0, s, static_cast<const uint16_t*>(a->q), a->q_stride,
                     static_cast<const uint16_t*>(c.k) + a->layer * c.layer_stride,
                     static_cast<const uint16_t*>(c.v) + a->layer * c.layer_stride, c.page_stride,
                     __builtin_ctz(c.page_size), c.n_pages, c.max_pages, c.page_table, a->q_offsets,
                     a->lengths, a->tree_mask, a->mask_words, c.B, a->T, a->max_nodes, a->Hq, c.Hkv,
                     a->scale, static_cast<uint16_t*>(a->out), a->out_stride);
  return hipGetLastError();
}

}  // namespace

size_t tree_attention_workspace_bytes(const tg_tree_attn_args* a) { return 256; }

hipError_t launch_tree_attention(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  if (a->T == 0 || a->cache.B == 0) return hipSuccess;
  const bool bf = a->cache.dtype == TG_BF16;
  switch (a->cache.D) {
    case 64: return bf ? launch<Bf16, 64>(a, s) : launch<F16, 64>(a, s);
    case 128: return bf ? launch<Bf16, 128>(a, s) : launch<F16, 128>(a, s);
    default: return bf ? launch<Bf16, 256>(a, s) : launch<F16, 256>(a, s);
  }
}

}  // namespace tg
