// Attention of a tree of drafted rows (or of single tokens) over a paged KV
// cache.
//
// The rows of one KV head (a request's nodes times the G query heads that
// share it) are the columns of two matrix products per 32 positions,
//   S^T = K Q^T   and   O^T = V^T P^T,
// with P = 2^(c S - m) between them (c = scale * log2 e, m a running maximum
// per row; 2^7 times that for f16). A lane holds, of S^T, exactly the positions
// that it feeds to the second product, so P never leaves the registers, and the
// only operand that needs a transpose is V, which comes out of LDS through
// ds_read_b64_tr_b16.
//
// Few rows (split kernel): the cache's bytes bound it. A wave takes 32
// positions at a time by itself, K straight from the cache into the operand's
// layout, V through the wave's own piece of LDS; no wave waits for another
// until the rows are finished, where the four waves of a block join their
// maxima, sums and outputs. 128 single tokens over contexts of up to 8192
// (heads 32 / 8 of 128): 436 us, 5.6 TB/s; two waves per SIMD without spilled
// registers are faster than three with (640 us). 7 rows over 131071 positions:
// 111 us, 4.8 TB/s (482 of the 512 blocks get 17 units, one 6, 29 none).
// Many rows (shared kernel): the products and the vector unit bound it. The
// four waves of a block take different rows and share each tile of 64
// positions through LDS, which the split kernel would read per wave. Eight
// trees of up to 64 rows over up to 16384 positions (heads 64 / 8 of 128):
// 215 us on average of 30 traced launches and 185 at best, 520 to 600 TFLOP/s
// (196 us with the join, among other calls); the matrix unit works in 35 % of the
// time, the vector unit (exp, maxima, conversions) in 44 %, LDS in 18 % without
// bank conflicts, and a wave, of which two fit a SIMD, waits in 42 %.
//
// The work is dealt by its amount, whatever the lengths: all (request, KV head,
// row tile) items are laid end to end in units of positions, and the blocks take
// runs of ceil(units / blocks) of them in turn, as far as they go: the last ones
// may have none, and a call of few units runs on the first XCDs alone. Items that
// end up in several blocks leave their parts (float32, not normalised, with m and
// the sum) in the workspace, and a second kernel joins those.
#include "tg_attn.h"

namespace tg {
namespace {

// Joins the parts of the items that several blocks had (3 to 14 us; with a
// grid of one block per item and pair of rows 17 to 45). As many blocks join an
// item as had a part of it, each an equal share of its rows, so that every
// block reads about as much as it left. A wave takes 256 / D rows at a time:
// the waves take different rows, kPass at once, or, where a block has few (one
// long context), every fourth part of the same ones.
template <class T, int D, int kRows>
__global__ __launch_bounds__(kBlock) void join_kernel(const Params p) {
  constexpr int kLine = D / 4, kAt = kWave / kLine;  // lanes per row, rows per wave
  constexpr int kPass = 4, kU = 8;
  __shared__ f32x4 os[kWaves][kWave];
  __shared__ float2 mls[kWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Split s = p.split[blockIdx.x];
  if (s.parts == 0) return;
  const int rows = min(kRows, s.lines - s.row0), ch = lane % kLine;
  const int each = (rows + s.parts - 1) / s.parts;
  const int begin = s.at * each, end = min(rows, begin + each);
  if (begin >= end) return;
  auto write = [&](int row, f32x4 o, float sum) {
    const float inv = inverse(sum);
    const int line = s.row0 + row, nd = line / p.G;
    *reinterpret_cast<uint2*>(p.out + (int64_t)(s.first + nd) * p.out_stride +
                              (int64_t)(s.g * p.G + line - nd * p.G) * D + ch * 4) =
        make_uint2(T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv));
  };
  auto part_of = [&](int k, int row) -> int64_t {  // the k-th part's row
    return (2 * (int64_t)(s.k0 + k) + (k == 0 ? s.slot : 0)) * kRows + row;
  };
  if (end - begin > 2 * kAt) {
    for (int r0 = begin + wave * kPass * kAt; r0 < end; r0 += kWaves * kPass * kAt) {
      const int row0 = r0 + lane / kLine;
      f32x4 o[kPass];
      float m[kPass], sum[kPass];
#pragma unroll
      for (int i = 0; i < kPass; ++i) {
        o[i] = f32x4{0, 0, 0, 0};
        m[i] = -INFINITY;
        sum[i] = 0.0f;
      }
#pragma unroll 2
      for (int k = 0; k < s.parts; ++k) {
        float2 t[kPass];
        f32x4 x[kPass];
#pragma unroll
        for (int i = 0; i < kPass; ++i) {
          const int64_t at = part_of(k, min(row0 + i * kAt, end - 1));
          t[i] = p.part_ml[at];
          x[i] = *reinterpret_cast<const f32x4*>(p.part + at * D + ch * 4);
        }
#pragma unroll
        for (int i = 0; i < kPass; ++i) {
          const float next = fmaxf(m[i], t[i].x), a = grow(m[i], next), e = grow(t[i].x, next);
          m[i] = next;
          sum[i] = sum[i] * a + t[i].y * e;
          o[i] = o[i] * a + x[i] * e;
        }
      }
#pragma unroll
      for (int i = 0; i < kPass; ++i)
        if (row0 + i * kAt < end) write(row0 + i * kAt, o[i], sum[i]);
    }
    return;
  }
  for (int r0 = begin; r0 < end; r0 += kAt) {
    const int row = min(r0 + lane / kLine, end - 1);
    f32x4 o = f32x4{0, 0, 0, 0};
    float m = -INFINITY, sum = 0.0f;
    for (int k = wave; k < s.parts; k += kU * kWaves) {
      float2 t[kU];
      f32x4 x[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t at = part_of(min(k + u * kWaves, s.parts - 1), row);
        t[u] = p.part_ml[at];
        x[u] = *reinterpret_cast<const f32x4*>(p.part + at * D + ch * 4);
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        if (k + u * kWaves >= s.parts) break;
        const float next = fmaxf(m, t[u].x), a = grow(m, next), e = grow(t[u].x, next);
        m = next;
        sum = sum * a + t[u].y * e;
        o = o * a + x[u] * e;
      }
    }
    os[wave][lane] = o;
    mls[wave][lane] = make_float2(m, sum);
    __syncthreads();
    if (wave == 0 && r0 + lane / kLine < end) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, mls[w][lane].x);
      sum = 0.0f;
      o = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float a = grow(mls[w][lane].x, top);
        sum += mls[w][lane].y * a;
        o += os[w][lane] * a;
      }
      write(row, o, sum);
    }
    __syncthreads();
  }
}

struct Layout {
  size_t part_ml, part, bytes;
};

Layout layout(const tg_tree_attn_args* a) {
  const Shape sh = shape_of(a);
  const int D = a->cache.D;
  const size_t blocks = (size_t)kCus * occupancy(D, sh.q);
  const size_t slots = 2 * blocks * rows_of(sh);
  Layout L;
  L.part_ml = (2 * blocks * sizeof(Split) + 255) & ~(size_t)255;
  L.part = L.part_ml + slots * 8;
  L.bytes = L.part + slots * D * 4;
  return L;
}

template <class T, int D, int kQ, bool kShared>
hipError_t launch(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  constexpr int kRows = rows_of(Shape{kQ, kShared});
  const Layout L = layout(a);
  char* w = static_cast<char*>(ws);
  Params p;
  fill(&p, a);
  p.split = reinterpret_cast<Split*>(w);
  p.part_ml = reinterpret_cast<float2*>(w + L.part_ml);
  p.part = reinterpret_cast<float*>(w + L.part);
  const hipError_t e = launch_items<T, D, kQ, kShared, kAll>(p, a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((join_kernel<T, D, kRows>), dim3(2 * kCus * occupancy(D, kQ)), dim3(kBlock), 0,
                     s, p);
  return hipGetLastError();
}

template <class T, int D>
hipError_t launch_shape(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  const Shape sh = shape_of(a);
  if (sh.q == 1) return sh.shared ? launch<T, D, 1, true>(a, ws, s) : launch<T, D, 1, false>(a, ws, s);
  if constexpr (D < 256)
    return sh.shared ? launch<T, D, 2, true>(a, ws, s) : launch<T, D, 2, false>(a, ws, s);
  return hipErrorInvalidValue;  // shape_of() gives no other
}

template <class T>
hipError_t launch_type(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  switch (a->cache.D) {
    case 64: return launch_shape<T, 64>(a, ws, s);
    case 128: return launch_shape<T, 128>(a, ws, s);
    default: return launch_shape<T, 256>(a, ws, s);
  }
}

}  // namespace

size_t tree_attention_workspace_bytes(const tg_tree_attn_args* a) { return layout(a).bytes; }

hipError_t launch_tree_attention(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  if (a->T == 0 || a->cache.B == 0) return hipSuccess;
  return a->cache.dtype == TG_BF16 ? launch_type<Bf16>(a, ws, s) : launch_type<F16>(a, ws, s);
}

}  // namespace tg
