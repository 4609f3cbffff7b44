// Attention of a tree of drafted rows (or of single tokens) over a paged KV
// cache.
//
// The rows of one KV head (a request's nodes times the G query heads that
// share it) are the columns of two matrix products per tile of positions,
//   S^T = K Q^T   and   O^T = V^T P^T,
// with P = 2^(c S - m) between them (c = scale * log2 e, m a running maximum
// per row). A wave takes 32 positions at a time by itself: its lanes hold, of
// S^T, exactly the positions that they feed to the second product, so P never
// leaves the registers, and the only operand that needs a transpose is V,
// which goes through the wave's own 32 x D piece of LDS and comes out through
// ds_read_b64_tr_b16. K comes from the cache straight into the operand's
// layout. The next tile's loads are issued before the softmax of this one;
// no wave waits for another until the rows are finished, where the four waves
// of a block join their maxima, sums and outputs through LDS.
//
// The work is dealt evenly whatever the lengths: all (request, KV head, row
// tile) items are laid end to end, 128 positions a unit, and every block takes
// an equal run of units. Items that end up in several blocks leave their
// parts (float32, not normalised, with m and the sum) in the workspace, and a
// second kernel joins those.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / kWave;
constexpr int kTile = 32;               // positions per wave and step
constexpr int kUnit = kWaves * kTile;   // positions per unit of work
constexpr int kCus = 256;
constexpr float kLazy = 8.0f;  // how far (in powers of two) a score may pass m

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <class T>
__device__ __forceinline__ f32x4 mfma(const uint4& a, const uint4& b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mfma<Bf16>(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 mfma<F16>(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Whether a pair of values holds an infinity or a NaN.
template <class T>
__device__ __forceinline__ bool odd_pair(uint32_t u);
template <>
__device__ __forceinline__ bool odd_pair<Bf16>(uint32_t u) {
  return (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
}
template <>
__device__ __forceinline__ bool odd_pair<F16>(uint32_t u) {
  return (u & 0x7c00u) == 0x7c00u || (u & 0x7c000000u) == 0x7c000000u;
}

// Over the four lanes that share a row of S (they differ in lane / 16).
__device__ __forceinline__ float max4(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum4(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

struct Params {
  const uint16_t *q, *k, *v;
  int64_t q_stride, out_stride, page_stride;
  const int32_t *table, *off, *lengths;
  const uint64_t* mask;
  uint16_t* out;
  int64_t* plan;   // [B + 1] units before each request, then units per block
  float* part;     // [2 * blocks][rows][D] float32
  float2* part_ml; // [2 * blocks][rows] maximum and sum
  int page_shift, n_pages, max_pages, words, B, T, max_nodes, Hkv, G;
  float c;
};

struct Request {
  int first, n, L;
  int64_t end;  // positions, the rows' own included
  int units, tiles;
};

template <int kRows>
__device__ __forceinline__ Request request_of(const Params& p, int b) {
  Request r;
  request_rows(p.off, b, p.T, p.max_nodes, &r.first, &r.n);
  r.L = max(0, p.lengths[b]);
  r.end = min((int64_t)r.L + r.n, (int64_t)p.max_pages << p.page_shift);
  r.units = (int)((r.end + kUnit - 1) / kUnit);
  r.tiles = (r.n * p.G + kRows - 1) / kRows;
  return r;
}

// 2^(a - b) with 0 where a is -infinity.
__device__ __forceinline__ float grow(float a, float b) {
  return a == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - b);
}

// kQ: columns of 16 rows per wave; kWhole: pages hold whole tiles of 32.
template <class T, int D, int kQ, bool kWhole, int kOcc>
__global__ __launch_bounds__(kBlock, kOcc) void tree_attention_kernel(const Params p) {
  constexpr int kRows = 16 * kQ;
  constexpr int kSteps = D / 32;          // of the first product
  constexpr int kCols = D / 16;           // of the second
  constexpr int kLanes = D / 8;           // lanes that load a row of V
  constexpr int kPer = kWave / kLanes;    // rows of V per load
  constexpr int kLoads = kTile / kPer;
  constexpr int kChunks = D / 8;          // 16-byte chunks of a row of V
  extern __shared__ __attribute__((aligned(16))) char smem[];
  uint16_t* const vt = reinterpret_cast<uint16_t*>(smem) + (threadIdx.x / kWave) * kTile * D;
  float2* const ml = reinterpret_cast<float2*>(smem + kWaves * kTile * D * 2);  // [kWaves][kRows]
  int64_t* const pre = reinterpret_cast<int64_t*>(ml + kWaves * kRows);         // [B + 1]
  __shared__ int64_t carry[kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int col = lane & 15, quad = lane >> 4;

  // Units before each request.
  {
    int64_t base = 0;
    for (int b0 = 0; b0 < p.B; b0 += kBlock) {
      const int b = b0 + threadIdx.x;
      int64_t x = 0;
      if (b < p.B) {
        const Request r = request_of<kRows>(p, b);
        x = (int64_t)r.units * r.tiles * p.Hkv;
      }
#pragma unroll
      for (int m = 1; m < kWave; m *= 2) {
        const int64_t o = __shfl_up(x, m);
        if (lane >= m) x += o;
      }
      __syncthreads();
      if (lane == kWave - 1) carry[wave] = x;
      __syncthreads();
      int64_t before = base;
      for (int i = 0; i < kWaves; ++i) {
        if (i < wave) before += carry[i];
        base += carry[i];
      }
      if (b < p.B) pre[b + 1] = before + x;
    }
    if (threadIdx.x == 0) pre[0] = 0;
    __syncthreads();
  }
  const int64_t total = pre[p.B];
  const int blocks = gridDim.x;
  // Blocks of one XCD (they are dealt out in turn) take neighbouring runs.
  const int me = (blockIdx.x % 8) * (blocks / 8) + blockIdx.x / 8;
  const int64_t share = max((int64_t)1, (total + blocks - 1) / blocks);
  if (blockIdx.x == 0) {
    for (int b = threadIdx.x; b <= p.B; b += kBlock) p.plan[b] = pre[b];
    if (threadIdx.x == 0) p.plan[p.B + 1] = share;
  }
  const int64_t begin = me * share, stop = min(total, begin + share);

  for (int64_t at = begin; at < stop;) {
    int b = 0;
    for (int hi = p.B; hi - b > 1;) {  // last b with pre[b] <= at
      const int mid = (b + hi) / 2;
      if (pre[mid] <= at) b = mid;
      else hi = mid;
    }
    // Requests without units share their start with the next one.
    const Request r = request_of<kRows>(p, b);
    const int64_t rest = at - pre[b];
    const int item = (int)(rest / r.units), u0 = (int)(rest - (int64_t)item * r.units);
    const int u1 = (int)min((int64_t)r.units, u0 + (stop - at));
    const int g = item / r.tiles, rt = item % r.tiles;
    const bool whole_item = u0 == 0 && u1 == r.units;
    const int32_t* const table = p.table + (int64_t)b * p.max_pages;

    // Q: column `col` of each group of 16 rows, elements step * 32 + quad * 8.
    uint4 q[kQ][kSteps];
    int node[kQ];
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      const int row = min(rt * kRows + c * 16 + col, r.n * p.G - 1);
      node[c] = row / p.G;
      const uint16_t* src = p.q + (int64_t)(r.first + node[c]) * p.q_stride +
                            (int64_t)(g * p.G + row - node[c] * p.G) * D + quad * 8;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) q[c][s] = *reinterpret_cast<const uint4*>(src + s * 32);
    }

    float m[kQ], sum[kQ];
    f32x4 o[kQ][kCols];
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      m[c] = -INFINITY;
      sum[c] = 0.0f;
#pragma unroll
      for (int d = 0; d < kCols; ++d) o[c][d] = f32x4{0, 0, 0, 0};
    }

    // Page of position p0 + lane % 32 (kWhole: of the tile), -1 for none.
    auto page_at = [&](int64_t p0) -> int {
      const int64_t pos = kWhole ? p0 : p0 + (lane & 31);
      if (pos >= r.end) return -1;
      const int g0 = table[pos >> p.page_shift];
      return g0 >= 0 && g0 < p.n_pages ? g0 : -1;
    };
    const int width = p.Hkv * D, page_mask = (1 << p.page_shift) - 1;
    uint4 kn[2][kSteps], vn[kLoads];
    // Loads of the tile at p0; rows without a page come from page 0, row 0
    // of the cache and are masked.
    auto load_tile = [&](int64_t p0, int page) {
      const int in_page = (int)(p0 & page_mask);
      const int64_t head = (int64_t)g * D;
      if (kWhole) {
        const int pg = __builtin_amdgcn_readfirstlane(max(page, 0));
        const int64_t base = pg * p.page_stride + (int64_t)in_page * width + head;
        const uint16_t* ks = p.k + base + quad * 8;
        const uint16_t* vs = p.v + base + (lane % kLanes) * 8;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
            kn[t][s] = *reinterpret_cast<const uint4*>(ks + (t * 16 + col) * width + s * 32);
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          vn[j] = *reinterpret_cast<const uint4*>(vs + (j * kPer + lane / kLanes) * width);
      } else {
        const int pos = (in_page + (lane & 31)) & page_mask;
        const int64_t mine = page < 0 ? head : page * p.page_stride + (int64_t)pos * width + head;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint16_t* ks = p.k + __shfl(mine, t * 16 + col) + quad * 8;
#pragma unroll
          for (int s = 0; s < kSteps; ++s) kn[t][s] = *reinterpret_cast<const uint4*>(ks + s * 32);
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          vn[j] = *reinterpret_cast<const uint4*>(p.v + __shfl(mine, j * kPer + lane / kLanes) +
                                                  (lane % kLanes) * 8);
      }
    };
    // Place of a 16-byte chunk of V in LDS: neighbouring rows' columns lie in
    // different banks for the transposing reads of four rows at a time.
    auto chunk_at = [](int row, int chunk) -> int {
      const int turn = D == 64 ? (row >> 1) & 3 : row & 7;
      return row * kChunks + (chunk ^ (turn * 2));
    };

    int64_t p0 = ((int64_t)u0 * kWaves + wave) * kTile;
    const int64_t p_end = min(r.end, (int64_t)u1 * kUnit);
    int page = page_at(p0);
    if (p0 < p_end) load_tile(p0, page);
    int page_next = page_at(p0 + kUnit);
    for (; p0 < p_end; p0 += kUnit) {
      // Bits of the tile's positions that are there at all.
      uint32_t there = ~0u;
      const bool inner = p0 + kTile <= r.L && __all(page >= 0);
      uint32_t odd = 0;  // rows of V past L that hold infinities or NaN
      if (!inner) {
        there = kWhole ? (page >= 0 ? ~0u : 0u) : (uint32_t)__ballot(page >= 0);
        if (r.end - p0 < kTile) there &= (1u << (int)(r.end - p0)) - 1;
        const int64_t ctx = r.L - p0;
        const uint32_t own = ctx <= 0 ? ~0u : ctx >= 32 ? 0u : ~((1u << (int)ctx) - 1);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int row = j * kPer + lane / kLanes;
          const bool bad = (there & own) >> row & 1 &&
                           (odd_pair<T>(vn[j].x) || odd_pair<T>(vn[j].y) || odd_pair<T>(vn[j].z) ||
                            odd_pair<T>(vn[j].w));
          const uint64_t any = __ballot(bad);
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (any >> (i * kLanes) & ((2ull << (kLanes - 1)) - 1)) odd |= 1u << (j * kPer + i);
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          if (!((there & ~odd) >> (j * kPer + lane / kLanes) & 1)) vn[j] = make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        *reinterpret_cast<uint4*>(vt + 8 * chunk_at(j * kPer + lane / kLanes, lane % kLanes)) = vn[j];

      f32x4 s[kQ][2];
#pragma unroll
      for (int c = 0; c < kQ; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          s[c][t] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int st = 0; st < kSteps; ++st) s[c][t] = mfma<T>(kn[t][st], q[c][st], s[c][t]);
        }

      const int64_t pn = p0 + kUnit;
      const int page_now = page;
      page = page_next;
      if (pn < p_end) {
        load_tile(pn, page);
        page_next = page_at(pn + kUnit);
      }

      uint32_t see[kQ];
      if (!inner) {
        const int64_t j0 = p0 - r.L;  // node at the tile's first position
#pragma unroll
        for (int c = 0; c < kQ; ++c) {
          uint32_t bits;
          if (j0 <= -32) {
            bits = ~0u;
          } else {
            const int ctx = j0 < 0 ? (int)-j0 : 0, n0 = j0 < 0 ? 0 : (int)j0;
            uint32_t own;
            if (p.mask) {
              const uint64_t* w = p.mask + (int64_t)(r.first + node[c]) * p.words + n0 / 64;
              const int sh = n0 % 64;
              uint64_t x = w[0] >> sh;
              if (sh > 32 && n0 / 64 + 1 < p.words) x |= w[1] << (64 - sh);
              own = (uint32_t)x;
            } else {
              const int k = node[c] - n0 + 1;
              own = k >= 32 ? ~0u : k > 0 ? (1u << k) - 1 : 0u;
            }
            if (r.n - n0 < 32) own &= (1u << max(r.n - n0, 0)) - 1;
            bits = ctx ? own << ctx | ((1u << ctx) - 1) : own;
          }
          see[c] = bits & there;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!(see[c] >> (t * 16 + quad * 4 + i) & 1)) s[c][t][i] = -INFINITY;
        }
      }

      uint4 pr[kQ];
#pragma unroll
      for (int c = 0; c < kQ; ++c) {
        float mx = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])),
                         fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3])));
        mx = max4(mx) * p.c;
        // m follows the maximum only when a row has passed it by 2^kLazy.
        if (__any(mx > m[c] + kLazy || (m[c] == -INFINITY && mx > -INFINITY))) {
          const float next = fmaxf(m[c], mx), a = grow(m[c], next);
          m[c] = next;
          sum[c] *= a;
#pragma unroll
          for (int d = 0; d < kCols; ++d) o[c][d] *= a;
        }
        const float base = m[c] == -INFINITY ? 0.0f : m[c];
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          e[i] = __builtin_amdgcn_exp2f(fmaf(s[c][i / 4][i % 4], p.c, -base));
        sum[c] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        pr[c] = pack8<T>(e);
      }

#pragma unroll
      for (int d = 0; d < kCols; ++d) {
        s16x8 a;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = h * 16 + quad * 4 + col / 4;
          const uint16_t* src =
              vt + 8 * chunk_at(row, d * 2 + (col & 3) / 2) + (col & 1) * 4;
          const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)src);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[h * 4 + i] = x[i];
        }
        const uint4 va = __builtin_bit_cast(uint4, a);
#pragma unroll
        for (int c = 0; c < kQ; ++c) o[c][d] = mfma<T>(va, pr[c], o[c][d]);
      }

      // Rows of V with infinities or NaN reach only the rows that see them.
      while (odd) {
        const int row = __ffs(odd) - 1;
        odd &= odd - 1;
        const int64_t pos = p0 + row;
        const int pg = kWhole ? page_now : __shfl(page_now, row);
        const uint16_t* src = p.v + pg * p.page_stride + (pos & page_mask) * width +
                              (int64_t)g * D + quad * 4;
        const int from = (row % 16) / 4 * 16 + col;
#pragma unroll
        for (int c = 0; c < kQ; ++c) {
          const uint32_t w = row / 16 ? (row & 2 ? pr[c].w : pr[c].z) : (row & 2 ? pr[c].y : pr[c].x);
          const uint32_t mine = (uint32_t)__shfl((int)w, from);
          const float e = row & 1 ? T::hi(mine) : T::lo(mine);
          if (!(see[c] >> row & 1)) continue;
#pragma unroll
          for (int d = 0; d < kCols; ++d) {
            const uint2 x = *reinterpret_cast<const uint2*>(src + d * 16);
            o[c][d][0] = fmaf(e, T::lo(x.x), o[c][d][0]);
            o[c][d][1] = fmaf(e, T::hi(x.x), o[c][d][1]);
            o[c][d][2] = fmaf(e, T::lo(x.y), o[c][d][2]);
            o[c][d][3] = fmaf(e, T::hi(x.y), o[c][d][3]);
          }
        }
      }
    }

    // The waves' parts joined, 16 rows at a time through the V tiles' place.
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      sum[c] = sum4(sum[c]);
      if (quad == 0) ml[wave * kRows + c * 16 + col] = make_float2(m[c], sum[c]);
    }
    __syncthreads();
    const int64_t slot = 2 * (int64_t)me + (at == begin ? 0 : 1);
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w * kRows + c * 16 + col].x);
      const float a = grow(m[c], top);
      float* const mine = reinterpret_cast<float*>(vt);
#pragma unroll
      for (int d = 0; d < kCols; ++d)
        *reinterpret_cast<f32x4*>(mine + col * D + (((d * 4 + quad) ^ (col & 7)) * 4)) = o[c][d] * a;
      __syncthreads();
      for (int i = threadIdx.x; i < 16 * D / 4; i += kBlock) {
        const int row = i / (D / 4), ch = i % (D / 4);
        f32x4 x = f32x4{0, 0, 0, 0};
        float peak = -INFINITY, whole = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          x += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem) +
                                               w * (kTile * D / 2) + row * D + ((ch ^ (row & 7)) * 4));
          peak = fmaxf(peak, ml[w * kRows + c * 16 + row].x);
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float2 t = ml[w * kRows + c * 16 + row];
          whole += t.y * grow(t.x, peak);
        }
        const int line = rt * kRows + c * 16 + row;
        if (line >= r.n * p.G) continue;
        if (whole_item) {
          const float inv = whole > 0.0f ? 1.0f / whole : whole == 0.0f ? 0.0f : whole;
          const int nd = line / p.G;
          *reinterpret_cast<uint2*>(p.out + (int64_t)(r.first + nd) * p.out_stride +
                                    (int64_t)(g * p.G + line - nd * p.G) * D + ch * 4) =
              make_uint2(T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv));
        } else {
          *reinterpret_cast<f32x4*>(p.part + (slot * kRows + c * 16 + row) * D + ch * 4) = x;
          if (ch == 0) p.part_ml[slot * kRows + c * 16 + row] = make_float2(peak, whole);
        }
      }
      __syncthreads();
    }
    at += u1 - u0;
  }
}

// Joins the parts of the items that several blocks had: a block takes 256 / D
// rows of an item, its waves every fourth part.
template <class T, int D, int kRows>
__global__ __launch_bounds__(kBlock) void join_kernel(const Params p, int max_tiles) {
  constexpr int kLine = D / 4, kAt = kWave / kLine;  // lanes per row, rows per block
  __shared__ f32x4 os[kWaves][kWave];
  __shared__ float2 mls[kWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int i = blockIdx.x;
  const int rt = i % max_tiles;
  i /= max_tiles;
  const int g = i % p.Hkv, b = i / p.Hkv;
  const int64_t share = p.plan[p.B + 1];
  const Request r = request_of<kRows>(p, b);
  if (rt >= r.tiles) return;
  const int64_t a0 = p.plan[b] + ((int64_t)g * r.tiles + rt) * r.units, a1 = a0 + r.units;
  const int64_t k0 = a0 / share, k1 = (a1 - 1) / share;
  if (k0 == k1) return;
  const int row = blockIdx.y * kAt + lane / kLine, ch = lane % kLine;
  const int line = rt * kRows + row;
  const bool valid = row < kRows && line < r.n * p.G;
  f32x4 o = f32x4{0, 0, 0, 0};
  float m = -INFINITY, sum = 0.0f;
  if (valid) {
    constexpr int kU = 4;
    for (int64_t k = k0 + wave; k <= k1; k += kU * kWaves) {
      float2 t[kU];
      f32x4 x[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t kk = k + u * kWaves;
        if (kk <= k1) {
          const int64_t at =
              (2 * kk + (kk == k0 && a0 != k0 * share ? 1 : 0)) * kRows + row;
          t[u] = p.part_ml[at];
          x[u] = *reinterpret_cast<const f32x4*>(p.part + at * D + ch * 4);
        } else {
          t[u] = make_float2(-INFINITY, 0.0f);
          x[u] = f32x4{0, 0, 0, 0};
        }
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const float next = fmaxf(m, t[u].x), a = grow(m, next), e = grow(t[u].x, next);
        m = next;
        sum = sum * a + t[u].y * e;
        o = o * a + x[u] * e;
      }
    }
  }
  os[wave][lane] = o;
  mls[wave][lane] = make_float2(m, sum);
  __syncthreads();
  if (wave != 0 || !valid) return;
  float top = -INFINITY, whole = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, mls[w][lane].x);
  f32x4 x = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float a = grow(mls[w][lane].x, top);
    whole += mls[w][lane].y * a;
    x += os[w][lane] * a;
  }
  const float inv = whole > 0.0f ? 1.0f / whole : whole == 0.0f ? 0.0f : whole;
  const int nd = line / p.G;
  *reinterpret_cast<uint2*>(p.out + (int64_t)(r.first + nd) * p.out_stride +
                            (int64_t)(g * p.G + line - nd * p.G) * D + ch * 4) =
      make_uint2(T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv));
}

// Row columns per wave, and waves per SIMD that the registers leave.
int columns(const tg_tree_attn_args* a) {
  const int rows = a->max_nodes * (a->Hq / a->cache.Hkv);
  return rows <= 16 ? 1 : rows <= 32 || a->cache.D == 256 ? 2 : 4;
}

constexpr int occupancy(int D, int q) {
  return D == 64 ? (q == 4 ? 2 : 3) : D == 128 ? (q == 1 ? 3 : q == 2 ? 2 : 1) : (q == 1 ? 2 : 1);
}

struct Layout {
  size_t plan, part_ml, part, bytes;
};

Layout layout(const tg_tree_attn_args* a) {
  const int q = columns(a), D = a->cache.D;
  const size_t slots = 2 * (size_t)kCus * occupancy(D, q) * 16 * q;
  Layout L;
  L.plan = 0;
  L.part_ml = ((size_t)(a->cache.B + 2) * 8 + 255) & ~(size_t)255;
  L.part = L.part_ml + slots * 8;
  L.bytes = L.part + slots * D * 4;
  return L;
}

template <class T, int D, int kQ>
hipError_t launch(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  constexpr int kOcc = occupancy(D, kQ), kRows = 16 * kQ;
  const tg_kv_cache& c = a->cache;
  const Layout L = layout(a);
  char* w = static_cast<char*>(ws);
  Params p;
  p.q = static_cast<const uint16_t*>(a->q);
  p.k = static_cast<const uint16_t*>(c.k) + a->layer * c.layer_stride;
  p.v = static_cast<const uint16_t*>(c.v) + a->layer * c.layer_stride;
  p.q_stride = a->q_stride;
  p.out_stride = a->out_stride;
  p.page_stride = c.page_stride;
  p.table = c.page_table;
  p.off = a->q_offsets;
  p.lengths = a->lengths;
  p.mask = a->tree_mask;
  p.out = static_cast<uint16_t*>(a->out);
  p.plan = reinterpret_cast<int64_t*>(w + L.plan);
  p.part_ml = reinterpret_cast<float2*>(w + L.part_ml);
  p.part = reinterpret_cast<float*>(w + L.part);
  p.page_shift = __builtin_ctz(c.page_size);
  p.n_pages = c.n_pages;
  p.max_pages = c.max_pages;
  p.words = a->mask_words;
  p.B = c.B;
  p.T = a->T;
  p.max_nodes = a->max_nodes;
  p.Hkv = c.Hkv;
  p.G = a->Hq / c.Hkv;
  p.c = a->scale * 1.4426950408889634f;
  const size_t lds = kWaves * kTile * D * 2 + kWaves * kRows * 8 + (size_t)(c.B + 1) * 8;
  auto* kernel = c.page_size >= kTile ? tree_attention_kernel<T, D, kQ, true, kOcc>
                                      : tree_attention_kernel<T, D, kQ, false, kOcc>;
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3(kCus * kOcc), dim3(kBlock), lds, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = a->max_nodes * p.G, tiles = (rows + kRows - 1) / kRows;
  const int line = rows < kRows ? rows : kRows, at = 256 / D;
  hipLaunchKernelGGL((join_kernel<T, D, kRows>), dim3(c.B * c.Hkv * tiles, (line + at - 1) / at),
                     dim3(kBlock), 0, s, p, tiles);
  return hipGetLastError();
}

template <class T>
hipError_t launch_type(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  const int q = columns(a);
  switch (a->cache.D) {
    case 64: return q == 1 ? launch<T, 64, 1>(a, ws, s) : q == 2 ? launch<T, 64, 2>(a, ws, s) : launch<T, 64, 4>(a, ws, s);
    case 128: return q == 1 ? launch<T, 128, 1>(a, ws, s) : q == 2 ? launch<T, 128, 2>(a, ws, s) : launch<T, 128, 4>(a, ws, s);
    default: return q == 1 ? launch<T, 256, 1>(a, ws, s) : launch<T, 256, 2>(a, ws, s);
  }
}

}  // namespace

size_t tree_attention_workspace_bytes(const tg_tree_attn_args* a) { return layout(a).bytes; }

hipError_t launch_tree_attention(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  if (a->T == 0 || a->cache.B == 0) return hipSuccess;
  return a->cache.dtype == TG_BF16 ? launch_type<Bf16>(a, ws, s) : launch_type<F16>(a, ws, s);
}

}  // namespace tg
