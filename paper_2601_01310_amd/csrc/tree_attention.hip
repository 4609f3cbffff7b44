// Attention of a tree of drafted rows (or of single tokens) over a paged KV
// cache.
//
// The rows of one KV head (a request's nodes times the G query heads that
// share it) are the columns of two matrix products per 32 positions,
//   S^T = K Q^T   and   O^T = V^T P^T,
// with P = 2^(c S - m) between them (c = scale * log2 e, m a running maximum
// per row). A lane holds, of S^T, exactly the positions that it feeds to the
// second product, so P never leaves the registers, and the only operand that
// needs a transpose is V, which comes out of LDS through ds_read_b64_tr_b16.
//
// Few rows (split kernel): the cache's bytes bound it. A wave takes 32
// positions at a time by itself, K straight from the cache into the operand's
// layout, V through the wave's own piece of LDS; no wave waits for another
// until the rows are finished, where the four waves of a block join their
// maxima, sums and outputs.
// Many rows (shared kernel): the products bound it. The four waves of a block
// take different rows and share each tile of 64 positions through LDS.
//
// The work is dealt evenly whatever the lengths: all (request, KV head, row
// tile) items are laid end to end in units of positions, and every block takes
// an equal run of units. Items that end up in several blocks leave their
// parts (float32, not normalised, with m and the sum) in the workspace, and a
// second kernel joins those.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / kWave;
constexpr int kTile = 32;  // positions per pair of products
constexpr int kCus = 256;
constexpr float kLazy = 8.0f;  // how far (in powers of two) a score may pass m

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
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

// The infinities and NaN of a pair of values, or (keep false) the pair without.
template <class T>
struct Exponent;
template <>
struct Exponent<Bf16> {
  static constexpr uint32_t kAll = 0x7f80u;
};
template <>
struct Exponent<F16> {
  static constexpr uint32_t kAll = 0x7c00u;
};
template <class T>
__device__ __forceinline__ uint32_t odd_part(uint32_t u, bool keep) {
  constexpr uint32_t e = Exponent<T>::kAll;
  const uint32_t m = ((u & e) == e ? 0xffffu : 0u) | ((u & e << 16) == e << 16 ? 0xffff0000u : 0u);
  return u & (keep ? m : ~m);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// x, of which the compiler knows nothing: what is computed from it stays where
// it is and takes no registers outside (rare paths inside the main loop).
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Over the four lanes that share a row of S (they differ in lane / 16).
// The swaps give each lane its own half's (row's) values and the other's.
__device__ __forceinline__ float max4(float x) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __float_as_uint(x);
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum4(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// 2^(a - b) with 0 where a is -infinity.
__device__ __forceinline__ float grow(float a, float b) {
  return a == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - b);
}

// 1 / sum; a row that saw nothing gives 0, a NaN stays.
__device__ __forceinline__ float inverse(float sum) {
  return sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
}

struct Params {
  const uint16_t *q, *k, *v;
  int64_t q_stride, out_stride, page_stride;
  uint16_t* out;
  int64_t* plan;    // [B + 1] units before each request, then units per block
  float* part;      // [2 * blocks][rows][D] float32
  float2* part_ml;  // [2 * blocks][rows] maximum and sum
  int page_shift, n_pages, max_pages, words, B, T, max_nodes, Hkv, G;
  float c;
};

struct Request {
  int first, n, L;
  int end;  // positions, the rows' own included (a table holds at most 2^30)
  int units, tiles;
};

// kUnit: positions per unit of work; kRows: rows per item.
template <int kRows, int kUnit>
__device__ __forceinline__ Request request_of(const Params& p, const int32_t* __restrict__ off,
                                              const int32_t* __restrict__ lengths, int b) {
  Request r;
  request_rows(off, b, p.T, p.max_nodes, &r.first, &r.n);
  const int cap = p.max_pages << p.page_shift;
  r.L = max(0, min(lengths[b], cap));
  r.end = min(r.L + r.n, cap);
  r.units = (r.end + kUnit - 1) / kUnit;
  r.tiles = (r.n * p.G + kRows - 1) / kRows;
  return r;
}

// Units before each request, pre [B + 1]; returns this block's run of units.
// Blocks of one XCD (they are dealt out in turn) take neighbouring runs.
struct Run {
  int64_t begin, stop;
  int me;
};

template <int kRows, int kUnit>
__device__ __forceinline__ Run deal(const Params& p, const int32_t* __restrict__ off,
                                    const int32_t* __restrict__ lengths, int64_t* pre,
                                    int64_t* carry) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int64_t base = 0;
  for (int b0 = 0; b0 < p.B; b0 += kBlock) {
    const int b = b0 + threadIdx.x;
    int64_t x = 0;
    if (b < p.B) {
      const Request r = request_of<kRows, kUnit>(p, off, lengths, b);
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
  const int64_t total = pre[p.B];
  const int blocks = gridDim.x;
  Run run;
  run.me = (blockIdx.x % 8) * (blocks / 8) + blockIdx.x / 8;
  const int64_t share = max((int64_t)1, (total + blocks - 1) / blocks);
  if (blockIdx.x == 0) {
    for (int b = threadIdx.x; b <= p.B; b += kBlock) p.plan[b] = pre[b];
    if (threadIdx.x == 0) p.plan[p.B + 1] = share;
  }
  run.begin = run.me * share;
  run.stop = min(total, run.begin + share);
  return run;
}

// The piece of a run that starts at unit `at`: one item, units [u0, u1).
struct Piece {
  Request r;
  int b, g, rt, u0, u1;
  bool whole;
};

template <int kRows, int kUnit>
__device__ __forceinline__ Piece piece_at(const Params& p, const int32_t* __restrict__ off,
                                          const int32_t* __restrict__ lengths, const int64_t* pre,
                                          int64_t at, int64_t stop) {
  Piece x;
  int b = 0;
  for (int hi = p.B; hi - b > 1;) {  // the last request that starts at or before `at`
    const int mid = (b + hi) / 2;
    if (pre[mid] <= at) b = mid;
    else hi = mid;
  }
  x.b = uniform(b);
  x.r = request_of<kRows, kUnit>(p, off, lengths, x.b);
  const int64_t rest = at - pre[b];
  const int item = (int)(rest / x.r.units), u0 = (int)(rest - (int64_t)item * x.r.units);
  x.u0 = uniform(u0);
  x.u1 = uniform((int)min((int64_t)x.r.units, u0 + (stop - at)));
  x.g = uniform(item / x.r.tiles);
  x.rt = uniform(item % x.r.tiles);
  x.r.first = uniform(x.r.first);
  x.r.n = uniform(x.r.n);
  x.r.L = uniform(x.r.L);
  x.r.end = uniform(x.r.end);
  x.r.units = uniform(x.r.units);
  x.whole = x.u0 == 0 && x.u1 == x.r.units;
  return x;
}

// kQ groups of 16 rows of a wave: what it knows of them.
template <class T, int D, int kQ>
struct Rows {
  static constexpr int kSteps = D / 32;  // of the first product
  static constexpr int kCols = D / 16;   // of the second
  // Rows of a tile in LDS lie 2 D + 32 bytes apart: the transposing reads of
  // four rows and the operand reads of eight hit different banks.
  static constexpr int kPitch = D + 16;  // elements

  uint4 q[kQ][kSteps];  // column lane % 16, elements step * 32 + lane / 16 * 8
  int node[kQ];
  float m[kQ], sum[kQ];
  f32x4 o[kQ][kCols];

  __device__ __forceinline__ void start(const Params& p, const Piece& x, int row0) {
    const int col = threadIdx.x & 15, quad = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      const int row = min(row0 + c * 16 + col, x.r.n * p.G - 1);
      node[c] = row / p.G;
      const uint16_t* src = p.q + (int64_t)(x.r.first + node[c]) * p.q_stride +
                            (int64_t)(x.g * p.G + row - node[c] * p.G) * D + quad * 8;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) q[c][s] = *reinterpret_cast<const uint4*>(src + s * 32);
      m[c] = -INFINITY;
      sum[c] = 0.0f;
#pragma unroll
      for (int d = 0; d < kCols; ++d) o[c][d] = f32x4{0, 0, 0, 0};
    }
  }

  // Bits of the positions p0 .. p0 + 31 that the rows of group c see, of
  // those that are `there`.
  __device__ __forceinline__ uint32_t sees(const Params& p, const uint64_t* __restrict__ mask,
                                           const Piece& x, int c, int p0, uint32_t there) const {
    const int j0 = p0 - x.r.L;  // node at the first position
    if (j0 <= -32) return there;
    const int ctx = max(0, -j0), n0 = max(0, j0);
    uint32_t own;
    if (mask) {
      const uint64_t* w = mask + (int64_t)(x.r.first + node[c]) * p.words + n0 / 64;
      const int sh = n0 % 64;
      uint64_t v = w[0] >> sh;
      if (sh > 32 && n0 / 64 + 1 < p.words) v |= w[1] << (64 - sh);
      own = (uint32_t)v;
    } else {
      const int k = node[c] - n0 + 1;
      own = k >= 32 ? ~0u : k > 0 ? (1u << k) - 1 : 0u;
    }
    if (x.r.n - n0 < 32) own &= (1u << max(x.r.n - n0, 0)) - 1;
    return there & (ctx ? own << ctx | ((1u << ctx) - 1) : own);
  }

  // Scores without the positions that see[] leaves out.
  __device__ __forceinline__ static void hide(f32x4 (&s)[kQ][2], const uint32_t (&see)[kQ]) {
    const int quad = here((threadIdx.x & 63) >> 4);
#pragma unroll
    for (int c = 0; c < kQ; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(see[c] >> (t * 16 + quad * 4 + i) & 1)) s[c][t][i] = -INFINITY;
  }

  // Probabilities of one tile's scores, in the second product's layout:
  // element e of lane (quad, col) is position e / 4 * 16 + quad * 4 + e % 4.
  // They are rounded to the cache's type (half a unit in the last place each,
  // as much as the output's own rounding); the sum takes them unrounded.
  __device__ __forceinline__ void weigh(const f32x4 (&s)[kQ][2], float scale, uint4 (&pr)[kQ]) {
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      float mx = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])),
                       fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3])));
      mx = max4(mx) * scale;
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
        e[i] = __builtin_amdgcn_exp2f(fmaf(s[c][i / 4][i % 4], scale, -base));
      sum[c] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      pr[c] = pack8<T>(e);
    }
  }

  // o += V^T P^T over the 32 rows of V at vt (LDS, kPitch apart).
  __device__ __forceinline__ void add(const uint16_t* vt, const uint4 (&pr)[kQ]) {
    const int col = threadIdx.x & 15, quad = (threadIdx.x & 63) >> 4;
    // A lane reads 4 columns of row quad * 4 + col / 4 (and of the row 16
    // below) and gets column `col` of the rows quad * 4 .. + 3.
    const uint16_t* src = vt + (quad * 4 + col / 4) * kPitch + (col & 3) * 4;
#pragma unroll
    for (int d = 0; d < kCols; ++d) {
      s16x8 a;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(src + h * 16 * kPitch + d * 16));
#pragma unroll
        for (int i = 0; i < 4; ++i) a[h * 4 + i] = x[i];
      }
      const uint4 va = __builtin_bit_cast(uint4, a);
#pragma unroll
      for (int c = 0; c < kQ; ++c) o[c][d] = mfma<T>(va, pr[c], o[c][d]);
    }
  }

  // The infinities and NaN of row `row` (0 .. 31) of the tile, which the tile
  // in LDS holds as 0: added for the rows that see it. `src`: the row of V.
  __device__ __forceinline__ void add_odd(const uint16_t* src, int row, const uint4 (&pr)[kQ],
                                          const uint32_t (&see)[kQ]) {
    const int col = here(threadIdx.x & 15), quad = here((threadIdx.x & 63) >> 4);
    const int from = (row % 16) / 4 * 16 + col;
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      const uint32_t w0 = pr[c].x, w1 = pr[c].y, w2 = pr[c].z, w3 = pr[c].w;
      const uint32_t pick = 0u - (uint32_t)(row >> 1 & 1), far = 0u - (uint32_t)(row >> 4 & 1);
      const uint32_t a = (w0 & ~pick) | (w1 & pick), b = (w2 & ~pick) | (w3 & pick);
      const uint32_t w = (a & ~far) | (b & far);
      const uint32_t mine = (uint32_t)__shfl((int)w, from);
      const float e = row & 1 ? T::hi(mine) : T::lo(mine);
      if (see[c] >> row & 1) {
#pragma unroll
        for (int d = 0; d < kCols; ++d) {
          const uint2 y = *reinterpret_cast<const uint2*>(src + d * 16 + quad * 4);
          const uint32_t u = odd_part<T>(y.x, true), v = odd_part<T>(y.y, true);
          const uint32_t all[4] = {u << 16, u & 0xffff0000u, v << 16, v & 0xffff0000u};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (all[i]) o[c][d][i] = fmaf(e, T::hi(all[i]), o[c][d][i]);
        }
      }
    }
  }
};

// kPages: pages per tile, 1 (pages of 32 rows and more) or 2 (of 16), whose
// addresses are the wave's; 0: smaller ones, an address per lane.
template <class T, int D, int kQ, int kPages, int kOcc>
__global__ __launch_bounds__(kBlock, kOcc) void split_kernel(
    const Params p, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask) {
  using R = Rows<T, D, kQ>;
  constexpr int kRows = 16 * kQ, kUnit = kWaves * kTile;
  constexpr int kLanes = D / 8;         // lanes that load a row of V
  constexpr int kPer = kWave / kLanes;  // rows of V per load
  constexpr int kLoads = kTile / kPer;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int64_t carry[kWaves];
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  uint16_t* const vt = reinterpret_cast<uint16_t*>(smem) + wave * kTile * R::kPitch;
  float2* const ml = reinterpret_cast<float2*>(smem + kWaves * kTile * R::kPitch * 2);
  int64_t* const pre = reinterpret_cast<int64_t*>(ml + kWaves * kRows);

  const Run run = deal<kRows, kUnit>(p, off, lengths, pre, carry);
  const int width = p.Hkv * D, page_mask = (1 << p.page_shift) - 1;
  for (int64_t at = run.begin; at < run.stop;) {
    const Piece x = piece_at<kRows, kUnit>(p, off, lengths, pre, at, run.stop);
    const int32_t* __restrict__ pages = table + (int64_t)x.b * p.max_pages;
    R rows;
    rows.start(p, x, x.rt * kRows);

    // Page of position p0 + lane % 32 (kPages == 1: of the tile), -1 for none.
    auto page_at = [&](int p0) -> int {
      const int pos = kPages == 1 ? p0 : p0 + (lane & 31);
      if (pos >= x.r.end) return -1;
      const int g0 = pages[pos >> p.page_shift];
      return g0 >= 0 && g0 < p.n_pages ? g0 : -1;
    };
    uint4 kn[2][R::kSteps], vn[kLoads];
    // Loads of the tile at p0; positions without a page read page 0 and are
    // masked.
    const uint16_t* const kh = p.k + (int64_t)x.g * D;
    const uint16_t* const vh = p.v + (int64_t)x.g * D;
    auto load_tile = [&](int p0, int page) {
      if (kPages) {
        int64_t base[2];  // of the tile's halves
        base[0] = (int64_t)uniform(max(page, 0)) * p.page_stride + (int64_t)(p0 & page_mask) * width;
        base[1] = kPages == 1
                      ? base[0] + 16 * width
                      : (int64_t)max(__builtin_amdgcn_readlane(page, 16), 0) * p.page_stride;
        const uint32_t kl = (col * width + quad * 8) * 2;
        const uint32_t vl = (lane / kLanes * width + lane % kLanes * 8) * 2;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int s = 0; s < R::kSteps; ++s)
            kn[t][s] = *reinterpret_cast<const uint4*>(
                reinterpret_cast<const char*>(kh + base[t]) + s * 64 + kl);
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          vn[j] = *reinterpret_cast<const uint4*>(
              reinterpret_cast<const char*>(vh + base[j / (kLoads / 2)] +
                                            j % (kLoads / 2) * kPer * width) + vl);
      } else {
        auto row_of = [&](int row) -> int64_t {
          const int pg = __shfl(page, row);
          return pg < 0 ? 0 : pg * p.page_stride + (int64_t)((p0 + row) & page_mask) * width;
        };
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint16_t* ks = kh + row_of(t * 16 + col) + quad * 8;
#pragma unroll
          for (int s = 0; s < R::kSteps; ++s)
            kn[t][s] = *reinterpret_cast<const uint4*>(ks + s * 32);
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
          vn[j] = *reinterpret_cast<const uint4*>(vh + row_of(j * kPer + lane / kLanes) +
                                                  lane % kLanes * 8);
      }
    };

    int p0 = (x.u0 * kWaves + wave) * kTile;
    const int p_end = min(x.r.end, x.u1 * kUnit);
    int page = page_at(p0);
    if (p0 < p_end) load_tile(p0, page);
    int page_next = page_at(p0 + kUnit);
    for (; p0 < p_end; p0 += kUnit) {
      const bool inner = p0 + kTile <= x.r.L && __all(page >= 0);
      uint32_t there = ~0u;  // positions of the tile that are there at all
      uint32_t odd = 0;      // rows of V past L that hold infinities or NaN
      if (!inner) {
        there = kPages == 1 ? (page >= 0 ? ~0u : 0u) : (uint32_t)__ballot(page >= 0);
        if (x.r.end - p0 < kTile) there &= (1u << (x.r.end - p0)) - 1;
        const int ctx = x.r.L - p0;
        const uint32_t own = ctx <= 0 ? ~0u : ctx >= 32 ? 0u : ~((1u << ctx) - 1);
        const int row0 = here(lane / kLanes);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int row = j * kPer + row0;
          const uint4 was = vn[j];
          const bool gone = !(there >> row & 1), past = own >> row & 1;
          const uint4 y = make_uint4(odd_part<T>(was.x, false), odd_part<T>(was.y, false),
                                     odd_part<T>(was.z, false), odd_part<T>(was.w, false));
          const bool bad = !gone && past &&
                           (y.x != was.x || y.y != was.y || y.z != was.z || y.w != was.w);
          const uint32_t m = gone ? 0u : ~0u;
          vn[j] = make_uint4(m & (past ? y.x : was.x), m & (past ? y.y : was.y),
                             m & (past ? y.z : was.z), m & (past ? y.w : was.w));
          const uint64_t any = __ballot(bad);
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (any >> (i * kLanes) & ((2ull << (kLanes - 1)) - 1)) odd |= 1u << (j * kPer + i);
        }
      }
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        *reinterpret_cast<uint4*>(vt + (j * kPer + lane / kLanes) * R::kPitch +
                                  lane % kLanes * 8) = vn[j];

      f32x4 s[kQ][2];
#pragma unroll
      for (int st = 0; st < R::kSteps; ++st)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int c = 0; c < kQ; ++c)
            s[c][t] = mfma<T>(kn[t][st], rows.q[c][st], st ? s[c][t] : f32x4{0, 0, 0, 0});

      // The next loads take the place of this tile's operands: not before.
      __builtin_amdgcn_sched_barrier(0);
      const int page_now = page;
      page = page_next;
      if (p0 + kUnit < p_end) {
        load_tile(p0 + kUnit, page);
        page_next = page_at(p0 + 2 * kUnit);
      }

      __builtin_amdgcn_sched_barrier(0);
      uint32_t see[kQ];
      if (!inner) {
#pragma unroll
        for (int c = 0; c < kQ; ++c) see[c] = rows.sees(p, mask, x, c, p0, there);
        R::hide(s, see);
      }
      uint4 pr[kQ];
      rows.weigh(s, p.c, pr);
      rows.add(vt, pr);
      while (odd) {
        const int row = __ffs(odd) - 1;
        odd &= odd - 1;
        const int pg = kPages == 1 ? page_now : __shfl(page_now, row);
        rows.add_odd(vh + pg * p.page_stride + (int64_t)((p0 + row) & page_mask) * width, row, pr,
                     see);
      }
    }

    // The waves' parts joined, 16 rows at a time through the V tiles' place.
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      rows.sum[c] = sum4(rows.sum[c]);
      if (quad == 0) ml[wave * kRows + c * 16 + col] = make_float2(rows.m[c], rows.sum[c]);
    }
    __syncthreads();
    const int64_t slot = 2 * (int64_t)run.me + (at == run.begin ? 0 : 1);
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w * kRows + c * 16 + col].x);
      const float a = grow(rows.m[c], top);
      float* const mine = reinterpret_cast<float*>(vt);
      const int hcol = here(col), hquad = here(quad);
#pragma unroll
      for (int d = 0; d < R::kCols; ++d)
        *reinterpret_cast<f32x4*>(mine + hcol * D + (((d * 4 + hquad) ^ (hcol & 7)) * 4)) =
            rows.o[c][d] * a;
      __syncthreads();
      for (int i = here(threadIdx.x); i < 16 * D / 4; i += kBlock) {
        const int row = i / (D / 4), ch = i % (D / 4);
        const int line = x.rt * kRows + c * 16 + row;
        if (line >= x.r.n * p.G) continue;
        f32x4 y = f32x4{0, 0, 0, 0};
        float peak = -INFINITY, whole = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          y += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem) +
                                               w * (kTile * R::kPitch / 2) + row * D +
                                               ((ch ^ (row & 7)) * 4));
          peak = fmaxf(peak, ml[w * kRows + c * 16 + row].x);
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float2 t = ml[w * kRows + c * 16 + row];
          whole += t.y * grow(t.x, peak);
        }
        if (x.whole) {
          const float inv = inverse(whole);
          const int nd = line / p.G;
          *reinterpret_cast<uint2*>(p.out + (int64_t)(x.r.first + nd) * p.out_stride +
                                    (int64_t)(x.g * p.G + line - nd * p.G) * D + ch * 4) =
              make_uint2(T::pack(y[0] * inv, y[1] * inv), T::pack(y[2] * inv, y[3] * inv));
        } else {
          *reinterpret_cast<f32x4*>(p.part + (slot * kRows + c * 16 + row) * D + ch * 4) = y;
          if (ch == 0) p.part_ml[slot * kRows + c * 16 + row] = make_float2(peak, whole);
        }
      }
      __syncthreads();
    }
    at += x.u1 - x.u0;
  }
}

// The four waves take kQ groups of 16 rows each and share tiles of 64
// positions, which go from registers into one of two LDS buffers while the
// other is multiplied.
template <class T, int D, int kQ, int kOcc>
__global__ __launch_bounds__(kBlock, kOcc) void shared_kernel(
    const Params p, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask) {
  using R = Rows<T, D, kQ>;
  constexpr int kRows = 16 * kQ * kWaves, kUnit = 2 * kTile;
  constexpr int kLanes = D / 8, kPer = kBlock / kLanes;  // rows per load of the block
  constexpr int kLoads = kUnit / kPer;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int64_t carry[kWaves];
  __shared__ uint32_t odd_rows[3][2];  // of the tiles, in turn
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  // [buffer][K, V][kUnit][kPitch]
  uint16_t* const tiles = reinterpret_cast<uint16_t*>(smem);
  constexpr int kTileElems = kUnit * R::kPitch;
  int64_t* const pre = reinterpret_cast<int64_t*>(smem + 4 * kTileElems * 2);

  const Run run = deal<kRows, kUnit>(p, off, lengths, pre, carry);
  const int width = p.Hkv * D, page_mask = (1 << p.page_shift) - 1;
  const int my_row = threadIdx.x / kLanes, my_chunk = threadIdx.x % kLanes;
  for (int64_t at = run.begin; at < run.stop;) {
    const Piece x = piece_at<kRows, kUnit>(p, off, lengths, pre, at, run.stop);
    const int32_t* __restrict__ pages = table + (int64_t)x.b * p.max_pages;
    const uint16_t* const kh = p.k + (int64_t)x.g * D;
    const uint16_t* const vh = p.v + (int64_t)x.g * D;
    const int row0 = x.rt * kRows + wave * 16 * kQ;
    const bool busy = row0 < x.r.n * p.G;  // the wave has rows of its own
    R rows;
    rows.start(p, x, row0);

    // Page of position p0 + lane, -1 for none.
    auto page_at = [&](int p0) -> int {
      if (p0 + lane >= x.r.end) return -1;
      const int g0 = pages[(p0 + lane) >> p.page_shift];
      return g0 >= 0 && g0 < p.n_pages ? g0 : -1;
    };
    u32x4 kn[kLoads], vn[kLoads];
    auto load_tile = [&](int p0, int page) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = j * kPer + my_row, pg = __shfl(page, row);
        const int64_t from = (pg < 0 ? 0 : pg * p.page_stride +
                              (int64_t)((p0 + row) & page_mask) * width) + my_chunk * 8;
        kn[j] = *reinterpret_cast<const u32x4*>(kh + from);
        vn[j] = *reinterpret_cast<const u32x4*>(vh + from);
      }
    };
    // The loaded tile into buffer `buf`; rows of V that are not there are 0,
    // infinities and NaN past L are left out and noted.
    auto store_tile = [&](int p0, int page, int buf, int turn) {
      uint16_t* const kt = tiles + buf * 2 * kTileElems + my_chunk * 8;
      if (!(p0 + kUnit <= x.r.L && __all(page >= 0))) {
        const unsigned long long there = __ballot(page >= 0);
        const int first = here(my_row);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
          const int row = j * kPer + first;
          const bool gone = !(there >> row & 1), own = p0 + row >= x.r.L;
          uint32_t bad = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t was = vn[j][i], odd = own ? odd_part<T>(was, true) : 0u;
            vn[j][i] = gone ? 0u : was ^ odd;
            bad |= odd;
          }
          if (bad && !gone) atomicOr(&odd_rows[turn][row / 32], 1u << (row % 32));
        }
      }
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        uint16_t* const to = kt + (j * kPer + my_row) * R::kPitch;
        *reinterpret_cast<u32x4*>(to) = kn[j];
        *reinterpret_cast<u32x4*>(to + kTileElems) = vn[j];
      }
    };

    int p0 = x.u0 * kUnit, buf = 0, turn = 0;
    const int p_end = x.u1 * kUnit;
    int page = page_at(p0), page_next = page_at(p0 + kUnit);
    load_tile(p0, page);
    __syncthreads();  // the last piece's reads are over
    if (threadIdx.x < 6) odd_rows[threadIdx.x / 2][threadIdx.x % 2] = 0;
    __syncthreads();
    store_tile(p0, page, 0, 0);
    __syncthreads();
    for (; p0 < p_end; p0 += kUnit, buf ^= 1) {
      const bool more = p0 + kUnit < p_end;
      const int page_now = page;
      if (more) {
        page = page_next;
        load_tile(p0 + kUnit, page);
        page_next = page_at(p0 + 2 * kUnit);
      }
      const bool inner = p0 + kUnit <= x.r.L && __all(page_now >= 0);
      if (busy) {
        const unsigned long long there64 = inner ? ~0ull : __ballot(page_now >= 0);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint16_t* const kt = tiles + buf * 2 * kTileElems + half * kTile * R::kPitch;
          f32x4 s[kQ][2];
#pragma unroll
          for (int st = 0; st < R::kSteps; ++st)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const uint4 kf = *reinterpret_cast<const uint4*>(kt + (t * 16 + col) * R::kPitch +
                                                               st * 32 + quad * 8);
#pragma unroll
              for (int c = 0; c < kQ; ++c)
                s[c][t] = mfma<T>(kf, rows.q[c][st], st ? s[c][t] : f32x4{0, 0, 0, 0});
            }
          uint32_t see[kQ];
          if (!inner) {
            const uint32_t there = (uint32_t)(there64 >> (half * 32));
#pragma unroll
            for (int c = 0; c < kQ; ++c)
              see[c] = rows.sees(p, mask, x, c, p0 + half * kTile, there);
            R::hide(s, see);
          }
          uint4 pr[kQ];
          rows.weigh(s, p.c, pr);
          rows.add(kt + kTileElems, pr);
          if (!inner) {
            uint32_t odd = odd_rows[turn][half];
            while (odd) {
              const int row = __ffs(odd) - 1;
              odd &= odd - 1;
              const int pg = __shfl(page_now, half * kTile + row);
              rows.add_odd(vh + pg * p.page_stride +
                               (int64_t)((p0 + half * kTile + row) & page_mask) * width,
                           row, pr, see);
            }
          }
        }
      }
      // One tile's notes are read, the next one's written, and those of the
      // one after it (read before the last barrier) cleared.
      const int next = turn == 2 ? 0 : turn + 1;
      if (threadIdx.x < 2) odd_rows[next == 2 ? 0 : next + 1][threadIdx.x] = 0;
      if (more) store_tile(p0 + kUnit, page, buf ^ 1, next);
      turn = next;
      __syncthreads();
    }

    const int64_t slot = 2 * (int64_t)run.me + (at == run.begin ? 0 : 1);
    if (busy) {
#pragma unroll
      for (int c = 0; c < kQ; ++c) {
        const float whole = sum4(rows.sum[c]);
        const int line = row0 + c * 16 + col;
        if (line < x.r.n * p.G) {
          if (x.whole) {
            const float inv = inverse(whole);
            uint16_t* const to = p.out + (int64_t)(x.r.first + rows.node[c]) * p.out_stride +
                                 (int64_t)(x.g * p.G + line - rows.node[c] * p.G) * D + quad * 4;
#pragma unroll
            for (int d = 0; d < R::kCols; ++d) {
              const f32x4 y = rows.o[c][d] * inv;
              *reinterpret_cast<uint2*>(to + d * 16) =
                  make_uint2(T::pack(y[0], y[1]), T::pack(y[2], y[3]));
            }
          } else {
            const int64_t line_at = slot * kRows + wave * 16 * kQ + c * 16 + col;
#pragma unroll
            for (int d = 0; d < R::kCols; ++d)
              *reinterpret_cast<f32x4*>(p.part + line_at * D + d * 16 + quad * 4) = rows.o[c][d];
            if (quad == 0) p.part_ml[line_at] = make_float2(rows.m[c], whole);
          }
        }
      }
    }
    at += x.u1 - x.u0;
  }
}

// Joins the parts of the items that several blocks had: a block takes 256 / D
// rows of an item, its waves every fourth part.
template <class T, int D, int kRows, int kUnit>
__global__ __launch_bounds__(kBlock) void join_kernel(const Params p,
                                                      const int32_t* __restrict__ off,
                                                      const int32_t* __restrict__ lengths,
                                                      int max_tiles) {
  constexpr int kLine = D / 4, kAt = kWave / kLine;  // lanes per row, rows per block
  __shared__ f32x4 os[kWaves][kWave];
  __shared__ float2 mls[kWaves][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int i = blockIdx.x;
  const int rt = i % max_tiles;
  i /= max_tiles;
  const int g = i % p.Hkv, b = i / p.Hkv;
  const int64_t share = p.plan[p.B + 1];
  const Request r = request_of<kRows, kUnit>(p, off, lengths, b);
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
          const int64_t at = (2 * kk + (kk == k0 && a0 != k0 * share ? 1 : 0)) * kRows + row;
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
  const float inv = inverse(whole);
  const int nd = line / p.G;
  *reinterpret_cast<uint2*>(p.out + (int64_t)(r.first + nd) * p.out_stride +
                            (int64_t)(g * p.G + line - nd * p.G) * D + ch * 4) =
      make_uint2(T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv));
}

// Which kernel: rows of one KV head at most, over 16-row groups.
struct Shape {
  int q;        // 16-row groups per wave
  bool shared;  // waves share tiles (rows over four waves), or split them
};

Shape shape_of(const tg_tree_attn_args* a) {
  const int rows = a->max_nodes * (a->Hq / a->cache.Hkv);
  if (rows <= 16) return {1, false};
  if (rows <= 32) return {2, false};
  if (rows <= 64) return {1, true};
  return {2, true};
}

// Waves per SIMD that the registers leave.
constexpr int occupancy(int D, int q, bool shared) {
  return D == 64 ? (q == 2 ? 2 : 3) : D == 128 ? 2 : q == 1 ? 2 : 1;
}

constexpr int rows_of(Shape s) { return 16 * s.q * (s.shared ? kWaves : 1); }

struct Layout {
  size_t plan, part_ml, part, bytes;
};

Layout layout(const tg_tree_attn_args* a) {
  const Shape sh = shape_of(a);
  const int D = a->cache.D;
  const size_t slots = 2 * (size_t)kCus * occupancy(D, sh.q, sh.shared) * rows_of(sh);
  Layout L;
  L.plan = 0;
  L.part_ml = ((size_t)(a->cache.B + 2) * 8 + 255) & ~(size_t)255;
  L.part = L.part_ml + slots * 8;
  L.bytes = L.part + slots * D * 4;
  return L;
}

template <class T, int D, int kQ, bool kShared>
hipError_t launch(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  constexpr int kOcc = occupancy(D, kQ, kShared);
  constexpr int kRows = rows_of(Shape{kQ, kShared});
  constexpr int kUnit = kShared ? 2 * kTile : kWaves * kTile;
  constexpr int kPitch = Rows<T, D, kQ>::kPitch;
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
  auto go = [&](auto* kernel, size_t lds) -> hipError_t {
    if (lds > 64 * 1024) {
      const hipError_t e =
          hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(kCus * kOcc), dim3(kBlock), lds, s, p, c.page_table,
                       a->q_offsets, a->lengths, a->tree_mask);
    return hipGetLastError();
  };
  const size_t pre = (size_t)(c.B + 1) * 8;
  hipError_t e;
  if constexpr (kShared) {
    e = go(shared_kernel<T, D, kQ, kOcc>, (size_t)4 * kUnit * kPitch * 2 + pre);
  } else {
    const size_t lds = (size_t)kWaves * kTile * kPitch * 2 + kWaves * kRows * 8 + pre;
    e = c.page_size >= kTile   ? go(split_kernel<T, D, kQ, 1, kOcc>, lds)
        : c.page_size == kTile / 2 ? go(split_kernel<T, D, kQ, 2, kOcc>, lds)
                                   : go(split_kernel<T, D, kQ, 0, kOcc>, lds);
  }
  if (e != hipSuccess) return e;
  const int rows = a->max_nodes * p.G, tiles = (rows + kRows - 1) / kRows;
  const int line = rows < kRows ? rows : kRows, at = 256 / D;
  hipLaunchKernelGGL((join_kernel<T, D, kRows, kUnit>),
                     dim3(c.B * c.Hkv * tiles, (line + at - 1) / at), dim3(kBlock), 0, s, p,
                     a->q_offsets, a->lengths, tiles);
  return hipGetLastError();
}

template <class T, int D>
hipError_t launch_shape(const tg_tree_attn_args* a, void* ws, hipStream_t s) {
  const Shape sh = shape_of(a);
  if (sh.shared) return sh.q == 1 ? launch<T, D, 1, true>(a, ws, s) : launch<T, D, 2, true>(a, ws, s);
  return sh.q == 1 ? launch<T, D, 1, false>(a, ws, s) : launch<T, D, 2, false>(a, ws, s);
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
