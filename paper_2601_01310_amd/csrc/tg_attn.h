// Attention over a paged KV cache: the two kernels that tree_attention.hip (all of
// a request's positions) and prefix_attention.hip (a group's shared ones, and the
// others) are made of, with what they deal their work by.
#pragma once

#include <type_traits>

#include "tg_kv.h"
#include "tg_tree.h"

namespace tg {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / kWave;
constexpr int kTile = 32;  // positions per pair of products
constexpr int kCus = 256;
constexpr int kMostUnits = (1 << 30) - 1;
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

// Of a type: the bits of the exponent that infinities and NaN have, and how many
// powers of two probabilities are held above their value. f16 loses precision
// below 2^-14 and all of it below 2^-25, where a long context after one large
// score would vanish; bf16 has float32's range.
template <class T>
struct Exponent;
template <>
struct Exponent<Bf16> {
  static constexpr uint32_t kAll = 0x7f80u;
  static constexpr float kUp = 0.0f;
};
template <>
struct Exponent<F16> {
  static constexpr uint32_t kAll = 0x7c00u;
  static constexpr float kUp = 7.0f;  // with kLazy 2^15 at most: below 65504
};
// The infinities and NaN of a pair of values, or (keep false) the pair without.
template <class T>
__device__ __forceinline__ uint32_t odd_part(uint32_t u, bool keep) {
  constexpr uint32_t e = Exponent<T>::kAll;
  const uint32_t m = ((u & e) == e ? 0xffffu : 0u) | ((u & e << 16) == e << 16 ? 0xffff0000u : 0u);
  return u & (keep ? m : ~m);
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// load_lds16() from an address per lane. (The compiler waits for these before
// any later LDS read; for those of load_lds16() it leaves the wait to us.)
__device__ __forceinline__ void load_lds(const uint16_t* from, lds_u16* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// x, of which the compiler knows nothing: what is computed from it stays where
// it is and takes no registers outside (rare paths inside the main loop).
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The larger one, NaN if either is (one instruction for three values; fmaxf
// costs another per value that comes out of a matrix product).
__device__ __forceinline__ float most(float a, float b) {
  return __builtin_elementwise_maximum(a, b);
}

// Over the four lanes that share a row of S (they differ in lane / 16).
// The swaps give each lane its own half's (row's) values and the other's.
__device__ __forceinline__ float max4(float x) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __float_as_uint(x);
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  const uint32_t v = __float_as_uint(most(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(v, v, false, false));
  return most(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum4(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Sums of units of work. The host's check keeps them below kMostUnits for
// offsets that ascend; others, whose requests overlap, stay inside all arrays.
__device__ __forceinline__ int add_units(int a, int b) { return min(a + b, kMostUnits); }

// 2^(a - b) with 0 where a is -infinity.
__device__ __forceinline__ float grow(float a, float b) {
  return a == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a - b);
}

// 1 / sum; a row that saw nothing gives 0, a NaN stays.
__device__ __forceinline__ float inverse(float sum) {
  return sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
}

// A block's share in joining an item that several blocks had: entry 0 of a
// block for the item that it went on with, entry 1 for the one that it began.
struct Split {
  int parts;  // 0: there is none
  int at;     // this block's number among the parts
  int k0, slot;  // the first part: block, and its slot there (then slot 0s)
  int first, lines, g, row0;
};

struct Params {
  const uint16_t *q, *k, *v;
  int64_t q_stride, out_stride, page_stride;
  uint16_t* out;
  Split* split;         // [blocks][2]
  float* part;          // [2 * blocks][rows][D] float32
  float2* part_ml;      // [2 * blocks][rows] maximum and sum
  int page_shift, n_pages, max_pages, words, B, T, max_nodes, Hkv, G;
  float c;
};

// Which positions a kernel attends over: all of each request's; those of each
// request behind its group's shared ones; or the shared ones, for all rows of a
// group, which it then takes for a request.
enum Kind { kAll, kTail, kPrefix };

struct Group {
  int first, n;  // rows
  int positions;
  int request;   // whose table holds the pages
};

// What the last two need besides: what they leave is joined afterwards, also that
// of items which one block had.
struct GroupedParams : Params {
  const int32_t* pre;   // [B + 1] units of work before each request (group)
  const int32_t* from;  // [B] positions that others take
  const Group* groups;  // [B]
  float* whole;         // [T * Hq][D], and
  float2* whole_ml;     // [T * Hq]: rows of items that one block had
};

template <Kind kKind>
using ParamsOf = std::conditional_t<kKind == kAll, Params, GroupedParams>;

struct Request {
  int first, n, L;
  int end;  // positions, the rows' own included (a table holds at most 2^30)
  int units, tiles;
  int from, table;  // the first position, and the row of the page table
};

// kUnit: positions per unit of work; kRows: rows per item.
template <int kRows, int kUnit, Kind kKind>
__device__ __forceinline__ Request request_of(const ParamsOf<kKind>& p,
                                              const int32_t* __restrict__ off,
                                              const int32_t* __restrict__ lengths, int b) {
  Request r;
  r.from = 0;
  r.table = b;
  if constexpr (kKind == kPrefix) {
    const Group g = p.groups[b];
    r.first = g.first;
    r.n = g.n;
    r.L = r.end = g.positions;
    r.table = g.request;
    r.units = (r.end + kUnit - 1) / kUnit;
    r.tiles = (r.n * p.G + kRows - 1) / kRows;
    return r;
  }
  request_rows(off, b, p.T, p.max_nodes, &r.first, &r.n);
  const int cap = p.max_pages << p.page_shift;
  r.L = max(0, min(lengths[b], cap));
  r.end = min(r.L + r.n, cap);
  if constexpr (kKind == kTail) r.from = p.from[b];
  r.units = (r.end - r.from + kUnit - 1) / kUnit;
  r.tiles = (r.n * p.G + kRows - 1) / kRows;
  return r;
}

// The piece of a block's run of units that starts at one of them: units [u0,
// u1) of one item.
struct Piece {
  Request r;
  int b, g, rt, u0, u1;
  bool whole;
};

// Which of `all` blocks this one is; neighbours lie on `xcds` XCDs in turn.
struct Blocks {
  int block, all, xcds;
};
__device__ __forceinline__ Blocks whole_grid() { return {(int)blockIdx.x, (int)gridDim.x, 8}; }

// Deals the units to the blocks in runs of one length; the units before each request
// are kept in LDS. Up to 64 requests are summed in the lanes of each wave, so
// that the first piece needs one round of loads.
template <int kRows, int kUnit, Kind kKind>
struct Dealer {
  const ParamsOf<kKind>& p;
  const int32_t* __restrict__ off;
  const int32_t* __restrict__ lengths;
  int* pre;  // LDS, [B + 1]
  Blocks at_work;
  int begin, stop, share, me;

  __device__ __forceinline__ Dealer(const ParamsOf<kKind>& p_, const int32_t* __restrict__ off_,
                                    const int32_t* __restrict__ lengths_, int* pre_, Blocks at_work_)
      : p(p_), off(off_), lengths(lengths_), pre(pre_), at_work(at_work_) {}

  __device__ __forceinline__ void runs(int total) {
    const int blocks = at_work.all, x = at_work.xcds;
    // Blocks of one XCD (they are dealt out in turn) take neighbouring runs.
    me = (at_work.block % x) * (blocks / x) + at_work.block / x;
    share = max(1, (total + blocks - 1) / blocks);
    begin = (int)min((int64_t)total, (int64_t)me * share);
    stop = min(total, begin + share);
  }

  // The block's first piece; begin == stop if it has none.
  __device__ __forceinline__ Piece first(int* carry) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    if constexpr (kKind != kAll) {
      for (int b = threadIdx.x; b <= p.B; b += kBlock) pre[b] = p.pre[b];
      __syncthreads();
      runs(uniform(pre[p.B]));
      return begin < stop ? at(begin) : Piece{};
    }
    if (p.B <= kWave) {
      const Request mine = request_of<kRows, kUnit, kKind>(p, off, lengths, min(lane, p.B - 1));
      const int units = lane < p.B ? mine.units * mine.tiles * p.Hkv : 0;
      int sum = units;
#pragma unroll
      for (int m = 1; m < kWave; m *= 2) {
        const int o = __shfl_up(sum, m);
        if (lane >= m) sum = add_units(sum, o);
      }
      const int before = sum - units;
      if (wave == 0 && lane < p.B) pre[lane + 1] = sum;
      if (threadIdx.x == 0) pre[0] = 0;
      runs(__builtin_amdgcn_readlane(sum, kWave - 1));
      // The last lane with units whose request starts at or before `begin`.
      const uint64_t m = __ballot(before <= begin && units > 0);
      Piece x;
      x.b = m ? 63 - __clzll(m) : 0;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, x.b); };
      x.r.first = of(mine.first);
      x.r.n = of(mine.n);
      x.r.L = of(mine.L);
      x.r.end = of(mine.end);
      x.r.units = of(mine.units);
      x.r.tiles = of(mine.tiles);
      x.r.from = 0;
      x.r.table = x.b;
      return cut(x, begin, of(before));
    }
    int base = 0;
    for (int b0 = 0; b0 < p.B; b0 += kBlock) {
      const int b = b0 + threadIdx.x;
      int x = 0;
      if (b < p.B) {
        const Request r = request_of<kRows, kUnit, kKind>(p, off, lengths, b);
        x = r.units * r.tiles * p.Hkv;
      }
#pragma unroll
      for (int m = 1; m < kWave; m *= 2) {
        const int o = __shfl_up(x, m);
        if (lane >= m) x = add_units(x, o);
      }
      __syncthreads();
      if (lane == kWave - 1) carry[wave] = x;
      __syncthreads();
      int front = base;
      for (int i = 0; i < kWaves; ++i) {
        if (i < wave) front = add_units(front, carry[i]);
        base = add_units(base, carry[i]);
      }
      if (b < p.B) pre[b + 1] = add_units(front, x);
    }
    if (threadIdx.x == 0) pre[0] = 0;
    __syncthreads();
    runs(uniform(pre[p.B]));
    return at(begin);
  }

  __device__ __forceinline__ Piece cut(Piece x, int unit, int start) const {
    const int rest = unit - start, item = rest / max(1, x.r.units);
    x.u0 = rest - item * x.r.units;
    x.u1 = min(x.r.units, x.u0 + (stop - unit));
    x.g = item / max(1, x.r.tiles);
    x.rt = item - x.g * x.r.tiles;
    x.whole = x.u0 == 0 && x.u1 == x.r.units;
    return x;
  }

  // The piece that starts at `unit`; pre[] is complete (a barrier lies behind).
  __device__ __forceinline__ Piece at(int unit) const {
    Piece x;
    int b = 0;
    for (int hi = p.B; hi - b > 1;) {  // the last request that starts at or before it
      const int mid = (b + hi) / 2;
      if (pre[mid] <= unit) b = mid;
      else hi = mid;
    }
    x.b = uniform(b);
    x.r = request_of<kRows, kUnit, kKind>(p, off, lengths, x.b);
    x.r.first = uniform(x.r.first);
    x.r.n = uniform(x.r.n);
    x.r.L = uniform(x.r.L);
    x.r.end = uniform(x.r.end);
    x.r.units = uniform(x.r.units);
    x.r.tiles = uniform(x.r.tiles);
    if constexpr (kKind != kAll) {
      x.r.from = uniform(x.r.from);
      x.r.table = uniform(x.r.table);
    }
    return cut(x, unit, uniform(pre[x.b]));
  }

  // What the join has to know of a piece.
  __device__ __forceinline__ void leave(const Piece& x, int unit) const {
    if (kKind != kAll || threadIdx.x != 0) return;
    const bool last = unit + x.u1 - x.u0 == stop;
    if (unit == begin && x.u0 == 0) p.split[2 * me].parts = 0;
    if (last && (x.u0 > 0 || x.whole)) p.split[2 * me + 1].parts = 0;
    if (x.whole) return;
    Split s;
    const int start = unit - x.u0;  // the item's first unit
    s.k0 = start / share;
    s.parts = min((start + x.r.units - 1) / share, at_work.all - 1) - s.k0 + 1;
    s.at = me - s.k0;
    s.slot = start == s.k0 * share ? 0 : 1;
    s.first = x.r.first;
    s.lines = x.r.n * p.G;
    s.g = x.g;
    s.row0 = x.rt * kRows;
    p.split[2 * me + (x.u0 > 0 ? 0 : 1)] = s;
  }
  __device__ __forceinline__ void leave_none() const {
    if (kKind == kAll && threadIdx.x < 2) p.split[2 * me + threadIdx.x].parts = 0;
  }
};

// Where the rows of an item that one block had lie: line `line` of its head.
__device__ __forceinline__ int64_t whole_row(const GroupedParams& p, const Piece& x, int line) {
  const int nd = line / p.G;
  return (int64_t)(x.r.first + nd) * p.Hkv * p.G + x.g * p.G + line - nd * p.G;
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
    return seen_bits(mask ? mask + (int64_t)(x.r.first + node[c]) * p.words : mask, p.words, node[c],
                     x.r.n, x.r.L, p0, there);
  }

  // Scores of a tile of 64 positions in LDS, rows D apart: `kt` is the lane's
  // row of the first 16, `chunk` its chunk of the first step. `apart`, here and
  // below, is only named: reads beside a restricted pointer are ones for which
  // the compiler does not wait for loads on their way into LDS (into the other
  // buffer; a barrier lies between these and this tile's).
  __device__ __forceinline__ void scores(const uint16_t* kt, int chunk, f32x4 (&s)[kQ][4],
                                         const uint16_t* __restrict__ apart) const {
#pragma unroll
    for (int st = 0; st < kSteps; ++st)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 raw =
            *reinterpret_cast<const u32x4*>(kt + t * 16 * D + (chunk ^ (st * 4)) * 8);
        const uint4 kf = __builtin_bit_cast(uint4, raw);
#pragma unroll
        for (int c = 0; c < kQ; ++c)
          s[c][t] = mfma<T>(kf, q[c][st], st ? s[c][t] : f32x4{0, 0, 0, 0});
      }
    asm volatile("" ::"s"(apart));
  }

  // Scores without the positions that see[] leaves out.
  template <int kN>
  __device__ __forceinline__ static void hide(f32x4 (&s)[kQ][kN], const uint32_t (&see)[kQ],
                                              int half) {
    const int quad = here((threadIdx.x & 63) >> 4);
#pragma unroll
    for (int c = 0; c < kQ; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(see[c] >> (t * 16 + quad * 4 + i) & 1)) s[c][half * 2 + t][i] = -INFINITY;
  }

  // Probabilities of kN / 2 tiles' scores, in the second product's layout:
  // element e of lane (quad, col) is position e / 4 * 16 + quad * 4 + e % 4 of
  // a tile. They are rounded to the cache's type (half a unit in the last
  // place each, as much as the output's own rounding; of f16, where that is
  // more, 2^-32 of the largest); the sum takes them unrounded. Probabilities,
  // their sum and o are 2^kUp times as large, which 1 / sum takes back.
  template <int kN>
  __device__ __forceinline__ void weigh(const f32x4 (&s)[kQ][kN], float scale,
                                        uint4 (&pr)[kN / 2][kQ]) {
#pragma unroll
    for (int c = 0; c < kQ; ++c) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < kN; ++t)
        mx = most(most(most(mx, s[c][t][0]), s[c][t][1]), most(s[c][t][2], s[c][t][3]));
      mx = max4(mx) * scale;
      // m follows the maximum only when a row has passed it by 2^kLazy.
      if (__any(mx > m[c] + kLazy || (m[c] == -INFINITY && mx > -INFINITY))) {
        const float next = fmaxf(m[c], mx), a = grow(m[c], next);
        m[c] = next;
        sum[c] *= a;
#pragma unroll
        for (int d = 0; d < kCols; ++d) o[c][d] *= a;
      }
      const float base = m[c] == -INFINITY ? 0.0f : m[c] - Exponent<T>::kUp;
#pragma unroll
      for (int h = 0; h < kN / 2; ++h) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          e[i] = __builtin_amdgcn_exp2f(fmaf(s[c][2 * h + i / 4][i % 4], scale, -base));
        sum[c] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        pr[h][c] = pack8<T>(e);
      }
    }
  }

  // o += V^T P^T over 32 rows of V in LDS; at(h, d): where the lane reads 4
  // columns, from 16 d on, of row quad * 4 + col / 4 of half h (it gets column
  // `col` of the rows quad * 4 .. + 3).
  template <class At>
  __device__ __forceinline__ void add(At at, const uint4 (&pr)[kQ],
                                      const uint16_t* __restrict__ apart) {
#pragma unroll
    for (int d = 0; d < kCols; ++d) {
      s16x8 a;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at(h, d));
#pragma unroll
        for (int i = 0; i < 4; ++i) a[h * 4 + i] = x[i];
      }
      const uint4 va = __builtin_bit_cast(uint4, a);
#pragma unroll
      for (int c = 0; c < kQ; ++c) o[c][d] = mfma<T>(va, pr[c], o[c][d]);
    }
    asm volatile("" ::"s"(apart));
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
template <class T, int D, int kQ, int kPages, Kind kKind>
__device__ __forceinline__ void split_items(const ParamsOf<kKind>& p,
                                            const int32_t* __restrict__ table,
                                            const int32_t* __restrict__ off,
                                            const int32_t* __restrict__ lengths,
                                            const uint64_t* __restrict__ mask, char* smem,
                                            Blocks at_work) {
  using R = Rows<T, D, kQ>;
  constexpr int kRows = 16 * kQ, kUnit = kWaves * kTile;
  constexpr int kLanes = D / 8;         // lanes that load a row of V
  constexpr int kPer = kWave / kLanes;  // rows of V per load
  constexpr int kLoads = kTile / kPer;
  __shared__ int carry[kWaves];
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  uint16_t* const vt = reinterpret_cast<uint16_t*>(smem) + wave * kTile * R::kPitch;
  float2* const ml = reinterpret_cast<float2*>(smem + kWaves * kTile * R::kPitch * 2);
  int* const pre = reinterpret_cast<int*>(ml + kWaves * kRows);

  Dealer<kRows, kUnit, kKind> run(p, off, lengths, pre, at_work);
  Piece x = run.first(carry);
  if (run.begin >= run.stop) {
    run.leave_none();
    return;
  }
  const int width = p.Hkv * D, page_mask = (1 << p.page_shift) - 1;
  for (int at = run.begin; at < run.stop;) {
    if (at != run.begin) x = run.at(at);
    run.leave(x, at);
    const int32_t* __restrict__ pages = table + (int64_t)x.r.table * p.max_pages;
    R rows;
    rows.start(p, x, x.rt * kRows);

    // The table's entry for position p0 + lane % 32 (kPages == 1: of the tile),
    // and the page that it is, -1 for none: looked at only where it is used,
    // since waiting for it means waiting for all loads before it.
    auto entry_at = [&](int p0) -> int {
      const int pos = kPages == 1 ? p0 : p0 + (lane & 31);
      return pages[min(pos, x.r.end - 1) >> p.page_shift];
    };
    auto page_of = [&](int entry, int p0) -> int {
      const int pos = kPages == 1 ? p0 : p0 + (lane & 31);
      return pos < x.r.end && entry >= 0 && entry < p.n_pages ? entry : -1;
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

    int p0 = x.r.from + (x.u0 * kWaves + wave) * kTile;
    const int p_end = min(x.r.end, x.r.from + x.u1 * kUnit);
    int page = page_of(entry_at(p0), p0);
    if (p0 < p_end) load_tile(p0, page);
    int entry = entry_at(p0 + kUnit);
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
      if (p0 + kUnit < p_end) {
        page = page_of(entry, p0 + kUnit);
        load_tile(p0 + kUnit, page);
        entry = entry_at(p0 + 2 * kUnit);
      }

      __builtin_amdgcn_sched_barrier(0);
      uint32_t see[kQ];
      if (!inner) {
#pragma unroll
        for (int c = 0; c < kQ; ++c) see[c] = rows.sees(p, mask, x, c, p0, there);
        R::hide(s, see, 0);
      }
      uint4 pr[1][kQ];
      rows.weigh(s, p.c, pr);
      const uint16_t* const vr = vt + (quad * 4 + col / 4) * R::kPitch + (col & 3) * 4;
      rows.add([&](int h, int d) { return vr + h * 16 * R::kPitch + d * 16; }, pr[0], vh);
      while (odd) {
        const int row = __ffs(odd) - 1;
        odd &= odd - 1;
        const int pg = kPages == 1 ? page_now : __shfl(page_now, row);
        rows.add_odd(vh + pg * p.page_stride + (int64_t)((p0 + row) & page_mask) * width, row,
                     pr[0], see);
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
        if (x.whole && (kKind == kAll || (kKind == kTail && x.r.from == 0))) {
          const float inv = inverse(whole);
          const int nd = line / p.G;
          *reinterpret_cast<uint2*>(p.out + (int64_t)(x.r.first + nd) * p.out_stride +
                                    (int64_t)(x.g * p.G + line - nd * p.G) * D + ch * 4) =
              make_uint2(T::pack(y[0] * inv, y[1] * inv), T::pack(y[2] * inv, y[3] * inv));
        } else {
          float* to = p.part + (slot * kRows + c * 16 + row) * D;
          float2* to_ml = p.part_ml + slot * kRows + c * 16 + row;
          if constexpr (kKind != kAll)
            if (x.whole) {
              const int64_t at = whole_row(p, x, line);
              to = p.whole + at * D;
              to_ml = p.whole_ml + at;
            }
          *reinterpret_cast<f32x4*>(to + ch * 4) = y;
          if (ch == 0) *to_ml = make_float2(peak, whole);
        }
      }
      __syncthreads();
    }
    at += x.u1 - x.u0;
  }
}

template <class T, int D, int kQ, int kPages, int kOcc, Kind kKind>
__global__ __launch_bounds__(kBlock, kOcc) void split_kernel(
    const ParamsOf<kKind> p, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  split_items<T, D, kQ, kPages, kKind>(p, table, off, lengths, mask, smem, whole_grid());
}
template <class T, int D, int kQ>
constexpr size_t split_lds() {
  return (size_t)kWaves * kTile * Rows<T, D, kQ>::kPitch * 2 + kWaves * 16 * kQ * 8;
}

// The four waves take kQ groups of 16 rows each and share tiles of 64
// positions, which go straight from the cache into one of two LDS buffers
// (no registers, no LDS instructions) while the other is multiplied. A row of
// a tile is D / 8 chunks of 16 bytes, chunk c at place c ^ turn(row): the
// transposing reads of four rows and the operand reads of eight hit different
// banks, as rows of other lengths would do, which these loads cannot write.
// kEven: a page holds the rows that a wave loads at once, whose address is the
// wave's then.
template <class T, int D, int kQ, bool kEven, Kind kKind>
__device__ __forceinline__ void shared_items(const ParamsOf<kKind>& p,
                                             const int32_t* __restrict__ table,
                                             const int32_t* __restrict__ off,
                                             const int32_t* __restrict__ lengths,
                                             const uint64_t* __restrict__ mask, uint16_t* tiles,
                                             int* pre, Blocks at_work) {
  using R = Rows<T, D, kQ>;
  constexpr int kRows = 16 * kQ * kWaves, kUnit = 2 * kTile;
  constexpr int kLanes = D / 8;            // lanes per row
  constexpr int kHave = kWave / kLanes;    // rows per load of a wave
  constexpr int kLoads = kUnit / (kHave * kWaves);
  constexpr int kTileElems = kUnit * D;
  // tiles: [buffer][K, V][kUnit][D]
  __shared__ int carry[kWaves];
  __shared__ uint32_t odd_rows[3][2];  // of the tiles, in turn
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  auto turn_of = [](int row) { return (D == 64 ? row >> 1 & 3 : row & 7) * 2; };

  Dealer<kRows, kUnit, kKind> run(p, off, lengths, pre, at_work);
  Piece x = run.first(carry);
  if (run.begin >= run.stop) {
    run.leave_none();
    return;
  }
  const int width = p.Hkv * D, page_mask = (1 << p.page_shift) - 1;
  // The lane's row and chunk in a wave's load (load j: rows j * kHave * kWaves
  // on; a multiple of 8 rows, so that the chunk is the same in all of them).
  const int my_row = wave * kHave + lane / kLanes;
  const int my_chunk = lane % kLanes ^ turn_of(my_row);
  const uint32_t my_at = (lane / kLanes * width + my_chunk * 8) * 2;
  // Where the lane reads K (first step) and V (first columns) of a tile.
  const int k_chunk = quad ^ turn_of(col), v_row = quad * 4 + col / 4;
  const int v_chunk = (col & 3) / 2 ^ turn_of(v_row);
  for (int at = run.begin; at < run.stop;) {
    if (at != run.begin) x = run.at(at);
    run.leave(x, at);
    const int32_t* __restrict__ pages = table + (int64_t)x.r.table * p.max_pages;
    const uint16_t* const kh = p.k + (int64_t)x.g * D;
    const uint16_t* const vh = p.v + (int64_t)x.g * D;
    const int row0 = x.rt * kRows + wave * 16 * kQ;
    const bool busy = row0 < x.r.n * p.G;  // the wave has rows of its own
    R rows;
    rows.start(p, x, row0);

    // The table's entry for position p0 + lane and the page that it is, as above.
    auto entry_at = [&](int p0) -> int {
      return pages[min(p0 + lane, x.r.end - 1) >> p.page_shift];
    };
    auto page_of = [&](int entry, int p0) -> int {
      return p0 + lane < x.r.end && entry >= 0 && entry < p.n_pages ? entry : -1;
    };
    // Starts the loads of the tile at p0 into buffer `buf`; positions without
    // a page read page 0.
    auto load_tile = [&](int p0, int page, int buf) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = (j * kWaves + wave) * kHave;  // the wave's first
        lds_u16* const to = (lds_u16*)(tiles + buf * 2 * kTileElems + row * D);
        if (kEven) {
          const int64_t from =
              (int64_t)max(__builtin_amdgcn_readlane(page, row), 0) * p.page_stride +
              (int64_t)((p0 + row) & page_mask) * width;
          load_lds16(make_rsrc(kh + from, kHave * width * 2), to, my_at, 0);
          load_lds16(make_rsrc(vh + from, kHave * width * 2), to + kTileElems, my_at, 0);
        } else {
          const int mine = row + lane / kLanes, pg = __shfl(page, mine);
          const int64_t from = (pg < 0 ? 0 : pg * p.page_stride +
                                (int64_t)((p0 + mine) & page_mask) * width) + my_chunk * 8;
          load_lds(kh + from, to);
          load_lds(vh + from, to + kTileElems);
        }
      }
    };
    // Waits for the wave's own loads of the tile at p0 and mends its rows of V:
    // those that are not there become 0, infinities and NaN past L too, noted.
    auto finish_tile = [&](int p0, int page, int buf, int turn) {
      TG_WAIT_VM(0);
      asm volatile("" ::: "memory");
      if (p0 + kUnit <= x.r.L && __all(page >= 0)) return;
      const unsigned long long there = __ballot(page >= 0);
#pragma unroll 1
      for (int j = 0; j < kLoads; ++j) {
        const int row = (j * kWaves + wave) * kHave + lane / kLanes;
        const bool gone = !(there >> row & 1), own = p0 + row >= x.r.L;
        u32x4* const place = reinterpret_cast<u32x4*>(
            tiles + (buf * 2 + 1) * kTileElems + (j * kWaves + wave) * kHave * D + lane * 8);
        u32x4 y = *place;
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t odd = own ? odd_part<T>(y[i], true) : 0u;
          y[i] = gone ? 0u : y[i] ^ odd;
          bad |= odd;
        }
        if (bad && !gone) atomicOr(&odd_rows[turn][row / 32], 1u << (row % 32));
        *place = y;
      }
    };

    int p0 = x.r.from + x.u0 * kUnit, buf = 0, turn = 0;
    const int p_end = x.r.from + x.u1 * kUnit;
    int page = page_of(entry_at(p0), p0), entry = entry_at(p0 + kUnit);
    __syncthreads();  // the last piece's reads are over
    if (threadIdx.x < 6) odd_rows[threadIdx.x / 2][threadIdx.x % 2] = 0;
    load_tile(p0, page, 0);
    __syncthreads();
    finish_tile(p0, page, 0, 0);
    __syncthreads();
    for (; p0 < p_end; p0 += kUnit, buf ^= 1) {
      const bool more = p0 + kUnit < p_end;
      const int page_now = page;
      const uint16_t* const kt = tiles + buf * 2 * kTileElems;
      f32x4 s[kQ][4];
      if (busy) rows.scores(kt + col * D, k_chunk, s, kh);
      if (more) {
        page = page_of(entry, p0 + kUnit);
        load_tile(p0 + kUnit, page, buf ^ 1);
        entry = entry_at(p0 + 2 * kUnit);
      }
      const bool inner = p0 + kUnit <= x.r.L && __all(page_now >= 0);
      if (busy) {
        const unsigned long long there64 = inner ? ~0ull : __ballot(page_now >= 0);
        uint32_t see[2][kQ];
        if (!inner) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t there = (uint32_t)(there64 >> (half * 32));
#pragma unroll
            for (int c = 0; c < kQ; ++c)
              see[half][c] = rows.sees(p, mask, x, c, p0 + half * kTile, there);
            R::hide(s, see[half], half);
          }
        }
        uint4 pr[2][kQ];
        rows.weigh(s, p.c, pr);
        const uint16_t* const vr = kt + kTileElems + v_row * D + (col & 1) * 4;
#pragma unroll
        for (int half = 0; half < 2; ++half)
          rows.add([&](int h, int d) {
            return vr + (half * kTile + h * 16) * D + (v_chunk ^ (d * 2)) * 8;
          }, pr[half], vh);
        if (!inner) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t odd = odd_rows[turn][half];
            while (odd) {
              const int row = __ffs(odd) - 1;
              odd &= odd - 1;
              const int pg = __shfl(page_now, half * kTile + row);
              rows.add_odd(vh + pg * p.page_stride +
                               (int64_t)((p0 + half * kTile + row) & page_mask) * width,
                           row, pr[half], see[half]);
            }
          }
        }
      }
      // One tile's notes are read, the next one's written, and those of the
      // one after it (read before the last barrier) cleared.
      const int next = turn == 2 ? 0 : turn + 1;
      if (threadIdx.x < 2) odd_rows[next == 2 ? 0 : next + 1][threadIdx.x] = 0;
      if (more) finish_tile(p0 + kUnit, page, buf ^ 1, next);
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
          if (x.whole && (kKind == kAll || (kKind == kTail && x.r.from == 0))) {
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
            float* to = p.part + line_at * D;
            float2* to_ml = p.part_ml + line_at;
            if constexpr (kKind != kAll)
              if (x.whole) {
                const int64_t at = whole_row(p, x, line);
                to = p.whole + at * D;
                to_ml = p.whole_ml + at;
              }
#pragma unroll
            for (int d = 0; d < R::kCols; ++d)
              *reinterpret_cast<f32x4*>(to + d * 16 + quad * 4) = rows.o[c][d];
            if (quad == 0) *to_ml = make_float2(rows.m[c], whole);
          }
        }
      }
    }
    at += x.u1 - x.u0;
  }
}

template <class T, int D, int kQ, bool kEven, int kOcc, Kind kKind>
__global__ __launch_bounds__(kBlock, kOcc) void shared_kernel(
    const ParamsOf<kKind> p, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask) {
  __shared__ __attribute__((aligned(16))) uint16_t tiles[8 * kTile * D];
  extern __shared__ __attribute__((aligned(16))) int pre[];
  shared_items<T, D, kQ, kEven, kKind>(p, table, off, lengths, mask, tiles, pre, whole_grid());
}

// Which kernel: the rows of one KV head that requests have (at most, or as a
// caller who cannot say so expects), over 16-row groups. Up to 32 rows
// the split kernel reads the cache once per item; above, tiles of 64 rows in a
// wave by itself take too many registers (64-row trees: 822 us split, 384
// shared, in the kernels' first forms), and 128 rows per tile halve what is
// read again for the next 128 (64-row trees 224 us, with 64-row tiles 314).
// Heads of 256 leave registers for 16 rows a wave.
struct Shape {
  int q;        // 16-row groups per wave
  bool shared;  // waves share tiles (rows over four waves), or split them
};

Shape shape_for(long long rows, int D) {
  if (rows <= 16) return {1, false};
  if (D == 256) return {1, true};
  if (rows <= 32) return {2, false};
  if (rows <= 64) return {1, true};
  return {2, true};
}

Shape shape_of(const tg_tree_attn_args* a) {
  const int nodes = a->typical_nodes > 0 && a->typical_nodes < a->max_nodes ? a->typical_nodes
                                                                           : a->max_nodes;
  return shape_for((long long)nodes * (a->Hq / a->cache.Hkv), a->cache.D);
}

// Waves per SIMD that the registers leave without spills (heads of 256 with
// two: a decode batch of 64 takes 223 us instead of 122).
constexpr int occupancy(int D, int q) {
  return D == 64 ? (q == 2 ? 2 : 3) : D == 128 ? 2 : 1;
}

constexpr int rows_of(Shape s) { return 16 * s.q * (s.shared ? kWaves : 1); }
constexpr int unit_of(Shape s) { return s.shared ? 2 * kTile : kWaves * kTile; }

// The parameters that all calls have.
inline void fill(Params* p, const tg_tree_attn_args* a) {
  const tg_kv_cache& c = a->cache;
  p->q = static_cast<const uint16_t*>(a->q);
  p->k = static_cast<const uint16_t*>(c.k) + a->layer * c.layer_stride;
  p->v = static_cast<const uint16_t*>(c.v) + a->layer * c.layer_stride;
  p->q_stride = a->q_stride;
  p->out_stride = a->out_stride;
  p->page_stride = c.page_stride;
  p->out = static_cast<uint16_t*>(a->out);
  p->page_shift = __builtin_ctz(c.page_size);
  p->n_pages = c.n_pages;
  p->max_pages = c.max_pages;
  p->words = a->mask_words;
  p->B = c.B;
  p->T = a->T;
  p->max_nodes = a->max_nodes;
  p->Hkv = c.Hkv;
  p->G = a->Hq / c.Hkv;
  p->c = a->scale * 1.4426950408889634f;
}

// Launches the kernel for these rows; p.B: requests or groups.
template <class T, int D, int kQ, bool kShared, Kind kKind>
hipError_t launch_items(const ParamsOf<kKind>& p, const tg_tree_attn_args* a, hipStream_t s) {
  constexpr int kOcc = occupancy(D, kQ);
  const tg_kv_cache& c = a->cache;
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
  const size_t pre = (size_t)(p.B + 1) * 4;
  if constexpr (kShared) {
    return c.page_size >= 512 / D ? go(shared_kernel<T, D, kQ, true, kOcc, kKind>, pre)
                                  : go(shared_kernel<T, D, kQ, false, kOcc, kKind>, pre);
  } else {
    const size_t lds = split_lds<T, D, kQ>() + pre;
    return c.page_size >= kTile       ? go(split_kernel<T, D, kQ, 1, kOcc, kKind>, lds)
           : c.page_size == kTile / 2 ? go(split_kernel<T, D, kQ, 2, kOcc, kKind>, lds)
                                      : go(split_kernel<T, D, kQ, 0, kOcc, kKind>, lds);
  }
}

}  // namespace
}  // namespace tg
