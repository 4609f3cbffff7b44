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

// The blocks that work is dealt to: those of the grid, or every other one of them.
// Neighbours lie on kXcds XCDs in turn.
struct WholeGrid {
  static constexpr uint32_t kXcds = 8;
  static __device__ __forceinline__ uint32_t block() { return blockIdx.x; }
  static __device__ __forceinline__ int blocks() { return (int)gridDim.x; }
};
struct HalfGrid {
  static constexpr uint32_t kXcds = 4;
  static __device__ __forceinline__ uint32_t block() { return blockIdx.x / 2; }
  static __device__ __forceinline__ int blocks() { return (int)gridDim.x / 2; }
};

// Deals the units to the blocks in runs of one length; the units before each request
// are kept in LDS. Up to 64 requests are summed in the lanes of each wave, so
// that the first piece needs one round of loads.
template <int kRows, int kUnit, Kind kKind, class Grid>
struct Dealer {
  const ParamsOf<kKind>& p;
  const int32_t* __restrict__ off;
  const int32_t* __restrict__ lengths;
  int* pre;  // LDS, [B + 1]
  int begin, stop, share, me;

  __device__ __forceinline__ Dealer(const ParamsOf<kKind>& p_, const int32_t* __restrict__ off_,
                                    const int32_t* __restrict__ lengths_, int* pre_)
      : p(p_), off(off_), lengths(lengths_), pre(pre_) {}

  __device__ __forceinline__ void runs(int total) {
    const int blocks = Grid::blocks();
    share = max(1, (total + blocks - 1) / blocks);
    // Blocks of one XCD (they are dealt out in turn) take neighbouring runs.
    int each = blocks / (int)Grid::kXcds;
    // Few runs are spread over all XCDs: 8 requests behind 2048 positions 24 us (on two
    // of them) and 11.6.
    if constexpr (kKind != kAll) {
      const int used = (total + share - 1) / share;
      each = (used + (int)Grid::kXcds - 1) / (int)Grid::kXcds;
      if ((int)(Grid::block() / Grid::kXcds) >= each) {
        begin = stop = 0;
        return;
      }
    }
    me = (Grid::block() % Grid::kXcds) * each + Grid::block() / Grid::kXcds;
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
    s.parts = min((start + x.r.units - 1) / share, Grid::blocks() - 1) - s.k0 + 1;
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
template <class T, int D, int kQ, int kPages, int kOcc, Kind kKind>
__global__ __launch_bounds__(kBlock, kOcc) void split_kernel(
    const ParamsOf<kKind> p, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask) {
  using Grid = WholeGrid;
  extern __shared__ __attribute__((aligned(16))) char smem[];
#include "tg_attn_split.h"
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
template <class T, int D, int kQ, bool kEven, int kOcc, Kind kKind>
__global__ __launch_bounds__(kBlock, kOcc) void shared_kernel(
    const ParamsOf<kKind> p, const int32_t* __restrict__ table, const int32_t* __restrict__ off,
    const int32_t* __restrict__ lengths, const uint64_t* __restrict__ mask) {
  using Grid = WholeGrid;
  __shared__ __attribute__((aligned(16))) uint16_t tiles[8 * kTile * D];
  extern __shared__ __attribute__((aligned(16))) int pre[];
#include "tg_attn_shared.h"
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
