// Attention of a batch whose groups of requests share the pages of a prefix.
//
// The rows of a group (all its requests' nodes) see the prefix alike, so they are
// one item's rows there, and its keys and values are read once for up to 128 of
// them instead of once per request; each request's own rows then see its other
// positions. Both are the kernels of tg_attn.h, over a group's shared positions
// and over each request's from there on, and leave, for every row and for every
// run of positions that one block had, its maximum m_i, sum l_i and output o_i
// (float32); a row's output is sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i.
//
//   plan    one block: what each group really shares (not past any member's
//           length, whole units of 128 positions), and the units of work before
//           each group and request;
//   prefix, tail;
//   join    a block takes one to four heads of a row, a wave every fourth part.
//
// 128 tokens behind 8192 shared positions and up to 512 of their own (heads 32 / 8
// of 128, bf16): plan 5 us, prefixes and tails 63, join 10, among other calls 85 (433
// through each request's own table). The 63 us are neither the memory's (27 us at its
// rate) nor the matrix unit's (16 % of the time at work): the prefixes have half of the
// device (see both_kernel), and their 17.2 GFLOP would take it 56 us at half of the next
// case's rate. 16 trees of up to 12 rows behind 30000 positions: the prefix's kernel 95
// us, 610 TFLOP/s (matrix unit 32 %, vector unit 44 %, waits 37 %), tails 13, join 11.
#include "tg_attn.h"

namespace tg {
namespace {

constexpr int kMaxRequests = 4096;
constexpr int kWholeUnits = 128;  // positions; a multiple of both kernels' units

struct PlanParams {
  int B, groups, T, max_nodes, cap, G, Hkv;
  int prefix_rows, prefix_unit, tail_rows, tail_unit;  // of the two kernels
  const int32_t *off, *lengths, *group_off, *shared;
  int32_t *pre_prefix, *pre_tail;  // [groups + 1], [B + 1]
  int32_t *from, *group_of;        // [B]
  int32_t* request_of_row;         // [T], -1: none
  Group* group;                    // [groups]
};

// The last i in [0, n) with a[i] <= x, 0 if there is none.
__device__ __forceinline__ int last_at(const int* a, int n, int x) {
  int i = 0;
  for (int hi = n; hi - i > 1;) {
    const int mid = (i + hi) / 2;
    if (a[mid] <= x) i = mid;
    else hi = mid;
  }
  return i;
}

// Every thread has the requests and the groups tid, tid + kThreads and so on, kEach at
// most; what it reads of them is read at once.
template <int kThreads, int kEach>
__global__ __launch_bounds__(kThreads) void plan_kernel(const PlanParams p) {
  constexpr int kMost = kThreads * kEach, kPlanWaves = kThreads / kWave;
  __shared__ int starts[kMost + 1];  // of groups: a request
  __shared__ int rows[kMost + 1];    // of requests: a row
  __shared__ int least[kMost];       // of a group: its shared positions
  __shared__ int member[kMost];      // the first one with rows
  __shared__ int last[kMost];        // and the last
  __shared__ int carry[2][kPlanWaves];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  int first[kEach], next[kEach], length[kEach], group[kEach];
  // Offsets that do not ascend from 0 to B stay inside all arrays.
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = k * kThreads + tid;
    if (i < p.B) {
      first[k] = p.off[i];
      next[k] = p.off[i + 1];
      length[k] = p.lengths[i];
    }
    if (i < p.groups) {
      starts[i] = max(0, min(p.group_off[i], p.B));
      least[i] = max(0, min(p.shared[i], p.cap));
      member[i] = p.B;
      last[i] = -1;
    }
  }
  if (tid == 0) {
    rows[p.B] = max(0, min(p.off[p.B], p.T));
    starts[p.groups] = p.groups ? max(0, min(p.group_off[p.groups], p.B)) : 0;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int b = k * kThreads + tid;
    if (b >= p.B) break;
    int g = p.groups ? last_at(starts, p.groups, b) : -1;
    if (g >= 0 && (b < starts[g] || b >= starts[g + 1])) g = -1;
    p.group_of[b] = group[k] = g;
    first[k] = max(0, min(first[k], p.T));
    next[k] = max(0, min(next[k], p.T));
    rows[b] = first[k];
    if (g >= 0 && next[k] > first[k]) {
      atomicMin(&least[g], max(0, length[k]));
      atomicMin(&member[g], b);
      atomicMax(&last[g], b);
    }
  }
  __syncthreads();
  // One request alone shares nothing.
  int units[2][kEach] = {};  // of groups, of requests
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int g = k * kThreads + tid;
    if (g >= p.groups) break;
    const int shared = member[g] < last[g] ? least[g] / kWholeUnits * kWholeUnits : 0;
    least[g] = shared;
    Group x;
    const int b0 = starts[g], b1 = max(b0, starts[g + 1]);
    x.first = rows[b0];
    x.n = shared ? max(x.first, rows[b1]) - x.first : 0;
    x.positions = shared;
    x.request = min(member[g], p.B - 1);
    p.group[g] = x;
    units[0][k] = (x.positions + p.prefix_unit - 1) / p.prefix_unit *
                  ((x.n * p.G + p.prefix_rows - 1) / p.prefix_rows) * p.Hkv;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int b = k * kThreads + tid;
    if (b >= p.B) break;
    const int from = group[k] >= 0 ? least[group[k]] : 0;
    p.from[b] = from;
    const int n = max(0, min(next[k] - first[k], p.max_nodes));
    const int L = max(0, min(length[k], p.cap)), end = min(L + n, p.cap);
    units[1][k] = (end - from + p.tail_unit - 1) / p.tail_unit *
                  ((n * p.G + p.tail_rows - 1) / p.tail_rows) * p.Hkv;
  }
  // Both running sums.
  int base[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    if (k * kThreads >= max(p.B, p.groups)) break;
    int x[2] = {units[0][k], units[1][k]};
    for (int m = 1; m < kWave; m *= 2) {
      const int o[2] = {__shfl_up(x[0], m), __shfl_up(x[1], m)};
      if (lane >= m) x[0] = add_units(x[0], o[0]), x[1] = add_units(x[1], o[1]);
    }
    if (k) __syncthreads();
    if (lane == kWave - 1) carry[0][wave] = x[0], carry[1][wave] = x[1];
    __syncthreads();
    const int i = k * kThreads + tid;
    for (int j = 0; j < 2; ++j) {
      int front = base[j];
      for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) front = add_units(front, carry[j][w]);
        base[j] = add_units(base[j], carry[j][w]);
      }
      if (i < (j ? p.B : p.groups)) (j ? p.pre_tail : p.pre_prefix)[i + 1] = add_units(front, x[j]);
    }
  }
  if (tid == 0) p.pre_prefix[0] = p.pre_tail[0] = 0;
  for (int t = tid; t < p.T; t += kThreads) {
    const int b = last_at(rows, p.B, t);
    p.request_of_row[t] = t >= rows[b] && t < min(rows[b + 1], rows[b] + p.max_nodes) ? b : -1;
  }
}

// Where a kernel left its items.
struct Parts {
  const int32_t* pre;
  const float* part;
  const float2* part_ml;
  const float* whole;
  const float2* whole_ml;
  int row_bits, unit_bits, blocks;  // powers of two: rows of an item, positions of a unit
};

struct JoinParams {
  Parts prefix, tail;
  const int32_t *off, *lengths, *from, *group_of, *request_of_row;
  const Group* group;
  uint16_t* out;
  int64_t out_stride;
  int T, Hkv, G, cap, max_nodes, B, groups;
};

__device__ __forceinline__ int pieces(int n, int bits) { return (n + (1 << bits) - 1) >> bits; }

// A running join of a row's parts, four columns to a lane.
struct Joined {
  f32x4 o = f32x4{0, 0, 0, 0};
  float m = -INFINITY, sum = 0.0f;

  __device__ __forceinline__ void add(f32x4 x, float2 ml) {
    const float next = fmaxf(m, ml.x), a = grow(m, next), e = grow(ml.x, next);
    m = next;
    sum = sum * a + ml.y * e;
    o = o * a + x * e;
  }
};

// Adds the parts of a row: line `line` of head g of the items from unit `pre` of
// `total` on, `tiles` times `units` units a head; `row`: its place among whole items' rows.
// Every wave adds every fourth one.
template <int D>
__device__ __forceinline__ void add_parts(Joined& j, const Parts& s, int total, int pre, int g, int line,
                                          int units, int tiles, int64_t row, int ch, int wave) {
  if (units <= 0) return;
  constexpr int kU = 4;
  const int share = max(1, (total + s.blocks - 1) / s.blocks);
  const int start = pre + (g * tiles + (line >> s.row_bits)) * units;
  const int k0 = start / share, parts = (start + units - 1) / share - k0 + 1;
  if (parts == 1) {
    if (wave == 0) j.add(*reinterpret_cast<const f32x4*>(s.whole + row * D + ch * 4), s.whole_ml[row]);
    return;
  }
  const int slot = start == k0 * share ? 0 : 1, at = line & ((1 << s.row_bits) - 1);
  for (int k = wave; k < parts; k += kU * kWaves) {
    f32x4 x[kU];
    float2 ml[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = min(k + u * kWaves, parts - 1);
      const int block = min(k0 + i, s.blocks - 1);
      const int64_t place = ((2 * (int64_t)block + (i == 0 ? slot : 0)) << s.row_bits) + at;
      x[u] = *reinterpret_cast<const f32x4*>(s.part + place * D + ch * 4);
      ml[u] = s.part_ml[place];
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (k + u * kWaves < parts) j.add(x[u], ml[u]);
  }
}

template <class T, int D>
__global__ __launch_bounds__(kBlock) void join_parts_kernel(const JoinParams p) {
  constexpr int kLine = D / 4, kAt = kWave / kLine;  // lanes per row, rows per wave
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int t = blockIdx.x, Hq = p.Hkv * p.G, ch = lane % kLine;
  const int b = p.request_of_row[t];
  __shared__ f32x4 os[kWaves][kWave];
  __shared__ float2 mls[kWaves][kWave];
  if (b < 0) return;
  const int head0 = blockIdx.y * kAt + lane / kLine, head = min(head0, Hq - 1);
  const int g = head / p.G, jj = head - g * p.G;
  const int from = p.from[b], gr = p.group_of[b];
  int first, n;
  request_rows(p.off, b, p.T, p.max_nodes, &first, &n);
  const int L = max(0, min(p.lengths[b], p.cap)), end = min(L + n, p.cap);
  const int total = p.tail.pre[p.B], pre = p.tail.pre[b];
  const int units = pieces(end - from, p.tail.unit_bits);
  const int tiles = pieces(n * p.G, p.tail.row_bits);
  const int line = (t - first) * p.G + jj;
  const int64_t row = (int64_t)t * Hq + head;
  Joined j;
  bool there = false;  // one block's rows are in the output already
  if (from > 0) {
    const Group x = p.group[gr];
    if (t >= x.first && t < x.first + x.n)  // (offsets that do not ascend)
      add_parts<D>(j, p.prefix, p.prefix.pre[p.groups], p.prefix.pre[gr], g,
                   (t - x.first) * p.G + jj, pieces(x.positions, p.prefix.unit_bits),
                   pieces(x.n * p.G, p.prefix.row_bits), row, ch, wave);
  } else {
    const int share = max(1, (total + p.tail.blocks - 1) / p.tail.blocks);
    const int start = pre + (g * tiles + (line >> p.tail.row_bits)) * units;
    there = start / share == (start + units - 1) / share;
  }
  if (!there) add_parts<D>(j, p.tail, total, pre, g, line, units, tiles, row, ch, wave);
  os[wave][lane] = j.o;
  mls[wave][lane] = make_float2(j.m, j.sum);
  __syncthreads();
  if (wave > 0 || there || head0 >= Hq) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) j.add(os[w][lane], mls[w][lane]);
  const float inv = inverse(j.sum);
  *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.out_stride + (int64_t)head * D + ch * 4) =
      make_uint2(T::pack(j.o[0] * inv, j.o[1] * inv), T::pack(j.o[2] * inv, j.o[3] * inv));
}

// The kernel for the prefixes goes by the mean rows of a group.
Shape prefix_shape(const tg_prefix_attn_args* a) {
  const tg_tree_attn_args& x = a->attn;
  const int groups = a->n_groups > 0 ? a->n_groups : 1;
  return shape_for((long long)(x.T + groups - 1) / groups * (x.Hq / x.cache.Hkv), x.cache.D);
}

int blocks_of(Shape s, int D) { return kCus * occupancy(D, s.q); }
int least_blocks(Shape s, Shape t, int D) {
  return blocks_of(s, D) < blocks_of(t, D) ? blocks_of(s, D) : blocks_of(t, D);
}

struct Space {
  int32_t *pre_prefix, *pre_tail, *from, *group_of, *request_of_row;
  Group* group;
  float *part[2], *whole[2];  // of the prefixes, of the tails
  float2 *part_ml[2], *whole_ml[2];
};

Space carve(const tg_prefix_attn_args* a, char* base, size_t* bytes) {
  size_t off = 0;
  auto take = [&](size_t n) -> char* {
    char* p = base ? base + off : nullptr;
    off += (n + 255) & ~(size_t)255;
    return p;
  };
  const tg_tree_attn_args& x = a->attn;
  const size_t B = x.cache.B, G = a->n_groups, D = x.cache.D, rows = (size_t)x.T * x.Hq;
  Space s;
  s.pre_prefix = reinterpret_cast<int32_t*>(take((G + 1) * 4));
  s.pre_tail = reinterpret_cast<int32_t*>(take((B + 1) * 4));
  s.from = reinterpret_cast<int32_t*>(take(B * 4));
  s.group_of = reinterpret_cast<int32_t*>(take(B * 4));
  s.request_of_row = reinterpret_cast<int32_t*>(take((size_t)x.T * 4));
  s.group = reinterpret_cast<Group*>(take(G * sizeof(Group)));
  for (int i = 0; i < 2; ++i) {
    const Shape sh = i == 0 ? prefix_shape(a) : shape_of(&x);
    const size_t slots = 2 * (size_t)blocks_of(sh, x.cache.D) * rows_of(sh);
    s.part_ml[i] = reinterpret_cast<float2*>(take(slots * 8));
    s.part[i] = reinterpret_cast<float*>(take(slots * D * 4));
    s.whole_ml[i] = reinterpret_cast<float2*>(take(rows * 8));
    s.whole[i] = reinterpret_cast<float*>(take(rows * D * 4));
  }
  *bytes = off;
  return s;
}

// Both in one launch, for tails of at most 16 rows a KV head: every other block takes
// prefixes, the others tails. Blocks go to the XCDs in turn, so prefixes have four of
// the eight and tails the other four, and no CU has both. (One launch less: 128 requests
// behind 8192 tokens 100 us instead of 104, four behind 1000, a case now left to tree
// attention, 21 instead of 30.)
template <class T, int D, int kPrefixQ, bool kShared, int kPagesOf, int kOcc>
__global__ __launch_bounds__(kBlock, kOcc) void both_kernel(
    const GroupedParams prefix, const GroupedParams tail, const int32_t* __restrict__ table,
    const int32_t* __restrict__ off, const int32_t* __restrict__ lengths,
    const uint64_t* __restrict__ mask) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  using Grid = HalfGrid;
  if (blockIdx.x % 2) {
    constexpr Kind kKind = kTail;
    constexpr int kQ = 1, kPages = kPagesOf;
    const GroupedParams& p = tail;
#include "tg_attn_split.h"
  } else if constexpr (kShared) {
    constexpr Kind kKind = kPrefix;
    constexpr int kQ = kPrefixQ;
    constexpr bool kEven = kPagesOf != 0;
    const GroupedParams& p = prefix;
    uint16_t* const tiles = reinterpret_cast<uint16_t*>(smem);
    int* const pre = reinterpret_cast<int*>(smem + 8 * kTile * D * 2);
#include "tg_attn_shared.h"
  } else {
    constexpr Kind kKind = kPrefix;
    constexpr int kQ = kPrefixQ, kPages = kPagesOf;
    const GroupedParams& p = prefix;
#include "tg_attn_split.h"
  }
}

bool merged(const tg_prefix_attn_args* a) {
  const Shape tail = shape_of(&a->attn);
  return tail.q == 1 && !tail.shared;
}

template <class T, int D, int kQ, bool kShared>
hipError_t launch_both(const GroupedParams& prefix, const GroupedParams& tail,
                       const tg_tree_attn_args* a, hipStream_t s) {
  constexpr int kOcc = occupancy(D, kQ) < occupancy(D, 1) ? occupancy(D, kQ) : occupancy(D, 1);
  const tg_kv_cache& c = a->cache;
  const size_t one = (kShared ? (size_t)8 * kTile * D * 2 : split_lds<T, D, kQ>()) + (prefix.B + 1) * 4;
  const size_t two = split_lds<T, D, 1>() + (tail.B + 1) * 4, lds = one > two ? one : two;
  auto go = [&](auto* kernel) -> hipError_t {
    if (lds > 48 * 1024) {
      const hipError_t e =
          hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(2 * kCus * kOcc), dim3(kBlock), lds, s, prefix, tail,
                       c.page_table, a->q_offsets, a->lengths, a->tree_mask);
    return hipGetLastError();
  };
  return c.page_size >= kTile       ? go(both_kernel<T, D, kQ, kShared, 1, kOcc>)
         : c.page_size == kTile / 2 ? go(both_kernel<T, D, kQ, kShared, 2, kOcc>)
                                    : go(both_kernel<T, D, kQ, kShared, 0, kOcc>);
}

template <class T, int D, Kind kKind>
hipError_t launch_kind(Shape sh, const GroupedParams& p, const tg_tree_attn_args* a, hipStream_t s) {
  if (sh.q == 1 && sh.shared) return launch_items<T, D, 1, true, kKind>(p, a, s);
  if constexpr (kKind == kPrefix)  // (such tails go by launch_both)
    if (sh.q == 1) return launch_items<T, D, 1, false, kKind>(p, a, s);
  if constexpr (D < 256)
    return sh.shared ? launch_items<T, D, 2, true, kKind>(p, a, s)
                     : launch_items<T, D, 2, false, kKind>(p, a, s);
  return hipErrorInvalidValue;  // shape_for() gives no other
}

template <class T, int D>
hipError_t launch(const tg_prefix_attn_args* a, void* ws, hipStream_t s) {
  const tg_tree_attn_args& x = a->attn;
  const tg_kv_cache& c = x.cache;
  const Shape shapes[2] = {prefix_shape(a), shape_of(&x)};
  size_t bytes;
  const Space sp = carve(a, static_cast<char*>(ws), &bytes);
  const int cap = c.max_pages * c.page_size;
  PlanParams plan;
  plan.B = c.B;
  plan.groups = a->n_groups;
  plan.T = x.T;
  plan.max_nodes = x.max_nodes;
  plan.cap = cap;
  plan.G = x.Hq / c.Hkv;
  plan.Hkv = c.Hkv;
  plan.prefix_rows = rows_of(shapes[0]);
  plan.prefix_unit = unit_of(shapes[0]);
  plan.tail_rows = rows_of(shapes[1]);
  plan.tail_unit = unit_of(shapes[1]);
  plan.off = x.q_offsets;
  plan.lengths = x.lengths;
  plan.group_off = a->group_offsets;
  plan.shared = a->shared;
  plan.pre_prefix = sp.pre_prefix;
  plan.pre_tail = sp.pre_tail;
  plan.from = sp.from;
  plan.group_of = sp.group_of;
  plan.request_of_row = sp.request_of_row;
  plan.group = sp.group;
  // Fewer waves wait for each other sooner: 61 requests 3.8 us, by 16 waves 4.5.
  if (c.B <= 256 && a->n_groups <= 256 && x.T <= 1024)
    hipLaunchKernelGGL((plan_kernel<256, 1>), dim3(1), dim3(256), 0, s, plan);
  else
    hipLaunchKernelGGL((plan_kernel<1024, kMaxRequests / 1024>), dim3(1), dim3(1024), 0, s, plan);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  JoinParams j;
  GroupedParams both[2];
  const bool merge = merged(a);
  for (int i = 0; i < 2; ++i) {
    GroupedParams& p = both[i];
    fill(&p, &x);
    p.split = nullptr;
    p.from = sp.from;
    p.groups = sp.group;
    p.pre = i ? sp.pre_tail : sp.pre_prefix;
    p.part = sp.part[i];
    p.part_ml = sp.part_ml[i];
    p.whole = sp.whole[i];
    p.whole_ml = sp.whole_ml[i];
    p.B = i ? c.B : a->n_groups;
    Parts& q = i ? j.tail : j.prefix;
    q = {p.pre, p.part, p.part_ml, p.whole, p.whole_ml, __builtin_ctz(rows_of(shapes[i])),
         __builtin_ctz(unit_of(shapes[i])),
         merge ? least_blocks(shapes[0], shapes[1], D) : blocks_of(shapes[i], D)};
    if (p.B == 0 || merge) continue;
    e = i ? launch_kind<T, D, kTail>(shapes[i], p, &x, s)
          : launch_kind<T, D, kPrefix>(shapes[i], p, &x, s);
    if (e != hipSuccess) return e;
  }
  if (merge) {
    const Shape sh = shapes[0];
    e = hipErrorInvalidValue;  // shape_for() gives no other
    if (sh.q == 1)
      e = sh.shared ? launch_both<T, D, 1, true>(both[0], both[1], &x, s)
                    : launch_both<T, D, 1, false>(both[0], both[1], &x, s);
    else if constexpr (D < 256)
      e = sh.shared ? launch_both<T, D, 2, true>(both[0], both[1], &x, s)
                    : launch_both<T, D, 2, false>(both[0], both[1], &x, s);
    if (e != hipSuccess) return e;
  }
  j.off = x.q_offsets;
  j.lengths = x.lengths;
  j.from = sp.from;
  j.group_of = sp.group_of;
  j.request_of_row = sp.request_of_row;
  j.group = sp.group;
  j.out = both[1].out;
  j.out_stride = x.out_stride;
  j.T = x.T;
  j.Hkv = c.Hkv;
  j.G = both[1].G;
  j.cap = cap;
  j.max_nodes = x.max_nodes;
  j.B = c.B;
  j.groups = a->n_groups;
  constexpr int kHeads = kWave / (D / 4);  // per block
  hipLaunchKernelGGL((join_parts_kernel<T, D>), dim3(x.T, (x.Hq + kHeads - 1) / kHeads), dim3(kBlock),
                     0, s, j);
  return hipGetLastError();
}

template <class T>
hipError_t launch_type(const tg_prefix_attn_args* a, void* ws, hipStream_t s) {
  switch (a->attn.cache.D) {
    case 64: return launch<T, 64>(a, ws, s);
    case 128: return launch<T, 128>(a, ws, s);
    default: return launch<T, 256>(a, ws, s);
  }
}

}  // namespace

// Whether reading a prefix once could save so little that the plan and the longer
// join cost more, by what the page tables can hold: heads 32 / 8 of 128, bf16, one
// token each behind 200 tokens of their own, tree attention and this one (us): 4
// requests behind 1000 shared positions 12.6 and 17.2, 8 behind 512 11.9 and 17.5; 4
// behind 2048 20.0 and 17.3, 8 behind 2048 21.5 and 18.9. Tables that can hold more than
// their requests have are taken for long ones: 32 behind 128 16.2 and 23.4, 32 behind 512
// 19.6 and 24, and the first two with tables for 8704 positions take the longer way too.
static bool little(const tg_prefix_attn_args* a) {
  const tg_kv_cache& c = a->attn.cache;
  return a->n_groups == 0 ||
         (long long)(c.B - 1) * c.max_pages * c.page_size * c.Hkv * c.D < 4096ll * 8 * 128;
}

size_t prefix_attention_workspace_bytes(const tg_prefix_attn_args* a) {
  if (little(a)) return tree_attention_workspace_bytes(&a->attn);
  size_t bytes;
  carve(a, nullptr, &bytes);
  return bytes;
}

hipError_t launch_prefix_attention(const tg_prefix_attn_args* a, void* ws, hipStream_t s) {
  if (a->attn.T == 0 || a->attn.cache.B == 0) return hipSuccess;
  if (little(a)) return launch_tree_attention(&a->attn, ws, s);
  return a->attn.cache.dtype == TG_BF16 ? launch_type<Bf16>(a, ws, s) : launch_type<F16>(a, ws, s);
}

}  // namespace tg
