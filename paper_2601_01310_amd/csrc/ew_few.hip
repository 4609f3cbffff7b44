// The expert-worker forward for a few tokens (at most TG_MAX_FEW): gate, routing
// table, SwiGLU experts and the gate-weighted sum, with
//   h[p] = bf16(silu(x W1^T) * (x W3^T)),   out[t] = bf16(sum_j w[t,j] h[t,j] W2^T)
// for the pairs p = (t, j) of tokens and their experts.
//
// The weights of the touched slots are read once, which is what bounds it; two
// kernels stream them past the rows. A step takes 16 or 32 weight rows as the
// first operand of v_mfma_f32_16x16x32_bf16 and up to 16 or 32 token rows as the
// second; the eight waves of a block split the long axis and add their sums in
// LDS, wave by wave, so that a token's result depends neither on the other tokens
// nor on which slot of an expert serves it.
//
// 16 tokens of a DeepSeek-V3 share (bf16): 206 us, 5.6 TB/s of weights; one token of
// a Mixtral layer with its gate 130 us, 5.4 TB/s; 32 tokens of it in 8 bits 276 us,
// 5.1 TB/s; one token of the share in 8 bits 21 us. (tg_ew_forward: one token of the
// share in bf16 46 us where this takes 40.5, of the Mixtral layer 147 and 130, 32
// tokens 488 and 477.) Layers of small d lose by the second kernel, up to 16 tokens of
// which have d / 16 blocks: 8 tokens with I = 8192 and 7 experts touched, d = 512 60 us
// (tg_ew_forward 52), 1024 91 (83), 2048 137 (175).
#include "tg_device.h"
#include "tg_launch.h"
#include "tg_route.h"
#include "tg_topk.h"

namespace tg {
namespace {

constexpr int kBlock = 512, kWaves = kBlock / kWave;
constexpr int kCus = 256;
constexpr int kMaxPairs = TG_MAX_FEW_PAIRS, kMaxSlots = 1024;
constexpr int kCols = 16;      // token rows per operand
constexpr int kTableInts = 2048;  // a routing table up to this size is kept in LDS
constexpr int kStep = 128;     // bytes of a weight row per step
constexpr int kStage = 16 * kStep / 2;  // 16-bit elements of 16 rows' step in LDS
constexpr int kGateLogits = 16;  // every block forms up to so many logits itself
// Up to so many tokens the second kernel forms the sums, with runs of 16 weight rows;
// above, a third one does, and runs may be taller. 16 tokens of a Mixtral layer in 8
// bits take 273 us the first way and 259 the second, 8 tokens 264 and 268, of a
// DeepSeek-V3 share 86 and 93; in bf16 the first is the faster one up to 16 tokens
// (share 205 and 208 us). (d is 4096 and 7168 there; for smaller ones the border, which
// goes by tokens alone, is not measured.)
template <bool kF8>
constexpr int fused_tokens() {
  return kF8 ? 8 : 16;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Up to 16 or 32 pairs of one slot: slot, first place in the list of pairs and
// number of them.
__device__ __forceinline__ uint32_t item_of(int slot, int first, int n) {
  return (uint32_t)slot << 22 | (uint32_t)first << 11 | (uint32_t)n;
}
__device__ __forceinline__ int slot_of(uint32_t item) { return (int)(item >> 22); }
__device__ __forceinline__ int first_of(uint32_t item) { return (int)(item >> 11 & 2047); }
__device__ __forceinline__ int rows_of(uint32_t item) { return (int)(item & 2047); }

// What the first kernel leaves for the others.
struct Plan {
  int32_t* head;       // [2]: number of items; which Shape
  uint32_t* items;     // [kMaxPairs]
  int32_t* pair_slot;  // [T * k]
  float* w;            // [T * k]
  uint16_t* pairs;     // [T * k], by slot
  uint16_t* h;         // [T * k, I]
  float* y;            // [T * k, d], where the sums have a kernel of their own
};

struct Params {
  int T, d, E, k, I, S, R, P;
  const uint16_t* x;
  const float* logits;  // or null
  const uint16_t* w_gate;  // or null; with neither, ids and w are given
  const int32_t* ids;
  const uint8_t* w13;
  const uint8_t* w2;
  const float* s13;
  const float* s2;
  const uint8_t* valid;  // or null
  int32_t* topk_ids;     // or null
  float* topk_w;         // or null
  int32_t* pair_slot;    // or null
  int32_t* n_unserved;   // or null
  uint16_t* out;
  Plan plan;
};

__device__ __forceinline__ float swiglu(float g, float u) {
  return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * u;
}

// A barrier that waits for the wave's LDS accesses but leaves its loads in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  block_barrier();
}

// Eight 8-bit values (e4m3, exact in bf16).
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b) {
  const bf16x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false);
  const bf16x2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  const bf16x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false);
  const bf16x2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// Where a run of kM * 16 weight rows and its other operand's rows lie.
template <int kM, int kQ>
struct Place {
  __amdgpu_buffer_rsrc_t rsrc;  // the slot's weights
  int voffset[2 * kM];          // bytes: the lane's row of each eight, its first element
  const uint16_t* b[kQ];        // the lane's row of the other operand
  const float* scale[kM];       // of the lane's four sums' rows, at its first block
};

// Streams runs of kM * 16 weight rows, `runs` of them, past their rows of the
// other operand. at(i, row of each eight, place) fills the place of the i-th;
// done(i, acc) gets the wave's sums: row 16 m + (lane / 16) * 4 + r of the
// weights, column lane % 16 + 16 q. A step takes 128 bytes of each row; its loads
// run kRing steps ahead, over the end of a run too. The weights go straight into
// the wave's own ring of LDS, eight lanes to a row's 128 bytes (read into
// registers in the operand's layout, every lane of a quarter wave is in another
// row, and the vector cache looks up a line for each: 4.3 TB/s where this takes
// 5.5). Chunk c of row r is at place c ^ (r & 7), so that operand reads hit
// different banks.
template <bool kF8, int kM, int kQ, int kRing, class At, class Done>
__device__ __forceinline__ void stream(uint16_t* lds, int row_bytes, int runs, At at, Done done) {
  constexpr int kEl = kF8 ? 128 : 64;  // elements per step
  constexpr int kB = kEl / 32;         // operands of the other rows per step
  // Loads of a step that are vector loads whatever the compiler does: 16 bytes a lane
  // from addresses of its own. It may take scales, the same for many lanes, as scalar
  // ones, which a wait for vector loads must not count.
  constexpr int kLoads = 2 * kM + kQ * kB;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id(), col = lane & 15, quad = lane >> 4;
  const int steps = row_bytes / kStep;
  const int n = (steps - wave + kWaves - 1) / kWaves;  // steps wave, wave + kWaves, ...
  f32x4 acc[kM][kQ];
  auto clear = [&]() {
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
      for (int q = 0; q < kQ; ++q) acc[m][q] = f32x4{0, 0, 0, 0};
  };
  clear();
  if (n <= 0) {  // fewer steps than waves
    for (int i = 0; i < runs; ++i) done(i, acc);
    return;
  }
  uint16_t* const ring = lds + wave * kRing * kM * kStage;
  u32x4 b[kRing][kQ][kB];
  float scale[kRing][kM];
  Place<kM, kQ> p;
  int ls = 0, lc = 0;  // of the loads: run and step
  auto place = [&]() {
    at(min(ls, runs - 1), lane / 8, &p);
#pragma unroll
    for (int i = 0; i < 2 * kM; ++i) p.voffset[i] += ((lane & 7) ^ (lane / 8)) * 16;
#pragma unroll
    for (int q = 0; q < kQ; ++q) p.b[q] += wave * kEl + quad * (kF8 ? 16 : 8);
  };
  auto issue = [&](int u) {
#pragma unroll
    for (int i = 0; i < 2 * kM; ++i)
      load_lds16(p.rsrc, (lds_u16*)(ring + (u * 2 * kM + i) * (kStage / 2)), p.voffset[i],
                 (wave + lc * kWaves) * kStep);
    // 16 bytes of an 8-bit row are elements of two operands, of a bf16 row one.
#pragma unroll
    for (int q = 0; q < kQ; ++q)
#pragma unroll
      for (int s = 0; s < kB; ++s)
        b[u][q][s] = *reinterpret_cast<const u32x4*>(p.b[q] + lc * kWaves * kEl +
                                                     (kF8 ? s / 2 * 64 + s % 2 * 8 : s * 32));
    if (kF8)
#pragma unroll
      for (int m = 0; m < kM; ++m) scale[u][m] = p.scale[m][wave + lc * kWaves];
    if (++lc == n) {
      lc = 0;
      ++ls;
      place();
    }
  };
  place();
#pragma unroll
  for (int u = 0; u < kRing; ++u) issue(u);
  int run = 0, left = n;
  while (run < runs) {
#pragma unroll
    for (int u = 0; u < kRing; ++u) {
      TG_WAIT_VM((kRing - 1) * kLoads);  // this step's loads have landed
      asm volatile("" ::: "memory");
      u32x4 a[kM][2];
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          a[m][j] = *reinterpret_cast<const u32x4*>(ring + (u * kM + m) * kStage +
                                                    col * (kStep / 2) +
                                                    ((j * 4 + quad) ^ (col & 7)) * 8);
      if (kF8) {
        f32x4 part[kM][kQ];
#pragma unroll
        for (int s = 0; s < kB; ++s)
#pragma unroll
          for (int m = 0; m < kM; ++m) {
            const bf16x8 av = widen(a[m][s / 2][2 * (s % 2)], a[m][s / 2][2 * (s % 2) + 1]);
#pragma unroll
            for (int q = 0; q < kQ; ++q)
              part[m][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  av, __builtin_bit_cast(bf16x8, b[u][q][s]),
                  s ? part[m][q] : f32x4{0, 0, 0, 0}, 0, 0, 0);
          }
#pragma unroll
        for (int m = 0; m < kM; ++m)
#pragma unroll
          for (int q = 0; q < kQ; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              acc[m][q][r] = fmaf(part[m][q][r], scale[u][m], acc[m][q][r]);
      } else {
#pragma unroll
        for (int s = 0; s < kB; ++s)
#pragma unroll
          for (int m = 0; m < kM; ++m)
#pragma unroll
            for (int q = 0; q < kQ; ++q)
              acc[m][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, a[m][s % 2]), __builtin_bit_cast(bf16x8, b[u][q][s]),
                  acc[m][q], 0, 0, 0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage has been read
      issue(u);
      if (--left == 0) {
        if (run < runs) done(run, acc);
        ++run;
        left = n;
        clear();
      }
    }
  }
}

// The waves' sums of a run in LDS, [kM][kQ][wave][column][row] float32. Two
// buffers in turn need one barrier per run; where only one fits (kM and kQ both
// 2), another barrier goes before it is written again.
constexpr int kPartsBytes = 4 * kWaves * kCols * 16 * 4;

template <int kM, int kQ>
struct Parts {
  static constexpr int kOne = kM * kQ * kWaves * kCols * 16;
  static constexpr bool kTwo = kM * kQ < 4;
  float* base;

  // Leaves the wave's sums of run i; afterwards all waves' are there.
  __device__ __forceinline__ void leave(int i, const f32x4 (&acc)[kM][kQ]) {
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    if (!kTwo) lds_barrier();
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
      for (int q = 0; q < kQ; ++q)
        *reinterpret_cast<f32x4*>(base + (kTwo ? i & 1 : 0) * kOne +
                                  (((m * kQ + q) * kWaves + wave) * kCols + (lane & 15)) * 16 +
                                  (lane >> 4) * 4) = acc[m][q];
    lds_barrier();
  }
  __device__ __forceinline__ float whole(int i, int m, int q, int col, int row) const {
    const float* const at =
        base + (kTwo ? i & 1 : 0) * kOne + ((m * kQ + q) * kWaves * kCols + col) * 16 + row;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += at[w * kCols * 16];
    return s;
  }
};

// Which form of stream() a batch takes: 16 weight rows a run where items have few
// token rows (more runs to deal out), 32 where they have many, whose loads then
// serve twice the weights; 32 token rows only where an item has more than 16.
enum Shape { kNarrow, kTall, kWide };

// Steps in flight per wave, and the LDS that they take: one block to a CU, or two
// of the fused second kernel.
constexpr int ring_of(Shape s) { return s == kNarrow ? 7 : 3; }
constexpr int kRingBytes = kWaves * 7 * kStage * 2;  // 112 KB; the others need 96
constexpr int kFusedRing = 3;

// Routing, by every block for itself: top-k of given logits, the pairs' slots,
// and the items, slots in order.
struct Tables {  // needed before the first loads of the ring, whose place they have
  int32_t table[kTableInts];
  uint32_t mask[kMaxSlots][kMaxPairs / 32];  // the pairs of each slot
  int first[kMaxSlots];
  float logits[kGateLogits];
  uint8_t alive[kMaxSlots];
};
static_assert(sizeof(Tables) <= kRingBytes, "the tables lie in the ring's place");

struct Route {
  int32_t ids[kMaxPairs];
  float w[kMaxPairs];
  int slot[kMaxPairs];
  uint32_t items[kMaxPairs];
  uint16_t pairs[kMaxPairs];
  int n_items, shape, unserved;
};

// The larger of each lane's key and its neighbour's, by DPP control.
template <int kCtrl>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, kCtrl, 0xF, 0xF, false));
}

// wave_topk with less work per round: a lane's values are order-preserving keys
// (0: none, or NaN), and a round takes the largest of the lanes' largest, then the
// lowest id that has it. 8 of 256: 0.5 us where wave_topk takes 4.
template <int kN>
__device__ __forceinline__ void quick_topk(const float* lg, int E, int k, int t, int32_t* ids,
                                           float* w) {
  const int lane = lane_id();
  uint32_t key[kN];
#pragma unroll
  for (int q = 0; q < kN; ++q) {
    const int e = lane + q * kWave;
    const float v = e < E ? lg[e] : __builtin_nanf("");
    const uint32_t u = __float_as_uint(v + 0.0f);  // -0 counts as 0
    key[q] = v != v ? 0u : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  }
  float my_v = 0.0f;
  int my_id = 0;
  for (int j = 0; j < k; ++j) {
    uint32_t best = key[0];
    int q = 0;
#pragma unroll
    for (int i = 1; i < kN; ++i)
      if (key[i] > best) {
        best = key[i];
        q = i;
      }
    uint32_t m = max_dpp<0xB1>(best);  // quad_perm [1,0,3,2]
    m = max_dpp<0x4E>(m);              // quad_perm [2,3,0,1]
    m = max_dpp<0x141>(m);             // row_half_mirror
    m = max_dpp<0x140>(m);             // row_mirror
    uint32_t top = (uint32_t)__builtin_amdgcn_readlane((int)m, 0);
#pragma unroll
    for (int r = 1; r < 4; ++r) top = max(top, (uint32_t)__builtin_amdgcn_readlane((int)m, 16 * r));
    int id = 0x7fffffff;
    if (top) {  // the lowest of equal ids: the least q, then the least lane
      uint64_t at = __ballot(best == top);
      int least = __builtin_amdgcn_readlane(q, __builtin_ctzll(at));
      if (kN > 1 && (at & (at - 1))) {
        least = kN;
        for (uint64_t a = at; a; a &= a - 1)
          least = min(least, __builtin_amdgcn_readlane(q, __builtin_ctzll(a)));
        at = __ballot(best == top && q == least);
      }
      const int from = __builtin_ctzll(at);
      id = least * kWave + from;
      if (lane == from)
#pragma unroll
        for (int i = 0; i < kN; ++i)
          if (i == q) key[i] = 0;
    }
    if (lane == j) {
      my_id = id;
      my_v = top ? __uint_as_float(top >> 31 ? top & 0x7fffffffu : ~top) : -__builtin_inff();
    }
  }
  store_topk(my_v, my_id, k, t, ids, w);
}

__device__ __forceinline__ void topk(const float* lg, int E, int k, int t, int32_t* ids, float* w) {
  if (E <= 64) quick_topk<1>(lg, E, k, t, ids, w);
  else if (E <= 256) quick_topk<4>(lg, E, k, t, ids, w);
  else quick_topk<16>(lg, E, k, t, ids, w);
}

template <bool kFused>
__device__ __forceinline__ void route(const Params& p, const int32_t* __restrict__ ert,
                                      const uint8_t* __restrict__ alive, Tables& tab, Route& r) {
  const int tid = threadIdx.x, wave = tid / kWave, lane = lane_id();
  const bool small_table = p.E * p.R <= kTableInts;
  if (small_table)
    for (int i = tid; i < p.E * p.R; i += kBlock) tab.table[i] = ert[i];
  for (int s = tid; s < p.S; s += kBlock) tab.alive[s] = alive[s];
  for (int i = tid; i < p.S * (kMaxPairs / 32); i += kBlock) (&tab.mask[0][0])[i] = 0;
  if (tid == 0) r.unserved = 0;
  if (p.w_gate) {
    for (int i = wave; i < p.T * p.E; i += kWaves) {
      const int t = i / p.E, e = i - t * p.E;
      float v;
      logits_of<1>(reinterpret_cast<const uint4*>(p.x + (int64_t)t * p.d), p.w_gate, p.d, &e, &v);
      if (lane == 0) tab.logits[i] = v;
    }
    __syncthreads();
    for (int t = wave; t < p.T; t += kWaves) topk(tab.logits + t * p.E, p.E, p.k, t, r.ids, r.w);
  } else if (p.logits) {
    for (int t = wave; t < p.T; t += kWaves)
      topk(p.logits + (size_t)t * p.E, p.E, p.k, t, r.ids, r.w);
  } else if (tid < p.P) {
    r.ids[tid] = p.ids[tid];
  }
  __syncthreads();
  if (tid < p.P) {
    bool unserved = false;
    int slot = -2;
    if (!p.valid || p.valid[tid / p.k]) {
      const int e = r.ids[tid];
      slot = small_table
                 ? resolve_expert<false>(e, 0, tab.table, p.E, p.R, tab.alive, p.S, &unserved)
                 : resolve_expert<false>(e, 0, ert, p.E, p.R, tab.alive, p.S, &unserved);
    }
    r.slot[tid] = slot;
    if (slot >= 0) atomicOr(&tab.mask[slot][tid / 32], 1u << (tid % 32));
    if (unserved) atomicAdd(&r.unserved, 1);
  }
  __syncthreads();
  if (wave == 0) {
    auto count = [&](int s) {
      int c = 0;
      if (s < p.S)
        for (int i = 0; i < (p.P + 31) / 32; ++i) c += __popc(tab.mask[s][i]);
      return c;
    };
    int most = 0, used = 0;
    for (int s0 = 0; s0 < p.S; s0 += kWave) {
      const int c = count(s0 + lane);
      most = max(most, c);
      used += __builtin_popcountll(__ballot(c > 0));
    }
    for (int o = 1; o < kWave; o *= 2) most = max(most, __shfl_xor(most, o));
    const int group = most > kCols && !kFused ? 2 * kCols : kCols;
    int rows = 0, items = 0;
    for (int s0 = 0; s0 < p.S; s0 += kWave) {
      const int s = s0 + lane, c = count(s), m = (c + group - 1) / group;
      int rs = c, is = m;
      for (int o = 1; o < kWave; o *= 2) {
        const int a = __shfl_up(rs, o), b = __shfl_up(is, o);
        if (lane >= o) {
          rs += a;
          is += b;
        }
      }
      const int row0 = rows + rs - c;
      if (s < p.S) tab.first[s] = row0;
      for (int i = 0; i < m; ++i)
        r.items[items + is - m + i] = item_of(s, row0 + i * group, min(group, c - i * group));
      rows += __shfl(rs, kWave - 1);
      items += __shfl(is, kWave - 1);
    }
    if (lane == 0) {
      r.n_items = items;
      r.shape = kFused           ? kNarrow
                : most > kCols    ? kWide
                : rows > 2 * used ? kTall
                                  : kNarrow;
    }
  }
  __syncthreads();
  if (tid < p.P && r.slot[tid] >= 0) {
    const uint32_t* const mask = tab.mask[r.slot[tid]];
    int rank = __popc(mask[tid / 32] & ((1u << (tid % 32)) - 1));
    for (int i = 0; i < tid / 32; ++i) rank += __popc(mask[i]);
    r.pairs[tab.first[r.slot[tid]] + rank] = (uint16_t)tid;
  }
  __syncthreads();
}

// Gate and up projection: half of a run's weight rows are of W1, the other half
// the same ones of W3.
template <bool kF8, int kM, int kQ, int kRing>
__device__ __forceinline__ void up(const Params& p, const Route& r, uint16_t* ring, float* sums) {
  constexpr int kOut = 8 * kM;  // columns of h per run
  const int tid = threadIdx.x, lane = lane_id();
  const int tiles = p.I / kOut, units = r.n_items * tiles, grid = gridDim.x;
  const int runs = units > (int)blockIdx.x ? (units - 1 - (int)blockIdx.x) / grid + 1 : 0;
  if (runs == 0) return;
  const int row_bytes = p.d * (kF8 ? 1 : 2);
  auto at = [&](int i, int row, Place<kM, kQ>* to) {
    const int u = (int)blockIdx.x + i * grid, item = u / tiles, tile = u - item * tiles;
    const uint32_t it = r.items[item], bytes = 2u * p.I * row_bytes;
    to->rsrc = make_rsrc(p.w13 + slot_of(it) * (int64_t)bytes, bytes);
#pragma unroll
    for (int j = 0; j < 2 * kM; ++j)
      to->voffset[j] = ((j / kM) * p.I + tile * kOut + (j % kM) * 8 + row) * row_bytes;
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      const int pair = r.pairs[first_of(it) + min((lane & 15) + q * kCols, rows_of(it) - 1)];
      to->b[q] = p.x + (int64_t)(pair / p.k) * p.d;
    }
    if (kF8)
#pragma unroll
      for (int m = 0; m < kM; ++m) {
        const int up = kM == 1 ? (lane >> 4) / 2 : m;  // a row of W3
        to->scale[m] = p.s13 + ((int64_t)slot_of(it) * (2 * p.I / 128) +
                                (up * p.I + tile * kOut) / 128) * (p.d / 128);
      }
  };
  Parts<kM, kQ> parts{sums};
  auto done = [&](int i, const f32x4 (&acc)[kM][kQ]) {
    parts.leave(i, acc);
    const int u = (int)blockIdx.x + i * grid, item = u / tiles, tile = u - item * tiles;
    const uint32_t it = r.items[item];
    const int row = tid % kOut, col = tid / kOut % kCols, q = tid / (kOut * kCols);
    const int n = q * kCols + col;
    if (q < kQ && n < rows_of(it)) {
      const float g = parts.whole(i, 0, q, col, row);
      const float v = kM == 1 ? parts.whole(i, 0, q, col, row + 8) : parts.whole(i, kM - 1, q, col, row);
      p.plan.h[(int64_t)r.pairs[first_of(it) + n] * p.I + tile * kOut + row] =
          f32_to_bf16(swiglu(g, v));
    }
  };
  stream<kF8, kM, kQ, kRing>(ring, row_bytes, runs, at, done);
}

template <bool kF8, bool kFused>
__global__ __launch_bounds__(kBlock, 2) void few_up_kernel(const Params p,
                                                           const int32_t* __restrict__ ert,
                                                           const uint8_t* __restrict__ alive) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  uint16_t* const ring = reinterpret_cast<uint16_t*>(smem);
  float* const sums = reinterpret_cast<float*>(smem + kRingBytes);
  Route& r = *reinterpret_cast<Route*>(smem + kRingBytes + kPartsBytes);
  const int tid = threadIdx.x;
  route<kFused>(p, ert, alive, *reinterpret_cast<Tables*>(smem), r);
  if (blockIdx.x == 0) {
    if (tid < p.P) {
      if (p.logits || p.w_gate) {
        if (p.topk_ids) p.topk_ids[tid] = r.ids[tid];
        if (p.topk_w) p.topk_w[tid] = r.w[tid];
        p.plan.w[tid] = r.w[tid];
      }
      if (p.pair_slot) p.pair_slot[tid] = r.slot[tid];
      p.plan.pair_slot[tid] = r.slot[tid];
      p.plan.pairs[tid] = r.pairs[tid];
    }
    if (tid < r.n_items) p.plan.items[tid] = r.items[tid];
    if (tid == 0) {
      p.plan.head[0] = r.n_items;
      p.plan.head[1] = r.shape;
      if (p.n_unserved) *p.n_unserved = r.unserved;
    }
  }
  if (kFused || r.shape == kNarrow) up<kF8, 1, 1, ring_of(kNarrow)>(p, r, ring, sums);
  else if (r.shape == kTall) up<kF8, 2, 1, ring_of(kTall)>(p, r, ring, sums);
  else up<kF8, 2, 2, ring_of(kWide)>(p, r, ring, sums);
}

// What the second kernel knows of the batch.
struct Batch {
  uint32_t items[kMaxPairs];
  int32_t slot[kMaxPairs];
  float w[kMaxPairs];
  uint16_t pairs[kMaxPairs];
  int n_items, shape;
};

__device__ __forceinline__ void load_batch(const Params& p, Batch& s) {
  const int tid = threadIdx.x;
  if (tid < p.P) {
    s.items[tid] = p.plan.items[tid];  // those past the last are not looked at
    s.slot[tid] = p.plan.pair_slot[tid];
    s.w[tid] = p.plan.w[tid];
    s.pairs[tid] = p.plan.pairs[tid];
  }
  if (tid == 0) s.n_items = p.plan.head[0];
  if (tid == 64) s.shape = p.plan.head[1];
  __syncthreads();
}

// Down projection: `runs` runs, the i-th being item item(i) of the kM * 16 output
// columns from tile(i) on; each pair's sum goes to put(i, pair, row).
// end(i) follows when all of the i-th's have been put.
template <bool kF8, int kM, int kQ, int kRing, class Tile, class Item, class Put, class End>
__device__ __forceinline__ void down(const Params& p, const Batch& s, uint16_t* ring, float* sums,
                                     int runs, Tile tile, Item item, Put put, End end) {
  const int tid = threadIdx.x, lane = lane_id();
  const int row_bytes = p.I * (kF8 ? 1 : 2);
  auto at = [&](int i, int row, Place<kM, kQ>* to) {
    const uint32_t it = s.items[item(i)], bytes = (uint32_t)p.d * row_bytes;
    to->rsrc = make_rsrc(p.w2 + slot_of(it) * (int64_t)bytes, bytes);
#pragma unroll
    for (int j = 0; j < 2 * kM; ++j)
      to->voffset[j] = (tile(i) * kM * 16 + j * 8 + row) * row_bytes;
#pragma unroll
    for (int q = 0; q < kQ; ++q)
      to->b[q] = p.plan.h + (int64_t)s.pairs[first_of(it) + min((lane & 15) + q * kCols,
                                                                rows_of(it) - 1)] * p.I;
    if (kF8)
#pragma unroll
      for (int m = 0; m < kM; ++m)
        to->scale[m] = p.s2 + ((int64_t)slot_of(it) * (p.d / 128) + tile(i) * kM * 16 / 128) *
                                  (p.I / 128);
  };
  Parts<kM, kQ> parts{sums};
  auto done = [&](int i, const f32x4 (&acc)[kM][kQ]) {
    parts.leave(i, acc);
    const uint32_t it = s.items[item(i)];
#pragma unroll
    for (int o = 0; o < kM * kQ * kCols * 16; o += kBlock) {
      const int row = (tid + o) % (kM * 16), n = (tid + o) / (kM * 16);  // n: column
      if (n < rows_of(it))
        put(i, s.pairs[first_of(it) + n], row,
            parts.whole(i, row / 16, n / kCols, n % kCols, row % 16));
    }
    end(i);
  };
  stream<kF8, kM, kQ, kRing>(ring, row_bytes, runs, at, done);
}

// A block takes 16 output columns through all items and forms the weighted sums.
template <bool kF8>
__global__ __launch_bounds__(kBlock, 4) void few_down_kernel(const Params p) {
  extern __shared__ __attribute__((aligned(16))) uint16_t ring[];
  __shared__ __attribute__((aligned(16))) float sums[2 * kWaves * kCols * 16];
  __shared__ Batch s;
  float(*const y)[16] = reinterpret_cast<float(*)[16]>(ring + kWaves * kFusedRing * kStage);  // [T * k]
  const int tid = threadIdx.x;
  load_batch(p, s);
  const int tiles = p.d / 16, grid = gridDim.x, n = s.n_items;
  const int mine = (tiles - 1 - (int)blockIdx.x) / grid + 1;  // grid <= tiles
  auto combine = [&](int tile) {  // one output element per thread
    const int row = tid & 15, t = tid >> 4;
    if (t >= p.T) return;
    float sum = 0.0f;
    for (int i = t * p.k; i < (t + 1) * p.k; ++i)
      if (s.slot[i] >= 0) sum = fmaf(s.w[i], y[i][row], sum);
    p.out[(int64_t)t * p.d + tile * 16 + row] = f32_to_bf16(sum);
  };
  auto tile = [&](int i) { return (int)blockIdx.x + i / n * grid; };
  if (n <= 0) {
    for (int i = 0; i < mine; ++i) combine((int)blockIdx.x + i * grid);
    return;
  }
  down<kF8, 1, 1, kFusedRing>(p, s, ring, sums, mine * n, tile, [&](int i) { return i % n; },
                              [&](int i, int pair, int row, float v) { y[pair][row] = v; },
                              [&](int i) {
                                if (i % n != n - 1) return;
                                lds_barrier();
                                combine(tile(i));
                              });
}

// The runs of all items and columns dealt out evenly; the sums have a kernel of
// their own.
template <bool kF8, int kM, int kQ, int kRing>
__device__ __forceinline__ void down_share(const Params& p, const Batch& s, uint16_t* ring,
                                           float* sums) {
  const int units = p.d / (16 * kM) * s.n_items, grid = gridDim.x;
  const int u0 = (int)((int64_t)blockIdx.x * units / grid);
  const int u1 = (int)(((int64_t)blockIdx.x + 1) * units / grid);
  if (u0 >= u1) return;
  auto tile = [&](int i) { return (u0 + i) / s.n_items; };
  down<kF8, kM, kQ, kRing>(p, s, ring, sums, u1 - u0, tile,
                           [&](int i) { return (u0 + i) % s.n_items; },
                           [&](int i, int pair, int row, float v) {
                             p.plan.y[(int64_t)pair * p.d + tile(i) * kM * 16 + row] = v;
                           },
                           [](int) {});
}

template <bool kF8>
__global__ __launch_bounds__(kBlock, 2) void few_down_share_kernel(const Params p) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ Batch s;
  uint16_t* const ring = reinterpret_cast<uint16_t*>(smem);
  float* const sums = reinterpret_cast<float*>(smem + kRingBytes);
  load_batch(p, s);
  if (s.shape == kNarrow) down_share<kF8, 1, 1, ring_of(kNarrow)>(p, s, ring, sums);
  else if (s.shape == kTall) down_share<kF8, 2, 1, ring_of(kTall)>(p, s, ring, sums);
  else down_share<kF8, 2, 2, ring_of(kWide)>(p, s, ring, sums);
}

// out[t] = bf16(sum_j w[t,j] y[t,j]), four columns a thread.
__global__ __launch_bounds__(256) void few_sum_kernel(const Params p) {
  const int at = (int)(blockIdx.x * 256 + threadIdx.x) * 4, t = blockIdx.y;
  if (at >= p.d) return;
  f32x4 sum = f32x4{0, 0, 0, 0};
  for (int i = t * p.k; i < (t + 1) * p.k; ++i) {
    if (p.plan.pair_slot[i] < 0) continue;
    const float w = p.plan.w[i];
    const f32x4 y = *reinterpret_cast<const f32x4*>(p.plan.y + (int64_t)i * p.d + at);
#pragma unroll
    for (int c = 0; c < 4; ++c) sum[c] = fmaf(w, y[c], sum[c]);
  }
  *reinterpret_cast<uint2*>(p.out + (int64_t)t * p.d + at) =
      make_uint2(pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3]));
}

struct Layout {
  Plan plan;
  int32_t* ids;
  size_t bytes;
};

bool fused(const tg_ew_few_args* a) {
  return a->ew.T <= (a->weights == TG_WEIGHTS_F8 ? fused_tokens<true>() : fused_tokens<false>());
}

Layout layout(const tg_ew_few_args* few, char* base) {
  const tg_ew_args* const a = &few->ew;
  size_t off = 0;
  const size_t np = (size_t)a->T * a->k;
  auto take = [&](size_t n) -> char* {
    char* p = base ? base + off : nullptr;
    off += (n + 255) & ~(size_t)255;
    return p;
  };
  Layout L;
  L.plan.head = reinterpret_cast<int32_t*>(take(8));
  L.plan.items = reinterpret_cast<uint32_t*>(take(kMaxPairs * 4));
  L.plan.pair_slot = reinterpret_cast<int32_t*>(take(np * 4));
  L.plan.w = reinterpret_cast<float*>(take(np * 4));
  L.plan.pairs = reinterpret_cast<uint16_t*>(take(np * 2));
  L.plan.h = reinterpret_cast<uint16_t*>(take(np * a->I * 2));
  L.plan.y = reinterpret_cast<float*>(take(fused(few) ? 0 : np * a->d * 4));
  L.ids = reinterpret_cast<int32_t*>(take(np * 4));
  L.bytes = off;
  return L;
}

template <class Kernel>
hipError_t more_lds(Kernel* kernel, size_t bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <bool kF8, bool kFused>
hipError_t launch(const Params& p, const tg_ew_args& e, hipStream_t s) {
  const size_t up_lds = kRingBytes + kPartsBytes + sizeof(Route);
  hipError_t err = more_lds(few_up_kernel<kF8, kFused>, up_lds);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL((few_up_kernel<kF8, kFused>), dim3(e.T ? kCus : 1), dim3(kBlock), up_lds, s, p,
                     e.ert, e.slot_alive);
  if ((err = hipGetLastError()) != hipSuccess || e.T == 0) return err;
  if (kFused) {
    const size_t lds = (size_t)kWaves * kFusedRing * kStage * 2 + (size_t)p.P * 16 * 4;
    if ((err = more_lds(few_down_kernel<kF8>, lds)) != hipSuccess) return err;
    const int tiles = p.d / 16;
    hipLaunchKernelGGL((few_down_kernel<kF8>), dim3(tiles < 2 * kCus ? tiles : 2 * kCus),
                       dim3(kBlock), lds, s, p);
    return hipGetLastError();
  }
  const size_t lds = kRingBytes + kPartsBytes;
  if ((err = more_lds(few_down_share_kernel<kF8>, lds)) != hipSuccess) return err;
  hipLaunchKernelGGL((few_down_share_kernel<kF8>), dim3(kCus), dim3(kBlock), lds, s, p);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  hipLaunchKernelGGL(few_sum_kernel, dim3((p.d / 4 + 255) / 256, p.T), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace

size_t ew_few_workspace_bytes(const tg_ew_few_args* a) { return layout(a, nullptr).bytes; }

hipError_t launch_ew_few(const tg_ew_few_args* a, void* ws, hipStream_t s) {
  const tg_ew_args& e = a->ew;
  Layout L = layout(a, static_cast<char*>(ws));
  Params p{};
  p.T = e.T, p.d = e.d, p.E = e.E, p.k = e.k, p.I = e.I, p.S = e.S, p.R = e.R, p.P = e.T * e.k;
  p.x = e.x;
  p.logits = e.logits_in;
  p.w13 = reinterpret_cast<const uint8_t*>(e.w13);
  p.w2 = reinterpret_cast<const uint8_t*>(e.w2);
  p.s13 = a->w13_scale;
  p.s2 = a->w2_scale;
  p.valid = e.token_valid;
  p.topk_ids = e.topk_ids;
  p.topk_w = e.topk_w;
  p.pair_slot = e.pair_slot;
  p.n_unserved = e.n_unserved;
  p.out = e.out;
  p.plan = L.plan;
  // Few logits are formed by every block for itself, which saves a launch: one token
  // of 8 experts of 4096, 136 us with a gate kernel before, 130 without.
  if (!e.logits_in && (long long)e.T * e.E <= kGateLogits) {
    p.w_gate = e.w_gate;
  } else if (!e.logits_in) {
    if (e.topk_w) p.plan.w = e.topk_w;
    int32_t* const ids = e.topk_ids ? e.topk_ids : L.ids;
    // h is written later: until then its place can hold the logits.
    const bool fits = (size_t)e.E * sizeof(float) <= (size_t)e.k * e.I * sizeof(uint16_t);
    const hipError_t err =
        launch_gate_topk(e.x, e.w_gate, nullptr, e.T, e.d, e.E, e.k, nullptr, ids, p.plan.w, s,
                         fits ? reinterpret_cast<float*>(p.plan.h) : nullptr);
    if (err != hipSuccess) return err;
    p.ids = ids;
  }
  if (a->weights == TG_WEIGHTS_F8)
    return fused(a) ? launch<true, true>(p, e, s) : launch<true, false>(p, e, s);
  return fused(a) ? launch<false, true>(p, e, s) : launch<false, false>(p, e, s);
}

}  // namespace tg
