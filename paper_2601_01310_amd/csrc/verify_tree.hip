// Verification of drafted tokens and the draw of the token after them.
//
// Probabilities count as whole numbers of 2^-36 (w = floor(p * 2^36), exact in
// float32), random numbers as whole numbers of 2^-24. Sums of w stay below
// 2^53, so float64 adds them exactly in any order: the answer is one, however
// the row is split.
//
// Whether a node would be accepted if its parent were (its "fit") depends on
// its parent's row and its earlier siblings alone, so all nodes are tested at
// once; a node stays if every bit of its tree mask is a node that fits and
// none of its earlier siblings does, and the deepest one that stays ends the
// path. The draw is a search in one row of V floats: the parts' masses are
// summed and the part that holds the drawn mass is split again, down to one
// wave's 256 elements.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 1024, kWaves = kBlock / kWave;
constexpr int kMaxN = TG_MAX_NODES;
constexpr double kUnit = 68719476736.0;  // 2^36

__device__ __forceinline__ float units(float p) {
  return truncf(fminf(fmaxf(p, 0.0f), 1.0f) * 68719476736.0f);  // fmaxf(NaN, 0) = 0
}

__device__ __forceinline__ uint64_t units24(float u) {
  return (uint64_t)(fminf(fmaxf(u, 0.0f), 0.99999994f) * 16777216.0f);
}

// What a row's elements weigh in a draw: p, max(p - q, 0), or p without the
// tokens of a list.
struct Weights {
  const float* p;
  const float* q;        // or null
  const int* drop_tok;   // LDS, n_drop of them
  const double* drop_w;  // their weights in p (0 for a token that occurs before)
  int n_drop;
};

__device__ __forceinline__ double weigh(float p, float q) {
  return fmax((double)units(p) - (double)units(q), 0.0);
}

// Mass of elements [lo, hi) summed over the lanes of a wave (dropped tokens
// included).
__device__ __forceinline__ double wave_mass(const Weights& w, int lo, int hi) {
  double s = 0.0;
  constexpr int kU = 8;
  for (int i0 = lo + (int)__lane_id(); i0 < hi; i0 += kU * kWave) {
    float p[kU], q[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u * kWave;
      p[u] = i < hi ? w.p[i] : 0.0f;
      q[u] = w.q && i < hi ? w.q[i] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) s += weigh(p[u], q[u]);
  }
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) s += __shfl_xor(s, m);
  return s;
}

// mass[0 .. kWaves) of the kWaves parts of [lo, hi), `step` elements each.
__device__ __forceinline__ void part_masses(const Weights& w, int lo, int hi, int step,
                                            double* mass) {
  const int wave = threadIdx.x / kWave;
  const int a = min(hi, lo + wave * step), b = min(hi, a + step);
  double m = wave_mass(w, a, b);
  for (int i = 0; i < w.n_drop; ++i)
    if (w.drop_tok[i] >= a && w.drop_tok[i] < b) m -= w.drop_w[i];
  __syncthreads();
  if (__lane_id() == 0) mass[wave] = m;
  __syncthreads();
}

// The lowest token of [lo, hi) whose cumulative mass exceeds `to`; the last
// one with any mass if `to` is not below the whole. One value for the block.
__device__ int find_token(const Weights& w, int lo, int hi, double to, double* mass, int* found) {
  while (hi - lo > 256) {
    const int step = ((hi - lo + kWaves - 1) / kWaves + 3) & ~3;
    part_masses(w, lo, hi, step, mass);
    double before = 0.0;
    int part = kWaves - 1;
    for (int i = 0; i < kWaves; ++i) {
      if (before + mass[i] > to) {
        part = i;
        break;
      }
      if (i < kWaves - 1) before += mass[i];
    }
    to -= before;
    lo = min(hi - 1, lo + part * step);
    hi = min(hi, lo + step);
  }
  __syncthreads();
  if (threadIdx.x < kWave) {
    double v[4], s = 0.0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = lo + (int)__lane_id() * 4 + u;
      v[u] = i < hi ? weigh(w.p[i], w.q ? w.q[i] : 0.0f) : 0.0;
      for (int j = 0; j < w.n_drop; ++j)
        if (w.drop_tok[j] == i) v[u] = 0.0;
      s += v[u];
    }
    double sum = s;
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) {
      const double o = __shfl_up(sum, m);
      if ((int)__lane_id() >= m) sum += o;
    }
    double run = sum - s;
    int at = 1 << 30;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      run += v[u];
      if (run > to) at = min(at, lo + (int)__lane_id() * 4 + u);
    }
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) at = min(at, __shfl_xor(at, m));
    if (threadIdx.x == 0) *found = min(at, hi - 1);
  }
  __syncthreads();
  return *found;
}

// floor(u * mass / 2^24): below mass for u < 2^24.
__device__ __forceinline__ double drawn_mass(uint64_t u, double mass) {
  return (double)(uint64_t)(((unsigned __int128)(uint64_t)mass * u) >> 24);
}

struct Shared {
  double w[kMaxN];  // the node's token in its parent's target row
  double q[kMaxN];  // and in its draft row
  int parent[kMaxN], token[kMaxN];
  int drop_tok[kMaxN];
  double drop_w[kMaxN];
  uint64_t good[kMaxN / 64];
  double mass[kWaves];
  uint32_t best;
  int n_drop, found, kids;
};

__global__ __launch_bounds__(kBlock) void verify_kernel(
    const float* __restrict__ target, int64_t ts, const float* __restrict__ draft, int64_t ds,
    const int32_t* __restrict__ tokens, const float* __restrict__ u_accept,
    const float* __restrict__ u_next, const int32_t* __restrict__ off,
    const uint64_t* __restrict__ mask, int words, int T, int V, int max_path, int max_nodes,
    int32_t* __restrict__ tokens_out, int32_t* __restrict__ path, int32_t* __restrict__ n_out) {
  __shared__ Shared sh;
  const int b = blockIdx.x, j = threadIdx.x;
  int first, n;
  request_rows(off, b, T, max_nodes, &first, &n);
  for (int i = j; i < max_path; i += kBlock) {
    path[(int64_t)b * max_path + i] = -1;
    tokens_out[(int64_t)b * max_path + i] = -1;
  }
  if (n == 0) {
    if (j == 0) n_out[b] = 0;
    return;
  }
  // Bits of the nodes above j, and their number with j itself.
  auto above = [&](int node, int wd) -> uint64_t {
    const int in = node - wd * 64;  // bits below `in` of this word
    const uint64_t m = in >= 64 ? ~0ull : in > 0 ? (1ull << in) - 1 : 0;
    if (!m) return 0;
    return (mask ? mask[(int64_t)(first + node) * words + wd] : ~0ull) & m;
  };
  const int used = min(words, (n + 63) / 64);
  int parent = -1, depth = 1;
  if (j < n) {
    for (int wd = 0; wd < used; ++wd) {
      const uint64_t m = above(j, wd);
      if (m) parent = wd * 64 + 63 - __clzll(m);
      depth += __popcll(m);
    }
    if (j == 0 || depth > max_path) parent = -1;
    const int tok = tokens[first + j];
    double w = 0.0, q = 0.0;
    if (parent >= 0 && tok >= 0 && tok < V) {
      w = units(target[(int64_t)(first + parent) * ts + tok]);
      if (draft) q = units(draft[(int64_t)(first + parent) * ds + tok]);
    }
    sh.w[j] = w;
    sh.q[j] = q;
    sh.parent[j] = parent;
    sh.token[j] = tok;
  }
  if (j < kMaxN / 64) sh.good[j] = 0;
  if (j == 0) {
    sh.best = 0;
    sh.n_drop = sh.kids = 0;
  }
  __syncthreads();
  // Earlier siblings: with the same token (this one weighs nothing then), and
  // their mass.
  bool again = false, eldest = true;
  if (parent >= 0)
    for (int i = parent + 1; i < j; ++i)
      if (sh.parent[i] == parent) {
        eldest = false;
        again |= sh.token[i] == sh.token[j];
      }
  __syncthreads();
  if (j < n && again) sh.w[j] = 0.0;
  __syncthreads();
  bool fits = false;
  if (parent >= 0) {
    const uint64_t u = units24(u_accept[first + j]), w = (uint64_t)sh.w[j];
    if (draft) {
      fits = eldest && u * (uint64_t)sh.q[j] < w << 24;
    } else {
      double left = kUnit;
      for (int i = parent + 1; i < j; ++i)
        if (sh.parent[i] == parent) left -= sh.w[i];
      fits = u * (uint64_t)fmax(left, 0.0) < w << 24;
    }
  }
  const uint64_t fit_bits = __ballot(fits);
  if (__lane_id() == 0) sh.good[j / kWave] = fit_bits;
  __syncthreads();
  bool good = fits || (j == 0);
  if (fits)
    for (int i = parent + 1; i < j; ++i)
      if (sh.parent[i] == parent && (sh.good[i / 64] >> (i % 64) & 1)) good = false;
  __syncthreads();
  const uint64_t good_bits = __ballot(good);
  if (__lane_id() == 0) sh.good[j / kWave] = good_bits;
  __syncthreads();
  if (j < n && good) {
    bool stays = true;
    for (int wd = 0; wd < used; ++wd) stays &= (above(j, wd) & ~sh.good[wd]) == 0;
    if (stays) atomicMax(&sh.best, (uint32_t)depth << 16 | (uint32_t)(kMaxN - j));
  }
  __syncthreads();
  const int last = kMaxN - (int)(sh.best & 0xffff), kept = (int)(sh.best >> 16);
  if (j == last) {  // the last node's ancestors in order, then itself
    int32_t* p = path + (int64_t)b * max_path;
    int i = 0;
    for (int wd = 0; wd < used; ++wd)
      for (uint64_t m = above(j, wd); m; m &= m - 1) {
        const int node = wd * 64 + __ffsll((unsigned long long)m) - 1;
        if (i > 0) tokens_out[(int64_t)b * max_path + i - 1] = sh.token[node];
        p[i++] = node;
      }
    if (i > 0) tokens_out[(int64_t)b * max_path + i - 1] = sh.token[j];
    p[i] = j;
    n_out[b] = kept;
  }
  if (j < n && parent == last) {
    sh.kids = 1;
    if (!draft) {
      const int i = atomicAdd(&sh.n_drop, 1);
      sh.drop_tok[i] = sh.token[j];
      sh.drop_w[i] = sh.w[j];
    }
  }
  __syncthreads();

  Weights w;
  w.p = target + (int64_t)(first + last) * ts;
  w.q = draft && sh.kids ? draft + (int64_t)(first + last) * ds : nullptr;
  w.drop_tok = sh.drop_tok;
  w.drop_w = sh.drop_w;
  w.n_drop = sh.n_drop;
  const uint64_t u = units24(u_next[b]);
  int token = 0;
  for (int turn = 0; turn < 2; ++turn) {
    const int step = ((V + kWaves - 1) / kWaves + 3) & ~3;
    part_masses(w, 0, V, step, sh.mass);
    double whole = 0.0;
    for (int i = 0; i < kWaves; ++i) whole += sh.mass[i];
    if (whole > 0.0) {
      token = find_token(w, 0, V, drawn_mass(u, whole), sh.mass, &sh.found);
      break;
    }
    w.q = nullptr;  // nothing is left: p as it is
    w.n_drop = 0;
  }
  if (j == 0) tokens_out[(int64_t)b * max_path + kept - 1] = token;
}

}  // namespace

size_t verify_workspace_bytes(const tg_verify_args* a) { return 256; }

hipError_t launch_verify_tree(const tg_verify_args* a, void* ws, hipStream_t s) {
  if (a->B == 0) return hipSuccess;
  hipLaunchKernelGGL(verify_kernel, dim3(a->B), dim3(kBlock), 0, s, a->target_probs,
                     a->target_stride, a->draft_probs, a->draft_stride, a->tokens, a->u_accept,
                     a->u_next, a->q_offsets, a->tree_mask,
                     a->tree_mask ? a->mask_words : kMaxN / 64, a->T, a->V, a->max_path,
                     a->max_nodes, a->tokens_out, a->path, a->n_out);
  return hipGetLastError();
}

}  // namespace tg
