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
// path.
//
// The draw needs one row of V floats (two after a refused sampled draft) read
// once, which is what bounds many requests: the row is split over blocks that
// all walk the tree themselves (a few loads) and leave the mass of every 1024
// elements; a second kernel finds the 1024 that hold the drawn mass in them,
// and the token among those. 128 sampled chains over 128000 tokens: 21 + 5 us
// (131 MB, 6.2 TB/s in the first kernel; one block per request and pass took
// 211); a tree of 8 nodes over 32000 tokens: 7 + 3 us of dependent loads.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / kWave;
constexpr int kMaxN = TG_MAX_NODES;
constexpr int kBin = 4 * kBlock;        // elements per mass
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
  const int* drop_tok;   // n_drop of them
  const double* drop_w;  // their weights in p (0 for a token that occurs before)
  int n_drop;
  int V;
};

__device__ __forceinline__ double weigh(float p, float q) {
  return fmax((double)units(p) - (double)units(q), 0.0);
}

__device__ __forceinline__ bool wide_rows(const Weights& w) {
  return ((reinterpret_cast<uintptr_t>(w.p) | reinterpret_cast<uintptr_t>(w.q)) & 15) == 0;
}

// Weights of the elements at, ..., at + 3 (dropped tokens included), 0 past V;
// one 16-byte load per row where its alignment allows it (`wide`).
__device__ __forceinline__ void weights4(const Weights& w, int at, bool wide, double* v) {
  float p[4], q[4];
  if (wide && at + 4 <= w.V) {
    const float4 x = *reinterpret_cast<const float4*>(w.p + at);
    const float4 y = w.q ? *reinterpret_cast<const float4*>(w.q + at) : make_float4(0, 0, 0, 0);
    p[0] = x.x, p[1] = x.y, p[2] = x.z, p[3] = x.w;
    q[0] = y.x, q[1] = y.y, q[2] = y.z, q[3] = y.w;
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      p[u] = at + u < w.V ? w.p[at + u] : 0.0f;
      q[u] = w.q && at + u < w.V ? w.q[at + u] : 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] = weigh(p[u], q[u]);
}

// Mass of a bin, in every lane of the wave.
__device__ __forceinline__ double bin_mass(const Weights& w, int bin, bool wide) {
  const int lane = (int)__lane_id(), lo = bin * kBin;
  double v[4][4], s = 0.0;
#pragma unroll
  for (int u = 0; u < 4; ++u) weights4(w, lo + (u * kWave + lane) * 4, wide, v[u]);
#pragma unroll
  for (int u = 0; u < 4; ++u) s += (v[u][0] + v[u][1]) + (v[u][2] + v[u][3]);
  for (int i = lane; i < w.n_drop; i += kWave)
    if (w.drop_tok[i] >= lo && w.drop_tok[i] < lo + kBin) s -= w.drop_w[i];
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) s += __shfl_xor(s, m);
  return s;
}

// Inclusive prefix sum over the block's threads; the whole in *total. lds:
// kWaves values.
__device__ __forceinline__ double block_scan(double x, double* lds, double* total) {
  const int lane = (int)__lane_id(), wave = threadIdx.x / kWave;
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) {
    const double o = __shfl_up(x, m);
    if (lane >= m) x += o;
  }
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  double before = 0.0, sum = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += lds[i];
    sum += lds[i];
  }
  *total = sum;
  return x + before;
}

// floor(u * mass / 2^24): below mass for u < 2^24.
__device__ __forceinline__ double drawn_mass(uint64_t u, double mass) {
  return (double)(uint64_t)(((unsigned __int128)(uint64_t)mass * u) >> 24);
}

// What the walk leaves for the draw of a request.
struct Drawn {
  int row, use_q, n_drop, kept;  // kept 0: the request has no rows, or no pages
};

struct Space {
  Drawn* drawn;      // [B]
  double* mass;      // [B][bins]
  double* drop_w;    // [B][max_nodes]
  int32_t* drop_tok; // [B][max_nodes]
};

struct Shared {
  double w[kMaxN];  // the node's token in its parent's target row
  double q[kMaxN];  // and in its draft row
  double drop_w[kMaxN];
  int parent[kMaxN], token[kMaxN];
  int drop_tok[kMaxN];
  uint64_t fits[kMaxN / 64], good[kMaxN / 64];
  uint32_t best;
  int n_drop, kids;
};

__global__ __launch_bounds__(kBlock) void walk_kernel(const tg_verify_args a, int words, int bins,
                                                      Space sp) {
  __shared__ Shared sh;
  const int b = blockIdx.y, part = (int)blockIdx.x, tid = threadIdx.x;
  const bool writes = part == 0;
  int first, n;
  request_rows(a.q_offsets, b, a.T, a.max_nodes, &first, &n);
  if (a.status && a.status[b] == 0) n = 0;
  int32_t* const path = a.path + (int64_t)b * a.max_path;
  int32_t* const out = a.tokens_out + (int64_t)b * a.max_path;
  if (writes)
    for (int i = tid; i < a.max_path; i += kBlock) path[i] = out[i] = -1;
  if (n == 0) {
    if (writes && tid == 0) {
      a.n_out[b] = 0;
      sp.drawn[b].kept = 0;
    }
    return;
  }
  // Bits of the nodes above `node`.
  auto above = [&](int node, int wd) -> uint64_t {
    const int in = node - wd * 64;  // bits below `in` of this word
    const uint64_t m = in >= 64 ? ~0ull : in > 0 ? (1ull << in) - 1 : 0;
    if (!m) return 0;
    return (a.tree_mask ? a.tree_mask[(int64_t)(first + node) * words + wd] : ~0ull) & m;
  };
  const int used = min(words, (n + 63) / 64), round = (n + 63) & ~63;
  for (int j = tid; j < n; j += kBlock) {
    int parent = -1, depth = 1;
    for (int wd = 0; wd < used; ++wd) {
      const uint64_t m = above(j, wd);
      if (m) parent = wd * 64 + 63 - __clzll(m);
      depth += __popcll(m);
    }
    if (j == 0 || depth > a.max_path) parent = -1;
    const int tok = a.tokens[first + j];
    double w = 0.0, q = 0.0;
    if (parent >= 0 && tok >= 0 && tok < a.V) {
      w = units(a.target_probs[(int64_t)(first + parent) * a.target_stride + tok]);
      if (a.draft_probs) q = units(a.draft_probs[(int64_t)(first + parent) * a.draft_stride + tok]);
    }
    sh.w[j] = w;
    sh.q[j] = q;
    sh.parent[j] = parent;
    sh.token[j] = tok;
  }
  if (tid == 0) {
    sh.best = 0;
    sh.n_drop = sh.kids = 0;
  }
  __syncthreads();
  // A child whose token an earlier sibling has weighs nothing; noted in q,
  // which is not needed where tokens matter.
  for (int j = tid; j < n; j += kBlock) {
    const int parent = sh.parent[j];
    bool again = false, eldest = true;
    if (parent >= 0)
      for (int i = parent + 1; i < j; ++i)
        if (sh.parent[i] == parent) {
          eldest = false;
          again |= sh.token[i] == sh.token[j];
        }
    if (!a.draft_probs) sh.q[j] = again;
    else if (!eldest) sh.q[j] = -1.0;  // not tested
  }
  __syncthreads();
  for (int j = tid; j < n; j += kBlock)
    if (!a.draft_probs && sh.q[j] != 0.0) sh.w[j] = 0.0;
  __syncthreads();
  for (int j = tid; j < round; j += kBlock) {
    bool fits = false;
    const int parent = j < n ? sh.parent[j] : -1;
    if (parent >= 0) {
      const uint64_t u = units24(a.u_accept[first + j]), w = (uint64_t)sh.w[j];
      if (a.draft_probs) {
        fits = sh.q[j] >= 0.0 && u * (uint64_t)sh.q[j] < w << 24;
      } else {
        double left = kUnit;
        for (int i = parent + 1; i < j; ++i)
          if (sh.parent[i] == parent) left -= sh.w[i];
        fits = u * (uint64_t)fmax(left, 0.0) < w << 24;
      }
    }
    const uint64_t bits = __ballot(fits);
    if (__lane_id() == 0) sh.fits[j / 64] = bits;
  }
  __syncthreads();
  for (int j = tid; j < round; j += kBlock) {
    bool good = j == 0;
    if (j < n && sh.fits[j / 64] >> (j % 64) & 1) {
      good = true;
      const int parent = sh.parent[j];
      for (int i = parent + 1; i < j; ++i)
        if (sh.parent[i] == parent && (sh.fits[i / 64] >> (i % 64) & 1)) good = false;
    }
    const uint64_t bits = __ballot(good);
    if (__lane_id() == 0) sh.good[j / 64] = bits;
  }
  __syncthreads();
  for (int j = tid; j < n; j += kBlock) {
    if (!(sh.good[j / 64] >> (j % 64) & 1)) continue;
    bool stays = true;
    int depth = 1;
    for (int wd = 0; wd < used; ++wd) {
      const uint64_t m = above(j, wd);
      stays &= (m & ~sh.good[wd]) == 0;
      depth += __popcll(m);
    }
    if (stays) atomicMax(&sh.best, (uint32_t)depth << 16 | (uint32_t)(kMaxN - j));
  }
  __syncthreads();
  const int last = kMaxN - (int)(sh.best & 0xffff), kept = (int)(sh.best >> 16);
  if (writes && tid == 0) {  // the last node's ancestors in order, then itself
    int i = 0;
    for (int wd = 0; wd < used; ++wd)
      for (uint64_t m = above(last, wd); m; m &= m - 1) {
        const int node = wd * 64 + __ffsll((unsigned long long)m) - 1;
        if (i > 0) out[i - 1] = sh.token[node];
        path[i++] = node;
      }
    if (i > 0) out[i - 1] = sh.token[last];
    path[i] = last;
    a.n_out[b] = kept;
  }
  for (int j = tid; j < n; j += kBlock)
    if (sh.parent[j] == last) {
      sh.kids = 1;
      if (!a.draft_probs) {
        const int i = atomicAdd(&sh.n_drop, 1);
        sh.drop_tok[i] = sh.token[j];
        sh.drop_w[i] = sh.w[j];
      }
    }
  __syncthreads();

  Weights w;
  w.p = a.target_probs + (int64_t)(first + last) * a.target_stride;
  const bool use_q = a.draft_probs && sh.kids;
  w.q = use_q ? a.draft_probs + (int64_t)(first + last) * a.draft_stride : nullptr;
  w.drop_tok = sh.drop_tok;
  w.drop_w = sh.drop_w;
  w.n_drop = sh.n_drop;
  w.V = a.V;
  const bool wide = wide_rows(w);
  const int wave = tid / kWave;
  for (int bin = part * kWaves + wave; bin < bins; bin += gridDim.x * kWaves) {
    const double m = bin_mass(w, bin, wide);
    if (__lane_id() == 0) sp.mass[(int64_t)b * bins + bin] = m;
  }
  if (!writes) return;
  if (tid == 0) sp.drawn[b] = Drawn{first + last, use_q, sh.n_drop, kept};
  for (int i = tid; i < sh.n_drop; i += kBlock) {
    sp.drop_tok[(int64_t)b * a.max_nodes + i] = sh.drop_tok[i];
    sp.drop_w[(int64_t)b * a.max_nodes + i] = sh.drop_w[i];
  }
}

// What the threads of a draw tell each other.
struct Found {
  double lds[kWaves], at;
  int bin, token;
};

// mass(bin) must be the bins' masses of w. Returns the lowest token whose
// cumulative mass exceeds that drawn by u, -1 if there is no mass. (Rows that
// sum to more than 2^17 are not added exactly: some token of theirs.)
template <class Mass>
__device__ int draw(const Weights& w, int bins, uint64_t u, Mass mass, Found* f) {
  const int each = (bins + kBlock - 1) / kBlock, b0 = threadIdx.x * each;
  double sum = 0.0, whole;
  for (int i = b0; i < min(bins, b0 + each); ++i) sum += mass(i);
  __syncthreads();
  if (threadIdx.x == 0) {
    f->bin = bins - 1;
    f->at = 0.0;
  }
  const double upto = block_scan(sum, f->lds, &whole);
  if (whole <= 0.0) return -1;
  const double to = drawn_mass(u, whole);
  if (upto > to && upto - sum <= to) {  // one thread's run of bins
    double run = upto - sum;
    int i = b0;
    for (; i < min(bins, b0 + each) - 1; ++i) {
      const double m = mass(i);
      if (run + m > to) break;
      run += m;
    }
    f->bin = i;
    f->at = to - run;
  }
  __syncthreads();
  const int lo = f->bin * kBin + threadIdx.x * 4;
  const double rest = f->at;
  if (threadIdx.x == 0) f->token = min(w.V, lo + kBin) - 1;
  double v[4], total;
  weights4(w, lo, wide_rows(w), v);
  for (int j = 0; j < w.n_drop; ++j) {
    const int t = w.drop_tok[j] - lo;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t == i) v[i] = 0.0;
  }
  const double mine = (v[0] + v[1]) + (v[2] + v[3]);
  double run = block_scan(mine, f->lds, &total) - mine;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (run <= rest && run + v[i] > rest) f->token = lo + i;
    run += v[i];
  }
  __syncthreads();
  return f->token;
}

__global__ __launch_bounds__(kBlock) void draw_kernel(const tg_verify_args a, int bins, Space sp) {
  __shared__ Found found;
  const int b = blockIdx.x;
  const Drawn d = sp.drawn[b];
  if (d.kept == 0) return;
  Weights w;
  w.p = a.target_probs + (int64_t)d.row * a.target_stride;
  w.q = d.use_q ? a.draft_probs + (int64_t)d.row * a.draft_stride : nullptr;
  w.drop_tok = sp.drop_tok + (int64_t)b * a.max_nodes;
  w.drop_w = sp.drop_w + (int64_t)b * a.max_nodes;
  w.n_drop = d.n_drop;
  w.V = a.V;
  const uint64_t u = units24(a.u_next[b]);
  double* const mass = sp.mass + (int64_t)b * bins;
  int token = draw(w, bins, u, [&](int i) { return mass[i]; }, &found);
  if (token < 0) {  // nothing is left: p as it is
    w.q = nullptr;
    w.n_drop = 0;
    const bool wide = wide_rows(w);
    for (int bin = threadIdx.x / kWave; bin < bins; bin += kWaves) {
      const double m = bin_mass(w, bin, wide);
      if (__lane_id() == 0) mass[bin] = m;
    }
    __syncthreads();
    token = max(0, draw(w, bins, u, [&](int i) { return mass[i]; }, &found));
  }
  if (threadIdx.x == 0) a.tokens_out[(int64_t)b * a.max_path + d.kept - 1] = token;
}

int bins_of(const tg_verify_args* a) { return (a->V + kBin - 1) / kBin; }

Space carve(const tg_verify_args* a, char* base, size_t* bytes) {
  size_t off = 0;
  auto take = [&](size_t n) -> char* {
    char* p = base ? base + off : nullptr;
    off += (n + 255) & ~(size_t)255;
    return p;
  };
  const size_t B = a->B;
  Space s;
  s.drawn = reinterpret_cast<Drawn*>(take(B * sizeof(Drawn)));
  s.mass = reinterpret_cast<double*>(take(B * bins_of(a) * sizeof(double)));
  s.drop_w = reinterpret_cast<double*>(take(B * a->max_nodes * sizeof(double)));
  s.drop_tok = reinterpret_cast<int32_t*>(take(B * a->max_nodes * sizeof(int32_t)));
  *bytes = off ? off : 256;
  return s;
}

}  // namespace

size_t verify_workspace_bytes(const tg_verify_args* a) {
  size_t bytes;
  carve(a, nullptr, &bytes);
  return bytes;
}

hipError_t launch_verify_tree(const tg_verify_args* a, void* ws, hipStream_t s) {
  if (a->B == 0) return hipSuccess;
  size_t bytes;
  const Space sp = carve(a, static_cast<char*>(ws), &bytes);
  // About four blocks per CU, a bin per wave at least.
  const int bins = bins_of(a);
  int parts = 1024 / a->B;
  if (parts > (bins + kWaves - 1) / kWaves) parts = (bins + kWaves - 1) / kWaves;
  if (parts < 1) parts = 1;
  hipLaunchKernelGGL(walk_kernel, dim3(parts, a->B), dim3(kBlock), 0, s, *a,
                     a->tree_mask ? a->mask_words : kMaxN / 64, bins, sp);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(draw_kernel, dim3(a->B), dim3(kBlock), 0, s, *a, bins, sp);
  return hipGetLastError();
}

}  // namespace tg
