// Pages of the KV cache: handed out, shared by forked requests, given back,
// and the rows that a verification kept moved together.
//
// The tables are a few kilobytes. One block does each call's bookkeeping, so
// that pages go out in a fixed order: a prefix sum of the pages that each
// request (or fork) needs, one pass over the reference counts that deals the
// free pages out in ascending order and stops with the last one needed, and
// a last step that takes back what went to requests that did not fit: 3 to 9
// us a call, a handful of dependent loads (64 requests, 8000 pages). The bytes
// (compaction, part pages of forks) move in kernels of their own over many
// blocks, every row read and written once: 29 us for 17 400 pieces of 2 KB in
// 32 layers and 14 us for 1024 part pages of up to 30 KB, both 2.5 TB/s read
// and written, whatever the pieces' size. What sets that rate is not shown; the
// compiler keeps the pieces in flight in scratch memory (144 bytes a lane of
// either kernel) instead of registers, which comes first in question.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kBlock = 1024, kWaves = kBlock / kWave;
constexpr int kMaxB = 4096;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Inclusive prefix sum over the block's threads; total in every thread.
// lds: kWaves + 1 words.
__device__ __forceinline__ int block_scan(int v, int* lds, int* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) {
    const int o = __shfl_up(v, m);
    if (lane >= m) v += o;
  }
  __syncthreads();  // lds may still be read from an earlier call
  if (lane == kWave - 1) lds[wave] = v;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const int t = lds[i];
    before += i < wave ? t : 0;
    sum += t;
  }
  *total = sum;
  return v + before;
}

// A thread's pages of the first round of deal_free(), loaded ahead of the sums
// that say how many are needed.
constexpr int kPer = 8;
struct FirstRefs {
  int r[kPer];
  __device__ __forceinline__ FirstRefs(const int32_t* refs, int n_pages) {
    const int p0 = threadIdx.x * kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) r[i] = p0 + i < n_pages ? refs[p0 + i] : 1;
  }
};

// Calls take(k, page) for the k-th free page, k < want, in ascending order of
// the page; returns how many there were (at most want). Uniform over the block.
template <class Take>
__device__ __forceinline__ int deal_free(const FirstRefs& ahead, const int32_t* refs, int n_pages,
                                         int want, int* lds, Take take) {
  int found = 0;
  for (int base = 0; base < n_pages && found < want; base += kBlock * kPer) {
    const int p0 = base + threadIdx.x * kPer;
    unsigned free = 0;
    int r[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      r[i] = base == 0 ? ahead.r[i] : p0 + i < n_pages ? refs[p0 + i] : 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) free |= (unsigned)(r[i] == 0) << i;
    int total;
    int k = found + block_scan(__popc(free), lds, &total) - __popc(free);
    while (free) {
      const int i = __ffs(free) - 1;
      free &= free - 1;
      if (k < want) take(k, p0 + i);
      ++k;
    }
    found += total;
  }
  return min(found, want);
}

// First i in [0, n) with end[i] > k (end ascending); n if there is none.
__device__ __forceinline__ int owner_of(const int* end, int n, int k) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (end[mid] > k) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Calls f(i, j, page) for the i-th of the pages that hold some of the positions
// [L, L + n) and that the request (`row` of the table, `held` pages) shares;
// returns their number. There is a new row in each, so i < n.
template <class F>
__device__ __forceinline__ int shared_pages(const int32_t* row, const int32_t* refs, int n_pages,
                                            int page_shift, int L, int n, int held, F f) {
  int i = 0;
  const int end = n > 0 ? min(held, ((L + n - 1) >> page_shift) + 1) : 0;
  for (int j = L >> page_shift; j < end; ++j) {
    const int p = row[j];
    if (p >= 0 && p < n_pages && refs[p] > 1) f(i++, j, p);
  }
  return i;
}

// New rows never land in a page that others hold too (after a fork, a request
// may go back to fewer tokens than it shares): such a page is replaced by a
// fresh one with the tokens in use copied. The counts before the call decide,
// so every request that would write gets a copy of its own, whatever the order.
// A rollback below a fork is rare: the block that keeps the tables copies too,
// a wave per layer's K or V (13 rows of 2 KB in 32 layers: 35 us a page).
__global__ __launch_bounds__(kBlock) void reserve_kernel(
    int32_t* table, int32_t* held, int32_t* refs, int n_pages, int page_shift, int B, int max_pages,
    const int32_t* __restrict__ lengths, const int32_t* __restrict__ off, int T, int32_t* slots,
    int32_t* __restrict__ status, uint16_t* k, uint16_t* v, int64_t layer_stride,
    int64_t page_stride, int n_layers, int width) {
  __shared__ int lds[kWaves + 1];
  __shared__ int end[kMaxB];        // pages needed up to and with request b
  __shared__ int first[kMaxB + 1];  // q_offsets
  __shared__ int len[kMaxB];        // lengths; -1: the request gets none
  __shared__ int copies[kMaxB];     // pages of request b to be replaced
  __shared__ int any_copies;
  const FirstRefs ahead(refs, n_pages);
  const int page = 1 << page_shift;
  // The shared pages among those of request b's new rows (of the n from row `at`
  // on, those that have slots). Until the rows' own slots are written,
  // slots[first[b] + i] keeps the page that replaces the i-th, then the page
  // that it replaced.
  auto shared_of = [&](int b, int at, int n, int L, int has, auto f) {
    const int rows = at >= 0 && at < T ? min(n, T - at) : 0;
    return shared_pages(table + (long)b * max_pages, refs, n_pages, page_shift, L, rows, has, f);
  };
  if (threadIdx.x == 0) any_copies = 0;
  int want = 0;
  for (int b0 = 0; b0 < B; b0 += kBlock) {
    const int b = b0 + threadIdx.x;
    int need = 0;
    if (b < B) {
      const int at = off[b], n = max(0, off[b + 1] - at);
      const int L = max(0, lengths[b]);
      const long pages = ((long)L + n + page - 1) >> page_shift;
      const int has = max(0, min(held[b], max_pages));
      first[b] = at;
      len[b] = pages <= max_pages ? L : -1;
      copies[b] = 0;
      if (pages <= max_pages) {
        copies[b] = shared_of(b, at, n, L, has, [](int, int, int) {});
        need = max(0, (int)pages - has) + copies[b];
      }
    }
    int total;
    const int sum = block_scan(need, lds, &total);
    if (b < B) end[b] = want + sum;
    want += total;
  }
  if (threadIdx.x == 0) first[B] = off[B];
  __syncthreads();
  const int got = deal_free(ahead, refs, n_pages, want, lds, [&](int k, int p) {
    const int b = owner_of(end, B, k), i = k - (b ? end[b - 1] : 0), c = copies[b];
    refs[p] = 1;
    if (i < c) slots[first[b] + i] = p;
    else table[(long)b * max_pages + max(0, held[b]) + (i - c)] = p;
  });
  __syncthreads();
  for (int b = threadIdx.x; b < B; b += kBlock) {
    const int k0 = b ? end[b - 1] : 0, need = end[b] - k0, c = copies[b];
    const bool fits = len[b] >= 0 && (need == 0 || end[b] <= got);
    const int has = need > c ? max(0, min(held[b], max_pages)) : 0;
    if (!fits) {  // pages dealt to it go back
      len[b] = -1;
      for (int i = 0; i < min(end[b], got) - k0; ++i) {
        int32_t* e = i < c ? &slots[first[b] + i] : &table[(long)b * max_pages + has + (i - c)];
        refs[*e] = 0;
        *e = -1;
      }
      copies[b] = 0;
    } else {
      if (need > c) held[b] = has + need - c;
      if (c) any_copies = 1;
    }
    status[b] = fits;
  }
  __syncthreads();
  if (any_copies) {
    const int lane = threadIdx.x % kWave;
    for (int b = 0; b < B; ++b) {
      if (copies[b] == 0) continue;
      shared_of(b, first[b], first[b + 1] - first[b], len[b], held[b], [&](int i, int j, int p) {
        const int rows = j == len[b] >> page_shift ? len[b] & (page - 1) : 0;
        const int fresh = slots[first[b] + i], chunks = rows * (width / 8);
        for (int l = threadIdx.x / kWave; l < 2 * n_layers; l += kWaves) {
          uint16_t* const base = (l & 1 ? v : k) + (int64_t)(l >> 1) * layer_stride;
          const u32x4* s = reinterpret_cast<const u32x4*>(base + p * page_stride);
          u32x4* o = reinterpret_cast<u32x4*>(base + fresh * page_stride);
          constexpr int kU = 8;
          for (int c0 = lane; c0 < chunks; c0 += kWave * kU) {
            u32x4 x[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) x[u] = s[min(c0 + u * kWave, chunks - 1)];
#pragma unroll
            for (int u = 0; u < kU; ++u)
              if (c0 + u * kWave < chunks) o[c0 + u * kWave] = x[u];
          }
        }
      });
    }
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += kBlock)
      if (copies[b])
        shared_of(b, first[b], first[b + 1] - first[b], len[b], held[b], [&](int i, int j, int p) {
          table[(long)b * max_pages + j] = slots[first[b] + i];
          slots[first[b] + i] = p;
        });
    __syncthreads();
    for (int b = threadIdx.x; b < B; b += kBlock)
      for (int i = 0; i < copies[b]; ++i) atomicSub(&refs[slots[first[b] + i]], 1);
    __syncthreads();
  }
  for (int r = threadIdx.x; r < T; r += kBlock) {
    const int b = owner_of(first + 1, B, r);
    int slot = -1;
    if (b < B && r >= first[b] && len[b] >= 0) {
      const int pos = len[b] + r - first[b];
      const int p = table[(long)b * max_pages + (pos >> page_shift)];
      if (p >= 0 && p < n_pages) slot = (p << page_shift) | (pos & (page - 1));
    }
    slots[r] = slot;
  }
}

__global__ __launch_bounds__(kBlock) void fork_kernel(
    int32_t* table, int32_t* held, int32_t* refs, int n_pages, int page_shift, int B, int max_pages,
    int32_t* lengths, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n,
    int32_t* __restrict__ status) {
  __shared__ int lds[kWaves + 1];
  __shared__ int to[TG_MAX_FORKS], from[TG_MAX_FORKS], len[TG_MAX_FORKS], fresh[TG_MAX_FORKS];
  const FirstRefs ahead(refs, n_pages);
  const int i = threadIdx.x, page = 1 << page_shift;
  if (i < n) {
    to[i] = dst[i];
    from[i] = src[i];
  }
  __syncthreads();
  bool good = false;
  int need = 0;
  if (i < n) {
    const int s = from[i], d = to[i];
    good = s >= 0 && s < B && d >= 0 && d < B;
    const int L = good ? max(0, lengths[s]) : 0;
    const int of_src = good ? held[s] : 0, of_dst = good ? held[d] : 1;
    for (int j = 0; j < n && good; ++j) good = to[j] != s && (j >= i || to[j] != d);
    const int pages = (int)(((long)L + page - 1) >> page_shift);
    good = good && of_dst == 0 && of_src >= pages && pages <= max_pages;
    need = good && (L & (page - 1));
    len[i] = L;
  }
  int want;
  const int sum = block_scan(need, lds, &want);
  const int got =
      deal_free(ahead, refs, n_pages, want, lds, [&](int k, int p) { fresh[k] = p; });
  __syncthreads();
  const bool fits = good && (need == 0 || sum <= got);
  if (i < n) {
    status[i] = fits;
    if (!fits) len[i] = 0;  // nothing is shared
    if (fits) {
      const int whole = len[i] >> page_shift;
      if (need) {
        const int p = fresh[sum - 1];
        refs[p] = 1;
        table[(long)to[i] * max_pages + whole] = p;
      }
      held[to[i]] = whole + need;
      lengths[to[i]] = len[i];
    }
  }
  __syncthreads();
  // Whole pages are shared: a wave takes a fork.
  for (int f = threadIdx.x / kWave; f < n; f += kWaves) {
    const int32_t* s = table + (long)from[f] * max_pages;
    int32_t* d = table + (long)to[f] * max_pages;
    for (int j = threadIdx.x % kWave; j < len[f] >> page_shift; j += kWave) {
      const int p = s[j];
      d[j] = p;
      if (p >= 0 && p < n_pages) atomicAdd(&refs[p], 1);
    }
  }
}

// The rows in use of a part page, one layer's K or V: one run of bytes.
__global__ __launch_bounds__(256) void fork_copy_kernel(
    const int32_t* __restrict__ table, int n_pages, int page_shift, int max_pages,
    const int32_t* __restrict__ lengths, const int32_t* __restrict__ src,
    const int32_t* __restrict__ dst, const int32_t* __restrict__ status, uint16_t* k, uint16_t* v,
    int64_t layer_stride, int64_t page_stride, int row) {
  const int f = blockIdx.x, done = status[f], from = src[f], d = dst[f];
  if (!done) return;
  const int L = lengths[d], rows = L & ((1 << page_shift) - 1);
  if (rows == 0) return;
  const int whole = L >> page_shift;
  const int ps = table[(long)from * max_pages + whole], pd = table[(long)d * max_pages + whole];
  if (ps < 0 || ps >= n_pages || pd < 0 || pd >= n_pages) return;
  uint16_t* base = (blockIdx.y & 1 ? v : k) + (int64_t)(blockIdx.y >> 1) * layer_stride;
  const uint4* s = reinterpret_cast<const uint4*>(base + ps * page_stride);
  uint4* o = reinterpret_cast<uint4*>(base + pd * page_stride);
  const int chunks = rows * (row / 8);
  constexpr int kU = 8;
  for (int c0 = blockIdx.z * 256 * kU + threadIdx.x; c0 < chunks; c0 += gridDim.z * 256 * kU) {
    uint4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (c0 + u * 256 < chunks) x[u] = s[c0 + u * 256];
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (c0 + u * 256 < chunks) o[c0 + u * 256] = x[u];
  }
}

__global__ __launch_bounds__(256) void trim_kernel(int32_t* table, int32_t* held, int32_t* refs,
                                                   int n_pages, int page_shift, int max_pages,
                                                   const int32_t* __restrict__ keep) {
  const int b = blockIdx.x;
  const int has = max(0, min(held[b], max_pages));
  const long pages = ((long)max(0, keep[b]) + (1 << page_shift) - 1) >> page_shift;
  __syncthreads();  // held[b] is read before it is written
  if (pages >= has) return;
  for (int j = (int)pages + threadIdx.x; j < has; j += 256) {
    int32_t* e = &table[(long)b * max_pages + j];
    const int p = *e;
    if (p >= 0 && p < n_pages) atomicSub(&refs[p], 1);
    *e = -1;
  }
  if (threadIdx.x == 0) held[b] = (int)pages;
}

// One block per request and layer; a thread takes a 16-byte column of K or V
// through the kept rows. Rows move down (path[i] >= i, ascending), so a batch
// of rows is read before any of them is written and later rows are still
// whole.
__global__ __launch_bounds__(256) void compact_kernel(
    const int32_t* __restrict__ table, int n_pages, int page_shift, int max_pages,
    const int32_t* __restrict__ path, int max_path, const int32_t* __restrict__ n_keep,
    const int32_t* __restrict__ lengths, int32_t* __restrict__ new_lengths, uint16_t* k, uint16_t* v,
    int64_t layer_stride, int64_t page_stride, int width) {
  // A table reaches at most 2^30 positions.
  const int b = blockIdx.x, L = max(0, min(lengths[b], 1 << 30));
  const int n = max(0, min(n_keep[b], max_path));
  if (blockIdx.y == 0 && threadIdx.x == 0) new_lengths[b] = max(0, lengths[b]) + n;
  const int32_t* row = table + (long)b * max_pages;
  path += (long)b * max_path;
  constexpr int kU = 8;
  const int in_page = (1 << page_shift) - 1;
  // Logical page of a position that the table reaches, -1 for others.
  auto page_of = [&](int pos) { return pos >> page_shift < max_pages ? pos >> page_shift : -1; };
  for (int i0 = 0; i0 < n; i0 += kU) {
    // The batch's places, each kind of load together: one after another they
    // cost a memory latency per row and kind.
    int j[kU], from[kU], at[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) j[u] = path[min(i0 + u, n - 1)];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u;
      // In its place already, or no place at all: not moved.
      const bool moves = i < n && j[u] > i && j[u] < (1 << 30);
      const int pf = moves ? page_of(L + j[u]) : -1, pt = moves ? page_of(L + i) : -1;
      from[u] = pf < 0 ? -1 : row[pf];
      at[u] = pt < 0 ? -1 : row[pt];
    }
#pragma unroll
    for (int u = 0; u < kU; ++u)
      if (from[u] >= n_pages || at[u] >= n_pages || at[u] < 0) from[u] = -1;
    for (int c = threadIdx.x * 8; c < 2 * width; c += 256 * 8) {
      uint16_t* const base =
          (c < width ? k : v - width) + (int64_t)blockIdx.y * layer_stride + c;
      uint4 x[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (from[u] >= 0)
          x[u] = *reinterpret_cast<const uint4*>(base + from[u] * page_stride +
                                                 (int64_t)((L + j[u]) & in_page) * width);
#pragma unroll
      for (int u = 0; u < kU; ++u)
        if (from[u] >= 0)
          *reinterpret_cast<uint4*>(base + at[u] * page_stride +
                                    (int64_t)((L + i0 + u) & in_page) * width) = x[u];
    }
  }
}

}  // namespace

hipError_t launch_kv_compact(const tg_kv_cache* c, const int32_t* path, int max_path,
                             const int32_t* n_keep, const int32_t* lengths, int32_t* new_lengths,
                             hipStream_t s) {
  if (c->B == 0) return hipSuccess;
  hipLaunchKernelGGL(compact_kernel, dim3(c->B, c->n_layers), dim3(256), 0, s, c->page_table,
                     c->n_pages, __builtin_ctz(c->page_size), c->max_pages, path, max_path, n_keep,
                     lengths, new_lengths, static_cast<uint16_t*>(c->k),
                     static_cast<uint16_t*>(c->v), c->layer_stride, c->page_stride, c->Hkv * c->D);
  return hipGetLastError();
}

hipError_t launch_kv_pages_reserve(const tg_kv_cache* c, const int32_t* lengths,
                                   const int32_t* q_offsets, int T, int32_t* slots, int32_t* status,
                                   hipStream_t s) {
  if (c->B == 0 && T == 0) return hipSuccess;  // T rows of nobody still get their -1
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kBlock), 0, s, c->page_table, c->held,
                     c->refcount, c->n_pages, __builtin_ctz(c->page_size), c->B, c->max_pages,
                     lengths, q_offsets, T, slots, status, static_cast<uint16_t*>(c->k),
                     static_cast<uint16_t*>(c->v), c->layer_stride, c->page_stride, c->n_layers,
                     c->Hkv * c->D);
  return hipGetLastError();
}

hipError_t launch_kv_pages_fork(const tg_kv_cache* c, int32_t* lengths, const int32_t* src,
                                const int32_t* dst, int n, int32_t* status, hipStream_t s) {
  if (n == 0) return hipSuccess;
  const int shift = __builtin_ctz(c->page_size), row = c->Hkv * c->D;
  hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kBlock), 0, s, c->page_table, c->held, c->refcount,
                     c->n_pages, shift, c->B, c->max_pages, lengths, src, dst, n, status);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t chunks = (int64_t)c->page_size * row / 8;
  const int z = (int)(chunks < 8 * 2048 ? (chunks + 2047) / 2048 : 8);
  hipLaunchKernelGGL(fork_copy_kernel, dim3(n, 2 * c->n_layers, z), dim3(256), 0, s, c->page_table,
                     c->n_pages, shift, c->max_pages, lengths, src, dst, status,
                     static_cast<uint16_t*>(c->k), static_cast<uint16_t*>(c->v), c->layer_stride,
                     c->page_stride, row);
  return hipGetLastError();
}

hipError_t launch_kv_pages_trim(const tg_kv_cache* c, const int32_t* keep, hipStream_t s) {
  if (c->B == 0) return hipSuccess;
  hipLaunchKernelGGL(trim_kernel, dim3(c->B), dim3(256), 0, s, c->page_table, c->held, c->refcount,
                     c->n_pages, __builtin_ctz(c->page_size), c->max_pages, keep);
  return hipGetLastError();
}

}  // namespace tg
