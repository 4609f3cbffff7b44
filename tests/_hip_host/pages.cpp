// The page table's kernels, run on the CPU.
#include <hip/hip_runtime.h>

namespace {
struct Block {
  unsigned x = 0, y = 0, z = 0;
} block_index;
}  // namespace
#define blockIdx block_index

inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
inline int __popc(unsigned v) { return __builtin_popcount(v); }
inline int __ffs(unsigned v) { return __builtin_ffs((int)v); }
inline int atomicSub(int* p, int v) {
  const int old = *p;
  *p -= v;
  return old;
}

#include "kv_pages.hip"

extern "C" {

// k and v: [layers, n_pages, page, width] of 16 bits.
void reserve(int32_t* table, int32_t* held, int32_t* refs, int n_pages, int page_shift, int B,
             int max_pages, const int32_t* lengths, const int32_t* off, int T, int32_t* slots,
             int32_t* status, uint16_t* k, uint16_t* v, int n_layers, int width) {
  const int64_t page_stride = (int64_t)width << page_shift;
  hip_host::run_block(0, 1, tg::kBlock, [&] {
    tg::reserve_kernel(table, held, refs, n_pages, page_shift, B, max_pages, lengths, off, T, slots,
                       status, k, v, page_stride * n_pages, page_stride, n_layers, width);
  });
}

}  // extern "C"
