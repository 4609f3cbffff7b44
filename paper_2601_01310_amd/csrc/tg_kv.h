// What the operators around the paged KV cache share.
#pragma once

#include "tg_device.h"
#include "tg_launch.h"

namespace tg {

// 16-bit activation types: 8 elements travel as one uint4.
struct Bf16 {
  static __device__ __forceinline__ float lo(uint32_t u) { return __uint_as_float(u << 16); }
  static __device__ __forceinline__ float hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16x2(a, b); }
};

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));

struct F16 {
  static __device__ __forceinline__ float lo(uint32_t u) {
    return (float)__builtin_bit_cast(f16x2_t, u)[0];
  }
  static __device__ __forceinline__ float hi(uint32_t u) {
    return (float)__builtin_bit_cast(f16x2_t, u)[1];
  }
  // Rounds to nearest even; beyond the type's range to infinity.
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const f16x2_t v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
};

template <class T>
__device__ __forceinline__ void unpack8(const uint4& u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = T::lo(w[i]);
    f[2 * i + 1] = T::hi(w[i]);
  }
}

template <class T>
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(T::pack(f[0], f[1]), T::pack(f[2], f[3]), T::pack(f[4], f[5]),
                    T::pack(f[6], f[7]));
}

// Rows of request b: first row and their number, at most max_nodes, inside
// [0, T) whatever the offsets hold.
__device__ __forceinline__ void request_rows(const int32_t* __restrict__ off, int b, int T,
                                             int max_nodes, int* first, int* n) {
  const int lo = max(0, min(off[b], T)), hi = max(lo, min(off[b + 1], T));
  *first = lo;
  *n = min(hi - lo, max_nodes);
}

}  // namespace tg
