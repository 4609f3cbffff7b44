// The next tokens from logits: temperature, top-k, top-p and min-p, and a draw from
// what they leave by given random numbers.
//
// A token's weight is 2^t over the row's largest, t = l log2 e / temperature, taken
// in float64 (whose FMA issues as fast as float32's) and counted in whole units, so
// that sums are the same in any order. Steps of 1/8 of a power of two order the
// tokens coarsely: the borders of top-k and top-p each lie in one step (or, of
// top-p within top-k, in a few), whose tokens alone have to be put in order.
//
//   part   4096 tokens a block, read once: their largest, the mass of every 1024,
//          and, for rows with filters, tokens and mass of every step;
//   cut    a row's steps added up: those that hold the borders;
//   keep   the logits again (from the last-level cache): the mass of every 1024 of
//          the tokens above the borders' steps; those in them are listed;
//   draw   the borders among the listed tokens (radix selection over logit and
//          index; the row itself where a list overflows), the 1024 that hold the
//          drawn mass, and the token in them;
//   probs  the distribution, where it is wanted.
// Rows without filters need the first and fourth only.
//
// 128 rows of 128000 tokens, bf16, temperature alone: part 17.6 us, draw 6, 22 in
// all (5.2 to read the logits); float32 with filters of all kinds: part 19, cut 9,
// keep 21, draw 16, 60 to 67 in all. part and keep are bound by the vector unit, which
// forms a weight in about 33 instructions and issues in 70 to 90 % of the time;
// cut and draw by their chains of barriers, one block to a row.
#include "tg_kv.h"

namespace tg {
namespace {

constexpr int kPart = 4096, kPartBlock = 256, kPartWaves = kPartBlock / kWave;
constexpr int kChunk = 1024;  // tokens that a wave takes at a time
constexpr int kEach = kChunk / kWave;
constexpr int kMine = kPart / (kChunk * kPartWaves);  // chunks of a wave of a part
constexpr int kSteps = 512;       // eighths of a power of two
constexpr int kNone = kSteps - 1;  // what is too small for a weight
constexpr int kBuckets = 1024;    // masses in token order, of the draw
constexpr int kDigits = 2048;     // of the radix selection
// Listed tokens of a row and border (what the draw's other tables leave of 64 KB of LDS),
// and of a part (12 KB, so that LDS holds more blocks of keep_kernel than a CU takes).
// Past either the draw's one block goes through the row itself, several times: 128 rows
// of 256000 tokens of deviation 2.5, top-p 0.95, 124 us at temperature 1 and 3700 at 1.3;
// of 128000 tokens 81 us at 1.75 and 1280 at 2.
constexpr int kList = 3328;
constexpr int kPartList = 768;
constexpr int kDrawBlock = 256, kDrawWaves = kDrawBlock / kWave;
// What a part whose tokens do not fit adds to their count: more than the list holds,
// and little enough that no number of parts comes to 2^32.
constexpr uint32_t kOverflow = kList + 1;
static_assert(kOverflow > kPartList && (1ull << 24) / kPart * kOverflow < 1ull << 32,
              "the tokens of all parts are counted in 32 bits");
// Rows of up to so many parts have no kernel for the cut: every block of keep_kernel finds
// it for itself, which saves a launch and repeats the work. 1 and 8 rows of 16384 tokens
// (4 parts), all filters, 23.1 and 23.3 us (26.2 and 26.0 with the kernel), of 32003 (8
// parts) 22.9 and 24.9 (24.3 and 25.9), of 64000 (16 parts) 25.6 and 27.8 (25.7 and 27.2).
// Batches lose by it: 64 and 192 rows of 32003 31.8 and 47.9 us (28.7 and 38.7).
constexpr int kFoldParts = 8;

typedef unsigned long long u64;

struct CutInfo {
  u64 best;               // key of the likeliest token; 0: the row has none
  double base;            // whole power of two at or above its t
  int first;              // tokens of steps before this one stay
  int k_step;             // the step with the top-k's border, -1: none
  int p_lo, p_hi;         // the steps that may hold the top-p's; p_lo > p_hi: none
  uint32_t k_before;      // tokens before k_step
  u64 k_mass, p_mass;     // mass before k_step, and before p_lo
  u64 all;
  // What the draw leaves for the distribution:
  u64 cut;                // keys from here on stay
  u64 whole;              // the kept mass
};

struct Space {
  u64* best;        // [T][parts]
  u64* chunk;       // [T][chunks]
  u64* mass;        // [T][parts][kSteps]
  uint32_t* count;  // [T][parts][kSteps]
  CutInfo* cut;     // [T]
  uint32_t* listed; // [T][2] of the next two lists; more than kList: not all are there
  u64* list_k;      // [T][kList]
  u64* list_p;      // [T][kList]
};

struct Params {
  int V, s, parts, chunks;
  int shift;  // a bucket is 2^shift chunks
  int64_t logits_stride, probs_stride;
  const float *u, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* tokens;
  float* probs;
  Space sp;
};

// A row's logits, 16 of a chunk in every lane.
template <class T>
struct Of;
template <>
struct Of<float> {
  static constexpr int kVec = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ float one(const uint8_t* p) {
    return *reinterpret_cast<const float*>(p);
  }
};
template <class T>
struct Of16 {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, float* f) { unpack8<T>(u, f); }
  static __device__ __forceinline__ float one(const uint8_t* p) {
    return T::lo(*reinterpret_cast<const uint16_t*>(p));
  }
};
template <>
struct Of<Bf16> : Of16<Bf16> {};
template <>
struct Of<F16> : Of16<F16> {};

// NaN is no token's logit, infinity the largest finite one: the median of three. With a
// NaN among them the instruction gives the least of the three by two minima in turn, of
// which the first makes a signalling NaN a quiet one and the second leaves that out:
// -infinity has to be the last operand. (The compiler, which makes a minimum of the
// builtin, would give the other bound.)
__device__ __forceinline__ float clean(float x) {
  float y;
  asm("v_med3_f32 %0, %1, %2, %3" : "=v"(y) : "v"(x), "v"(3.402823466e38f), "v"(-INFINITY));
  return y;
}

template <class T>
struct Row {
  static constexpr int kVec = Of<T>::kVec, kBytes = 16 / kVec;
  const uint8_t* p;
  int V;

  __device__ __forceinline__ Row(const uint8_t* logits, const Params& a, int t)
      : p(logits + (int64_t)t * a.logits_stride * kBytes), V(a.V) {}
  // Where the lane's e-th logit of a chunk lies in it.
  static __device__ __forceinline__ int place(int e) {
    return (e / kVec * kWave + (int)__lane_id()) * kVec + e % kVec;
  }
  __device__ __forceinline__ float at(int i) const {
    return i < V ? clean(Of<T>::one(p + (int64_t)i * kBytes)) : -INFINITY;
  }
  __device__ __forceinline__ void load(int chunk, float (&v)[kEach]) const {
#pragma unroll
    for (int j = 0; j < kEach / kVec; ++j) {
      const int i = chunk * kChunk + (j * kWave + (int)__lane_id()) * kVec;
      if (i + kVec <= V) {
        uint4 u;  // rows need not be aligned to 16 bytes
        __builtin_memcpy(&u, p + (int64_t)i * kBytes, 16);
        Of<T>::unpack(u, v + j * kVec);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[j * kVec + e] = at(i + e);
      }
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) v[e] = clean(v[e]);
  }
};

// What a row's filters are.
struct Filters {
  float hot;
  int k;
  float p, m;
  bool greedy, by_k, by_p, by_min;

  __device__ __forceinline__ Filters(const Params& a, int t) {
    hot = a.temperature ? a.temperature[t] : 1.0f;
    k = a.top_k ? a.top_k[t] : 0;
    p = a.top_p ? a.top_p[t] : 1.0f;
    m = a.min_p ? fminf(a.min_p[t], 1.0f) : 0.0f;
    greedy = !(hot > 0.0f);
    by_k = k > 0 && k < a.V;
    by_p = p < 1.0f;
    by_min = a.min_p && a.min_p[t] > 0.0f;
  }
  __device__ __forceinline__ bool any() const { return by_k || by_p || by_min; }
  // 64 log2 e / temperature
  __device__ __forceinline__ double c64() const { return 92.332482616893657 / (double)hot; }
};

// Larger logits have larger keys, of equal ones the lower index. 0: no token.
__device__ __forceinline__ uint32_t ordered(float l) {
  const uint32_t u = __float_as_uint(l + 0.0f);  // -0 counts as 0
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ u64 key_of(float l, int i) { return (u64)ordered(l) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float logit_of(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int index_of(u64 key) { return (int)~(uint32_t)key; }

// The whole power of two at or above 2^t of a key's logit.
__device__ __forceinline__ double base_of(u64 key, double c64) {
  return ceil((double)logit_of(key) * c64 * (1.0 / 64.0));
}

// x * mass for a share x, not rounded on the way, then down or up to a whole number
// (0 for x <= 0, mass for x >= 1): a border that equal weights meet exactly is met.
__device__ __forceinline__ u64 share_of(float x, u64 mass, bool up) {
  if (!(x > 0.0f)) return 0;
  if (x >= 1.0f) return mass;
  const uint32_t b = __float_as_uint(x), e = b >> 23;  // x is m 2^-shift
  const uint32_t m = e ? (b & 0x7fffffu) | 0x800000u : b;
  const int shift = e ? 150 - (int)e : 149;
  if (shift > 90) return up ? 1 : 0;  // m * mass is below 2^87
  const unsigned __int128 y = (unsigned __int128)mass * m;
  const u64 whole = (u64)(y >> shift);
  return whole + (up && (y & (((unsigned __int128)1 << shift) - 1)) != 0);
}

// 2^(-j/64)
constexpr int kTable = 64;
__device__ const double kPowers[kTable] = {
    0x1.0000000000000p+0, 0x1.fa7c1819e90d8p-1, 0x1.f50765b6e4540p-1, 0x1.efa1bee615a27p-1,
    0x1.ea4afa2a490dap-1, 0x1.e502ee78b3ff6p-1, 0x1.dfc97337b9b5fp-1, 0x1.da9e603db3285p-1,
    0x1.d5818dcfba487p-1, 0x1.d072d4a07897cp-1, 0x1.cb720dcef9069p-1, 0x1.c67f12e57d14bp-1,
    0x1.c199bdd85529cp-1, 0x1.bcc1e904bc1d2p-1, 0x1.b7f76f2fb5e47p-1, 0x1.b33a2b84f15fbp-1,
    0x1.ae89f995ad3adp-1, 0x1.a9e6b5579fdbfp-1, 0x1.a5503b23e255dp-1, 0x1.a0c667b5de565p-1,
    0x1.9c49182a3f090p-1, 0x1.97d829fde4e50p-1, 0x1.93737b0cdc5e5p-1, 0x1.8f1ae99157736p-1,
    0x1.8ace5422aa0dbp-1, 0x1.868d99b4492edp-1, 0x1.82589994cce13p-1, 0x1.7e2f336cf4e62p-1,
    0x1.7a11473eb0187p-1, 0x1.75feb564267c9p-1, 0x1.71f75e8ec5f74p-1, 0x1.6dfb23c651a2fp-1,
    0x1.6a09e667f3bcdp-1, 0x1.6623882552225p-1, 0x1.6247eb03a5585p-1, 0x1.5e76f15ad2148p-1,
    0x1.5ab07dd485429p-1, 0x1.56f4736b527dap-1, 0x1.5342b569d4f82p-1, 0x1.4f9b2769d2ca7p-1,
    0x1.4bfdad5362a27p-1, 0x1.486a2b5c13cd0p-1, 0x1.44e086061892dp-1, 0x1.4160a21f72e2ap-1,
    0x1.3dea64c123422p-1, 0x1.3a7db34e59ff7p-1, 0x1.371a7373aa9cbp-1, 0x1.33c08b26416ffp-1,
    0x1.306fe0a31b715p-1, 0x1.2d285a6e4030bp-1, 0x1.29e9df51fdee1p-1, 0x1.26b4565e27cddp-1,
    0x1.2387a6e756238p-1, 0x1.2063b88628cd6p-1, 0x1.1d4873168b9aap-1, 0x1.1a35beb6fcb75p-1,
    0x1.172b83c7d517bp-1, 0x1.1429aaea92de0p-1, 0x1.11301d0125b51p-1, 0x1.0e3ec32d3d1a2p-1,
    0x1.0b5586cf9890fp-1, 0x1.0874518759bc8p-1, 0x1.059b0d3158574p-1, 0x1.02c9a3e778061p-1,
};
// 2^(-j/64 + s)
__device__ __forceinline__ void fill_table(double* table, int s) {
  if (threadIdx.x < kTable) {
    const double x = kPowers[threadIdx.x];
    table[threadIdx.x] = __hiloint2double(__double2hiint(x) + (s << 20), __double2loint(x));
  }
}

// Weights round(2^s 2^(t - base)) and steps of logits. D = 64 (base - t) is split
// into a whole number n and a rest of at most 1/2 by adding 3 * 2^51, whose low
// bits n then is; 2^(-D/64) is a table's entry with n / 64 taken off its exponent
// times a polynomial (to 2^-44), and adding 2^52 rounds the product to a whole
// number, in the low bits too. 16 instructions of float64, where conversions,
// floor and ldexp, at half the rate, took 2.6 times as long.
// Distances go by the difference to the likeliest token, which is exact however
// large the logits and small the temperature are.
struct Weigh {
  double top, at, c64;  // the likeliest logit, its distance
  const double* table;

  // best: the likeliest token's key, 0 if there is none.
  __device__ __forceinline__ Weigh(u64 best, double c, const double* tab)
      : top(best ? (double)logit_of(best) : 0.0), c64(c), table(tab) {
    at = best ? fmin(fmax(fma(-c64, top, base_of(best, c64) * 64.0), 0.0), 64.0) : 0.0;
  }

  __device__ __forceinline__ double distance(float l) const {
    const double D = fma(c64, top - (double)l, at), most = 8.0 * kSteps - 1.0;
    double d;  // the lesser, `most` if D is NaN (a logit of -infinity at temperature infinity)
    asm("v_min_f64 %0, %1, %2" : "=v"(d) : "v"(D), "v"(most));
    return d;
  }
  static constexpr double kSplit = 6755399441055744.0;  // 3 * 2^51
  static constexpr u64 kBias = 0x4330000000000000ull;   // of 2^52

  // The step of a logit; kNone: no weight.
  __device__ __forceinline__ int step(float l) const {
    return __double2loint(distance(l) + kSplit) >> 3;
  }
  // Below the logit of every token of the steps up to `last`: a unit more than they
  // take stands for the roundings to float64 (where they are more than one, the next
  // float32 below the likeliest is further than any step), the rest for that to
  // float32. May be NaN: !(l < bound) then holds for all.
  __device__ __forceinline__ float bound(int last) const {
    const float y = (float)(top - (8.0 * (last + 1) + 1.0 - at) / c64);
    return y - fabsf(y) * 0x1p-23f - 0x1p-126f;
  }
  // The weight plus kBias.
  __device__ __forceinline__ u64 biased(float l, int* at) const {
    const double D = distance(l), m = D + kSplit;
    const int n = __double2loint(m);
    const double g = D - (m - kSplit);
    constexpr double k = -0.010830424696249145;  // -ln 2 / 64
    double r = k * k * k * k / 24.0;
    r = fma(r, g, k * k * k / 6.0);
    r = fma(r, g, k * k / 2.0);
    r = fma(r, g, k);
    r = fma(r, g, 1.0);
    const double e = table[n & (kTable - 1)];
    const double scale = __hiloint2double(__double2hiint(e) - ((n >> 6) << 20), __double2loint(e));
    *at = n >> 3;
    return (u64)__double_as_longlong(fma(r, scale, 4503599627370496.0));
  }
  __device__ __forceinline__ u64 operator()(float l, int* at) const { return biased(l, at) - kBias; }
  __device__ __forceinline__ u64 operator()(float l) const {
    int n;
    return (*this)(l, &n);
  }
  // The least weight that min-p leaves: that of the likeliest times m, which the
  // likeliest itself has.
  __device__ __forceinline__ u64 floor_of(const Filters& f, u64 best) const {
    if (!f.by_min) return 1;
    return max((u64)1, share_of(f.m, (*this)(logit_of(best)), true));
  }
};

// Scans and reductions over a wave's lanes by DPP (12 instructions and 6 operations,
// where shuffles through LDS have six of its latencies in a row: the draw of one row
// took 10.6 us and takes 9.5). All lanes take part; `none`: what op leaves as it is.
template <int kCtrl, int kRows>
__device__ __forceinline__ u64 dpp64(u64 x, u64 none) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, kCtrl, kRows, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp((int)(none >> 32), (int)(x >> 32), kCtrl,
                                                            kRows, 0xF, false);
  return (u64)hi << 32 | lo;
}
template <class Op>
__device__ __forceinline__ u64 wave_scan(u64 x, u64 none, Op op) {
  x = op(x, dpp64<0x111, 0xF>(x, none));  // row_shr:1
  x = op(x, dpp64<0x112, 0xF>(x, none));
  x = op(x, dpp64<0x114, 0xF>(x, none));
  x = op(x, dpp64<0x118, 0xF>(x, none));
  x = op(x, dpp64<0x142, 0xA>(x, none));  // row_bcast:15
  x = op(x, dpp64<0x143, 0xC>(x, none));  // row_bcast:31
  return x;
}
template <class Op>
__device__ __forceinline__ u64 wave_all(u64 x, u64 none, Op op) {
  x = wave_scan(x, none, op);
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), kWave - 1) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)x, kWave - 1);
}
struct Add {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a + b; }
};
struct Max {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return max(a, b); }
};
struct Min {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return min(a, b); }
};
__device__ __forceinline__ u64 wave_sum(u64 x) { return wave_all(x, 0, Add{}); }
__device__ __forceinline__ u64 wave_max(u64 x) { return wave_all(x, 0, Max{}); }
__device__ __forceinline__ u64 wave_min(u64 x) { return wave_all(x, ~0ull, Min{}); }

// Inclusive sums over the block's threads; the whole in *total. lds, lds_n: an
// entry per wave; n and lds_n may be null.
template <int kWaves>
__device__ __forceinline__ void scan(u64* lds, uint32_t* lds_n, u64* x, uint32_t* n, u64* total) {
  const int lane = (int)__lane_id(), wave = threadIdx.x / kWave;
  *x = wave_scan(*x, 0, Add{});
  if (n) *n = (uint32_t)wave_scan(*n, 0, Add{});
  __syncthreads();
  if (lane == kWave - 1) {
    lds[wave] = *x;
    if (n) lds_n[wave] = *n;
  }
  __syncthreads();
  u64 sum = 0;
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) {
      *x += lds[i];
      if (n) *n += lds_n[i];
    }
    sum += lds[i];
  }
  *total = sum;
}

template <class T>
__global__ __launch_bounds__(kPartBlock) void part_kernel(const uint8_t* __restrict__ logits,
                                                          const Params p) {
  __shared__ u64 mass[kSteps], tops[kPartWaves];
  __shared__ uint32_t count[kSteps];
  __shared__ double table[kTable];
  const int tid = threadIdx.x, wave = tid / kWave;
  const int t = (int)(blockIdx.x / (uint32_t)p.parts), part = (int)(blockIdx.x % (uint32_t)p.parts);
  const Row<T> row(logits, p, t);
  const Filters f(p, t);
  const int c0 = part * (kPart / kChunk) + wave * kMine;
  float v[kMine][kEach];
#pragma unroll
  for (int j = 0; j < kMine; ++j) row.load(c0 + j, v[j]);
  fill_table(table, p.s);
  for (int i = tid; i < kSteps; i += kPartBlock) {
    mass[i] = 0;
    count[i] = 0;
  }
  float most = -INFINITY;
#pragma unroll
  for (int j = 0; j < kMine; ++j)
#pragma unroll
    for (int e = 0; e < kEach; ++e) most = fmaxf(most, v[j][e]);
  u64 best = 0;
  if (most > -INFINITY) {
    int first = 0;
    if (f.greedy) {  // of equal logits the first: from the last on, the one set last
#pragma unroll
      for (int j = kMine - 1; j >= 0; --j)
#pragma unroll
        for (int e = kEach - 1; e >= 0; --e)
          if (v[j][e] == most) first = (c0 + j) * kChunk + row.place(e);
    }
    best = key_of(most, first);
  }
  best = wave_max(best);
  if (__lane_id() == 0) tops[wave] = best;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPartWaves; ++i) best = max(best, tops[i]);
  const int64_t at = (int64_t)t * p.parts + part;
  if (tid == 0) p.sp.best[at] = best;
  if (part == 0 && tid < 2) p.sp.listed[2 * t + tid] = 0;
  if (f.greedy) return;
  const double c64 = f.c64();
  const Weigh weigh(best, c64, table);
  if (!f.any()) {
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      u64 sum = 0;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        int n;
        sum += weigh.biased(v[j][e], &n);
      }
      sum = wave_sum(sum - kEach * Weigh::kBias);
      if (__lane_id() == 0 && c0 + j < p.chunks) p.sp.chunk[(int64_t)t * p.chunks + c0 + j] = sum;
    }
    return;
  }
  if (f.by_k) {
#pragma unroll
    for (int j = 0; j < kMine; ++j)
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int n = weigh.step(v[j][e]);
        if (n < kNone) atomicAdd(&count[n], 1u);
      }
  }
  if (f.by_p) {
#pragma unroll
    for (int j = 0; j < kMine; ++j)
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        int n;
        const u64 w = weigh(v[j][e], &n);
        if (w) atomicAdd(&mass[n], w);
      }
  }
  __syncthreads();
  for (int i = tid; i < kSteps; i += kPartBlock) {
    if (f.by_p) p.sp.mass[at * kSteps + i] = mass[i];
    if (f.by_k) p.sp.count[at * kSteps + i] = count[i];
  }
}

// A row's steps added up over its parts, and the ones that hold the borders.
struct CutShared {
  u64 scan[kSteps / kWave], tops[kSteps / kWave];
  uint32_t scan_n[kSteps / kWave];
  int below[kSteps];
  CutInfo c;
};

template <int kThreads, int kUnroll>
__device__ __forceinline__ void find_cut(const Params& p, const Filters& f, int t, CutShared& sh) {
  constexpr int kPer = kSteps / kThreads, kWaves = kThreads / kWave;
  const int tid = threadIdx.x;
  CutInfo& c = sh.c;
  const u64* const bests = p.sp.best + (int64_t)t * p.parts;
  u64 best = 0;
  for (int i = tid; i < p.parts; i += kThreads) best = max(best, bests[i]);
  best = wave_max(best);
  if (__lane_id() == 0) sh.tops[tid / kWave] = best;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) best = max(best, sh.tops[i]);
  const double c64 = f.c64(), base = best ? base_of(best, c64) : 0.0;
  if (tid == 0) {
    c.best = best;
    c.base = base;
    c.first = kSteps;
    c.k_step = -1;
    c.p_lo = kSteps;
    c.p_hi = -1;
    c.k_mass = c.p_mass = c.all = 0;
    c.k_before = 0;
  }
  // A part's steps begin at its own power of two, where its units are smaller.
  u64 m[kPer] = {};
  uint32_t n[kPer] = {};
  if (f.by_k || f.by_p)
    for (int i0 = 0; i0 < p.parts; i0 += kThreads) {
      const int parts = min(kThreads, p.parts - i0);
      const u64 b = tid < parts ? bests[i0 + tid] : 0;
      __syncthreads();
      sh.below[tid] = b ? (int)fmin(base - base_of(b, c64), 64.0) : 64;
      __syncthreads();
#pragma unroll kUnroll
      for (int i = 0; i < parts; ++i) {
        const int down = sh.below[i];
        const int64_t at = ((int64_t)t * p.parts + i0 + i) * kSteps;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
          const int from = tid * kPer + j - 8 * down;
          const u64 mass = f.by_p ? p.sp.mass[at + max(from, 0)] : 0;
          const uint32_t count = f.by_k ? p.sp.count[at + max(from, 0)] : 0;
          if (from >= 0 && down < 64) {
            m[j] += mass >> down;
            n[j] += count;
          }
        }
      }
    }
  u64 upto = 0, all;
  uint32_t upto_n = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    upto += m[j];
    upto_n += n[j];
  }
  u64 before = upto;
  uint32_t before_n = upto_n;
  scan<kWaves>(sh.scan, sh.scan_n, &upto, &upto_n, &all);
  before = upto - before;
  before_n = upto_n - before_n;
  u64 mb = before;
  uint32_t nb = before_n;
  if (f.by_k)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (nb < (uint32_t)f.k && nb + n[j] >= (uint32_t)f.k) {
        c.first = c.k_step = tid * kPer + j;
        c.k_before = nb;
        c.k_mass = mb;
        sh.tops[0] = mb;  // the top-k's mass is between these
        sh.tops[1] = mb + m[j];
      }
      nb += n[j];
      mb += m[j];
    }
  __syncthreads();
  if (tid == 0) c.all = all;
  if (f.by_p) {
    const u64 lo = c.k_step >= 0 ? sh.tops[0] : all, hi = c.k_step >= 0 ? sh.tops[1] : all;
    const u64 to_lo = max((u64)1, share_of(f.p, lo, true));
    const u64 to_hi = max((u64)1, share_of(f.p, hi, true));
    mb = before;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (mb < to_lo && mb + m[j] >= to_lo) {
        c.p_lo = tid * kPer + j;
        c.p_mass = mb;
      }
      if (mb < to_hi && mb + m[j] >= to_hi) c.p_hi = tid * kPer + j;
      mb += m[j];
    }
    __syncthreads();
    if (tid == 0) c.first = min(c.first, c.p_lo);
  }
  __syncthreads();
}

__global__ __launch_bounds__(kSteps) void cut_kernel(const Params p) {
  __shared__ CutShared sh;
  const int t = blockIdx.x;
  const Filters f(p, t);
  if (f.greedy || !f.any()) return;
  find_cut<kSteps, 8>(p, f, t, sh);
  if (threadIdx.x == 0) p.sp.cut[t] = sh.c;
}

// kFold: the row has few parts, and every block finds the cut for itself.
template <class T, bool kFold>
__global__ __launch_bounds__(kPartBlock) void keep_kernel(const uint8_t* __restrict__ logits,
                                                          const Params p) {
  __shared__ double table[kTable];
  __shared__ u64 list[2][kPartList];
  __shared__ uint32_t n[2], to[2];
  __shared__ CutShared cut;
  const int tid = threadIdx.x, wave = tid / kWave;
  const int t = (int)(blockIdx.x / (uint32_t)p.parts), part = (int)(blockIdx.x % (uint32_t)p.parts);
  const Filters f(p, t);
  if (f.greedy || !f.any()) return;
  const Row<T> row(logits, p, t);
  const int c0 = part * (kPart / kChunk) + wave * kMine;
  float v[kMine][kEach];
#pragma unroll
  for (int j = 0; j < kMine; ++j) row.load(c0 + j, v[j]);
  fill_table(table, p.s);
  if (tid < 2) n[tid] = 0;
  if constexpr (kFold) {
    find_cut<kPartBlock, 2>(p, f, t, cut);
    if (part == 0 && tid == 0) p.sp.cut[t] = cut.c;
  } else {
    if (tid == 0) cut.c = p.sp.cut[t];
    __syncthreads();
  }
  const u64 best = cut.c.best;
  const int first = cut.c.first, k_step = cut.c.k_step, p_lo = cut.c.p_lo, p_hi = cut.c.p_hi;
  const Weigh weigh(best, f.c64(), table);
  const u64 floor_w = weigh.floor_of(f, best);
  const int last = min(kNone - 1, max(first - 1, max(k_step, p_hi)));
  const float bound = weigh.bound(last);
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    u64 sum = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const float l = v[j][e];
      if (!__any(!(l < bound))) continue;
      int step;
      const u64 w = weigh(l, &step);
      if (step < first && w >= floor_w) sum += w;
      const bool in_k = step == k_step, in_p = step >= p_lo && step <= p_hi;
      if ((in_k || in_p) && w) {
        const u64 key = key_of(l, (c0 + j) * kChunk + row.place(e));
        if (in_k) {
          const uint32_t i = atomicAdd(&n[0], 1u);
          if (i < kPartList) list[0][i] = key;
        }
        if (in_p) {
          const uint32_t i = atomicAdd(&n[1], 1u);
          if (i < kPartList) list[1][i] = key;
        }
      }
    }
    sum = wave_sum(sum);
    if (__lane_id() == 0 && c0 + j < p.chunks) p.sp.chunk[(int64_t)t * p.chunks + c0 + j] = sum;
  }
  __syncthreads();
  if (tid < 2 && n[tid])
    to[tid] = atomicAdd(&p.sp.listed[2 * t + tid], n[tid] > kPartList ? kOverflow : n[tid]);
  __syncthreads();
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (n[which] == 0 || n[which] > kPartList) continue;
    u64* const out = (which ? p.sp.list_p : p.sp.list_k) + (int64_t)t * kList;
    for (uint32_t i = tid; i < n[which]; i += kPartBlock)
      if (to[which] + i < kList) out[to[which] + i] = list[which][i];
  }
}

struct DrawShared {
  u64 mass[kDigits];
  uint32_t count[kDigits];
  u64 list[kList];
  u64 bucket[kBuckets];
  double table[kTable];
  u64 scan[kDrawWaves];
  uint32_t scan_n[kDrawWaves];
  int index, digit;
  u64 before_mass, in_mass, rest, key, lo, hi;
  uint32_t before, in, n_pick, lo32, hi32;
  u64 pick[kWave];
};

// The tokens of the steps lo .. hi: n listed ones, or, if those are not all, the
// row's.
template <class T>
struct Border {
  const Row<T>& row;
  const Weigh& weigh;
  const u64* list;
  uint32_t n;
  int lo, hi;

  template <class F>
  __device__ __forceinline__ void each(F use) const {
    if (n <= kList) {
      for (uint32_t i = threadIdx.x; i < n; i += kDrawBlock) use(list[i], weigh(logit_of(list[i])));
      return;
    }
#pragma unroll 1
    for (int i0 = threadIdx.x; i0 < row.V; i0 += 8 * kDrawBlock) {
      float l[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) l[j] = row.at(i0 + j * kDrawBlock);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        int step;
        const u64 w = weigh(l[j], &step);
        if (w && step >= lo && step <= hi) use(key_of(l[j], i0 + j * kDrawBlock), w);
      }
    }
  }
};

// Any border. Of its tokens in the order of their keys, with `before` tokens and
// `before_mass` before them all: those from `cut` on with fewer than `most` tokens
// and less than `mass` before them. Returns the key from which on they stay, the mass
// before it and its own in *kept. If all of the border do, that is their last one's: the
// border ends at it, and what is less likely never stays. (A step's tokens, each in whole
// units of the row, may come to less than their mass in the smaller units of their parts,
// by which the border's steps were found.)
template <class T>
__device__ __attribute__((noinline)) u64 select(DrawShared& sh, const Border<T>& border, u64 cut,
                                                uint32_t before, u64 before_mass, uint32_t most,
                                                u64 mass, u64* kept) {
  constexpr int kPer = kDigits / kDrawBlock;
  const int tid = threadIdx.x;
  u64 found = 0;  // the digits of the border so far
  // The digits that all keys share are left out.
  if (tid == 0) {
    sh.lo = ~0ull;
    sh.hi = 0;
  }
  __syncthreads();
  u64 lo = ~0ull, hi = 0;
  border.each([&](u64 key, u64) {
    lo = min(lo, key);
    hi = max(hi, key);
  });
  if (lo <= hi) {
    atomicMin(&sh.lo, lo);
    atomicMax(&sh.hi, hi);
  }
  __syncthreads();
  lo = sh.lo;
  hi = sh.hi;
  *kept = before_mass;
  if (lo > hi) return cut;  // none
  int shift = lo == hi ? 1 : 64 - __clzll((long long)(lo ^ hi)), next;
  if (shift < 64) found = hi >> shift;
  for (;; shift = next) {
    next = max(0, shift - 11);
    const int bits = shift - next;
    for (int i = tid; i < kDigits; i += kDrawBlock) {
      sh.mass[i] = 0;
      sh.count[i] = 0;
    }
    if (tid == 0) sh.digit = -1;
    __syncthreads();
    border.each([&](u64 key, u64 w) {
      if (w == 0 || key < cut || (shift < 64 && key >> shift != found)) return;
      const int digit = (int)(key >> next & ((1u << bits) - 1));
      atomicAdd(&sh.mass[digit], w);
      atomicAdd(&sh.count[digit], 1u);
    });
    __syncthreads();
    // Digits from the largest on, kPer to a thread.
    const int d0 = kDigits - 1 - kPer * tid;
    u64 own = 0, all;
    uint32_t own_n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      own += sh.mass[d0 - i];
      own_n += sh.count[d0 - i];
    }
    u64 m = own;
    uint32_t n = own_n;
    scan<kDrawWaves>(sh.scan, sh.scan_n, &m, &n, &all);
    auto stays = [&](uint32_t nb, u64 mb) { return before + nb < most && before_mass + mb < mass; };
    if (own_n && stays(n - own_n, m - own) && !stays(n, m)) {  // one thread has the border
      u64 mb = m - own;
      uint32_t nb = n - own_n;
      int d = d0;
      for (;; --d) {
        const u64 dm = sh.mass[d];
        const uint32_t dn = sh.count[d];
        if (dn && !stays(nb + dn, mb + dm)) break;
        mb += dm;
        nb += dn;
      }
      sh.digit = d;
      sh.before = nb;
      sh.before_mass = mb;
      sh.in = sh.count[d];
      sh.in_mass = sh.mass[d];
    }
    __syncthreads();
    const int digit = sh.digit;
    if (digit < 0) {  // all of them stay (or none)
      if (!stays(0, 0)) return ~0ull;
      *kept = before_mass + all;
      return max(cut, lo);
    }
    before += sh.before;
    before_mass += sh.before_mass;
    const uint32_t in = sh.in;
    *kept = before_mass + sh.in_mass;
    found = (shift < 64 ? found << bits : 0) | (u64)digit;
    if (in == 1 || next == 0) break;
    __syncthreads();
  }
  border.each([&](u64 key, u64 w) {  // one token, which stays: its whole key
    if (w && key >= cut && key >> next == found) sh.key = key;
  });
  __syncthreads();
  return sh.key;
}

// The same by the first wave, for up to 64 tokens in sh.pick: the key of the last
// one that stays in sh.key, the mass before them and of those that stay in sh.rest.
__device__ __forceinline__ void settle_picked(DrawShared& sh, const Weigh& weigh, int n, u64 cut,
                                              uint32_t before, u64 before_mass, uint32_t most,
                                              u64 mass) {
  const int lane = (int)__lane_id();
  const u64 key = lane < n ? sh.pick[lane] : 0;
  const u64 w = key && key >= cut ? weigh(logit_of(key)) : 0;
  uint32_t nb = before;
  u64 mb = before_mass;
  for (int i = 0; i < n; ++i) {
    const u64 k = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), i) << 32 |
                  (uint32_t)__builtin_amdgcn_readlane((int)key, i);
    const u64 v = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(w >> 32), i) << 32 |
                  (uint32_t)__builtin_amdgcn_readlane((int)w, i);
    if (k > key) {
      nb += v != 0;
      mb += v;
    }
  }
  const bool stays = w && nb < most && mb < mass;
  u64 least = wave_min(stays ? key : ~0ull);
  if (least == ~0ull) least = cut;  // the border is among tokens without weight
  const u64 sum = wave_sum(stays ? w : 0);
  if (lane == 0) {
    sh.key = least;
    sh.rest = before_mass + sum;
  }
}

// select() in the usual case, a list: one round of digits over the list's range
// leaves a few tokens in the border's digit, which one wave settles.
template <class T>
__device__ __forceinline__ u64 settle(DrawShared& sh, const Border<T>& border, u64 cut,
                                      uint32_t before, u64 before_mass, uint32_t most, u64 mass,
                                      u64* kept) {
  const int tid = threadIdx.x;
  const uint32_t n = border.n;
  if (n > kList) return select<T>(sh, border, cut, before, before_mass, most, mass, kept);
  uint32_t picked = n;
  if (n <= kWave) {
    if (tid < (int)n) sh.pick[tid] = border.list[tid];
  } else {
    constexpr int kPer = kDigits / kDrawBlock;
    if (tid == 0) {
      sh.lo32 = 0xffffffffu;
      sh.hi32 = 0;
      sh.n_pick = 0;
    }
    for (int i = tid; i < kDigits; i += kDrawBlock) {
      sh.mass[i] = 0;
      sh.count[i] = 0;
    }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0;
    for (uint32_t i = tid; i < n; i += kDrawBlock) {
      const uint32_t o = (uint32_t)(border.list[i] >> 32);
      lo = min(lo, o);
      hi = max(hi, o);
    }
    lo = (uint32_t)wave_min(lo);
    hi = (uint32_t)wave_max(hi);
    if (__lane_id() == 0) {
      atomicMin(&sh.lo32, lo);
      atomicMax(&sh.hi32, hi);
    }
    __syncthreads();
    lo = sh.lo32;
    const int shift = max(0, 32 - __clz((int)(sh.hi32 - lo)) - 11);
    auto digit_of = [&](u64 key) { return (int)(((uint32_t)(key >> 32) - lo) >> shift); };
    border.each([&](u64 key, u64 w) {
      if (w == 0 || key < cut) return;
      atomicAdd(&sh.mass[digit_of(key)], w);
      atomicAdd(&sh.count[digit_of(key)], 1u);
    });
    __syncthreads();
    // Digits from the largest on, kPer to a thread.
    const int d0 = kDigits - 1 - kPer * tid;
    u64 own = 0, all;
    uint32_t own_n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      own += sh.mass[d0 - i];
      own_n += sh.count[d0 - i];
    }
    u64 m = own;
    uint32_t c = own_n;
    scan<kDrawWaves>(sh.scan, sh.scan_n, &m, &c, &all);
    auto stays = [&](uint32_t nb, u64 mb) { return before + nb < most && before_mass + mb < mass; };
    if (tid == 0) sh.digit = -1;
    __syncthreads();
    if (own_n && stays(c - own_n, m - own) && !stays(c, m)) {  // one thread has the border
      u64 mb = m - own;
      uint32_t nb = c - own_n;
      int d = d0;
      for (;; --d) {
        const u64 dm = sh.mass[d];
        const uint32_t dn = sh.count[d];
        if (dn && !stays(nb + dn, mb + dm)) break;
        mb += dm;
        nb += dn;
      }
      sh.digit = d;
      sh.before = nb;
      sh.before_mass = mb;
      sh.in = sh.count[d];
    }
    __syncthreads();
    const int digit = sh.digit;
    if (digit < 0 || sh.in > kWave)
      return select<T>(sh, border, cut, before, before_mass, most, mass, kept);
    for (uint32_t i = tid; i < n; i += kDrawBlock) {
      const u64 key = border.list[i];
      if (digit_of(key) != digit || key < cut) continue;
      const uint32_t at = atomicAdd(&sh.n_pick, 1u);
      if (at < kWave) sh.pick[at] = key;
    }
    before += sh.before;
    before_mass += sh.before_mass;
  }
  __syncthreads();
  if (n > kWave) picked = sh.n_pick;
  if (picked > kWave)  // tokens without weight among them
    return select<T>(sh, border, cut, before, before_mass, most, mass, kept);
  if (tid < kWave)
    settle_picked(sh, border.weigh, (int)picked, cut, before, before_mass, most, mass);
  __syncthreads();
  *kept = sh.rest;
  const u64 key = sh.key;
  __syncthreads();
  return key;
}

template <class T>
__global__ __launch_bounds__(kDrawBlock) void draw_kernel(const uint8_t* __restrict__ logits,
                                                          const Params p) {
  constexpr int kPer = kBuckets / kDrawBlock, kTokens = kChunk / kDrawBlock;
  __shared__ DrawShared sh;
  const int tid = threadIdx.x, t = blockIdx.x;
  const Row<T> row(logits, p, t);
  const Filters f(p, t);
  const bool any = f.any();
  const u64* const bests = p.sp.best + (int64_t)t * p.parts;
  const u64* const chunk = p.sp.chunk + (int64_t)t * p.chunks;
  CutInfo* const info = p.sp.cut + t;
  fill_table(sh.table, p.s);
  for (int i = tid; i < kBuckets; i += kDrawBlock) sh.bucket[i] = 0;
  u64 best = 0;
  if (any && !f.greedy) {
    best = info->best;
    __syncthreads();
  } else {
    for (int i = tid; i < p.parts; i += kDrawBlock) best = max(best, bests[i]);
    best = wave_max(best);
    if (__lane_id() == 0) sh.scan[tid / kWave] = best;
    __syncthreads();
    for (int i = 0; i < kDrawWaves; ++i) best = max(best, sh.scan[i]);
  }
  if (best == 0 || f.greedy) {
    if (tid == 0) {
      p.tokens[t] = best ? index_of(best) : -1;
      info->best = best;
    }
    return;
  }
  const double c64 = f.c64(), base = base_of(best, c64);
  const Weigh weigh(best, c64, sh.table);
  const u64 floor_w = weigh.floor_of(f, best);
  for (int i = tid; i < p.chunks; i += kDrawBlock) {
    int below = 0;  // without filters, in units of the part
    if (!any) {
      const u64 b = bests[i / (kPart / kChunk)];
      below = b ? (int)fmin(base - base_of(b, c64), 63.0) : 63;
    }
    const u64 m = chunk[i] >> below;
    if (m) atomicAdd(&sh.bucket[i >> p.shift], m);
  }
  u64 cut = 0;
  if (f.by_k || f.by_p) {
    const CutInfo c = *info;
    u64 kept = c.all;
    // top-k (round 0), then top-p in what it leaves. What stays of the last border
    // is added to the masses. (A row may have fewer tokens than top-k takes.)
    for (int round = c.k_step >= 0 ? 0 : 1; round < (f.by_p ? 2 : 1); ++round) {
      const u64* const from = (round ? p.sp.list_p : p.sp.list_k) + (int64_t)t * kList;
      const uint32_t n = p.sp.listed[2 * t + round];
      __syncthreads();
      if (n <= kList)
        for (uint32_t i0 = tid; i0 < n; i0 += 8 * kDrawBlock) {
          u64 x[8];  // loads together
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = from[min(i0 + j * kDrawBlock, n - 1)];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (i0 + j * kDrawBlock < n) sh.list[i0 + j * kDrawBlock] = x[j];
        }
      __syncthreads();
      const Border<T> border{row, weigh, sh.list, n, round ? c.p_lo : c.k_step,
                             round ? c.p_hi : c.k_step};
      const u64 to = share_of(f.p, kept, true);
      cut = settle<T>(sh, border, cut, round ? 0 : c.k_before, round ? c.p_mass : c.k_mass,
                      round ? 0xffffffffu : (uint32_t)f.k, round ? max((u64)1, to) : ~0ull, &kept);
      if (round == (f.by_p ? 1 : 0))
        border.each([&](u64 key, u64 w) {
          if (key >= cut && w >= floor_w)
            atomicAdd(&sh.bucket[index_of(key) / kChunk >> p.shift], w);
        });
    }
  }
  __syncthreads();

  // The bucket that holds the drawn mass.
  u64 own = 0, whole;
#pragma unroll
  for (int i = 0; i < kPer; ++i) own += sh.bucket[tid * kPer + i];
  u64 upto = own;
  scan<kDrawWaves>(sh.scan, sh.scan_n, &upto, (uint32_t*)nullptr, &whole);
  // (The likeliest token stays whatever the filters are: whole is not 0.)
  const u64 to = min(share_of(p.u[t], whole, false), whole - 1);
  if (upto > to && upto - own <= to) {
    u64 at = upto - own;
    int i = tid * kPer;
    while (at + sh.bucket[i] <= to) at += sh.bucket[i++];
    sh.index = i;
    sh.rest = to - at;
  }
  __syncthreads();
  // And the token in it.
  const int first = sh.index << p.shift;
  u64 rest = sh.rest;
  for (int c = first; c < min(first + (1 << p.shift), p.chunks); ++c) {
    // Without filters a chunk's mass is that of its part's units, cut to the row's.
    const u64 b = any ? best : bests[c / (kPart / kChunk)];
    const int below = b ? (int)fmin(base - base_of(b, c64), 63.0) : 63;
    const Weigh here(b, c64, sh.table);
    u64 w[kTokens], mine = 0, sum;
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
      const int i = c * kChunk + tid * kTokens + j;
      const float l = row.at(i);
      w[j] = here(l);
      if (w[j] < floor_w || key_of(l, i) < cut) w[j] = 0;
      mine += w[j];
    }
    u64 x = mine;
    scan<kDrawWaves>(sh.scan, sh.scan_n, &x, (uint32_t*)nullptr, &sum);
    if (sum >> below > rest) {
      u64 at = x - mine;
      const u64 target = rest << below;
#pragma unroll
      for (int j = 0; j < kTokens; ++j) {
        if (at <= target && at + w[j] > target) p.tokens[t] = c * kChunk + tid * kTokens + j;
        at += w[j];
      }
      break;
    }
    rest -= sum >> below;
  }
  if (tid == 0) {
    info->best = best;
    info->base = base;
    info->cut = cut;
    info->whole = whole;
  }
}

template <class T>
__global__ __launch_bounds__(kPartBlock) void probs_kernel(const uint8_t* __restrict__ logits,
                                                           const Params p) {
  __shared__ double table[kTable];
  const int t = (int)(blockIdx.x / (uint32_t)p.parts), part = (int)(blockIdx.x % (uint32_t)p.parts);
  const int wave = threadIdx.x / kWave, c0 = part * (kPart / kChunk) + wave * kMine;
  const Row<T> row(logits, p, t);
  const Filters f(p, t);
  float v[kMine][kEach];
#pragma unroll
  for (int j = 0; j < kMine; ++j) row.load(c0 + j, v[j]);
  fill_table(table, p.s);
  __syncthreads();
  const CutInfo* const c = p.sp.cut + t;
  const u64 best = c->best, cut = c->cut;
  const bool one = f.greedy || best == 0;
  const Weigh weigh(one ? 0 : best, one ? 0.0 : f.c64(), table);
  const u64 floor_w = one ? 0 : weigh.floor_of(f, best);
  const double scale = one ? 0.0 : 1.0 / (double)c->whole;
  float* const probs = p.probs + (int64_t)t * p.probs_stride;
#pragma unroll
  for (int j = 0; j < kMine; ++j)
#pragma unroll
    for (int q = 0; q < kEach; q += 4) {
      float y[4];
      const int i = (c0 + j) * kChunk + row.place(q);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float l = v[j][q + e];
        const u64 key = key_of(l, i + e);
        if (one) {
          y[e] = key == best && l > -INFINITY ? 1.0f : 0.0f;
        } else {
          y[e] = 0.0f;
          if (__any(key >= cut)) {
            const u64 w = weigh(l);
            if (w >= floor_w && key >= cut) y[e] = (float)((double)w * scale);
          }
        }
      }
      if (i + 4 <= p.V) {  // (rows are aligned to 4 bytes only)
        __builtin_memcpy(probs + i, y, 16);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i + e < p.V) probs[i + e] = y[e];
      }
    }
}

int parts_of(const tg_sample_args* a) { return (a->V + kPart - 1) / kPart; }
int chunks_of(const tg_sample_args* a) { return (a->V + kChunk - 1) / kChunk; }

Space carve(const tg_sample_args* a, char* base, size_t* bytes) {
  size_t off = 0;
  auto take = [&](size_t n) -> char* {
    char* p = base ? base + off : nullptr;
    off += (n + 255) & ~(size_t)255;
    return p;
  };
  const size_t T = a->T, parts = T * parts_of(a);
  Space s;
  s.best = reinterpret_cast<u64*>(take(parts * 8));
  s.chunk = reinterpret_cast<u64*>(take(T * chunks_of(a) * 8));
  s.cut = reinterpret_cast<CutInfo*>(take(T * sizeof(CutInfo)));
  s.listed = reinterpret_cast<uint32_t*>(take(T * 2 * sizeof(uint32_t)));
  s.mass = reinterpret_cast<u64*>(take(a->top_p ? parts * kSteps * 8 : 0));
  s.count = reinterpret_cast<uint32_t*>(take(a->top_k ? parts * kSteps * 4 : 0));
  s.list_k = reinterpret_cast<u64*>(take(a->top_k ? T * kList * 8 : 0));
  s.list_p = reinterpret_cast<u64*>(take(a->top_p ? T * kList * 8 : 0));
  *bytes = off ? off : 256;
  return s;
}

template <class T>
hipError_t launch(const tg_sample_args* a, const Params& p, hipStream_t s) {
  const uint8_t* const logits = static_cast<const uint8_t*>(a->logits);
  const dim3 parts((uint32_t)p.parts * (uint32_t)a->T), rows(a->T);
  hipError_t e;
  hipLaunchKernelGGL(part_kernel<T>, parts, dim3(kPartBlock), 0, s, logits, p);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a->top_k || a->top_p || a->min_p) {
    if (p.parts <= kFoldParts) {
      hipLaunchKernelGGL((keep_kernel<T, true>), parts, dim3(kPartBlock), 0, s, logits, p);
    } else {
      hipLaunchKernelGGL(cut_kernel, rows, dim3(kSteps), 0, s, p);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL((keep_kernel<T, false>), parts, dim3(kPartBlock), 0, s, logits, p);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(draw_kernel<T>, rows, dim3(kDrawBlock), 0, s, logits, p);
  if ((e = hipGetLastError()) != hipSuccess || !a->probs) return e;
  hipLaunchKernelGGL(probs_kernel<T>, parts, dim3(kPartBlock), 0, s, logits, p);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(const tg_sample_args* a) {
  size_t bytes;
  carve(a, nullptr, &bytes);
  return bytes;
}

hipError_t launch_sample(const tg_sample_args* a, void* ws, hipStream_t s) {
  if (a->T == 0) return hipSuccess;
  size_t bytes;
  Params p;
  p.sp = carve(a, static_cast<char*>(ws), &bytes);
  p.V = a->V;
  p.parts = parts_of(a);
  p.chunks = chunks_of(a);
  int log2v = 0;
  while ((1 << log2v) < a->V) ++log2v;
  p.s = 62 - log2v < 45 ? 62 - log2v : 45;
  p.shift = log2v > 20 ? log2v - 20 : 0;
  p.logits_stride = a->logits_stride;
  p.probs_stride = a->probs_stride;
  p.u = a->u;
  p.temperature = a->temperature;
  p.top_p = a->top_p;
  p.min_p = a->min_p;
  p.top_k = a->top_k;
  p.tokens = a->tokens;
  p.probs = a->probs;
  switch (a->dtype) {
    case TG_F32: return launch<float>(a, p, s);
    case TG_BF16: return launch<Bf16>(a, p, s);
    default: return launch<F16>(a, p, s);
  }
}

}  // namespace tg
