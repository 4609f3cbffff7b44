// Body of split_kernel and of a part of both_kernel (prefix_attention.hip).
// (Text and no function: called as one, inlined, the same statements are scheduled
// in another order, and trees of 64 rows take 207 us instead of 196.) It uses T, D,
// kQ, kPages, kKind, Grid, p, table, off, lengths, mask and smem.
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

  Dealer<kRows, kUnit, kKind, Grid> run(p, off, lengths, pre);
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
