// Body of shared_kernel and of a part of both_kernel (prefix_attention.hip).
// (Text and no function: called as one, inlined, the same statements are scheduled
// in another order, and trees of 64 rows take 207 us instead of 196.) It uses T, D,
// kQ, kEven, kKind, Grid, p, table, off, lengths, mask, tiles and pre.
  using R = Rows<T, D, kQ>;
  constexpr int kRows = 16 * kQ * kWaves, kUnit = 2 * kTile;
  constexpr int kLanes = D / 8;            // lanes per row
  constexpr int kHave = kWave / kLanes;    // rows per load of a wave
  constexpr int kLoads = kUnit / (kHave * kWaves);
  constexpr int kTileElems = kUnit * D;
  // tiles: [buffer][K, V][kUnit][D]
  __shared__ int carry[kWaves];
  __shared__ uint32_t odd_rows[3][2];  // of the tiles, in turn
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  auto turn_of = [](int row) { return (D == 64 ? row >> 1 & 3 : row & 7) * 2; };

  Dealer<kRows, kUnit, kKind, Grid> run(p, off, lengths, pre);
  Piece x = run.first(carry);
  if (run.begin >= run.stop) {
    run.leave_none();
    return;
  }
  const int width = p.Hkv * D, page_mask = (1 << p.page_shift) - 1;
  // The lane's row and chunk in a wave's load (load j: rows j * kHave * kWaves
  // on; a multiple of 8 rows, so that the chunk is the same in all of them).
  const int my_row = wave * kHave + lane / kLanes;
  const int my_chunk = lane % kLanes ^ turn_of(my_row);
  const uint32_t my_at = (lane / kLanes * width + my_chunk * 8) * 2;
  // Where the lane reads K (first step) and V (first columns) of a tile.
  const int k_chunk = quad ^ turn_of(col), v_row = quad * 4 + col / 4;
  const int v_chunk = (col & 3) / 2 ^ turn_of(v_row);
  for (int at = run.begin; at < run.stop;) {
    if (at != run.begin) x = run.at(at);
    run.leave(x, at);
    const int32_t* __restrict__ pages = table + (int64_t)x.r.table * p.max_pages;
    const uint16_t* const kh = p.k + (int64_t)x.g * D;
    const uint16_t* const vh = p.v + (int64_t)x.g * D;
    const int row0 = x.rt * kRows + wave * 16 * kQ;
    const bool busy = row0 < x.r.n * p.G;  // the wave has rows of its own
    R rows;
    rows.start(p, x, row0);

    // The table's entry for position p0 + lane and the page that it is, as above.
    auto entry_at = [&](int p0) -> int {
      return pages[min(p0 + lane, x.r.end - 1) >> p.page_shift];
    };
    auto page_of = [&](int entry, int p0) -> int {
      return p0 + lane < x.r.end && entry >= 0 && entry < p.n_pages ? entry : -1;
    };
    // Starts the loads of the tile at p0 into buffer `buf`; positions without
    // a page read page 0.
    auto load_tile = [&](int p0, int page, int buf) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int row = (j * kWaves + wave) * kHave;  // the wave's first
        lds_u16* const to = (lds_u16*)(tiles + buf * 2 * kTileElems + row * D);
        if (kEven) {
          const int64_t from =
              (int64_t)max(__builtin_amdgcn_readlane(page, row), 0) * p.page_stride +
              (int64_t)((p0 + row) & page_mask) * width;
          load_lds16(make_rsrc(kh + from, kHave * width * 2), to, my_at, 0);
          load_lds16(make_rsrc(vh + from, kHave * width * 2), to + kTileElems, my_at, 0);
        } else {
          const int mine = row + lane / kLanes, pg = __shfl(page, mine);
          const int64_t from = (pg < 0 ? 0 : pg * p.page_stride +
                                (int64_t)((p0 + mine) & page_mask) * width) + my_chunk * 8;
          load_lds(kh + from, to);
          load_lds(vh + from, to + kTileElems);
        }
      }
    };
    // Waits for the wave's own loads of the tile at p0 and mends its rows of V:
    // those that are not there become 0, infinities and NaN past L too, noted.
    auto finish_tile = [&](int p0, int page, int buf, int turn) {
      TG_WAIT_VM(0);
      asm volatile("" ::: "memory");
      if (p0 + kUnit <= x.r.L && __all(page >= 0)) return;
      const unsigned long long there = __ballot(page >= 0);
#pragma unroll 1
      for (int j = 0; j < kLoads; ++j) {
        const int row = (j * kWaves + wave) * kHave + lane / kLanes;
        const bool gone = !(there >> row & 1), own = p0 + row >= x.r.L;
        u32x4* const place = reinterpret_cast<u32x4*>(
            tiles + (buf * 2 + 1) * kTileElems + (j * kWaves + wave) * kHave * D + lane * 8);
        u32x4 y = *place;
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t odd = own ? odd_part<T>(y[i], true) : 0u;
          y[i] = gone ? 0u : y[i] ^ odd;
          bad |= odd;
        }
        if (bad && !gone) atomicOr(&odd_rows[turn][row / 32], 1u << (row % 32));
        *place = y;
      }
    };

    int p0 = x.r.from + x.u0 * kUnit, buf = 0, turn = 0;
    const int p_end = x.r.from + x.u1 * kUnit;
    int page = page_of(entry_at(p0), p0), entry = entry_at(p0 + kUnit);
    __syncthreads();  // the last piece's reads are over
    if (threadIdx.x < 6) odd_rows[threadIdx.x / 2][threadIdx.x % 2] = 0;
    load_tile(p0, page, 0);
    __syncthreads();
    finish_tile(p0, page, 0, 0);
    __syncthreads();
    for (; p0 < p_end; p0 += kUnit, buf ^= 1) {
      const bool more = p0 + kUnit < p_end;
      const int page_now = page;
      const uint16_t* const kt = tiles + buf * 2 * kTileElems;
      f32x4 s[kQ][4];
      if (busy) rows.scores(kt + col * D, k_chunk, s, kh);
      if (more) {
        page = page_of(entry, p0 + kUnit);
        load_tile(p0 + kUnit, page, buf ^ 1);
        entry = entry_at(p0 + 2 * kUnit);
      }
      const bool inner = p0 + kUnit <= x.r.L && __all(page_now >= 0);
      if (busy) {
        const unsigned long long there64 = inner ? ~0ull : __ballot(page_now >= 0);
        uint32_t see[2][kQ];
        if (!inner) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint32_t there = (uint32_t)(there64 >> (half * 32));
#pragma unroll
            for (int c = 0; c < kQ; ++c)
              see[half][c] = rows.sees(p, mask, x, c, p0 + half * kTile, there);
            R::hide(s, see[half], half);
          }
        }
        uint4 pr[2][kQ];
        rows.weigh(s, p.c, pr);
        const uint16_t* const vr = kt + kTileElems + v_row * D + (col & 1) * 4;
#pragma unroll
        for (int half = 0; half < 2; ++half)
          rows.add([&](int h, int d) {
            return vr + (half * kTile + h * 16) * D + (v_chunk ^ (d * 2)) * 8;
          }, pr[half], vh);
        if (!inner) {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t odd = odd_rows[turn][half];
            while (odd) {
              const int row = __ffs(odd) - 1;
              odd &= odd - 1;
              const int pg = __shfl(page_now, half * kTile + row);
              rows.add_odd(vh + pg * p.page_stride +
                               (int64_t)((p0 + half * kTile + row) & page_mask) * width,
                           row, pr[half], see[half]);
            }
          }
        }
      }
      // One tile's notes are read, the next one's written, and those of the
      // one after it (read before the last barrier) cleared.
      const int next = turn == 2 ? 0 : turn + 1;
      if (threadIdx.x < 2) odd_rows[next == 2 ? 0 : next + 1][threadIdx.x] = 0;
      if (more) finish_tile(p0 + kUnit, page, buf ^ 1, next);
      turn = next;
      __syncthreads();
    }

    const int64_t slot = 2 * (int64_t)run.me + (at == run.begin ? 0 : 1);
    if (busy) {
#pragma unroll
      for (int c = 0; c < kQ; ++c) {
        const float whole = sum4(rows.sum[c]);
        const int line = row0 + c * 16 + col;
        if (line < x.r.n * p.G) {
          if (x.whole && (kKind == kAll || (kKind == kTail && x.r.from == 0))) {
            const float inv = inverse(whole);
            uint16_t* const to = p.out + (int64_t)(x.r.first + rows.node[c]) * p.out_stride +
                                 (int64_t)(x.g * p.G + line - rows.node[c] * p.G) * D + quad * 4;
#pragma unroll
            for (int d = 0; d < R::kCols; ++d) {
              const f32x4 y = rows.o[c][d] * inv;
              *reinterpret_cast<uint2*>(to + d * 16) =
                  make_uint2(T::pack(y[0], y[1]), T::pack(y[2], y[3]));
            }
          } else {
            const int64_t line_at = slot * kRows + wave * 16 * kQ + c * 16 + col;
            float* to = p.part + line_at * D;
            float2* to_ml = p.part_ml + line_at;
            if constexpr (kKind != kAll)
              if (x.whole) {
                const int64_t at = whole_row(p, x, line);
                to = p.whole + at * D;
                to_ml = p.whole_ml + at;
              }
#pragma unroll
            for (int d = 0; d < R::kCols; ++d)
              *reinterpret_cast<f32x4*>(to + d * 16 + quad * 4) = rows.o[c][d];
            if (quad == 0) *to_ml = make_float2(rows.m[c], whole);
          }
        }
      }
    }
    at += x.u1 - x.u0;
  }
