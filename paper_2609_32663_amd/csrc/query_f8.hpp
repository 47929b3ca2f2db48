// One item of the query tiles over quantised pools: query tile qt of segment s
// over key tiles [t_lo, t_hi), as query_item does it for bf16 pools (included by
// query_attn.hip, whose items, tables and records these are).
//
// A SIMD issues vector instructions of one wave at half its rate (2.3 ns each, 1.0
// with two waves at it), so the two waves of a SIMD must not take turns between
// products and vector work, as the bf16 tiles' waves do: a vector phase is then as
// long as both waves' vector work together.  Here every wave runs through its keys
// by itself and meets the others once per 64-key tile, so that the two waves' vector
// phases can share the unit (24 tokens of 16 requests over 16K in turns 152 us, so
// 133).  What bounds it is this schedule.  Scores, conversion, softmax and outputs
// of a wave are one chain, in that order (the fences below keep it), and the two
// waves of a SIMD start every tile together at the meeting, so little of the
// matrix work lies beside vector work: for 512 tokens over 32K (8 heads of 128, 371 to
// 398 us with plan and merge, by card) the matrix units are busy 56% of the time,
// 52% for trees of 48, and the parts' times nearly add up (without the products of V 128 us
// less, all of their matrix time, without the softmax 114, without the conversion
// 25).  Three products a pair of key and query take 200 us at the rate that a loop
// of matrix instructions alone reaches (2.08 PFLOP/s).  With up to 128 rows a SIMD
// has one wave or two at work, and a tile is as long as their chain of phases (1.3
// us with 32 rows, 1.6 with 96).  Two tiles' rows on their way, in registers, gain
// 6% with 64 dims or up to 64 rows and lose 4% at 96 rows of 128 dims to spills.
//
//   * Waves are 32 query rows each: eight of them, or, with at most 128 rows, four
//     times two that share the rows and take a tile's halves (a key half each),
//     and are folded through LDS at the end.
//   * Wave w brings rows 8w .. 8w + 7 of the tile after the next, and their exponent
//     bytes, to LDS of its own, and a tile later converts them: K's values, exact
//     in bf16, and V's codes, exact in fp16, go to the tile buffers, the exponents
//     as numbers to where the softmax reads them.  Every row is converted once.
//   * S^T = K Q^T with v_mfma_f32_32x32x16_bf16 (a twelfth more per watt than
//     16x16x32): lane (query n = lane % 32, h = lane / 32) receives the scores of
//     keys 8i + 4h .. 8i + 4h + 3, i < 4, of 32 keys, so a row's maximum, sum and
//     mask are one lane's pair's.
//   * O += P V with v_mfma_f32_32x32x16_f16: K slot e of lane half h is key 16s +
//     8 (e / 4) + 4h + e % 4 of product s, the lane's scores in their order, and the
//     transpose reads of V fetch the same keys.  Weights: dkv_f8.hpp.
#pragma once

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int D>
__device__ __forceinline__ void f8_item(const QueryParams& p, const QueryItem& item, uint16_t* k0, uint16_t* k1,
                                        uint16_t* v0, uint16_t* v1, uint8_t* raw_k, uint8_t* raw_v, uint8_t* exps,
                                        float* keys0, float* keys1, u32x4* table, int* counts) {
  using C = QCfg<D>;
  constexpr int NU = D / 16;  // products of a score
  constexpr int NB = D / 32;  // 32-column output blocks
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int n32 = lane & 31;
  const int h = lane >> 5;

  // uniform: pages are looked up with scalar arithmetic
  const int s = __builtin_amdgcn_readfirstlane(item.s), qt = __builtin_amdgcn_readfirstlane(item.qt);
  const int64_t t_lo = q_uniform64(item.t_lo), t_hi = q_uniform64(item.t_hi);
  const PagedBlock blk{__builtin_amdgcn_readfirstlane(item.blk.tok0), __builtin_amdgcn_readfirstlane(item.blk.n),
                       __builtin_amdgcn_readfirstlane(item.blk.pos0)};
  const int32_t seen = __builtin_amdgcn_readfirstlane(item.seen);
  const int rows = blk.n * p.G;
  const int bseq = s / p.Hkv;
  const int g = s - bseq * p.Hkv;
  const int64_t tok_row0 = blk.tok0;

  // This wave's rows and key half (-1: both).  Waves w and w + 4 share a SIMD: the
  // halves of the same rows go to different ones, so that up to 64 rows use all
  // four (16 requests of 4 to 256 rows over up to 16K keys 206 us, so 199; of 64 rows over
  // 16K, in these tiles, 197 and 179).
  const bool halves = rows - qt * kQRows <= kQRows / 2;
  const int row_wave = halves ? (wave_u + 2 * (wave_u >> 2)) & 3 : wave_u;
  const int my_half = halves ? wave_u >> 2 : -1;
  const int wave_row0 = qt * kQRows + 32 * row_wave;
  const bool some = wave_row0 < rows;
  const int r = wave_row0 + n32;
  const bool row_ok = r < rows;
  const int tok = row_ok ? r / p.G : 0;
  const int32_t cut = paged_pos(blk, tok) + 1;  // positions below it are seen without a mask
  const int64_t k_lo = q_uniform64(t_lo * kQKeys);
  const int64_t k_end = t_hi * kQKeys < seen ? t_hi * kQKeys : seen;
  const int64_t k_hi = q_uniform64(k_end > k_lo ? k_end : k_lo);

  // |scale| and B operand of QK, as in query_item: query n32, dims 16u + 8h .. + 7
  const bool qneg = p.scale_log2 < 0.f;
  const float cpos = fmaxf(fabsf(p.scale_log2), 1.17549435e-38f);
  u32x4 qb[NU];
  {
    const char* qrow = static_cast<const char*>(p.q) + (tok_row0 + tok) * p.q_stride +
                       ((int64_t)g * p.G + (row_ok ? r - tok * p.G : 0)) * C::kRowBytes;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      qb[u] = row_ok ? *reinterpret_cast<const u32x4*>(qrow + 32 * u + 16 * h) : z;
      if (qneg) qb[u] ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    }
  }
  f32x16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) o[b] = f32x16{};
  float m = kF8None, l = 0.f;  // of query n32: reference (log2 units), this lane's share of the sum

  // ---- runs, raw rows and their conversion -----------------------------------
  TileRun run[2][2] = {}, ahead[2] = {};
  u32x4 coming[2];
  const PagedSegment seg =
      paged_segment(p, s, 0, (int32_t)k_hi, blk.pos0 >= 0 ? paged_pos(blk, blk.n - 1) + 1 : 0);
  auto fill_table = [&](int64_t from) __attribute__((always_inline)) {
    const int64_t left = (k_hi - from + kRun - 1) / kRun;
    const int n = (int)(left < 0 ? 0 : (left < kTableRuns ? left : kTableRuns));
    const i32x4* entries = reinterpret_cast<const i32x4*>(p.entries) + (int64_t)s * p.max_entries;
    for (int i = tid; i < n + kTablePad; i += kQThreads) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (i < n) {
        const int32_t at = (int32_t)from + i * kRun;
        w = tile_run_word(paged_run(seg, entries[at >> seg.shift], at), D);
      }
      table[i] = w;
    }
  };
  auto read_runs = [&](int at) __attribute__((always_inline)) {
    coming[0] = table[at];
    coming[1] = table[at + 1];
  };
  auto take_runs = [&](TileRun (&u)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      u[i] = TileRun{(uint32_t)__builtin_amdgcn_readfirstlane(coming[i][0]),
                     (uint32_t)__builtin_amdgcn_readfirstlane(coming[i][1]),
                     (uint32_t)__builtin_amdgcn_readfirstlane(coming[i][2]),
                     (uint32_t)__builtin_amdgcn_readfirstlane(coming[i][3])};
  };
  // lane l: row l % 8 of the wave's eight, 16 bytes l / 8 of it (64 dims: the first 32 lanes)
  auto raw_rows = [&](const TileRun (&u)[2]) __attribute__((always_inline)) {
    const TileRun& x = wave_u >= 4 ? u[1] : u[0];
    const uint64_t at = (uint64_t)(x.off_hi & 0xFFFF) << 32 | x.off;  // of the run's first slot that counts
    const uint32_t row = (uint32_t)(8 * (wave_u & 3));
    const uint32_t off = (row + (lane & 7) - x.lo()) * D + 16 * (lane >> 3);
    const __amdgpu_buffer_rsrc_t ks = q_rsrc(static_cast<const char*>(p.k) + at, x.bytes);
    const __amdgpu_buffer_rsrc_t vs = q_rsrc(static_cast<const char*>(p.v) + at, x.bytes);
    if (D == 128 || lane < 32) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          ks, (__attribute__((address_space(3))) void*)(raw_k + 8 * D * wave_u), 16, off, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          vs, (__attribute__((address_space(3))) void*)(raw_v + 8 * D * wave_u), 16, off, 0, 0, 0);
    }
    if (lane == 0)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          q_rsrc(reinterpret_cast<const char*>(p.scales) + 2 * (at / D - x.lo()), x.bytes > 0 ? 2 * kRun : 0),
          (__attribute__((address_space(3))) void*)(exps + 16 * wave_u), 16, 2 * row, 0, 0, 0);
  };
  // Row l % 8, D / 8 codes l / 8.  K's layout, in 16-byte chunks: ((R / 32) *
  // kRowChunks + c) * 32 + (R + 8 (c % 2)) % 32, so that a product's lanes read 32 in a
  // row; V's: ((R / 8) * kRowChunks / 2 + c / 2) * 16 + 2 (R % 8 ^ 4 (c / 2 % 2)) + c % 2.  The
  // turn by 8 rows and the exchange of 4, and odd columns' eights in the other order,
  // keep the lanes that write or read together in different banks (a tenth of the
  // kernel's cycles were conflicts, a third of that is left; trees of 48 over 32K 432 -> 427 us).
  const int swap = D == 128 ? (lane >> 3) & 1 : 0;
  uint2 rk[D / 64], rv[D / 64];
  uint32_t rx;
  auto read_raw = [&]() __attribute__((always_inline)) {
    const int row = lane & 7, col = lane >> 3;
    const int at = 8 * D * wave_u + (D == 128 ? 16 * lane : 16 * (row + 8 * (col >> 1)) + 8 * (col & 1));
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      rk[i] = *reinterpret_cast<const uint2*>(raw_k + at + 8 * (i ^ swap));
      rv[i] = *reinterpret_cast<const uint2*>(raw_v + at + 8 * (i ^ swap));
    }
    rx = *reinterpret_cast<const uint16_t*>(exps + 16 * wave_u + 2 * row);
  };
  auto convert = [&](uint16_t* kb, uint16_t* vb, float* keys) __attribute__((always_inline)) {
    const int col = lane >> 3, R = 8 * wave_u + (lane & 7);
    // a byte that belongs to no slot of the entry may be that of an infinity
    const float power = f8_power((rx & 0xFF) < 254u ? rx & 0xFF : 254u);
    if (col == 0) {
      const uint32_t byte = rx >> 8 > kF8MinByte ? rx >> 8 : kF8MinByte;  // rows of zeros may come with any
      keys[R] = (float)byte;
      keys[kQKeys + R] = __builtin_amdgcn_ldexpf(1.f, 127 - (int)byte);
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const int c = D / 64 * col + (i ^ swap);  // eight columns
      *reinterpret_cast<u32x4*>(kb + 8 * (((R / 32) * C::kRowChunks + c) * 32 + (R + 8 * (c & 1)) % 32)) =
          u32x4{f8_pair<false>(rk[i].x, power), f8_pair<true>(rk[i].x, power), f8_pair<false>(rk[i].y, power),
                f8_pair<true>(rk[i].y, power)};
      *reinterpret_cast<u32x4*>(vb + 8 * (((R / 8) * (C::kRowChunks / 2) + c / 2) * 16 + (R % 8 ^ 4 * (c / 2 & 1)) * 2 + c % 2)) =
          u32x4{f8_pair_f16<false>(rv[i].x), f8_pair_f16<true>(rv[i].x), f8_pair_f16<false>(rv[i].y),
                f8_pair_f16<true>(rv[i].y)};
    }
  };

  // ---- 32 keys -----------------------------------------------------------------
  const int32_t pos_all = p.mask != nullptr ? blk.pos0 : paged_pos(blk, min(wave_row0, rows - 1) / p.G) + 1;
  // LDS reads go out well before their products: K's of 32 keys at once, V's two
  // groups of products ahead.  The fences keep the compiler from gathering them in
  // front of their uses again.
  u32x4 kf[NU];
  auto load_k = [&](const uint16_t* kb, int half) __attribute__((always_inline)) {
    const uint16_t* kr = kb + 8 * ((half * C::kRowChunks + h) * 32 + ((n32 + 8 * h) & 31));
#pragma unroll
    for (int u = 0; u < NU; ++u) kf[u] = *reinterpret_cast<const u32x4*>(kr + 8 * 64 * u);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto scores = [&]() __attribute__((always_inline)) {
    f32x16 a = {};
#pragma unroll
    for (int u = 0; u < NU; ++u)
      a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[u]), __builtin_bit_cast(bf16x8, qb[u]), a, 0,
                                                  0, 0);
    __builtin_amdgcn_sched_barrier(0);
    return a;
  };
  constexpr int NG = NB;  // groups of V: two blocks of one of the two products
  u32x4 vf[2][2];
  auto load_v = [&](const uint16_t* vb, int half, int n) __attribute__((always_inline)) {
    const int j = lane & 15, ch = (lane >> 4) & 1;
    const uint16_t* vr = vb + (4 * half * (C::kRowChunks / 2) + ch) * 128 + (4 * (h ^ ch) + (j >> 2)) * 16 + (j & 3) * 4;
    const int t = n / (NB / 2), b0 = n % (NB / 2) * 2;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint16_t* at = vr + (2 * t * (C::kRowChunks / 2) + 2 * (b0 + b)) * 128;
      const uint2 w0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at));
      const uint2 w1 = __builtin_bit_cast(
          uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + (C::kRowChunks / 2) * 128)));
      vf[n % 2][b] = u32x4{w0.x, w0.y, w1.x, w1.y};
    }
  };
  u32x4 pp[2][2];  // [part][product]
  auto softmax = [&](f32x16 sc, const TileRun& u, const float* keys, const uint16_t* vb, int half) __attribute__((always_inline)) {
    // slots outside the entry, or that one of the wave's rows does not see
    if (!u.whole() || (int32_t)u.pos + kRun > pos_all) {
      asm volatile("");  // keeps this a branch
      const uint32_t sees =
          tree_sees(p, tok_row0 + tok, cut, blk.pos0, (int32_t)u.pos, (int32_t)u.lo(), (int32_t)u.hi()) >> 4 * h;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(sees >> (8 * (i >> 2) + (i & 3)) & 1)) sc[i] = -INFINITY;
    }
    float x[16], mx = kF8None;
    auto exponents = [&]() __attribute__((always_inline)) {
      const float base = m - kF8Up;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 byte = *reinterpret_cast<const f32x4*>(keys + 8 * i + 4 * h);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          x[4 * i + v] = __builtin_fmaf(sc[4 * i + v], cpos, byte[v] - base);
          mx = fmaxf(mx, x[4 * i + v]);
        }
      }
    };
    exponents();
    if (__builtin_amdgcn_ballot_w64(mx > kF8Up + kLazy)) {
      float mt = kF8None;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 byte = *reinterpret_cast<const f32x4*>(keys + 8 * i + 4 * h);
#pragma unroll
        for (int v = 0; v < 4; ++v) mt = fmaxf(mt, __builtin_fmaf(sc[4 * i + v], cpos, byte[v]));
      }
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
      mt = __builtin_ceilf(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
      const bool grow = mt > m + kLazy;
      const float alpha = fast_exp2(grow ? m - mt : 0.f);
      m = grow ? mt : m;
      l *= alpha;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float a = __shfl(alpha, 8 * (i >> 2) + 4 * h + (i & 3), 64);
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b][i] *= a;
      }
      exponents();
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = fminf(x[i], kF8Top);
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) load_v(vb, half, n);
    __builtin_amdgcn_sched_barrier(0);
    float ps = l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 back = *reinterpret_cast<const f32x4*>(keys + kQKeys + 8 * i + 4 * h);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        x[4 * i + v] = fast_exp2(x[4 * i + v]);
        ps = __builtin_fmaf(x[4 * i + v], back[v], ps);
      }
#pragma unroll
      for (int v = 0; v < 4; v += 2) {
        uint32_t w[2];
        f16_parts(x[4 * i + v], x[4 * i + v + 1], w[0], w[1]);
        pp[0][i >> 1][2 * (i & 1) + v / 2] = w[0];
        pp[1][i >> 1][2 * (i & 1) + v / 2] = w[1];
      }
    }
    l = ps;
    asm volatile("" : "+v"(l));
  };
  auto outputs = [&](const uint16_t* vb, int half) __attribute__((always_inline)) {
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const int t = n / (NB / 2), b0 = n % (NB / 2) * 2;
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int b = 0; b < 2; ++b)
          o[b0 + b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, pp[part][t]),
                                                             __builtin_bit_cast(f16x8_t, vf[n % 2][b]), o[b0 + b], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (n + 2 < NG) load_v(vb, half, n + 2);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // ---- the walk ------------------------------------------------------------------
  auto meet = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_sched_barrier(0);
  };
  uint16_t* const kbuf[2] = {k0, k1};
  uint16_t* const vbuf[2] = {v0, v1};
  float* const kkeys[2] = {keys0, keys1};
  fill_table(k_lo);
  __syncthreads();
  int64_t ntile = (k_hi - k_lo + kQKeys - 1) / kQKeys;
  if (item.gaps && k_hi - k_lo <= kTableRuns * kRun) {
    ntile = (drop_gaps(table, counts, (int)((k_hi - k_lo + kRun - 1) / kRun)) + 1) / 2;
    __syncthreads();
  }
  ntile = q_uniform64(ntile);
  read_runs(0);
  take_runs(run[0]);
  read_runs(2);
  take_runs(run[1]);
  raw_rows(run[0]);
  __builtin_amdgcn_s_waitcnt(0x0F70);
  __builtin_amdgcn_sched_barrier(0);
  read_raw();
  convert(kbuf[0], vbuf[0], kkeys[0]);
  __builtin_amdgcn_sched_barrier(0);
  raw_rows(run[1]);
  int at = 4;  // where the table holds the tile whose rows set out next
  int64_t from = k_lo;
  // Tile t in buffers i.  After the meeting everybody has left tile t - 1, whose
  // buffers take tile t + 1, and tile t is written.
  auto tile = [&](auto par, auto any, auto two) __attribute__((always_inline)) {
    constexpr int i = decltype(par)::value;
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the wave's rows of tile t are written
    meet();
    read_runs(at);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // those of tile t + 1 have arrived
    __builtin_amdgcn_sched_barrier(0);
    read_raw();
    const int first = decltype(two)::value ? 0 : my_half;
    f32x16 sc;
    if constexpr (decltype(any)::value) {
      load_k(kbuf[i], first);
      sc = scores();
    }
    take_runs(ahead);
    convert(kbuf[1 - i], vbuf[1 - i], kkeys[1 - i]);
    __builtin_amdgcn_sched_barrier(0);
    raw_rows(ahead);
    if constexpr (decltype(any)::value) {
      softmax(sc, first ? run[i][1] : run[i][0], kkeys[i] + 32 * first, vbuf[i], first);
      if constexpr (decltype(two)::value) load_k(kbuf[i], 1);
      outputs(vbuf[i], first);
      if constexpr (decltype(two)::value) {
        sc = scores();
        softmax(sc, run[i][1], kkeys[i] + 32, vbuf[i], 1);
        outputs(vbuf[i], 1);
      }
    }
    run[i][0] = ahead[0];
    run[i][1] = ahead[1];
    at += 2;
    from += kQKeys;
  };
  auto walk = [&](auto any, auto two) __attribute__((always_inline)) {
    for (int64_t t = 0; t < ntile; t += 2) {
      if (at + 4 > kTableRuns) {
        // nobody reads the table between the meeting and this
        meet();
        fill_table(from + 2 * kQKeys);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        meet();
        at = 0;
      }
      tile(std::integral_constant<int, 0>{}, any, two);
      if (t + 1 < ntile) tile(std::integral_constant<int, 1>{}, any, two);
    }
  };
  if (!some) walk(std::false_type{}, std::true_type{});
  else if (halves) walk(std::true_type{}, std::false_type{});
  else walk(std::true_type{}, std::true_type{});
  // no direct load may still be writing LDS when the workgroup goes on
  __builtin_amdgcn_s_waitcnt(0x0F70);

  // ---- the two key halves' waves; row totals; the output or this range's record ----
  if (halves) {
    __syncthreads();  // nobody reads tiles any more
    // The second half's waves hand theirs over: 16 KB (8 with 64 dims) of accumulators through a tile
    // buffer, maximum and sum through the codes' room.
    f32x4* const hand = reinterpret_cast<f32x4*>((row_wave & 2) ? ((row_wave & 1) ? v1 : v0) : ((row_wave & 1) ? k1 : k0));
    float* const ml = reinterpret_cast<float*>(raw_k) + 128 * row_wave;
    if (some && my_half == 1) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          hand[(4 * b + i) * 64 + lane] = f32x4{o[b][4 * i], o[b][4 * i + 1], o[b][4 * i + 2], o[b][4 * i + 3]};
      ml[lane] = m;
      ml[64 + lane] = l;
    }
    __syncthreads();
    if (some && my_half == 0) {
      const float m1 = ml[lane], l1 = ml[64 + lane];
      const float M = fmaxf(m, m1);
      const float f0 = fast_exp2(m - M), f1 = fast_exp2(m1 - M);
      l = l * f0 + l1 * f1;
      m = M;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a0[4], a1[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          a0[v] = __shfl(f0, 8 * i + 4 * h + v, 64);
          a1[v] = __shfl(f1, 8 * i + 4 * h + v, 64);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const f32x4 c = hand[(4 * b + i) * 64 + lane];
#pragma unroll
          for (int v = 0; v < 4; ++v) o[b][4 * i + v] = o[b][4 * i + v] * a0[v] + c[v] * a1[v];
        }
      }
    }
  }
  if (!some || my_half == 1) return;
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int at_row = 8 * (i >> 2) + 4 * h + (i & 3);
    const float lq = __shfl(l, at_row, 64), mq = __shfl(m, at_row, 64);
    const int rr = 32 * row_wave + at_row, rq = qt * kQRows + rr;
    if (rq >= rows) continue;
    if (item.single) {
      const int tq = rq / p.G;
      float* orow = p.out + ((tok_row0 + tq) * p.Hq + (int64_t)g * p.G + (rq - tq * p.G)) * D;
      const float inv = lq > 0.f ? 1.f / lq : 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b) orow[32 * b + n32] = o[b][i] * inv;
    } else {
      float* rrow = item.rec + (int64_t)rr * C::kRec;
      if (n32 == 0) {
        rrow[0] = mq;
        rrow[1] = lq;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) rrow[2 + 32 * b + n32] = o[b][i];
    }
  }
}
