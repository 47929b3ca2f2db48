// Query-block attention over the packed Distance-KV cache (Sec. 3.4: after
// the one-time compaction the query tokens attend to the compressed context,
// while their own K/V are appended like every new token and kept).
//
// Rows.  Segment s = (sequence b, KV head g) has R = n_q * G query rows; row
// r is token r / G of query head g * G + r % G and sees the segment's first
// seg_len + n_tail + r / G + 1 rows (the packed context, the tokens appended
// before the block, and the block causally up to its own token).
//
// Work split.  A workgroup (8 waves of 32 rows) takes one item: 256 query
// rows (a query tile) of one segment and one key range.  Each segment's
// keys are cut into max(1, round(tiles / C)) near-equal ranges of whole
// 64-key tiles, C the same for every segment, so items are about equally
// long however unequal the segments are.  A one-workgroup plan kernel counts
// the ranges and lays the items out segment by segment, range by range,
// query tile fastest; the workgroups of one hardware L2 domain (ids equal
// mod 8) take consecutive items, so the query tiles of a key range read it
// through the same L2.  With one range a workgroup writes the output; with
// several, each range writes (max, sum, unnormalised output) per row and a
// combine kernel folds the ranges in order.  When the keys are too few to
// split at all there is no plan: one workgroup per (segment, query tile).
//
// Per 64-key tile, K and V go from memory straight into LDS (16 bytes per
// lane, two buffers per matrix, a whole tile ahead); every wave then works
// on 32-key halves:
//   * S^T = K Q^T with v_mfma_f32_16x16x32_bf16: 16 K rows from LDS are the
//     A operand, the wave's two 16-row groups (registers) two B operands, so
//     lane (query n, group kg) receives the scores of keys 4kg..4kg+3 of each
//     16-key block.
//   * Online softmax per query row: max over the lane's scores, then over the
//     row's 4 lanes (permlane swaps); probabilities 2^(c s - m) stay fp32
//     until the product.  The reference max m moves only when a half's max
//     exceeds it by more than 2^8, so the accumulators are rarely rescaled.
//   * O += P V with v_mfma_f32_16x16x32_bf16 per 32 keys: the probabilities
//     are the A operand as the scores sit in the lanes (lane (query n, kg)
//     holds keys 4kg..4kg+3 of two 16-key blocks: its eight K slots), split
//     into a bf16 high part and a bf16 remainder (two products, ~16
//     significant bits kept).  The B operand needs, per lane, the same eight
//     keys of one V column; two ds_read_b64_tr_b16 transpose reads fetch them
//     (within each 16-lane group, lanes 4r..4r+3 address row r of a 4 x 16
//     block and lane i receives its column i).
// The two waves on a SIMD play ping-pong: while one issues the products of
// its half, the other runs the softmax and bf16 split of its own, so the
// matrix and the vector units of a SIMD work at once.  Attention here is a
// dense contraction (G * n_q query rows against every key), so it is MFMA
// work, unlike the one-query decode step.
//
// Paged calls (dkv_paged_query_attn) run the same tiles over a segment's pages,
// for sequences whose chunks differ in length: the split into slices and the
// kernel that plans it are described further down, tile addresses come from a
// table of 32-row runs in LDS, the products of a phase are one pipeline of LDS
// reads and matrix instructions, and a probability has three bf16 parts.  A
// workgroup takes 6,540 cycles for a 64-key tile, of which its matrix
// instructions fill 4,096: 512 tokens of an 8B layer over 32K keys 423 us (655
// TFLOP/s of the 4 d flops per query row and key, 1,310 with the further
// parts'), two prompts of 4K 261 us (565 and 1,130).
//
// This file is compiled with IEEE mode off and no NaN semantics
// (-mno-amdgpu-ieee -fno-honor-nans): the maxima then need no NaN
// canonicalisation.  With finite inputs no NaN arises anywhere (masked keys
// are -inf and every -inf - x difference feeds a factor of 0 or 1); for NaN
// inputs the outputs are unspecified.

#include <hip/hip_runtime.h>

#include <type_traits>

#include "dkv_device.hpp"
#include "../../include/dkv.h"
#include "dkv_query_device.hpp"

namespace dkv {

namespace {

constexpr int kQThreads = 512;
constexpr int kRG = 2;                   // 16-row groups per wave
constexpr int kQRows = kQueryRowsPerWG;  // query rows per workgroup
static_assert(kQRows == kQThreads / kWave * 16 * kRG, "rows per workgroup");
constexpr int kQKeys = 64;               // keys per tile
constexpr int kPlanThreads = 1024;

template <int D>
struct QCfg {
  static constexpr int kRowBytes = D * 2;
  static constexpr int kChunks = D / 32;    // 16-byte chunks of a row per lane (QK)
  static constexpr int kBlocks = D / 16;    // 16-column output blocks per lane
  static constexpr int kRowChunks = D / 8;  // 16-byte chunks per row
  static constexpr int kDma = kQKeys * kRowChunks / kWave / (kQThreads / kWave);  // loads per wave per matrix
  static constexpr int kRec = D + 2;        // floats per partial record row
  static_assert(kDma >= 1, "a tile needs one direct load per wave at least");
};

// Key tiles of segment s for its last query row (the most any row sees).
// A negative length marks a segment dkv_compact could not pack: no tiles.
__device__ __forceinline__ int64_t seg_tiles(const QueryParams& p, int s) {
  const int32_t len = p.seg_len[s];
  return len < 0 ? 0 : ((int64_t)len + p.n_tail + p.n_q + kQKeys - 1) / kQKeys;
}

__device__ __forceinline__ int64_t seg_ranges(int64_t tiles, int64_t c) {
  const int64_t r = (tiles + c / 2) / c;
  return r < 1 ? 1 : r;
}

// Plan of the split: with C tiles per range (raised if the ranges would not
// fit the records the workspace holds), ranges per segment and the first
// item of every segment.
__global__ __launch_bounds__(kPlanThreads) void query_plan_kernel(QueryParams p) {
  __shared__ int64_t red[kPlanThreads / kWave + 1];
  const int tid = threadIdx.x;
  int64_t part = 0;
  for (int s = tid; s < p.nseg; s += kPlanThreads) part += seg_tiles(p, s);
  int64_t total_tiles;
  block_exclusive_scan<kPlanThreads>(part, red, &total_tiles);
  // qtiles * sum_s max(1, round(T_s / C)) <= qtiles * (total / C + nseg) <= max_items
  const int64_t room = p.max_items / p.qtiles - p.nseg;  // >= 1 (host)
  int64_t c = p.tiles_per_range;
  const int64_t cmin = (total_tiles + room - 1) / room;
  if (c < cmin) c = cmin;
  int64_t base = 0;
  for (int s0 = 0; s0 < p.nseg; s0 += kPlanThreads) {
    const int s = s0 + tid;
    const int64_t r = s < p.nseg ? seg_ranges(seg_tiles(p, s), c) : 0;
    int64_t sum;
    const int64_t ex = block_exclusive_scan<kPlanThreads>(r, red, &sum);
    if (s < p.nseg) p.plan[kQueryPlanHead + s] = (int32_t)((base + ex) * p.qtiles);
    base += sum;
  }
  if (tid == 0) {
    p.plan[kQueryPlanHead + p.nseg] = (int32_t)(base * p.qtiles);
    p.plan[0] = (int32_t)(base * p.qtiles);
    p.plan[1] = (int32_t)(c < INT32_MAX ? c : INT32_MAX);  // for inspection; no kernel reads it
  }
}

// One item of a workgroup: query tile qt of segment s over key tiles [t_lo,
// t_hi), which writes the output (`single`) or a record.
struct QueryItem {
  int s, qt;
  int64_t t_lo, t_hi;
  bool single;
  float* rec;
  PagedBlock blk;  // paged: the sequence's block, and the segment's rows that the tile's rows see
  int32_t seen;
  bool gaps;  // among them may be slots of no key
};

// Paged: the next kTableRuns runs of a segment's rows, decoded side by side into
// LDS before they are walked: a wave's scalar instructions take its issue slots
// like any other, and finding a tile's pages entry by entry (some 200 of them)
// took a seventh of its time.  A word is the run's byte offset in the pools
// (48 bits), its first and last slot, its first position and its bytes.
constexpr int kTableRuns = 2048;
constexpr int kTablePad = 8;  // empty runs behind the span: tiles are read ahead

struct TileRun {
  uint32_t off, off_hi, pos, bytes;  // off_hi: offset bits 32 .. 47 | lo << 16 | hi << 24

  __device__ __forceinline__ uint32_t lo() const { return (off_hi >> 16) & 0xFF; }
  __device__ __forceinline__ uint32_t hi() const { return off_hi >> 24; }
  __device__ __forceinline__ bool whole() const { return off_hi >> 16 == kRun << 8; }
};

__device__ __forceinline__ u32x4 tile_run_word(const PagedRun& u, int row_bytes) {
  const uint64_t off = (uint64_t)(u.row + u.lo()) * row_bytes;
  return u32x4{(uint32_t)off, (uint32_t)(off >> 32) | (uint32_t)u.lohi << 16, (uint32_t)u.pos,
               (uint32_t)((u.hi() - u.lo()) * row_bytes)};
}

template <int D, bool PAGED>
__device__ __forceinline__ void query_item(const QueryParams& p, const QueryItem& item, uint16_t* k0, uint16_t* k1,
                                           uint16_t* v0, uint16_t* v1, u32x4* table, int* counts) {
  using C = QCfg<D>;
  // bf16 parts of a probability.  Packed: two, 17 bits.  Paged: three, its 24
  // bits, at any length: two err by 2.1e-6 to 2.5e-6 of the output's norm at
  // 1,000 keys as at 131,072, three by 2.0e-7 to 5.2e-7, attention in plain fp32
  // by 3.3e-7 to 4.0e-6 (q, K, V Gaussian, one head; 64 dimensions at 131,072 keys
  // 2.5e-6, 5.2e-7 and 1.8e-6; the more keys a workgroup adds up, the more the fp32
  // sums err: 8 heads, 512 tokens at 32K, three parts 1.0e-6).  The third product
  // costs what it computes, as the kernel runs at the rate that the matrix units
  // reach under the power limit (two / three parts, us, 8B layer: 512 tokens at 32K
  // 349 / 423, 256 over 45K rows 277 / 330).
  constexpr int kParts = PAGED ? 3 : 2;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  const int n16 = lane & 15;
  const int kg = lane >> 4;

  int s = item.s, qt = item.qt;
  int64_t t_lo = item.t_lo, t_hi = item.t_hi;
  PagedBlock blk = item.blk;
  int32_t seen = item.seen;
  if constexpr (PAGED) {  // uniform: pages are looked up with scalar loads and arithmetic
    s = __builtin_amdgcn_readfirstlane(s);
    qt = __builtin_amdgcn_readfirstlane(qt);
    t_lo = q_uniform64(t_lo);
    t_hi = q_uniform64(t_hi);
    blk.tok0 = __builtin_amdgcn_readfirstlane(blk.tok0);
    blk.n = __builtin_amdgcn_readfirstlane(blk.n);
    blk.pos0 = __builtin_amdgcn_readfirstlane(blk.pos0);
    seen = __builtin_amdgcn_readfirstlane(seen);
  }
  const int rows = PAGED ? blk.n * p.G : p.rows;  // query rows of the segment
  const int bseq = s / p.Hkv;
  const int g = s - bseq * p.Hkv;
  int64_t base_len = 0, row0 = 0;
  if constexpr (!PAGED) {
    if (p.seg_len[s] < 0) {
      // a segment dkv_compact could not pack (one range, so this workgroup
      // owns its query tile's output): no rows to attend, zeros
      for (int i = tid; i < kQRows * D; i += kQThreads) {
        const int rq = qt * kQRows + i / D;
        if (rq >= p.rows) break;
        const int tq = rq / p.G;
        p.out[(((int64_t)bseq * p.n_q + tq) * p.Hq + (int64_t)g * p.G + (rq - tq * p.G)) * D + i % D] = 0.f;
      }
      return;
    }
    base_len = q_uniform64((int64_t)p.seg_len[s] + p.n_tail);  // rows every query row sees
    row0 = q_uniform64(p.seg_off[s]);
  }
  // where the block starts in the token-major arrays
  const int64_t tok_row0 = PAGED ? (int64_t)blk.tok0 : (int64_t)bseq * p.n_q;

  // Paged: up to 128 rows are spread over the waves, one row group each: a wave's
  // phases halve, and they bound a tile of few rows (32 sequences of 8,000 keys:
  // 32 rows 264 -> 198 us, 64 278 -> 224, 128 324 -> 309).
  const bool spread = PAGED && rows - qt * kQRows <= kQRows / 2;
  const int wave_rows = spread ? 16 : 16 * kRG;
  // this lane's query rows (one per row group) in the score layout, and the keys they see
  int r[kRG], tok[kRG];
  bool row_ok[kRG];
  int64_t limit[kRG];
#pragma unroll
  for (int q = 0; q < kRG; ++q) {
    r[q] = qt * kQRows + wave * wave_rows + 16 * q + n16;
    row_ok[q] = r[q] < rows && 16 * q < wave_rows;
    tok[q] = row_ok[q] ? r[q] / p.G : 0;
    limit[q] = base_len + tok[q] + 1;
  }
  // this workgroup's keys: the range, up to what its last row sees
  // (all workgroup-uniform; readfirstlane keeps them in scalar registers)
  const int r_last = min(rows - 1, qt * kQRows + kQRows - 1);
  const int64_t lim_max = PAGED ? (int64_t)seen : base_len + r_last / p.G + 1;
  const int64_t k_lo = q_uniform64(t_lo * kQKeys);
  const int64_t k_end = t_hi * kQKeys < lim_max ? t_hi * kQKeys : lim_max;
  const int64_t k_hi = q_uniform64(k_end > k_lo ? k_end : k_lo);
  // packed: keys [k_lo, k_lo + cut) count for the row (cut <= the range length);
  // paged: keys at positions below cut
  int32_t cut[kRG];
#pragma unroll
  for (int q = 0; q < kRG; ++q)
    cut[q] = PAGED ? paged_pos(blk, tok[q]) + 1 : (int32_t)((limit[q] < k_hi ? limit[q] : k_hi) - k_lo);
  // every row of the workgroup sees all keys below this one
  const int64_t all_see = q_uniform64(base_len + 1 < k_hi ? base_len + 1 : k_hi);

  // Scores are taken with |scale| (a negative scale negates the queries,
  // exactly); a zero scale becomes the smallest normal float, so masked keys
  // (-inf) stay at -inf after scaling.
  const bool qneg = p.scale_log2 < 0.f;
  const float cpos = fmaxf(fabsf(p.scale_log2), 1.17549435e-38f);
  // B operand of QK: query row r, dims 32u + 8kg .. +7
  u32x4 qb[kRG][C::kChunks];
#pragma unroll
  for (int q = 0; q < kRG; ++q) {
    const int hh = r[q] - tok[q] * p.G;
    const char* qrow = reinterpret_cast<const char*>(p.q);
    if constexpr (PAGED)
      qrow += (tok_row0 + tok[q]) * p.q_stride + ((int64_t)g * p.G + (row_ok[q] ? hh : 0)) * C::kRowBytes;
    else
      qrow += ((tok_row0 + tok[q]) * p.Hq + (int64_t)g * p.G + (row_ok[q] ? hh : 0)) * C::kRowBytes;
#pragma unroll
    for (int u = 0; u < C::kChunks; ++u) {
      const u32x4 z = {0u, 0u, 0u, 0u};
      qb[q][u] = row_ok[q] ? *reinterpret_cast<const u32x4*>(qrow + 64 * u + 16 * kg) : z;
      if (qneg) qb[q][u] ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
    }
  }

  // output accumulators as scalars: a rescale in a branch then updates them
  // in place instead of in a second set of registers
  float o[kRG][C::kBlocks][4];
  float m[kRG], l[kRG];  // reference max of query row n16 (log2 units), this lane's share of its sum
#pragma unroll
  for (int q = 0; q < kRG; ++q) {
#pragma unroll
    for (int b = 0; b < C::kBlocks; ++b) o[q][b][0] = o[q][b][1] = o[q][b][2] = o[q][b][3] = 0.f;
    m[q] = -INFINITY;
    l[q] = 0.f;
  }

  const char* kbase = reinterpret_cast<const char*>(p.k) + row0 * C::kRowBytes;
  const char* vbase = reinterpret_cast<const char*>(p.v) + row0 * C::kRowBytes;
  // LDS layouts (16-byte chunk units; chunk c of key row R is bytes 16c..16c+15):
  //   K: ((R / 16) * kRowChunks + c) * 16 + R % 16   -- 16 rows of one chunk column together
  //   V: ((R / 8) * kRowChunks / 2 + c / 2) * 16 + (R % 8) * 2 + c % 2
  //      -- 8 rows of one 32-byte column pair together
  // The score product's lanes then read 16 consecutive chunks (K) and the
  // transpose reads 32 consecutive 8-byte halves (V): no bank conflicts, and
  // every read is a per-lane base plus a constant.  One wave instruction of
  // the direct loads fills 64 consecutive chunks (lane l chunk l).
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  // byte offsets of this lane's chunk within a tile for the wave's first
  // instruction; instruction i covers the chunks 1 KiB x (waves) x i further
  // on in both layouts, in LDS and in memory alike (the layouts are made of
  // whole 16-row / 8-row blocks)
  uint32_t koff, voff;
  {
    const int qk_ = 4 * wave + (lane >> 4);  // K: (R / 16) * kRowChunks + c
    const int rk = 16 * (qk_ / C::kRowChunks) + (lane & 15);
    koff = (uint32_t)(rk * C::kRowBytes + 16 * (qk_ % C::kRowChunks));
    const int qv = 4 * wave + (lane >> 4);  // V: (R / 8) * kRowChunks / 2 + c / 2
    const int rv = 8 * (qv / (C::kRowChunks / 2)) + ((lane >> 1) & 7);
    voff = (uint32_t)(rv * C::kRowBytes + 16 * (2 * (qv % (C::kRowChunks / 2)) + (lane & 1)));
  }
  // Global -> LDS: K or V rows [kt, kt + kQKeys) of the segment into a tile
  // buffer.  Keys past k_hi (a whole tile past it included) read zeros
  // without touching memory, so the loads are issued unconditionally.  (The
  // range check of a raw buffer counts the scalar offset too, which
  // tests/test_gpu_query_room.py holds with NaN behind every segment; the
  // displacement in the vector offset cost 4 registers and 1% of a 256-token
  // call at 128K.)
  // Paged: the two 32-row runs of a tile lie in pages of their own, each with
  // a descriptor over its slots [lo, hi): slots outside them (and runs past
  // the range) read zeros.  A wave instruction stays within one run.  `run`
  // holds the runs of tile t (parity t % 2) from its K loads on, in scalar
  // registers.
  TileRun run[2][2] = {};
  TileRun ahead[2] = {};  // the runs of the tile whose K is loaded next
  u32x4 coming[2];        // the same, on their way from the table
  const PagedSegment seg = PAGED ? paged_segment(p, s, 0, (int32_t)k_hi,
                                                 blk.pos0 >= 0 ? paged_pos(blk, blk.n - 1) + 1 : 0)
                                 : PagedSegment{};
  if (PAGED && D == 64) {  // one instruction per wave: waves 4-7 fill the second run
    koff -= (uint32_t)((wave_u >> 2) * kRun * C::kRowBytes);
    voff -= (uint32_t)((wave_u >> 2) * kRun * C::kRowBytes);
  }
  // the runs from row `from` on, up to the range's end and kTablePad empty ones
  auto fill_table = [&](int64_t from) __attribute__((always_inline)) {
    const int64_t left = (k_hi - from + kRun - 1) / kRun;
    const int n = (int)(left < 0 ? 0 : (left < kTableRuns ? left : kTableRuns));
    const i32x4* entries = reinterpret_cast<const i32x4*>(p.entries) + (int64_t)s * p.max_entries;
    for (int i = tid; i < n + kTablePad; i += kQThreads) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (i < n) {
        const int32_t r = (int32_t)from + i * kRun;
        w = tile_run_word(paged_run(seg, entries[r >> seg.shift], r), C::kRowBytes);
      }
      table[i] = w;
    }
  };
  // The runs with slots moved to the table's front, in order; returns their
  // number (256 tokens over the 35% of 131,072 positions that a selection kept,
  // in 128-row pages 333 -> 323 us, in 256-row pages 369 -> 324, in 1,024-row pages
  // 613 -> 372; 512 tokens over whole pages, without gaps, 417 -> 420).  A word moves
  // to its own index or a lower one, after the words up to it have been read.
  auto drop_gaps = [&](int n) __attribute__((always_inline)) {
    int at = 0;
    for (int i0 = 0, turn = 0; i0 < n; i0 += kQThreads, turn ^= 1) {
      const int i = i0 + tid;
      u32x4 w = {0u, 0u, 0u, 0u};
      if (i < n) w = table[i];
      const uint64_t some = __builtin_amdgcn_ballot_w64(w[3] != 0u);
      if (lane == 0) counts[8 * turn + wave] = __popcll(some);
      __syncthreads();
      int to = at;
      for (int k = 0; k < kQThreads / kWave; ++k) {
        const int c = counts[8 * turn + k];
        to += k < wave ? c : 0;
        at += c;
      }
      if (w[3] != 0u) table[to + __popcll(some & ((1ull << lane) - 1))] = w;
    }
    __syncthreads();
    if (tid < kTablePad) table[at + tid] = u32x4{0u, 0u, 0u, 0u};
    return __builtin_amdgcn_readfirstlane(at);
  };
  auto read_runs = [&](int at) __attribute__((always_inline)) {
    coming[0] = table[at];
    coming[1] = table[at + 1];
  };
  auto take_runs = [&](TileRun (&u)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      u[h] = TileRun{(uint32_t)__builtin_amdgcn_readfirstlane(coming[h][0]),
                     (uint32_t)__builtin_amdgcn_readfirstlane(coming[h][1]),
                     (uint32_t)__builtin_amdgcn_readfirstlane(coming[h][2]),
                     (uint32_t)__builtin_amdgcn_readfirstlane(coming[h][3])};
  };
  auto issue_runs = [&](const void* pool, uint32_t off, const TileRun (&u)[2], uint16_t* buf)
                        __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::kDma; ++i) {
      const int mi = i * (kQThreads / kWave) + wave_u;
      const bool second = D == 64 ? wave_u >= 4 : i == 1;
      const TileRun& x = second ? u[1] : u[0];
      const __amdgpu_buffer_rsrc_t rs =
          q_rsrc(static_cast<const char*>(pool) + ((uint64_t)(x.off_hi & 0xFFFF) << 32 | x.off), x.bytes);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(buf + 512 * mi), 16,
                                               off - x.lo() * C::kRowBytes, 0, 0, 0);
    }
  };
  auto issue = [&](const char* base, uint32_t off, int64_t kt, uint16_t* buf) __attribute__((always_inline)) {
    const int64_t left = k_hi - kt;
    const uint32_t nk = (uint32_t)(left <= 0 ? 0 : (left < kQKeys ? left : kQKeys));
    const __amdgpu_buffer_rsrc_t rs = q_rsrc(base + kt * C::kRowBytes, nk * C::kRowBytes);
#pragma unroll
    for (int i = 0; i < C::kDma; ++i) {
      const int mi = i * (kQThreads / kWave) + wave_u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(buf + 512 * mi), 16, off,
                                               1024 * (kQThreads / kWave) * i, 0, 0);
    }
  };

  // Scores S^T = K Q^T of half h (keys 32h .. 32h + 31) of the tile in kb:
  // lane (n16, kg) reads K row 16j + n16, chunk 4u + kg, i.e. chunk index
  // (j * kRowChunks + 4u + kg) * 16 + n16 = lane + 16 (j kRowChunks + 4u).
  // Four independent accumulation chains (two key blocks x two row groups).
  auto qk = [&](const uint16_t* kb, int h, float (&sc)[kRG][2][4]) __attribute__((always_inline)) {
    f32x4 acc[2][kRG];
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int q = 0; q < kRG; ++q) acc[jj][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < C::kChunks; ++u)
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const int j = 2 * h + jj;
        const u32x4 a = *reinterpret_cast<const u32x4*>(&kb[8 * (lane + 16 * (j * C::kRowChunks + 4 * u))]);
#pragma unroll
        for (int q = 0; q < kRG; ++q)
          acc[jj][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                               __builtin_bit_cast(bf16x8, qb[q][u]), acc[jj][q], 0, 0, 0);
      }
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
#pragma unroll
      for (int q = 0; q < kRG; ++q)
#pragma unroll
        for (int v = 0; v < 4; ++v) sc[q][jj][v] = acc[jj][q][v];
  };

  // Online softmax of a half whose first key is kh: the raw scores become
  // the probabilities 2^(c s - m), m and l move on.  The reference max m is
  // lazy: it moves only when a half's max exceeds it by more than kLazy (log2
  // units), so probabilities stay below 2^kLazy.  One of a row's four lanes
  // sees that by itself, so the row max across lanes, the factors and the
  // rescale of m, l and the accumulators (output rows of a lane are queries
  // 4kg + v of the group: their factors live in the lanes of those rows) run
  // only in waves where some lane does: 256 tokens of an 8B layer at 128K
  // 259.4 -> 253.0 us a call, at 32K 99.9 -> 96.6 (medians of 20 turns, which
  // spread by 1 to 2 us on either side; taking the bf16 remainders by dot products
  // as well, 16 instructions fewer per half, gave nothing: the kernel runs at the
  // power limit).
  const int32_t pos_all = PAGED ? paged_pos(blk, min(qt * kQRows + wave_rows * wave_u, rows - 1) / p.G) + 1 : 0;
  auto softmax = [&](auto masked, auto rgs, float (&sc)[kRG][2][4], int64_t kh, const TileRun& u) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      // slots outside the entry, or past the position of one of the wave's rows
      if (!u.whole() || (int32_t)u.pos + kRun > pos_all) {
        asm volatile("");  // keeps this a branch: the selects would run for every half
#pragma unroll
        for (int q = 0; q < decltype(rgs)::value; ++q) {
          const int32_t see = cut[q] - (int32_t)u.pos, last = (int32_t)u.hi(), lim = see < last ? see : last;
#pragma unroll
          for (int jj = 0; jj < 2; ++jj)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const int key = 16 * jj + 4 * kg + v;
              if (key >= lim || key < (int32_t)u.lo()) sc[q][jj][v] = -INFINITY;
            }
        }
      }
    }
#pragma unroll
    for (int q = 0; q < decltype(rgs)::value; ++q) {
      // keys past a row's causal limit or past the range: only in the
      // halves that reach min over rows of that limit
      if (!PAGED && decltype(masked)::value && kh + 32 > all_see) {
        const int32_t lim = cut[q] - (int32_t)(kh - k_lo);  // keys [0, lim) of this half count
#pragma unroll
        for (int jj = 0; jj < 2; ++jj)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (16 * jj + 4 * kg + v >= lim) sc[q][jj][v] = -INFINITY;
      }
      float mx = sc[q][0][0];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int v = 0; v < 4; ++v) mx = fmaxf(mx, sc[q][jj][v]);
      mx *= cpos;
      if (__builtin_amdgcn_ballot_w64(mx > m[q] + kLazy)) {
        mx = row4_max(mx);
        const bool grow = mx > m[q] + kLazy;
        const float alpha = fast_exp2(grow ? m[q] - mx : 0.f);
        m[q] = grow ? mx : m[q];
        l[q] *= alpha;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float av = __shfl(alpha, 4 * kg + v, 64);
#pragma unroll
          for (int b = 0; b < C::kBlocks; ++b) o[q][b][v] *= av;
        }
      }
      const float m_use = m[q] == -INFINITY ? 0.f : m[q];
      float ps = 0.f;
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          sc[q][jj][v] = fast_exp2(__builtin_fmaf(sc[q][jj][v], cpos, -m_use));
          ps += sc[q][jj][v];
        }
      l[q] += ps;
      // an empty operand barrier: the sum is formed here, in the vector
      // phase, instead of being sunk into a later one (which unbalances the
      // phases and keeps the probabilities alive across them)
      asm volatile("" : "+v"(l[q]));
    }
  };

  // Probabilities of a half as the A operand of P V: K slot e of lane group
  // kg is key 4kg + e (e < 4) or 16 + 4kg + (e - 4) of the half, the lane's
  // scores of its two 16-key blocks; high part and remainder.
  auto split = [&](auto rgs, const float (&sc)[kRG][2][4], u32x4 (&pp)[kParts][kRG]) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < decltype(rgs)::value; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t x[kParts];
        if constexpr (PAGED) bf16_parts(sc[q][e >> 1][2 * (e & 1)], sc[q][e >> 1][2 * (e & 1) + 1], x);
        else bf16_split(sc[q][e >> 1][2 * (e & 1)], sc[q][e >> 1][2 * (e & 1) + 1], x[0], x[1]);
#pragma unroll
        for (int part = 0; part < kParts; ++part) pp[part][q][e] = x[part];
      }
  };

  // O += P V over half h of the tile whose V is in vb; each V fragment
  // serves both row groups.  Transpose-read addresses: lane 4r + q of group
  // kg reads row R = 32h + 4kg + r (and R + 16), columns 16b + 4q .. +3, i.e.
  // chunk c = 2b + q / 2, half q % 2: chunk index
  // ((4h + kg / 2) * kRowChunks / 2 + b) * 16 + (4 (kg % 2) + r) * 2 + q / 2.
  // Two V blocks at a time: the high parts of both, then the remainders, so
  // a product never waits for the one just before it.
  auto pv = [&](auto rgs, const uint16_t* vb, int h, const u32x4 (&pp)[kParts][kRG]) __attribute__((always_inline)) {
    const uint16_t* vr0 = &vb[8 * ((4 * h + (kg >> 1)) * (C::kRowChunks / 2) * 16 + (4 * (kg & 1) + (n16 >> 2)) * 2 +
                                   ((n16 >> 1) & 1)) + 4 * (n16 & 1)];
#pragma unroll
    for (int b0 = 0; b0 < C::kBlocks; b0 += 2) {
      u32x4 vbo[2];
#pragma unroll
      for (int bb = 0; bb < 2; ++bb) {
        const int b = b0 + bb;
        const s16x4 t0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vr0 + 8 * 16 * b));
        const s16x4 t1 =
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vr0 + 8 * 16 * (2 * (C::kRowChunks / 2) + b)));
        const uint2 w0 = __builtin_bit_cast(uint2, t0);
        const uint2 w1 = __builtin_bit_cast(uint2, t1);
        vbo[bb] = u32x4{w0.x, w0.y, w1.x, w1.y};
      }
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int bb = 0; bb < 2; ++bb)
#pragma unroll
          for (int q = 0; q < decltype(rgs)::value; ++q) {
            const int b = b0 + bb;
            f32x4 c = {o[q][b][0], o[q][b][1], o[q][b][2], o[q][b][3]};
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pp[part][q]),
                                                        __builtin_bit_cast(bf16x8, vbo[bb]), c, 0, 0, 0);
            o[q][b][0] = c[0];
            o[q][b][1] = c[1];
            o[q][b][2] = c[2];
            o[q][b][3] = c[3];
          }
    }
  };

  // Paged: the products of a phase as one pipeline, every LDS read two groups
  // of products ahead of its use, so that the matrix unit does not wait for
  // one: O += P V of half hv (two V blocks at a time), then the scores of half
  // hk of the tile in kb.  The fences keep the compiler from gathering the
  // reads in front of their uses again.
  auto products = [&](auto rgs, const uint16_t* kb, int hk, const uint16_t* vb, int hv, bool do_pv, bool do_qk,
                      const u32x4 (&pp)[kParts][kRG], float (&sc)[kRG][2][4]) __attribute__((always_inline)) {
    constexpr int NP = C::kBlocks / 2;  // pairs of V blocks
    const uint16_t* vr0 = &vb[8 * ((4 * hv + (kg >> 1)) * (C::kRowChunks / 2) * 16 + (4 * (kg & 1) + (n16 >> 2)) * 2 +
                                   ((n16 >> 1) & 1)) + 4 * (n16 & 1)];
    auto read_v = [&](int b) __attribute__((always_inline)) {
      const uint2 w0 = __builtin_bit_cast(
          uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vr0 + 8 * 16 * b)));
      const uint2 w1 = __builtin_bit_cast(
          uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vr0 + 8 * 16 * (2 * (C::kRowChunks / 2) + b))));
      return u32x4{w0.x, w0.y, w1.x, w1.y};
    };
    auto read_k = [&](int jj, int u) __attribute__((always_inline)) {
      return *reinterpret_cast<const u32x4*>(&kb[8 * (lane + 16 * ((2 * hk + jj) * C::kRowChunks + 4 * u))]);
    };
    u32x4 vf[2][2], kf[C::kChunks][2];
    if (do_pv) {
#pragma unroll
      for (int n = 0; n < 2; ++n) vf[n][0] = read_v(2 * n), vf[n][1] = read_v(2 * n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < NP; ++n) {
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int bb = 0; bb < 2; ++bb)
#pragma unroll
            for (int q = 0; q < decltype(rgs)::value; ++q) {
              const int b = 2 * n + bb;
              f32x4 c = {o[q][b][0], o[q][b][1], o[q][b][2], o[q][b][3]};
              c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pp[part][q]),
                                                          __builtin_bit_cast(bf16x8, vf[n % 2][bb]), c, 0, 0, 0);
              o[q][b][0] = c[0];
              o[q][b][1] = c[1];
              o[q][b][2] = c[2];
              o[q][b][3] = c[3];
            }
        __builtin_amdgcn_sched_barrier(0);
        if (n + 2 < NP) {
          vf[n % 2][0] = read_v(2 * n + 4), vf[n % 2][1] = read_v(2 * n + 5);
        } else if (do_qk) {
          kf[n + 2 - NP][0] = read_k(0, n + 2 - NP), kf[n + 2 - NP][1] = read_k(1, n + 2 - NP);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) kf[u][0] = read_k(0, u), kf[u][1] = read_k(1, u);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (do_qk) {
#pragma unroll
      for (int u = 2; u < C::kChunks; ++u) kf[u][0] = read_k(0, u), kf[u][1] = read_k(1, u);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 acc[2][kRG];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int q = 0; q < decltype(rgs)::value; ++q) acc[jj][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < C::kChunks; ++u)
#pragma unroll
        for (int jj = 0; jj < 2; ++jj)
#pragma unroll
          for (int q = 0; q < decltype(rgs)::value; ++q)
            acc[jj][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[u][jj]),
                                                                 __builtin_bit_cast(bf16x8, qb[q][u]), acc[jj][q], 0, 0, 0);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int q = 0; q < decltype(rgs)::value; ++q)
#pragma unroll
          for (int v = 0; v < 4; ++v) sc[q][jj][v] = acc[jj][q][v];
    }
  };

  // Ping-pong over 32-key halves.  Each wave alternates a product phase
  // (P V products of half g, then score products of half g + 1) with a
  // vector phase (softmax, rescale and bf16 split of half g + 1), and the
  // waves meet after every phase.  Waves w and w + 4 share a SIMD (waves are
  // dealt to the four SIMDs in turn); waves 0-3 (lead) run one phase ahead
  // of waves 4-7 (follow), so on every SIMD one wave issues matrix products
  // while the other does vector work, and the product wave runs at raised
  // priority.  A meeting is a bare s_barrier that nothing is scheduled
  // across: LDS reads of a phase are consumed by its own products before the
  // meeting, and tile loads are made visible by each wave's own vmcnt wait
  // before the meeting that precedes their first reader (a workgroup fence
  // here would wait for every direct load in flight, including the tile
  // just issued).
  auto meet = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_barrier();
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_sched_barrier(0);
  };
  uint16_t* const kbuf[2] = {k0, k1};
  uint16_t* const vbuf[2] = {v0, v1};
  const bool lead = __builtin_amdgcn_readfirstlane(wave < 4 ? 1 : 0) != 0;
  float sc[kRG][2][4];
  u32x4 pp[kParts][kRG];
  constexpr int kWaitOne = 0x0F70 | C::kDma;  // vmcnt(kDma): the younger of two tiles may still be in flight
  auto vphase = [&](auto masked, auto rgs, int64_t kh, const TileRun& u) __attribute__((always_inline)) {
    softmax(masked, rgs, sc, kh, u);
    split(rgs, sc, pp);
    if constexpr (PAGED) {
      // the parts are formed here, not sunk into the product phase
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int q = 0; q < decltype(rgs)::value; ++q) asm volatile("" : "+v"(pp[part][q]));
    }
  };
  // P V first: the probabilities are dead before the new scores are formed
  auto mphase = [&](auto rgs, const uint16_t* kb, int hk, const uint16_t* vb, int hv, bool do_pv) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);
    if constexpr (PAGED) {
      if (do_pv) products(rgs, kb, hk, vb, hv, true, true, pp, sc);
      else products(rgs, kb, hk, vb, hv, false, true, pp, sc);
    } else {
      if (do_pv) pv(rgs, vb, hv, pp);
      __builtin_amdgcn_sched_barrier(0);
      qk(kb, hk, sc);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  int32_t live = -1;  // paged: runs with slots, where they are known
  if constexpr (PAGED) {
    fill_table(k_lo);
    __syncthreads();
    if (item.gaps && k_hi - k_lo <= kTableRuns * kRun) {
      live = drop_gaps((int)((k_hi - k_lo + kRun - 1) / kRun));
      __syncthreads();
    }
    read_runs(0);
    take_runs(run[0]);
    read_runs(2);
    take_runs(run[1]);
    issue_runs(p.k, koff, run[0], kbuf[0]);
    issue_runs(p.v, voff, run[0], vbuf[0]);
    issue_runs(p.k, koff, run[1], kbuf[1]);
  } else {
    issue(kbase, koff, k_lo, kbuf[0]);
    issue(vbase, voff, k_lo, vbuf[0]);
    issue(kbase, koff, k_lo + kQKeys, kbuf[1]);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
  const int64_t ntile = PAGED && live >= 0 ? (live + 1) / 2 : (k_hi > k_lo ? (k_hi - k_lo + kQKeys - 1) / kQKeys : 0);
  const int64_t nround = q_uniform64((ntile + (PAGED ? 0 : 1)) / 2);
  const bool odd = PAGED && (ntile & 1) != 0;  // a last tile without a second
  int at = 4;  // paged: where the table holds the tile whose K is loaded next
  // pairs of tiles whose halves (up to 32 keys past the pair) all lie below
  // every row's limit need no masking
  const int64_t clear = all_see - k_lo - 5 * 32;
  int64_t nclear = !PAGED && clear >= 0 ? clear / (2 * kQKeys) + 1 : 0;
  nclear = q_uniform64(nclear < nround ? nclear : nround);
  int64_t kt = k_lo;
  // Tile t (K in kbuf[i], V in vbuf[i]) takes phases 4t + 1 .. 4t + 4.  K of
  // tile t is read in phases 4t .. 4t + 3 and V in 4t + 2 .. 4t + 5; V of
  // tile t + 1 is loaded from phase 4t + 2 on and K of tile t + 2 from
  // 4t + 4 on, each a whole tile before its first reader.  Each group runs
  // its own copy of the loop, so no phase branches on the group (a branch
  // gave the accumulators a second register set).  Both groups meet equally
  // often: every wave passes the same number of barriers.
  auto one_tile = [&](auto masked, auto leadc, auto rgs, auto par) __attribute__((always_inline)) {
    constexpr bool L = decltype(leadc)::value;
    constexpr int i = decltype(par)::value;  // tile t's parity
    // 4t + 1: lead: vector phase of half 2t; follow: P V of half 2t - 1, scores of 2t
    if (PAGED && L) read_runs(at);
    if (L) vphase(masked, rgs, kt, run[i][0]);
    else mphase(rgs, kbuf[i], 0, vbuf[1 - i], 1, i == 1 || kt != k_lo);
    if (PAGED && L) take_runs(ahead);
    __builtin_amdgcn_s_waitcnt(kWaitOne);  // V of tile t
    meet();
    // 4t + 2: lead: P V of 2t, scores of 2t + 1; follow: vector phase of 2t
    if constexpr (PAGED) issue_runs(p.v, voff, run[1 - i], vbuf[1 - i]);
    else issue(vbase, voff, kt + kQKeys, vbuf[1 - i]);
    if (PAGED && !L) read_runs(at);
    if (L) mphase(rgs, kbuf[i], 1, vbuf[i], 0, true);
    else vphase(masked, rgs, kt, run[i][0]);
    if (PAGED && !L) take_runs(ahead);
    meet();
    // 4t + 3: lead: vector phase of 2t + 1; follow: P V of 2t, scores of 2t + 1
    const TileRun second = run[i][1];
    if (L) vphase(masked, rgs, kt + 32, second);
    else mphase(rgs, kbuf[i], 1, vbuf[i], 0, true);
    __builtin_amdgcn_s_waitcnt(kWaitOne);  // K of tile t + 1
    meet();
    // 4t + 4: lead: P V of 2t + 1, scores of 2t + 2; follow: vector phase of 2t + 1
    if constexpr (PAGED) {
      run[i][0] = ahead[0];
      run[i][1] = ahead[1];
      issue_runs(p.k, koff, run[i], kbuf[i]);
      at += 2;
    } else {
      issue(kbase, koff, kt + 2 * kQKeys, kbuf[i]);
    }
    if (L) mphase(rgs, kbuf[1 - i], 0, vbuf[i], 1, true);
    else vphase(masked, rgs, kt + 32, second);
    meet();
    kt += kQKeys;
  };
  auto tile_pair = [&](auto masked, auto leadc, auto rgs) __attribute__((always_inline)) {
    one_tile(masked, leadc, rgs, std::integral_constant<int, 0>{});
    one_tile(masked, leadc, rgs, std::integral_constant<int, 1>{});
  };
  // Between two pairs of tiles nobody reads the table: the last reads were two
  // meetings ago.
  auto next_table = [&]() __attribute__((always_inline)) {
    fill_table(kt + 2 * kQKeys);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    meet();
    at = 0;
  };
  auto walk = [&](auto leadc, auto rgs) __attribute__((always_inline)) {
    constexpr bool L = decltype(leadc)::value;
    if (L) mphase(rgs, kbuf[0], 0, vbuf[0], 0, false);  // scores of half 0
    meet();
    if constexpr (!PAGED)
      for (int64_t rd = 0; rd < nclear; ++rd) tile_pair(std::false_type{}, leadc, rgs);
    for (int64_t rd = nclear; rd < nround; ++rd) {
      if (PAGED && at + 4 > kTableRuns) next_table();
      tile_pair(std::true_type{}, leadc, rgs);
    }
    if (PAGED && odd) {
      one_tile(std::true_type{}, leadc, rgs, std::integral_constant<int, 0>{});
      if (!L) pv(rgs, vbuf[0], 1, pp);
      return;
    }
    // the follow group's P V products of the last half (tiles past k_hi hold
    // zeros and all their keys are masked, so the lead's last scores are unused)
    if (!L && nround > 0) pv(rgs, vbuf[1], 1, pp);
  };
  // Paged: waves without rows (a sequence of few tokens) load and meet only;
  // the others then have the matrix units and the power to themselves.
  auto attend_none = [&]() __attribute__((always_inline)) {
    meet();
    auto none = [&](auto par) __attribute__((always_inline)) {
      constexpr int i = decltype(par)::value;
      __builtin_amdgcn_s_waitcnt(kWaitOne);
      meet();
      issue_runs(p.v, voff, run[1 - i], vbuf[1 - i]);
      read_runs(at);
      take_runs(run[i]);
      at += 2;
      meet();
      __builtin_amdgcn_s_waitcnt(kWaitOne);
      meet();
      issue_runs(p.k, koff, run[i], kbuf[i]);
      meet();
      kt += kQKeys;
    };
    for (int64_t rd = 0; rd < nround; ++rd) {
      if (at + 4 > kTableRuns) next_table();
      none(std::integral_constant<int, 0>{});
      none(std::integral_constant<int, 1>{});
    }
    if (odd) none(std::integral_constant<int, 0>{});
  };
  if (PAGED && qt * kQRows + wave_rows * wave_u >= rows) attend_none();
  else if (spread && lead) walk(std::true_type{}, std::integral_constant<int, 1>{});
  else if (spread) walk(std::false_type{}, std::integral_constant<int, 1>{});
  else if (lead) walk(std::true_type{}, std::integral_constant<int, kRG>{});
  else walk(std::false_type{}, std::integral_constant<int, kRG>{});
  // no direct load may still be writing LDS when the workgroup ends
  __builtin_amdgcn_s_waitcnt(0x0F70);

  // ---- row totals; write the output or this range's record ------------------
  float* rec = item.rec;
#pragma unroll
  for (int q = 0; q < kRG; ++q) {
    l[q] = lane_xor_sum<16>(l[q]);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int rr = wave * wave_rows + 16 * q + 4 * kg + v;  // row within the tile
      const int rq = qt * kQRows + rr;
      const float lq = __shfl(l[q], 4 * kg + v, 64);
      const float mq = __shfl(m[q], 4 * kg + v, 64);
      if (rq < rows && 16 * q < wave_rows) {
        if (item.single) {
          const int tq = rq / p.G;
          float* orow = p.out + ((tok_row0 + tq) * p.Hq + (int64_t)g * p.G + (rq - tq * p.G)) * D;
          const float inv = lq > 0.f ? 1.f / lq : 0.f;
#pragma unroll
          for (int b = 0; b < C::kBlocks; ++b) orow[16 * b + n16] = o[q][b][v] * inv;
        } else {
          float* rrow = rec + (int64_t)rr * C::kRec;
          if (n16 == 0) {
            rrow[0] = mq;
            rrow[1] = lq;
          }
#pragma unroll
          for (int b = 0; b < C::kBlocks; ++b) rrow[2 + 16 * b + n16] = o[q][b][v];
        }
      }
    }
  }
}

// Two tile buffers per matrix (separate arrays: the compiler then tells the
// direct loads into one apart from the reads of the other).
#define DKV_QUERY_TILES(D)                                          \
  __shared__ __align__(1024) uint16_t k0[kQKeys * D], k1[kQKeys * D]; \
  __shared__ __align__(1024) uint16_t v0[kQKeys * D], v1[kQKeys * D]

template <int D>
__global__ __launch_bounds__(kQThreads) void query_attn_kernel(QueryParams p) {
  DKV_QUERY_TILES(D);
  // ---- this workgroup's item: segment, query tile, key tiles ---------------
  int item, s, qt;
  bool single;             // the segment has one range: write the output
  int64_t t_lo, t_hi;      // key tiles [t_lo, t_hi) of the range
  if (p.plan == nullptr) {
    item = blockIdx.x;
    s = item / p.qtiles;
    qt = item - s * p.qtiles;
    single = true;
    t_lo = 0;
    t_hi = seg_tiles(p, s);
  } else {
    // the grid is a multiple of 8 and at least the items, so every item
    // i = x * per + y (x < 8, y < per) has its workgroup 8y + x
    const int total = p.plan[0];
    const int per = (total + 7) / 8;  // items per L2 domain
    const int b = blockIdx.x;
    if (b / 8 >= per) return;
    item = (b % 8) * per + b / 8;
    if (item >= total) return;
    // the segment: the last s with first item <= item
    int lo = 0, hi = p.nseg;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.plan[kQueryPlanHead + mid] <= item) lo = mid;
      else hi = mid;
    }
    s = lo;
    const int first = p.plan[kQueryPlanHead + s];
    const int nr = (p.plan[kQueryPlanHead + s + 1] - first) / p.qtiles;
    const int r = (item - first) / p.qtiles;
    qt = item - first - r * p.qtiles;
    single = nr == 1;
    const int64_t tiles = seg_tiles(p, s);
    t_lo = (int64_t)r * tiles / nr;
    t_hi = (int64_t)(r + 1) * tiles / nr;
  }
  query_item<D, false>(p, QueryItem{s, qt, t_lo, t_hi, single, p.rec + (int64_t)item * kQRows * QCfg<D>::kRec,
                                    PagedBlock{0, 0, 0}, 0, false}, k0, k1, v0, v1, nullptr, nullptr);
}

// ---------------------------------------------------------------------------
// Paged calls.  A unit is one query tile of one segment (of a sequence's own
// number of them); its length is the cost of its key tiles (up to what its last
// row sees) and kUnitTiles more for what it takes by itself.  A tile costs
// kThinCost with up to 64 rows (one row group in each lead wave), kHalfCost with
// up to 128 (one in every wave), and else kTileCost: 32 sequences of 8,000 keys, 8
// heads, walked at 1.55 us a tile with 4 to 32 rows, 1.75 with 64, 2.2 with 96, 2.4
// with 128, 3.1 with 160, 3.7 with 256.
// The lengths of all units, laid end to end, are cut into P equal slices (up to
// the next whole tile), one per workgroup: however unequal the chunks and the
// contexts, every workgroup has the same work and all run at once.  A unit that
// lies in one slice is written directly.  A slice holds at
// most two parts of others, the rest of the unit it starts in (record slot 2w)
// and the head of the unit it ends in (2w + 1; a unit that starts with the
// slice is in slot 2w), and a combine kernel folds a unit's records in slice
// order.  Consecutive slices, which share keys, go to the same L2 domain.
//
// Prompts have many units, none longer than a slice.  There the plan deals the
// units by falling length, P at a time, the longest of a round to the workgroup
// with the least so far: when the longest share is at most kWholeTiles above
// the mean, units stay whole and no record is written (us, whole / slices, 32
// query heads on 8: two prompts of 4,096 tokens 436 / 490, eight of 1,500 304 / 324,
// of 1,000 162 / 174).  Not for units of fewer than kWholeMean tiles on average:
// a slice's many small units read the same keys, one after another (16 prompts of
// 700 207 / 188, 32 of 512 241 / 224).
// ---------------------------------------------------------------------------
constexpr int kUnitTiles = 2;
constexpr int kTileCost = 4, kHalfCost = 3, kThinCost = 2;
constexpr int kWholeTiles = 10, kWholeMean = 8;
constexpr int kSortBuckets = 1024;

struct PagedUnit {
  int32_t s, qt;
  int32_t rows;  // of the segment, up to the last that the tile sees
  int32_t cost;  // of a key tile
  PagedBlock blk;
  int32_t gaps;
};

// Words of the plan: slices and units, whether units stay whole,
// each slice's first unit and where it starts, the units that several slices
// share, what each unit is, where it starts, and for whole units the workgroups' units,
// round by round (-1: none).
struct PagedShared {
  int32_t slot, parts;  // slot of the first record, records (the others at slots 2w of the next slices)
  int32_t s, qt, tok0, rows, pad[2];
};

struct PagedPlan {
  int32_t* head;        // [4]: P, units, whole, shared units
  int32_t* first;       // [kPagedSlices] unit that holds the slice's start
  int64_t* cut;         // [kPagedSlices + 2] where each slice starts, the last one's end
  PagedShared* shared;  // [kPagedSlices]
  PagedUnit* unit;      // [units]
  int64_t* start;       // [units + 1]
  int32_t* order;       // [units, rounded up to rounds of kPagedSlices]
};

constexpr int kPagedPlanHead = 8;  // words before `first`

__host__ __device__ __forceinline__ PagedPlan paged_plan_of(int32_t* words, int64_t units) {
  PagedPlan x;
  x.head = words;
  x.first = words + kPagedPlanHead;
  x.cut = reinterpret_cast<int64_t*>(x.first + kPagedSlices);
  x.shared = reinterpret_cast<PagedShared*>(x.cut + kPagedSlices + 2);
  x.unit = reinterpret_cast<PagedUnit*>(x.shared + kPagedSlices);
  x.start = reinterpret_cast<int64_t*>(x.unit + units);
  x.order = reinterpret_cast<int32_t*>(x.start + units + 1);
  return x;
}

size_t paged_plan_bytes(int64_t units) {
  return (sizeof(int32_t) * (kPagedPlanHead + 2 * kPagedSlices + units) + sizeof(PagedShared) * kPagedSlices +
          sizeof(PagedUnit) * units + sizeof(int64_t) * (kPagedSlices + units + 3) + 255) / 256 * 256;
}

__device__ __forceinline__ int64_t unit_tiles(int32_t rows) {
  return ((int64_t)rows + kQKeys - 1) / kQKeys;
}

// Rows of segment s that query tile qt of a block sees.
__device__ __forceinline__ int32_t unit_rows(const QueryParams& p, const PagedBlock& k, int s, int qt, bool* gaps) {
  *gaps = false;
  if (k.pos0 < 0 || p.max_entries == 0) return 0;
  const int64_t last = (int64_t)(qt + 1) * kQRows < (int64_t)k.n * p.G ? (int64_t)(qt + 1) * kQRows : (int64_t)k.n * p.G;
  return paged_rows(p, s, paged_pos(k, (int32_t)((last - 1) / p.G)), gaps);
}

// One workgroup; bound by the chain of its dependent reads (offsets, counts)
// and scans, so what later steps read again stays in LDS.
constexpr int kPlanUnits = 4096;  // units whose starts fit LDS
constexpr int kWholeRounds = 32;  // rounds of whole units at most

__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(QueryParams p) {
  __shared__ int64_t red[3][kPlanThreads / kWave];
  __shared__ int32_t pre[DKV_MAX_SEGMENTS + 1];  // query tiles of the sequences before
  __shared__ PagedBlock blk[DKV_MAX_SEGMENTS];
  __shared__ int64_t start[kPlanUnits + 1];
  __shared__ int64_t cut[kPagedSlices + 1];
  __shared__ int32_t bucket[kSortBuckets];       // whole units: units per length, then where they go
  __shared__ int32_t size[kSortBuckets];         // the longest of each bucket
  __shared__ int32_t order[kPlanUnits];
  __shared__ __align__(16) int32_t load[kPagedSlices];
  static_assert(kPlanThreads == 4 * kPagedSlices, "four threads rank a workgroup's load");
  __shared__ int32_t longest, share, nshared;
  const int tid = threadIdx.x;
  const int B = p.nseg / p.Hkv;
  const PagedPlan plan = paged_plan_of(p.plan, p.max_items);
  int64_t base = 0;
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int64_t tiles = 0, sum;
    if (b < B) {
      const PagedBlock k = paged_block(p, b);
      blk[b] = k;
      tiles = ((int64_t)k.n * p.G + kQRows - 1) / kQRows;
    }
    if (b0 > 0) __syncthreads();
    const int64_t ex = block_scan<kPlanThreads>(tiles, red[0], &sum);
    if (b < B) pre[b] = (int32_t)(base + ex);
    base += sum;
  }
  if (tid == 0) {
    pre[B] = (int32_t)base;
    longest = share = nshared = 0;
  }
  __syncthreads();
  // offsets that overlap could name more units than the workspace holds
  const int64_t units = base * p.Hkv < p.max_items ? base * p.Hkv : p.max_items;
  const bool near = units <= kPlanUnits;
  int64_t len = 0;
  int32_t most = 0;
  for (int64_t u0 = 0; u0 < units; u0 += kPlanThreads) {
    const int64_t u = u0 + tid;
    int64_t mine = 0, sum;
    if (u < units) {
      int lo = 0, hi = B;  // the last sequence whose units start at or before u, and which has any
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)pre[mid] * p.Hkv <= u) lo = mid;
        else hi = mid;
      }
      const int tiles = pre[lo + 1] - pre[lo];
      const int in = (int)(u - (int64_t)pre[lo] * p.Hkv);
      const int g = in / tiles, qt = in - g * tiles;
      const int s = lo * p.Hkv + g;
      bool gaps;
      const int32_t rows = unit_rows(p, blk[lo], s, qt, &gaps);
      const int64_t left = (int64_t)blk[lo].n * p.G - (int64_t)qt * kQRows;
      const int32_t cost = left <= 64 ? kThinCost : (left <= kQRows / 2 ? kHalfCost : kTileCost);
      plan.unit[u] = PagedUnit{s, qt, rows, cost, blk[lo], gaps};
      mine = (unit_tiles(rows) + kUnitTiles) * cost;  // below 2^27
      most = max(most, (int32_t)mine);
    }
    if (u0 > 0) __syncthreads();
    const int64_t ex = block_scan<kPlanThreads>(mine, red[1], &sum);
    if (u < units) {
      plan.start[u] = len + ex;
      if (near) start[u] = len + ex;
    }
    len += sum;
  }
  // slices of two tiles at least, so that each has its own start
  const int64_t most_slices = len == 0 ? 0 : (len < 4 * kTileCost ? 1 : len / (2 * kTileCost));
  const int64_t P = most_slices < p.P ? most_slices : p.P;
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, kWave));
  if ((tid & (kWave - 1)) == 0) atomicMax(&longest, most);
  if (tid == 0) {
    plan.start[units] = len;
    if (near) start[units] = len;
    plan.head[0] = (int32_t)P;
    plan.head[1] = (int32_t)units;
  }
  __syncthreads();
  bool whole = near && units > P && len <= INT32_MAX && longest <= len / p.P &&
               units <= (int64_t)kWholeRounds * p.P && len >= units * (kWholeMean + kUnitTiles) * kTileCost;
  if (whole) {
    const int rounds = (int)((units + p.P - 1) / p.P);
    for (int i = tid; i < kSortBuckets; i += kPlanThreads) bucket[i] = size[i] = 0;
    if (tid < kPagedSlices) load[tid] = tid < p.P ? 0 : INT32_MAX;
    __syncthreads();
    // A counting sort.  Units of one bucket stand in the order of arrival, so
    // each counts as the bucket's longest: the shares, and whether units stay
    // whole, then depend on the lengths alone (counted by their own lengths, two
    // prompts of some 2,000 tokens after 66,000 each had a longest share of 8,468
    // or 8,472 by the order, against a limit of 8,471).  A bucket is at most a
    // thousandth of the longest unit wide, and one length up to 1,023.
    const float scale = (float)(kSortBuckets - 1) / (float)longest;
    auto bucket_of = [&](int64_t u) {
      const int b = (int)((float)(longest - (int32_t)(start[u + 1] - start[u])) * scale);
      return b < kSortBuckets ? b : kSortBuckets - 1;
    };
    for (int u = tid; u < units; u += kPlanThreads) {
      const int b = bucket_of(u);
      atomicAdd(&bucket[b], 1);
      atomicMax(&size[b], (int32_t)(start[u + 1] - start[u]));
    }
    __syncthreads();
    int64_t sum;
    const int64_t ex = block_scan<kPlanThreads>(tid < kSortBuckets ? bucket[tid] : 0, red[2], &sum);
    if (tid < kSortBuckets) bucket[tid] = (int32_t)ex;
    __syncthreads();
    for (int u = tid; u < units; u += kPlanThreads) order[atomicAdd(&bucket[bucket_of(u)], 1)] = u;
    __syncthreads();
    const int mine_of = tid / 4;  // the workgroup that this thread ranks, with its three neighbours
    for (int r = 0; r < rounds; ++r) {
      const int32_t mine = load[mine_of];
      // workgroups with less so far (or as much, and before this one): none in
      // the first round, all behind it in the second
      int rank = r == 0 ? mine_of : p.P - 1 - mine_of;
      if (r > 1) {
        rank = 0;
#pragma unroll
        for (int k = 0; k < kPagedSlices / 4; k += 4) {
          const int j = (tid & 3) * (kPagedSlices / 4) + k;
          const int4 x = *reinterpret_cast<const int4*>(&load[j]);
          rank += (x.x < mine || (x.x == mine && j < mine_of)) + (x.y < mine || (x.y == mine && j + 1 < mine_of)) +
                  (x.z < mine || (x.z == mine && j + 2 < mine_of)) + (x.w < mine || (x.w == mine && j + 3 < mine_of));
        }
        rank += __shfl_xor(rank, 1, kWave);
        rank += __shfl_xor(rank, 2, kWave);
      }
      const int i = r * p.P + rank;
      const int32_t unit = mine_of < p.P && i < units ? order[i] : -1;
      __syncthreads();
      if ((tid & 3) == 0 && mine_of < p.P) {
        if (unit >= 0) load[mine_of] = mine + size[bucket_of(unit)];
        plan.order[r * p.P + mine_of] = unit;
      }
      __syncthreads();
    }
    int32_t top = tid < p.P ? load[tid] : 0;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) top = max(top, __shfl_xor(top, o, kWave));
    if (tid < kPagedSlices && (tid & (kWave - 1)) == 0) atomicMax(&share, top);
    __syncthreads();
    whole = share <= len / p.P + kWholeTiles * kTileCost;
  }
  if (tid == 0) plan.head[2] = whole ? 1 : 0, plan.head[3] = 0;
  if (whole) return;
  int64_t x = 0, lo = 0, from = 0;  // this thread's slice: its start, the unit there, that unit's first tile
  PagedUnit u{};
  if (tid < P) {
    x = (int64_t)tid * len / P;
    int64_t hi = units;
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) >> 1;
      if ((near ? start[mid] : plan.start[mid]) <= x) lo = mid;
      else hi = mid;
    }
    u = plan.unit[lo];
    from = (near ? start[lo] : plan.start[lo]) + kUnitTiles * u.cost;
    if (x > from) x = from + (x - from + u.cost - 1) / u.cost * u.cost;
    cut[tid] = x;
    plan.first[tid] = (int32_t)lo;
    plan.cut[tid] = x;
  }
  if (tid == 0) plan.cut[P] = len;
  __syncthreads();
  if (tid > 0 && tid < P) {
    // the unit that this slice continues, by the first slice to do so
    const int64_t end = near ? start[lo + 1] : plan.start[lo + 1];
    const int64_t before = cut[tid - 1];
    if (from < x && x < end && from >= before) {
      int64_t last = owner_of(end - 1, len, P);
      if (cut[last] >= end) --last;
      const int i = atomicAdd(&nshared, 1);
      plan.shared[i] = PagedShared{2 * (tid - 1) + (from > before ? 1 : 0), (int)last - tid + 2, u.s, u.qt, u.blk.tok0,
                                   u.blk.n * p.G, {0, 0}};
    }
  }
  __syncthreads();
  if (tid == 0) plan.head[3] = nshared;
}

template <int D>
__global__ __launch_bounds__(kQThreads) void paged_query_kernel(QueryParams p) {
  DKV_QUERY_TILES(D);
  __shared__ __align__(16) u32x4 table[kTableRuns + kTablePad];
  __shared__ int counts[2 * kQThreads / kWave];  // runs with slots, per wave
  __shared__ PagedUnit own[kWholeRounds];  // whole units: this workgroup's
  // Without a plan (too few keys to split) one workgroup per (segment, query
  // tile): the loop's only unit.
  const bool split = p.plan != nullptr;
  const PagedPlan plan = paged_plan_of(p.plan, p.max_items);
  int w = blockIdx.x, u = 0, units = 1, rounds = 0;
  int64_t lo = 0, hi = 0;
  bool whole = false;
  if (split) {
    units = __builtin_amdgcn_readfirstlane(plan.head[1]);
    whole = __builtin_amdgcn_readfirstlane(plan.head[2]) != 0;
    if (whole) {
      rounds = (units + (int)gridDim.x - 1) / (int)gridDim.x;
      for (int i = threadIdx.x; i < rounds; i += kQThreads) {
        const int v = plan.order[i * gridDim.x + w];
        if (v >= 0) own[i] = plan.unit[v];
        else own[i].s = -1;
      }
      __syncthreads();
    } else {
      const int P = __builtin_amdgcn_readfirstlane(plan.head[0]);
      w = (blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;  // the grid is a multiple of 8
      if (w >= P) return;
      lo = q_uniform64(plan.cut[w]);
      hi = q_uniform64(plan.cut[w + 1]);
      u = __builtin_amdgcn_readfirstlane(plan.first[w]);
    }
  }
  for (int r = 0;; ++r, ++u) {
    QueryItem x;
    if (whole) {
      if (r >= rounds) break;
      const PagedUnit unit = own[r];
      if (__builtin_amdgcn_readfirstlane(unit.s) < 0) continue;
      x.s = unit.s;
      x.qt = unit.qt;
      x.seen = unit.rows;
      x.gaps = __builtin_amdgcn_readfirstlane(unit.gaps) != 0;
      x.blk = unit.blk;
      x.t_lo = 0;
      x.t_hi = unit_tiles(unit.rows);
      x.single = true;
      x.rec = nullptr;
    } else if (split) {
      if (u >= units) break;
      const PagedUnit unit = plan.unit[u];
      const int64_t begin = q_uniform64(plan.start[u]), end = q_uniform64(plan.start[u + 1]);
      const int32_t cost = __builtin_amdgcn_readfirstlane(unit.cost);
      const int64_t from = begin + kUnitTiles * cost;  // the unit's first key tile
      if (begin >= hi) break;
      const bool empty = from == end;  // no keys: zeros, by the slice that holds its start
      const int64_t a = lo > from ? lo : from, b = hi < end ? hi : end;
      if (empty ? begin < lo : a >= b) continue;
      x.s = __builtin_amdgcn_readfirstlane(unit.s);
      x.qt = __builtin_amdgcn_readfirstlane(unit.qt);
      x.seen = __builtin_amdgcn_readfirstlane(unit.rows);
      x.gaps = __builtin_amdgcn_readfirstlane(unit.gaps) != 0;
      x.blk = unit.blk;
      x.t_lo = (uint32_t)(a - from) / (uint32_t)cost;  // below 2^27
      x.t_hi = (uint32_t)(b - from) / (uint32_t)cost;
      x.single = empty || (a == from && b == end);
      x.rec = p.rec + (int64_t)(2 * w + (from > lo ? 1 : 0)) * kQRows * QCfg<D>::kRec;
    } else {
      if (r > 0) break;
      x.s = __builtin_amdgcn_readfirstlane(blockIdx.x / p.qtiles);
      x.qt = blockIdx.x - x.s * p.qtiles;
      x.blk = paged_block(p, x.s / p.Hkv);
      if ((int64_t)x.qt * kQRows >= (int64_t)x.blk.n * p.G) return;
      bool gaps;
      x.seen = __builtin_amdgcn_readfirstlane(unit_rows(p, x.blk, x.s, x.qt, &gaps));
      x.gaps = __builtin_amdgcn_readfirstlane(gaps ? 1 : 0) != 0;
      x.t_lo = 0;
      x.t_hi = unit_tiles(x.seen);
      x.single = true;
      x.rec = nullptr;
    }
    query_item<D, true>(p, x, k0, k1, v0, v1, table, counts);
    __syncthreads();  // the tile buffers are free for the next unit
  }
}

// Combine kernel: thread item (row, 4 columns) of one (segment, query tile);
// kMergeThreads items per workgroup.  Segments with one range were written
// by the attention kernel.  A thread loads the row's max, sum and 4 columns
// from eight ranges at once (one memory round trip per eight), then folds
// them in range order into
//   M = max_k m_k,  out = sum_k 2^(m_k - M) o_k / sum_k 2^(m_k - M) l_k.
constexpr int kMergeThreads = 256;
constexpr int kMergeBatch = 8;

template <int D>
__global__ __launch_bounds__(kMergeThreads) void query_merge_kernel(QueryParams p) {
  using C = QCfg<D>;
  constexpr int kItems = kQRows * (D / 4);        // items per query tile
  constexpr int kParts = kItems / kMergeThreads;  // workgroups per query tile
  const int tile = blockIdx.x / kParts;           // s * qtiles + qt
  const int it = (blockIdx.x - tile * kParts) * kMergeThreads + threadIdx.x;
  const int s = tile / p.qtiles;
  const int qt = tile - s * p.qtiles;
  const int rr = it / (D / 4);
  const int c4 = it - rr * (D / 4);
  const int rq = qt * kQRows + rr;
  if (rq >= p.rows) return;
  const int first = p.plan[kQueryPlanHead + s];
  const int nr = (p.plan[kQueryPlanHead + s + 1] - first) / p.qtiles;
  if (nr <= 1) return;
  const int bseq = s / p.Hkv;
  const int g = s - bseq * p.Hkv;
  // record of range k: item first + k * qtiles + qt
  const float* recs = p.rec + ((int64_t)first + qt) * kQRows * C::kRec + (int64_t)rr * C::kRec;
  const int64_t stride = (int64_t)p.qtiles * kQRows * C::kRec;
  float M = -INFINITY, L = 0.f;
  f32x4 A = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < nr; k0 += kMergeBatch) {
    float mk[kMergeBatch], lk[kMergeBatch];
    f32x4 ak[kMergeBatch];
#pragma unroll
    for (int k = 0; k < kMergeBatch; ++k) {
      if (k0 + k < nr) {
        const float* r = recs + (int64_t)(k0 + k) * stride;
        mk[k] = r[0];
        lk[k] = r[1];
        ak[k] = *reinterpret_cast<const f32x4*>(r + 2 + 4 * c4);
      } else {
        mk[k] = -INFINITY;
        lk[k] = 0.f;
        ak[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    float Mn = M;
#pragma unroll
    for (int k = 0; k < kMergeBatch; ++k) Mn = fmaxf(Mn, mk[k]);
    const float Mu = Mn == -INFINITY ? 0.f : Mn;
    const float fo = fast_exp2(M - Mu);
    L *= fo;
    A *= fo;
#pragma unroll
    for (int k = 0; k < kMergeBatch; ++k) {
      const float f = fast_exp2(mk[k] - Mu);
      L += f * lk[k];
      A += f * ak[k];
    }
    M = Mn;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  const int tq = rq / p.G;
  float* orow = p.out + (((int64_t)bseq * p.n_q + tq) * p.Hq + (int64_t)g * p.G + (rq - tq * p.G)) * D;
  *reinterpret_cast<f32x4*>(orow + 4 * c4) = A * inv;
}

// Combine kernel of paged calls: kParts workgroups per unit that several slices
// share, as the plan lists them.
template <int D>
__global__ __launch_bounds__(kMergeThreads, 5) void paged_merge_kernel(QueryParams p) {
  using C = QCfg<D>;
  constexpr int kParts = kQRows * (D / 4) / kMergeThreads;
  const int i = blockIdx.x / kParts;
  const PagedPlan plan = paged_plan_of(p.plan, p.max_items);
  if (i >= plan.head[3]) return;
  const PagedShared x = plan.shared[i];
  const int nr = x.parts;
  const int it = (blockIdx.x - i * kParts) * kMergeThreads + threadIdx.x;
  const int rr = it / (D / 4);
  const int c4 = it - rr * (D / 4);
  const int rq = x.qt * kQRows + rr;
  if (rq >= x.rows) return;
  // record k: slot x.slot for the first, 2w of the slices after its own for the others
  constexpr int64_t kSlot = (int64_t)kQRows * C::kRec;
  const float* head = p.rec + x.slot * kSlot + (int64_t)rr * C::kRec;
  const float* recs = p.rec + (x.slot & ~1) * kSlot + (int64_t)rr * C::kRec;
  float M = -INFINITY, L = 0.f;
  f32x4 A = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < nr; k0 += kMergeBatch) {
    float mk[kMergeBatch], lk[kMergeBatch];
    f32x4 ak[kMergeBatch];
#pragma unroll
    for (int k = 0; k < kMergeBatch; ++k) {
      mk[k] = -INFINITY;
      lk[k] = 0.f;
      ak[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (k0 + k < nr) {
        const float* r = k0 + k == 0 ? head : recs + (k0 + k) * 2 * kSlot;
        mk[k] = r[0];
        lk[k] = r[1];
        ak[k] = *reinterpret_cast<const f32x4*>(r + 2 + 4 * c4);
      }
    }
    float Mn = M;
#pragma unroll
    for (int k = 0; k < kMergeBatch; ++k) Mn = fmaxf(Mn, mk[k]);
    const float Mu = Mn == -INFINITY ? 0.f : Mn;
    const float fo = fast_exp2(M - Mu);
    L *= fo;
    A *= fo;
#pragma unroll
    for (int k = 0; k < kMergeBatch; ++k) {
      const float f = fast_exp2(mk[k] - Mu);
      L += f * lk[k];
      A += f * ak[k];
    }
    M = Mn;
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  const int tq = rq / p.G;
  const int g = x.s % p.Hkv;
  float* orow = p.out + (((int64_t)x.tok0 + tq) * p.Hq + (int64_t)g * p.G + (rq - tq * p.G)) * D;
  *reinterpret_cast<f32x4*>(orow + 4 * c4) = A * inv;
}

template <int D>
hipError_t launch_paged_d(const QueryParams& p, hipStream_t stream) {
  if (p.plan == nullptr) {
    hipLaunchKernelGGL((paged_query_kernel<D>), dim3((unsigned)((int64_t)p.nseg * p.qtiles)), dim3(kQThreads), 0, stream,
                       p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, p);
  hipLaunchKernelGGL((paged_query_kernel<D>), dim3((unsigned)p.P), dim3(kQThreads), 0, stream, p);
  if (p.P > 1)
    hipLaunchKernelGGL((paged_merge_kernel<D>), dim3((unsigned)((p.P - 1) * (kQRows * (D / 4) / kMergeThreads))),
                       dim3(kMergeThreads), 0, stream, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const QueryParams& p, int64_t grid, hipStream_t stream) {
  if (p.plan != nullptr) hipLaunchKernelGGL(query_plan_kernel, dim3(1), dim3(kPlanThreads), 0, stream, p);
  hipLaunchKernelGGL((query_attn_kernel<D>), dim3((unsigned)grid), dim3(kQThreads), 0, stream, p);
  if (p.plan != nullptr) {
    const int64_t parts = (int64_t)kQRows * (D / 4) / kMergeThreads;
    hipLaunchKernelGGL((query_merge_kernel<D>), dim3((unsigned)((int64_t)p.nseg * p.qtiles * parts)),
                       dim3(kMergeThreads), 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace

QueryPlanShape query_plan_shape(int32_t nseg, int32_t rows, int32_t head_dim, int64_t rows_hint) {
  QueryPlanShape sh;
  sh.qtiles = (rows + kQRows - 1) / kQRows;
  const int64_t units = (int64_t)nseg * sh.qtiles;
  // key tiles of all segments: the hint's rows, or (unknown) a long context
  const int64_t hint = rows_hint < ((int64_t)1 << 40) ? rows_hint : ((int64_t)1 << 40);
  const int64_t tiles = hint > 0 ? (hint + kQKeys - 1) / kQKeys + nseg : (int64_t)nseg * kQueryUnknownTiles;
  sh.tiles_per_range = (sh.qtiles * tiles + kQueryTargetItems - 1) / kQueryTargetItems;
  if (sh.tiles_per_range < kQueryMinTiles) sh.tiles_per_range = kQueryMinTiles;
  if (sh.tiles_per_range > ((int64_t)1 << 30)) sh.tiles_per_range = (int64_t)1 << 30;
  // segments of fewer than two ranges' worth of keys on average: no split
  if (tiles < (int64_t)nseg * 2 * kQueryMinTiles) {
    sh.max_items = units;
    sh.plan_bytes = 0;
    sh.rec_bytes = 0;
    return sh;
  }
  // sum_s max(1, round(T_s / C)) <= tiles / C + nseg for the hinted tiles;
  // the plan kernel raises C if the real keys would need more
  // (launched as a multiple of 8 workgroups: items are dealt to the 8 L2
  // domains in runs of ceil(items / 8))
  sh.max_items = (sh.qtiles * (tiles / sh.tiles_per_range + nseg + 1) + 7) / 8 * 8;
  sh.plan_bytes = ((size_t)(kQueryPlanHead + nseg + 1) * sizeof(int32_t) + 255) / 256 * 256;
  sh.rec_bytes = (size_t)sh.max_items * kQRows * (head_dim + 2) * sizeof(float);
  return sh;
}

hipError_t launch_query_attn(const QueryParams& p, int head_dim, int64_t grid, hipStream_t stream) {
  return head_dim == 64 ? launch_d<64>(p, grid, stream) : launch_d<128>(p, grid, stream);
}

constexpr int64_t kWholeTileRows = 2048, kWholeShortRows = 4096;

PagedPlanShape paged_plan_shape(int32_t batch, int32_t hkv, int32_t G, int32_t head_dim, int32_t num_tokens,
                                int32_t max_q, int64_t rows_hint) {
  PagedPlanShape sh;
  const int64_t nseg = (int64_t)batch * hkv;
  const int64_t qtiles = ((int64_t)max_q * G + kQRows - 1) / kQRows;
  // query tiles of all sequences: each has at most one that is not full
  const int64_t full = (int64_t)num_tokens * G / kQRows + batch;
  sh.units = hkv * (full < batch * qtiles ? full : batch * qtiles);
  const int64_t hint = rows_hint < ((int64_t)1 << 40) ? rows_hint : ((int64_t)1 << 40);
  const int64_t seg = hint > 0 ? (hint + nseg * kQKeys - 1) / (nseg * kQKeys) : kQueryUnknownTiles;  // tiles, on average
  sh.slices = 0;
  sh.plan_bytes = sh.rec_bytes = 0;
  const int64_t rows = (int64_t)max_q * G;
  sh.rec_rows = (int32_t)((rows + 3) / 4 * 4);
  sh.shorts = paged_takes_short(nseg, rows, rows_hint);
  // No split for segments of fewer than two ranges' worth of keys on average,
  // where it saves two launches or one, unless all sequences together have so
  // many rows that one long one among them would be a workgroup's alone (us,
  // whole / split, 32 query heads on 8: 8 prompts of 256 tokens 29 / 50, of 512
  // 75 / 64; steps of 8 sequences at 300 rows 15.0 / 18.1, of 64 at 100 21.9 /
  // 25.2; 4,096 rows of one sequence are 180 in query tiles and 45 in the kernels
  // for short blocks).
  if (seg < 2 * kQueryMinTiles && hint / hkv <= (sh.shorts ? kWholeShortRows : kWholeTileRows)) return sh;
  if (sh.shorts) {
    // at least 128 keys per workgroup, up to 256 workgroups
    const int64_t P = hint > 0 && hint < kPagedSlices * 128 ? (hint + 127) / 128 : kPagedSlices;
    sh.slices = (int32_t)P;
    sh.plan_bytes = ((size_t)nseg * 2 * sizeof(int32_t) + 255) / 256 * 256;
    sh.rec_bytes = (size_t)(P + nseg) * sh.rec_rows * (head_dim + 2) * sizeof(float);
    return sh;
  }
  const int64_t P = sh.units * (seg + kUnitTiles) / kQueryMinTiles;
  sh.slices = (int32_t)((P < kPagedSlices ? P + 8 : kPagedSlices) / 8 * 8);
  sh.plan_bytes = paged_plan_bytes(sh.units);
  sh.rec_bytes = (size_t)(2 * sh.slices) * kQRows * (head_dim + 2) * sizeof(float);
  return sh;
}

hipError_t launch_paged_query_attn(const QueryParams& p, int head_dim, hipStream_t stream) {
  return head_dim == 64 ? launch_paged_d<64>(p, stream) : launch_paged_d<128>(p, stream);
}

}  // namespace dkv
