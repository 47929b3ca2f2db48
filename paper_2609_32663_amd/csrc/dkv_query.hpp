// Launch interface of query-block attention (argument checks live in the
// C-ABI layer; the launcher assumes validated arguments).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace dkv {

constexpr int kQueryRowsPerWG = 256;     // query rows (tokens x heads of a group) per workgroup
constexpr int kQueryTargetItems = 512;   // workgroups a split call aims at: two per compute unit
constexpr int kQueryMinTiles = 8;        // 64-key tiles per key range at least
constexpr int kQueryUnknownTiles = 512;  // key tiles per segment assumed when the caller gives no hint
constexpr int kQueryPlanHead = 4;        // plan words before the first-item table

struct QueryParams {
  const void* q;           // [B][n_q][Hq][d] bf16
  const void* k;           // packed K rows (bf16)
  const void* v;
  const int64_t* seg_off;  // [B*Hkv]
  const int32_t* seg_len;  // [B*Hkv]
  int32_t n_tail;          // tokens appended before the block
  int32_t n_q;             // tokens in the block (already appended after them)
  int32_t nseg, Hkv, Hq, G;
  int32_t rows;            // query rows per segment: n_q * G
  int32_t qtiles;          // ceil(rows / kQueryRowsPerWG)
  int32_t tiles_per_range; // C before the plan kernel's check against max_items
  int32_t max_items;       // items the records hold
  float scale_log2;        // sm_scale * log2(e)
  float* out;              // [B][n_q][Hq][d] fp32
  // Split calls only (nullptr otherwise): plan words [0] items, [1] tiles per
  // range, then [kQueryPlanHead + s] first item of segment s (s <= nseg); and
  // the records [max_items][kQueryRowsPerWG][d + 2] (max, sum, output).
  int32_t* plan;
  float* rec;
  // Short blocks (rows <= kShortRows) only: workgroups of the split (0: no
  // split, one workgroup per segment), rows of a record (a multiple of 4;
  // record slot x holds rec_rows maxima, sums and then outputs of d floats),
  // and per segment the first record slot and the piece count.
  int32_t P, rec_rows;
  int32_t stream_once;     // load K and V past the caches
  int32_t* seg_meta;
  // Paged calls only.  q is [num_tokens][Hq][d] with tokens q_stride bytes
  // apart, out [num_tokens][Hq][d]; sequence b's block is tokens [tok_off[b],
  // tok_off[b + 1]), its first one at position first_pos[b].  k and v are page
  // pools; a segment's row space is the page_rows slots of each of its
  // entries, in entry order (rows of entry e: [e << page_shift, ...)), and a
  // slot counts when it lies in the entry's [lo, hi) and at or below the query
  // token's position.
  const int32_t* tok_off;    // [B + 1]
  const int32_t* first_pos;  // [B]
  const int32_t* entries;    // [nseg][max_entries][4]: page, logical page, lo, hi
  const int32_t* n_entries;  // [nseg]
  int64_t num_pages, q_stride;
  int32_t max_entries, page_shift, num_tokens, max_q;
  // Tree calls only.  mask: [num_tokens][mask_words], bit j of a token's row
  // says whether it sees its sequence's new token j (null: those up to itself);
  // everything before the new tokens is seen.  scales: quantised pools (rows of
  // d codes), the exponent bytes of the K and the V row [pool rows][2].
  const uint64_t* mask;
  const uint8_t* scales;
  int32_t mask_words;
};

// How a call is split, from the shapes and the caller's hint of the total
// rows (0 = unknown) only, so the workspace size is known before the call.
struct QueryPlanShape {
  int32_t qtiles;
  int64_t tiles_per_range;
  int64_t max_items;   // attention workgroups launched
  size_t plan_bytes;   // 0: no split, one workgroup per (segment, query tile)
  size_t rec_bytes;
};

QueryPlanShape query_plan_shape(int32_t nseg, int32_t rows, int32_t head_dim, int64_t rows_hint);
// Short blocks: most query rows per segment, and most segments of a call (the
// workgroups' prefix over them shares the LDS with the tiles).
constexpr int kShortRows = 256;
constexpr int kShortSegments = 512;
// Whether the short kernels take a call, where they are level or ahead; long /
// short, us, attention and combine.
//   * Up to 64 rows: always.
//   * Up to 128 rows: but for many segments of few keys, where a piece is little
//     more than its start and its record and the long kernel's items fit one
//     round of workgroups or, with more than 96 rows, nearly fill two (128 rows
//     of 64 dimensions: 128 segments of 960 keys 36 / 55, 80 of 1,400 33 / 41, 160
//     of 1,400 58 / 69; a started second round turns it: 160 of 1,000 66 / 59, 96
//     of 1,250 57 / 46; 65 rows, 256 unequal segments of 1,700 141 / 86).
//   * More rows leave one key wave and up to 133 KB of record per piece, so the
//     segments have to be long (240 rows: 128 segments of 1,050 keys 85.8 /
//     110.9, 8 of 11,500 54.7 / 41.2) and few; with 128 dimensions the long
//     kernel's overlapped products win again once all the keys are many (192
//     rows: 8 segments of 120,000 199 / 180, 16 of 45,000 151 / 147, of 120,000
//     341 / 371, 32 of 9,000 83 / 81, of 45,000 256 / 280, 128 of 9,000 214 /
//     261; of 64 dimensions 32 of 45,000 203 / 196).
constexpr int64_t kShortLongKeys = 8192;  // keys per segment on average
constexpr int kShortManySegments = 48;
constexpr int64_t kShortFewKeys = 2048;
inline bool query_takes_short(int32_t nseg, int32_t rows, int32_t head_dim, int64_t rows_hint,
                              const QueryPlanShape& sh) {
  if (rows > kShortRows || nseg > kShortSegments) return false;
  if (rows <= kShortRows / 4) return true;
  if (rows <= kShortRows / 2) {
    if (sh.plan_bytes == 0 || nseg < kShortManySegments || rows_hint <= 0 || rows_hint / kShortFewKeys >= nseg)
      return true;
    const int64_t tiles = (rows_hint / nseg + 63) / 64;  // of a segment, on average
    const int64_t items = nseg * ((tiles + sh.tiles_per_range / 2) / sh.tiles_per_range);
    return items > kQueryTargetItems / 2 && (items < 400 || rows <= 96);
  }
  return sh.plan_bytes > 0 && rows_hint / kShortLongKeys >= nseg && nseg <= 32 &&
         (head_dim == 64 || rows_hint <= (int64_t(1) << 24) / nseg);
}
// K and V of a call up to this size may still be in the 256 MB last-level
// cache from the call before (the block's append, the last step), so they are
// loaded normally; larger ones are streamed past the caches.
constexpr int64_t kShortCachedBytes = 96 << 20;
hipError_t launch_query_short(const QueryParams& p, int head_dim, hipStream_t stream);
hipError_t launch_query_attn(const QueryParams& p, int head_dim, int64_t grid, hipStream_t stream);

// Whether the kernels for short blocks take a paged call, whose longest block has
// `rows` query rows per segment; query tiles / short, us, attention with plan
// and combine, 128-row pages.
//   * Up to 32 rows: always (32 rows: 256 segments of 1,000 keys 41 / 38, 64 of
//     16,000 119 / 98).  The stream is the bound, and one wave's.
//   * Up to 128 rows: few segments or keys, where the plan and a tile's chain of
//     phases weigh most; the query tiles spread the rows over all waves (64 query
//     heads on 8, 64 rows: 8 segments of 16,000 keys 44 / 30, 16 of 16,000 50 / 46; 32
//     of 1,000 35 / 25, of 4,000 38 / 34, of 16,000 70 / 74; 64 of 1,000 39 / 34, of 4,000
//     49 / 55; 128 of 1,000 41 / 48; 128 rows: 16 of 16,000 59 / 56; 32 of 1,000 39 /
//     35, of 4,000 44 / 46; 128 of 300 41 / 33, of 1,000 48 / 72; 256 of 100 43 / 19, of
//     1,000 54 / 60).  Up to 16 segments longer ones would be level or ahead here
//     too (64 rows: 8 of 65,000 79 / 71, 16 of 65,000 130 / 124), but the hint counts
//     slots of no key, whose runs the short kernels walk and the tiles drop: of
//     131,072 positions, the 35% that a selection kept, 8 segments, 64 rows, are 69 /
//     57 in pages of 128 rows, 90 / 119 of 512 and 93 / 199 of 1,024.
//   * More rows: fewer still (28 heads on 4, 252 rows: 4 of 1,000 35 / 31; 64 on 8,
//     256 rows: 8 of 16,000 64 / 57, of 32,000 88 / 82, of 65,000 139 / 141; 16 of 4,000
//     55 / 49, of 16,000 83 / 87; 32 of 1,000 51 / 53).
//   * Without a hint, up to 128 rows: up to 16 segments, where they are ahead at
//     any length of whole pages (behind over a selection in large pages, as above;
//     64 query heads on 8; 16 segments, 64 rows: 100 keys 21 / 17, 4,000 35 / 27,
//     60,000 122 / 118; 128 rows: 25 / 23, 39 / 36, 157 / 142), and the query tiles
//     beyond, which lose with short segments only (64 rows, 32 segments: 100 keys 22 /
//     20, 4,000 38 / 37, 60,000 202 / 222; 128 segments: 25 / 21, 74 / 90, 759 / 839;
//     128 rows, 128 segments: 32 / 27, 1,000 keys 48 / 71, 4,000 96 / 118, 16,000 303 /
//     314).
inline bool paged_takes_short(int64_t nseg, int64_t rows, int64_t rows_hint) {
  if (rows <= kShortRows / 8) return true;
  if (rows <= kShortRows / 2 && rows_hint <= 0) return nseg <= 16;
  if (rows <= kShortRows / 2)
    return (nseg <= 16 && rows_hint < 1 << 18) || (nseg * rows <= 4096 && rows_hint <= 1 << 17) ||
           (nseg <= 256 && rows_hint <= 1 << 16);
  return rows <= kShortRows && nseg <= 16 && rows_hint > 0 && rows_hint <= 1 << 17;
}
// The same for a quantised cache (us, short blocks / query tiles, 32 query heads
// on 8 of 128 dims, 128-row pages).
//   * Up to 32 rows: always.  The short kernels read the codes at 6 TB/s, the tiles
//     hold one tile's codes on their way (8 rows: 256 segments of 8,000 keys 90 /
//     182).
//   * Up to 64 rows: as well (64 rows: 8 segments of 4,000 keys 24 / 32; 32 of 2,000
//     29 / 37; 128 of 300 28 / 36, of up to 16,000 105 / 121; 256 of 8,000 157 /
//     183), but where most segments are cut once or twice, each piece with its fold
//     and records, and are too short for that (128 of 1,000 47 / 35, of 2,000 54 /
//     43, of up to 2,000 47 / 43, of up to 4,000 59 / 56, of up to 8,000 75 / 79; 192
//     of up to 1,000 50 / 48, of up to 4,000 77 / 78; of one length 72 of 1,000 37 / 39, of
//     2,000 42 / 41, of 6,000 59 / 60; 96 of 1,000 42 / 39, of 4,000 59 / 56, of 7,900 82 /
//     82; 160 of 500 44 / 40, of 3,000 75 / 66; 248 of 500 54 / 43, of 2,000 83 / 69).
//     The bound is one of all rows: with more segments it ends at fewer keys of each
//     than the tiles are ahead at (128 of 6,000 85 / 77; 192 of 3,000 86 / 73, of
//     6,000 120 / 117; 248 of 4,000 117 / 106, of 6,000 148 / 146).
//   * Up to 128 rows: few keys, or few segments, whose keys the short kernels cut
//     evenly: the tiles convert a key once for all rows, the short kernels once in
//     each row group (96 rows: 8 segments of 2,000 keys 23 / 32, of 32,000 48 / 55,
//     of 100,000 107 / 100; 32 of 2,000 36 / 42, of 4,000 43 / 39, of 8,000 55 / 48; 128 of
//     300 31 / 42, of 2,000 78 / 50, of 8,000 159 / 123; 256 of 300 36 / 33).
//   * More rows: fewer still (192 rows: 8 segments of 300 keys 37 / 25, of 2,000
//     32 / 37, of 8,000 41 / 48, of 32,000 79 / 70; 32 of 2,000 54 / 48, of 8,000
//     94 / 65).
//   * Without a hint: up to 64 rows, and up to 128 over up to 16 segments.
inline bool paged_f8_takes_short(int64_t nseg, int64_t rows, int64_t rows_hint) {
  if (rows <= kShortRows / 8) return true;
  if (rows <= kShortRows / 4) return nseg <= 64 || nseg >= 256 || rows_hint <= 1 << 16 || rows_hint > 1 << 19;
  if (rows <= kShortRows / 2)
    return (rows_hint > 0 && rows_hint <= 1 << 16) || (nseg <= 16 && rows_hint < 1 << 19);
  return rows <= kShortRows && nseg <= 16 && rows_hint > 1 << 13 && rows_hint <= 1 << 17;
}

// How a paged call is split: the most units ((segment, query tile) pairs) it
// can have, and the slices its keys are cut into (0: no split).
constexpr int kPagedSlices = 256;  // one workgroup per compute unit
struct PagedPlanShape {
  bool shorts;  // the kernels for short blocks take the call
  int64_t units;
  int32_t slices;
  size_t plan_bytes, rec_bytes;  // short blocks: segment metadata, records of rec_rows rows
  int32_t rec_rows;
};
PagedPlanShape paged_plan_shape(int32_t batch, int32_t hkv, int32_t G, int32_t head_dim, int32_t num_tokens,
                                int32_t max_q, int64_t rows_hint, bool f8 = false);
hipError_t launch_paged_query_attn(const QueryParams& p, int head_dim, hipStream_t stream);
hipError_t launch_paged_query_short(const QueryParams& p, int head_dim, hipStream_t stream);
hipError_t launch_paged_tree_attn(const QueryParams& p, int head_dim, hipStream_t stream);
hipError_t launch_paged_tree_short(const QueryParams& p, int head_dim, hipStream_t stream);

}  // namespace dkv
