// Device helpers shared by the query-block attention kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dkv_device.hpp"
#include "dkv_query.hpp"

namespace dkv {

constexpr float kLazy = 8.f;  // log2 headroom of the lazy running max

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t q_rsrc(const char* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)a);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(((uint64_t)hi << 32) | lo), (short)0,
                                           (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

__device__ __forceinline__ int64_t q_uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Two probabilities as a bf16 pair (round to nearest even) and the bf16 pair
// of what that rounding left out: a + b carries ~16 significant bits.
__device__ __forceinline__ void bf16_split(float x0, float x1, uint32_t& a, uint32_t& b) {
  const f32x2 x = {x0, x1};
  const bf16x2 h = __builtin_convertvector(x, bf16x2);
  const bf16x2 l = __builtin_convertvector(x - __builtin_convertvector(h, f32x2), bf16x2);
  a = __builtin_bit_cast(uint32_t, h);
  b = __builtin_bit_cast(uint32_t, l);
}

// Two probabilities as N bf16 pairs, each the rounding of what the ones before
// left out: two carry 17 bits, three all 24.  (Remainders by dot products with
// (-1, 0), half the instructions, made a vector phase a tenth longer.)
template <int N>
__device__ __forceinline__ void bf16_parts(float x0, float x1, uint32_t (&part)[N]) {
  f32x2 x = {x0, x1};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const bf16x2 h = __builtin_convertvector(x, bf16x2);
    part[i] = __builtin_bit_cast(uint32_t, h);
    if (i + 1 < N) x = x - __builtin_convertvector(h, f32x2);
  }
}

// Maximum over the lanes that share (lane % 16).
__device__ __forceinline__ float row4_max(float x) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// ---------------------------------------------------------------------------
// Paged addressing.  The kernels walk a segment's row space in runs of 32 rows,
// which lie in one page (page sizes are multiples of 32).
// ---------------------------------------------------------------------------
constexpr int kRun = 32;

// A sequence's block: its first row in the token-major arrays, its tokens and
// the position of the first one (negative: the sequence attends nothing).
// Offsets that do not fit the arrays give fewer tokens.
struct PagedBlock {
  int32_t tok0, n, pos0;
};

__device__ __forceinline__ PagedBlock paged_block(const QueryParams& p, int b) {
  PagedBlock k;
  const int32_t lo = p.tok_off[b], hi = p.tok_off[b + 1];
  k.tok0 = lo < 0 ? 0 : (lo > p.num_tokens ? p.num_tokens : lo);
  const int64_t end = hi > p.num_tokens ? p.num_tokens : hi;
  const int64_t n = end - k.tok0;
  k.n = (int32_t)(n < 0 || lo < 0 ? 0 : (n > p.max_q ? p.max_q : n));
  k.pos0 = p.first_pos[b];
  return k;
}

// The same for a uniform b, in scalar registers.
__device__ __forceinline__ PagedBlock paged_block_uniform(const QueryParams& p, int b) {
  const PagedBlock k = paged_block(p, b);
  return PagedBlock{__builtin_amdgcn_readfirstlane(k.tok0), __builtin_amdgcn_readfirstlane(k.n),
                    __builtin_amdgcn_readfirstlane(k.pos0)};
}

// Position of token t of a block (positions stop below the largest int32).
__device__ __forceinline__ int32_t paged_pos(const PagedBlock& k, int32_t t) {
  return k.pos0 > INT32_MAX - 1 - t ? INT32_MAX - 1 : k.pos0 + t;
}

// Rows of segment s up to the last that a token at position `last` can see, in
// whole runs.  It sees slots of all entries, or, when the one after that
// position's page number starts behind it (as in an unpruned cache), of the
// ones before that; and the last of them up to its end or that position (half a
// page less to walk on average).  `gaps`: whether there may be slots of no key
// among them, as a selection's runs leave (not where the last entry seen is
// that of its page in a cache without any).
__device__ __forceinline__ int32_t paged_rows(const QueryParams& p, int s, int32_t last, bool* gaps) {
  const int32_t x = last >> p.page_shift;
  const i32x4* list = reinterpret_cast<const i32x4*>(p.entries) + (int64_t)s * p.max_entries;
  // an unpruned cache's last entry is x: these loads wait for nothing
  const int32_t n = p.n_entries[s];
  const int32_t page = x + 1 < p.max_entries ? list[x + 1][1] : 0;
  i32x4 e = list[x < p.max_entries ? x : 0];
  const int32_t all = n < 0 ? 0 : (n > p.max_entries ? p.max_entries : n);
  const int32_t held = x + 1 < all && page > x ? x + 1 : all;
  *gaps = held != x + 1 || e[1] != x;
  if (held == 0) return 0;
  if (held != x + 1) e = list[held - 1];
  // positions from 2^31 on are beyond every token
  const int64_t start = (int64_t)e[1] << p.page_shift;
  int64_t slots = last + 1 - start < e[3] ? last + 1 - start : e[3];
  slots = slots < 0 ? 0 : (slots > 1 << p.page_shift ? 1 << p.page_shift : slots);
  return (int32_t)(((int64_t)(held - 1) << p.page_shift) + (slots + kRun - 1) / kRun * kRun);
}

// A run of 32 rows: the pool row and the position of its first slot, and the
// slots [lo, hi) of it that hold keys of the segment (none: lo = hi = 0).  All
// uniform, so that it stays in scalar registers.
struct PagedRun {
  int64_t row;
  int32_t pos, lohi;  // lo | hi << 8

  __device__ __forceinline__ int32_t lo() const { return lohi & 0xFF; }
  __device__ __forceinline__ int32_t hi() const { return lohi >> 8; }
};

// What a workgroup needs of a segment's entries: the entries (constant while
// the kernel runs, so a uniform index reads them with scalar loads), their
// number, and where its rows and positions end.
struct PagedSegment {
  const __attribute__((address_space(4))) i32x4* entries;
  int32_t n, end, stop, shift, pages;
};

__device__ __forceinline__ PagedSegment paged_segment(const QueryParams& p, int s, int32_t n, int32_t end,
                                                      int32_t stop) {
  return PagedSegment{(const __attribute__((address_space(4))) i32x4*)(p.entries + 4 * (int64_t)s * p.max_entries), n, end,
                      stop, p.page_shift, (int32_t)p.num_pages};
}

// The entry that holds row r (the last one for rows past them).
__device__ __forceinline__ i32x4 paged_entry(const PagedSegment& g, int32_t r) {
  const int32_t e = r >> g.shift;
  return g.entries[e < g.n ? e : (g.n > 0 ? g.n - 1 : 0)];
}

// The run at row r (uniform, a multiple of 32) of entry x; empty past the end,
// for slots past the last position and for an entry that names a page outside
// the pool or slots outside a page.
__device__ __forceinline__ PagedRun paged_run(const PagedSegment& g, const i32x4& x, int32_t r) {
  const int32_t slot = r & ((1 << g.shift) - 1);
  // without branches: a chain of scalar selects
  const bool ok = (r < g.end) & ((uint32_t)x.x < (uint32_t)g.pages) &
                  ((uint32_t)x.y <= (uint32_t)(INT32_MAX - 1) >> g.shift) & (x.z >= 0) &
                  ((uint32_t)x.w <= 1u << g.shift);  // 0 <= x.w: no difference below wraps
  PagedRun u;
  u.row = ok ? ((int64_t)x.x << g.shift) + slot : 0;
  u.pos = ok ? (x.y << g.shift) + slot : 0;
  int32_t lo = x.z - slot, hi = x.w - slot;
  if (g.stop - u.pos < hi) hi = g.stop - u.pos;
  lo = lo < 0 ? 0 : lo;
  hi = hi > kRun ? kRun : hi;
  u.lohi = ok & (lo < hi) ? lo | hi << 8 : 0;
  return u;
}

// Which of the 32 slots of a run at position `pos` a token sees, as bits: those
// of [lo, hi) below its position (no mask), or before the new tokens and where
// its mask row has their bit.  `cut` is the position past the token's own, `first`
// that of its sequence's first new token.
__device__ __forceinline__ uint32_t tree_sees(const QueryParams& p, int64_t token, int32_t cut, int32_t first, int32_t pos,
                                              int32_t lo, int32_t hi) {
  uint32_t sees;
  if (p.mask != nullptr) {
    const uint32_t* row = reinterpret_cast<const uint32_t*>(p.mask) + token * 2 * p.mask_words;
    const int32_t rel = pos - first, w = rel >> 5, words = 2 * p.mask_words;
    const uint32_t a = w < 0 ? ~0u : (w < words ? row[w] : 0u);
    const uint32_t b = w + 1 < 0 ? ~0u : (w + 1 < words ? row[w + 1] : 0u);
    sees = __builtin_amdgcn_alignbit(b, a, (uint32_t)rel & 31u);
  } else {
    const int32_t n = cut - pos;
    sees = n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u);
  }
  const uint32_t below = hi >= 32 ? ~0u : (1u << hi) - 1u;
  return sees & below & (lo >= 32 ? 0u : ~0u << lo);
}

}  // namespace dkv
