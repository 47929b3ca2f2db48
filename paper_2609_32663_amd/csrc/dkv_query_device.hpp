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
typedef float f32x2 __attribute__((ext_vector_type(2)));

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

// The same in three bf16 pairs: a + b + c carries all 24 bits of x.
__device__ __forceinline__ void bf16_split3(float x0, float x1, uint32_t& a, uint32_t& b, uint32_t& c) {
  const f32x2 x = {x0, x1};
  const bf16x2 h = __builtin_convertvector(x, bf16x2);
  const f32x2 r = x - __builtin_convertvector(h, f32x2);
  const bf16x2 l = __builtin_convertvector(r, bf16x2);
  const bf16x2 t = __builtin_convertvector(r - __builtin_convertvector(l, f32x2), bf16x2);
  a = __builtin_bit_cast(uint32_t, h);
  b = __builtin_bit_cast(uint32_t, l);
  c = __builtin_bit_cast(uint32_t, t);
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

// Position of token t of a block (positions stop below the largest int32).
__device__ __forceinline__ int32_t paged_pos(const PagedBlock& k, int32_t t) {
  return k.pos0 > INT32_MAX - 1 - t ? INT32_MAX - 1 : k.pos0 + t;
}

// Entries of segment s that a token at position `last` can see any slot of:
// all of them, or, when the one after that position's page number starts
// behind it (as in an unpruned cache), the ones before that.
__device__ __forceinline__ int32_t paged_entries(const QueryParams& p, int s, int32_t last) {
  const int32_t n = p.n_entries[s];
  const int32_t all = n < 0 ? 0 : (n > p.max_entries ? p.max_entries : n);
  const int32_t x = (last >> p.page_shift) + 1;
  if (x < all && p.entries[4 * ((int64_t)s * p.max_entries + x) + 1] > (last >> p.page_shift)) return x;
  return all;
}

// 64 consecutive entries of a segment in a wave's registers, one per lane; an
// entry that names a page outside the pool or slots outside a page is empty.
struct PagedEntries {
  int32_t page, lpage, lohi;  // lohi: lo | hi << 16
  int32_t base;               // first entry held (uniform)

  __device__ __forceinline__ void load(const QueryParams& p, int s, int32_t n, int32_t first) {
    base = first;
    const int32_t e = first + (int)(threadIdx.x & (kWave - 1));
    page = lpage = lohi = 0;
    if (e < n) {
      const int4 x = *reinterpret_cast<const int4*>(p.entries + 4 * ((int64_t)s * p.max_entries + e));
      const int32_t rows = 1 << p.page_shift;
      if (x.x >= 0 && x.x < p.num_pages && x.y >= 0 && x.y <= (INT32_MAX - 1) >> p.page_shift && x.z >= 0 &&
          x.z < x.w && x.w <= rows) {
        page = x.x;
        lpage = x.y;
        lohi = x.z | x.w << 16;
      }
    }
  }
};

// A run of 32 rows: the pool row and the position of its first slot, and the
// slots [lo, hi) of it that hold keys of the segment (none: lo = hi = 0).
struct PagedRun {
  int64_t row;
  int32_t pos, lo, hi;
};

// The run at row r of the segment's row space (uniform, a multiple of 32), with
// rows from `end` on and positions from `stop` on left out.  `held` moves on
// when r passes it.
__device__ __forceinline__ PagedRun paged_run(const QueryParams& p, PagedEntries& held, int s, int32_t n, int32_t r,
                                              int32_t end, int32_t stop) {
  PagedRun u{0, 0, 0, 0};
  if (r >= end) return u;
  const int32_t e = r >> p.page_shift;
  if (e - held.base >= kWave) held.load(p, s, n, e);
  const int li = e - held.base;
  const int32_t slot = r & ((1 << p.page_shift) - 1);
  const int32_t lohi = __builtin_amdgcn_readlane(held.lohi, li);
  u.row = ((int64_t)__builtin_amdgcn_readlane(held.page, li) << p.page_shift) + slot;
  u.pos = (__builtin_amdgcn_readlane(held.lpage, li) << p.page_shift) + slot;
  int32_t lo = (lohi & 0xFFFF) - slot, hi = (lohi >> 16) - slot;
  if (stop - u.pos < hi) hi = stop - u.pos;
  lo = lo < 0 ? 0 : lo;
  hi = hi > kRun ? kRun : hi;
  if (lo < hi) {
    u.lo = lo;
    u.hi = hi;
  }
  return u;
}

}  // namespace dkv
