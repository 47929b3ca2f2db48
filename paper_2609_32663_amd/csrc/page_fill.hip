// Filling a paged cache on the GPU: page tables and slots from request lengths
// (extend), rows of K and V into their slots (append), pages back to the stack
// of free ones (release).
//
// Extend.  Unit n holds len positions and gets `new` more; its Hkv segments
// need per = ceil((len + new) / R) - ceil(len / R) pages each.  With exclusive
// sums over the units of new tokens (row of the unit's first token) and of
// Hkv * per (its first page in the order of the call), everything else is
// elementwise: page i of the call is stack[top - 1 - i], token at position pos
// of segment s has page pos / R, which is one of the call's pages when it
// starts at or past ceil(len / R) * R and stands in the table otherwise, and
// slot page * R + pos % R.  No thread reads what another one writes, so the
// call has two forms.  With few rows every workgroup sums all units and fills
// 128 rows, in one launch: such calls are bound by the kernel's chain of reads
// and scans, which goes over the units' lengths three times and sums rows before
// pages (2,048 units, a decode step of 64 sequences on 32 layers: 9.7 us a call,
// 7.9 of them the kernel; one unit 4.4; the other calls' kernels of one launch 2.6 to 2.8).
// With many rows one workgroup sums the units and a second kernel fills, whose
// stores each wait for a chain of reads, up to the page's word (four prompts of
// up to 8,192 tokens on 32 layers, 56 MB: 23.7 us, of them the sums 5.5 and the
// fill 18.2, 3 TB/s; 8.1 at the rate of stores alone).
//
// Release.  The pages to go, in table order, are pushed on the stack: a count
// per chunk of table words, then every chunk sums the counts before it and
// places its own.  One chunk needs no count.  Bound by its launches (a request
// of 4,100 positions 6.9 us, 2.8 of them the kernel; all layers of a 128K
// context, 3 MB, 10.2, the kernels 3.4 and 4.8).

#include "dkv_device.hpp"
#include "dkv_launch.hpp"

namespace dkv {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kFillThreads = 256;

// ------------------------------------------------------------------- extend

struct ExtendUnit {
  int32_t len, add;
  int64_t rows;  // rows of the token-major arrays that the unit takes
};

__device__ __forceinline__ ExtendUnit extend_unit(const PageExtendParams& p, int n) {
  ExtendUnit u;
  u.len = p.unit_len[n];
  u.add = p.unit_new[n];
  u.rows = u.add > 0 ? u.add : 0;
  return u;
}

__device__ __forceinline__ int64_t pages_of(int64_t rows, int shift) { return (rows + (1 << shift) - 1) >> shift; }

// Pages that each segment of the unit needs, or -1 when the unit cannot be
// served however many pages are free: an invalid length, a table that is too
// short, rows past max_tokens.
__device__ __forceinline__ int64_t extend_need(const PageExtendParams& p, const ExtendUnit& u, int64_t end) {
  const int64_t grown = (int64_t)u.len + u.add;
  if (u.len < 0 || u.add < 0 || grown > INT32_MAX || grown > ((int64_t)p.pages_per_seg << p.page_shift) ||
      end > p.max_tokens)
    return -1;
  return pages_of(grown, p.page_shift) - pages_of(u.len, p.page_shift);
}

// The new rows of one unit: where they start, the positions held before them,
// their number and the unit's first page of the call (-1: not served).
struct ExtendRows {
  int32_t n, first, len, add, base;
};

__device__ __forceinline__ void extend_slot(const PageExtendParams& p, const ExtendRows& u, int32_t top, int32_t row,
                                            int g, int64_t* to) {
  int64_t slot = -1;
  if (u.base >= 0) {
    const int sh = p.page_shift;
    const int32_t grown = u.len + u.add;
    const int32_t pos = u.len + (row - u.first);
    const int32_t lpage = pos >> sh, in_page = pos & ((1 << sh) - 1);
    const int32_t old = (int32_t)pages_of(u.len, sh);
    const int64_t s = (int64_t)u.n * p.Hkv + g;
    int32_t page;
    if (lpage >= old) {
      const int32_t per = (int32_t)pages_of(grown, sh) - old;
      page = p.free_pages[top - 1 - (u.base + g * per + (lpage - old))];
      if (in_page == 0) p.table[s * p.pages_per_seg + lpage] = page;
    } else {
      page = p.table[s * p.pages_per_seg + lpage];
    }
    if (page >= 0) slot = ((int64_t)page << sh) + in_page;
    if (in_page == 0 || row == u.first) {
      if (p.entries != nullptr && lpage < p.max_entries) {
        const int64_t end = (int64_t)grown - ((int64_t)lpage << sh);
        int32_t* e = p.entries + 4 * (s * p.max_entries + lpage);
        *reinterpret_cast<int4*>(e) = int4{page, lpage, 0, (int32_t)(end < (1 << sh) ? end : (1 << sh))};
      }
      if (p.n_entries != nullptr && row == u.first) p.n_entries[s] = (int32_t)pages_of(grown, sh);
    }
  }
  *to = slot;
}

// Thread t plans units [t * per, t * per + per): sums of its units' rows and
// pages, a scan of each over the workgroup, and its units again.  FILL: the
// workgroup then fills rows [kBlockRows * block, + kBlockRows); only the first
// one writes what the units share.
constexpr int kBlockRows = 128;
// One launch up to a workgroup per compute unit, two beyond; one / two, us: 32
// units of 64 rows 8.7 / 11.5, 2,048 of 16 rows 9.0 / 13.0, 8,191 of 4 rows 30 / 40; of
// more workgroups, each summing all units, 1 unit of 131,072 rows 14.4 / 11.5, 32 of
// 32,768 87 / 24.
constexpr int kOneLaunchBlocks = 256;

template <bool FILL>
__global__ __launch_bounds__(kPlanThreads) void page_extend_plan_kernel(PageExtendParams p) {
  __shared__ int64_t red[2][kPlanThreads / kWave];
  __shared__ int32_t given;  // pages handed out: those of the units before the first that finds too few
  // FILL: the units of the workgroup's rows, each where its first row lies
  __shared__ uint32_t head[kBlockRows / 32];
  __shared__ ExtendRows unit[FILL ? kBlockRows : 1];
  const int tid = threadIdx.x;
  const int N = p.num_units;
  const int per = (N + kPlanThreads - 1) / kPlanThreads;
  const int lo = min(N, tid * per), hi = min(N, lo + per);
  const bool writes = blockIdx.x == 0;
  const int64_t row_lo = (int64_t)blockIdx.x * kBlockRows;
  const int32_t height = *p.n_free;
  const int32_t top = height < 0 ? 0 : (height > p.free_cap ? p.free_cap : height);
  if (tid == 0) given = 0;
  if (tid < kBlockRows / 32) head[tid] = 0;
  int64_t rows = 0;
  for (int n = lo; n < hi; ++n) rows += extend_unit(p, n).rows;
  int64_t all_rows;
  const int64_t row0 = block_scan<kPlanThreads>(rows, red[0], &all_rows);
  int64_t row = row0, pages = 0;
  for (int n = lo; n < hi; ++n) {
    const ExtendUnit u = extend_unit(p, n);
    const int64_t need = extend_need(p, u, row += u.rows);
    if (need > 0) pages += need * p.Hkv;
  }
  int64_t all_pages;
  int64_t base = block_scan<kPlanThreads>(pages, red[1], &all_pages);
  row = row0;
  for (int n = lo; n < hi; ++n) {
    const ExtendUnit u = extend_unit(p, n);
    const int64_t first = row;
    row += u.rows;
    const int64_t need = extend_need(p, u, row);
    const int64_t all = need > 0 ? need * p.Hkv : 0;
    const bool served = need == 0 || (need > 0 && base + all <= top);
    const int32_t at = served ? (int32_t)(base < top ? base : top) : -1;
    if (writes) {
      p.tok_off[n] = (int32_t)(first < p.max_tokens ? first : p.max_tokens);
      p.first_pos[n] = served ? u.len : -1;
      p.new_len[n] = served ? u.len + u.add : u.len;
      if (!FILL) p.base[n] = at;
      if (served && all > 0) atomicMax(&given, (int32_t)(base + all));
    }
    if (FILL && u.rows > 0 && first < row_lo + kBlockRows && row > row_lo) {
      const int i = (int)(first > row_lo ? first - row_lo : 0);
      atomicOr(&head[i >> 5], 1u << (i & 31));
      unit[i] = ExtendRows{n, (int32_t)first, u.len, u.add, at};
    }
    base += all;
  }
  __syncthreads();
  if (writes && tid == 0) {
    p.tok_off[N] = (int32_t)(all_rows < p.max_tokens ? all_rows : p.max_tokens);
    if (!FILL) p.top[0] = top;
    p.n_free_out[0] = top - given;
    if (p.pages_needed != nullptr) p.pages_needed[0] = all_pages;
  }
  if constexpr (FILL) {
    const int slots = (int)min((int64_t)kBlockRows, p.max_tokens - row_lo) * p.Hkv;
    for (int i = tid; i < slots; i += kPlanThreads) {
      const int r = (int)((uint32_t)i / (uint32_t)p.Hkv);
      const int g = i - r * p.Hkv;
      int64_t* to = p.slots + (row_lo * p.Hkv + i);
      // the last unit that starts at or before the row, if the row is one of its
      int w = r >> 5;
      uint32_t m = head[w] & (0xFFFFFFFFu >> (31 - (r & 31)));
      while (m == 0 && w > 0) m = head[--w];
      if (m == 0 || row_lo + r >= all_rows) {
        *to = -1;
      } else {
        extend_slot(p, unit[32 * w + 31 - __clz(m)], top, (int32_t)row_lo + r, g, to);
      }
    }
  }
}

// Number of offsets off[1 .. n] that are <= row, i.e. the unit of a row below
// off[n] (units without rows are stepped over).
__device__ __forceinline__ int unit_of(const int32_t* off, int lo, int hi, int32_t row) {
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (off[mid + 1] <= row) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// unit_of by a wave: 64 offsets at a time.
__device__ __forceinline__ int wave_unit_of(const int32_t* off, int n, int32_t row) {
  const int lane = threadIdx.x & (kWave - 1);
  int lo = 0, hi = n;  // the answer is in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + kWave - 1) / kWave;
    const int64_t at = lo + (int64_t)(lane + 1) * step;  // offsets off[lo + step], ...
    const bool below = at <= hi && off[at] <= row;
    const int k = __popcll(__builtin_amdgcn_ballot_w64(below));
    lo += k * step;
    hi = min(hi, lo + step - 1);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Rows [kFillRows * block, + kFillRows) of the slots; most blocks of a prompt's
// rows lie in one unit.
constexpr int kFillRows = 128;

__global__ __launch_bounds__(kFillThreads) void page_extend_fill_kernel(PageExtendParams p) {
  const int32_t total = p.tok_off[p.num_units];
  const int32_t top = p.top[0];
  const int64_t row_lo = (int64_t)blockIdx.x * kFillRows;
  const int rows = (int)min((int64_t)kFillRows, p.max_tokens - row_lo);
  const int slots = rows * p.Hkv;
  int64_t* to = p.slots + row_lo * p.Hkv;
  const int32_t r0 = (int32_t)row_lo;
  if (r0 >= total) {
    for (int i = threadIdx.x; i < slots; i += kFillThreads) to[i] = -1;
    return;
  }
  const int32_t r_last = min(r0 + rows, total) - 1;
  const int u0 = wave_unit_of(p.tok_off, p.num_units, r0);
  const int32_t off0 = p.tok_off[u0], off1 = p.tok_off[u0 + 1];
  const ExtendRows one{u0, off0, p.first_pos[u0], off1 - off0, p.base[u0]};
  const int u1 = off1 > r_last ? u0 : wave_unit_of(p.tok_off, p.num_units, r_last);
  for (int i = threadIdx.x; i < slots; i += kFillThreads) {
    const int r = (int)((uint32_t)i / (uint32_t)p.Hkv);
    const int g = i - r * p.Hkv;
    const int32_t row = r0 + r;
    if (row > r_last) {
      to[i] = -1;
    } else if (u0 == u1) {
      extend_slot(p, one, top, row, g, to + i);
    } else {
      const int n = unit_of(p.tok_off, u0, u1, row);
      const int32_t first = p.tok_off[n];
      extend_slot(p, ExtendRows{n, first, p.first_pos[n], p.tok_off[n + 1] - first, p.base[n]}, top, row, g, to + i);
    }
  }
}

// ------------------------------------------------------------------ release

constexpr int kReleaseThreads = 256;
constexpr int kReleaseWords = 1024;    // table words of a chunk at least
constexpr int kReleaseChunks = 4096;   // chunks at most

int64_t release_chunk(int64_t words) {
  const int64_t c = (words + kReleaseChunks - 1) / kReleaseChunks;
  return c <= kReleaseWords ? kReleaseWords : (c + kReleaseThreads - 1) / kReleaseThreads * kReleaseThreads;
}

__device__ __forceinline__ bool released(const PageReleaseParams& p, int64_t i) {
  return p.table[i] >= 0 && (p.keep == nullptr || p.keep[i] == 0);
}

__device__ __forceinline__ int32_t release_top(const PageReleaseParams& p) {
  const int32_t height = *p.n_free;
  return height < 0 ? 0 : (height > p.free_cap ? p.free_cap : height);
}

__global__ __launch_bounds__(kReleaseThreads) void page_release_count_kernel(PageReleaseParams p, int64_t chunk) {
  __shared__ int64_t red[kReleaseThreads / kWave];
  const int64_t lo = blockIdx.x * chunk, hi = lo + chunk < p.words ? lo + chunk : p.words;
  int64_t n = 0;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kReleaseThreads) n += released(p, i) ? 1 : 0;
  int64_t all;
  block_scan<kReleaseThreads>(n, red, &all);
  if (threadIdx.x == 0) {
    p.counts[blockIdx.x] = (int32_t)all;
    if (blockIdx.x == 0) p.top[0] = release_top(p);
  }
}

__global__ __launch_bounds__(kReleaseThreads) void page_release_push_kernel(PageReleaseParams p, int64_t chunk) {
  // a scan's buffer is written again two scans later, one barrier after its last reader
  __shared__ int64_t red[3][kReleaseThreads / kWave];
  const int tid = threadIdx.x;
  int64_t before = 0, at = 0;
  if (gridDim.x > 1) {
    for (int c = tid; c < (int)blockIdx.x; c += kReleaseThreads) before += p.counts[c];
    block_scan<kReleaseThreads>(before, red[2], &at);
    at += p.top[0];
  } else {
    at = release_top(p);
  }
  const int64_t lo = blockIdx.x * chunk, hi = lo + chunk < p.words ? lo + chunk : p.words;
  // four neighbouring words per thread and scan
  int turn = 0;
  for (int64_t i0 = lo; i0 < hi; i0 += 4 * kReleaseThreads, turn ^= 1) {
    const int64_t i = i0 + 4 * tid;
    int32_t page[4];
    bool go[4];
    int n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      page[j] = i + j < hi ? p.table[i + j] : -1;
      go[j] = i + j < hi && page[j] >= 0 && (p.keep == nullptr || p.keep[i + j] == 0);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) n += go[j] ? 1 : 0;
    int64_t sum;
    int64_t to = at + block_scan<kReleaseThreads>(n, red[turn], &sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool push = go[j] && to < p.free_cap;  // a page that the stack has no room for stays
      if (push) p.free_pages[to] = page[j];
      if (i + j < hi) p.table_out[i + j] = push ? -1 : page[j];
      to += go[j] ? 1 : 0;
    }
    at += sum;
  }
  if (blockIdx.x == gridDim.x - 1 && tid == 0) p.n_free_out[0] = (int32_t)(at < p.free_cap ? at : p.free_cap);
}

// ------------------------------------------------------------------- append

// One 16-byte granule of K and of V per thread: a row is row_bytes / 16
// threads, rows of one token side by side.  Bound by moving the rows (8,192
// tokens of an 8B layer, 68 MB: 12.5 us, 5.4 TB/s, launch included; 96 tokens 6.9
// us, the launch).
__global__ __launch_bounds__(kFillThreads) void paged_append_kernel(PagedAppendParams p) {
  const int per_row = p.row_bytes / 16;
  const int64_t i = (int64_t)blockIdx.x * kFillThreads + threadIdx.x;
  const int64_t r = i / per_row;  // token * Hkv + head
  if (r >= (int64_t)p.tokens * p.Hkv) return;
  const int64_t slot = p.slots[r];
  if (slot < 0 || slot >= p.pool_rows) return;
  const int c = (int)(i - r * per_row) * 16;
  const int64_t tok = r / p.Hkv;
  const int64_t from = tok * p.token_bytes + (r - tok * p.Hkv) * p.row_bytes + c;
  const int64_t to = slot * p.row_bytes + c;
  const u32x4 k = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.k_new) + from);
  const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.v_new) + from);
  *reinterpret_cast<u32x4*>(static_cast<char*>(p.k_pages) + to) = k;
  *reinterpret_cast<u32x4*>(static_cast<char*>(p.v_pages) + to) = v;
}

}  // namespace

size_t page_extend_workspace_bytes(int64_t num_units) { return (size_t)(num_units + 1) * sizeof(int32_t); }

hipError_t launch_page_extend(const PageExtendParams& p, hipStream_t stream) {
  // One launch: every workgroup reads all the lengths, so with more than one
  // of them the outputs must be other buffers.
  const int64_t blocks = p.max_tokens > kBlockRows ? ((int64_t)p.max_tokens + kBlockRows - 1) / kBlockRows : 1;
  const bool apart = p.new_len != p.unit_len && p.n_free_out != p.n_free;
  if (blocks == 1 || (apart && blocks <= kOneLaunchBlocks)) {
    hipLaunchKernelGGL(page_extend_plan_kernel<true>, dim3((unsigned)blocks), dim3(kPlanThreads), 0, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(page_extend_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, stream, p);
  hipLaunchKernelGGL(page_extend_fill_kernel, dim3((unsigned)(((int64_t)p.max_tokens + kFillRows - 1) / kFillRows)),
                     dim3(kFillThreads), 0, stream, p);
  return hipGetLastError();
}

size_t page_release_workspace_bytes(int64_t words) {
  const int64_t chunks = (words + kReleaseWords - 1) / kReleaseWords;
  return (size_t)(2 + (chunks < kReleaseChunks ? chunks : kReleaseChunks)) * sizeof(int32_t);
}

hipError_t launch_page_release(const PageReleaseParams& p, hipStream_t stream) {
  const int64_t chunk = release_chunk(p.words);
  const unsigned chunks = p.words > 0 ? (unsigned)((p.words + chunk - 1) / chunk) : 1u;
  if (chunks > 1)
    hipLaunchKernelGGL(page_release_count_kernel, dim3(chunks), dim3(kReleaseThreads), 0, stream, p, chunk);
  hipLaunchKernelGGL(page_release_push_kernel, dim3(chunks), dim3(kReleaseThreads), 0, stream, p, chunk);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendParams& p, hipStream_t stream) {
  const int64_t n = (int64_t)p.tokens * p.Hkv * (p.row_bytes / 16);
  hipLaunchKernelGGL(paged_append_kernel, dim3((unsigned)((n + kFillThreads - 1) / kFillThreads)), dim3(kFillThreads),
                     0, stream, p);
  return hipGetLastError();
}

}  // namespace dkv
