// Drafted trees: ancestors and positions from parents, and the rows of an
// accepted path moved to the front of their request's new ones.

#include <hip/hip_runtime.h>

#include "dkv_device.hpp"
#include "dkv_tree.hpp"

namespace dkv {

namespace {

constexpr int kTreeThreads = 256;

// One workgroup per sequence (and one for the rows of none).  A token walks up
// its parents, which lie in LDS; they come before it, so its mask words fill
// from the token's own down.  Latency bounds it: a link of the longest path is
// one LDS read.
__global__ __launch_bounds__(kTreeThreads) void tree_plan_kernel(TreePlanParams p) {
  __shared__ int32_t up[kMaxTree];
  const int tid = threadIdx.x;
  auto in_range = [&](int64_t x) { return x < 0 ? (int64_t)0 : (x > p.tokens ? (int64_t)p.tokens : x); };
  auto none = [&](int64_t from, int64_t to) {
    for (int64_t t = from + tid; t < to; t += kTreeThreads) p.pos[t] = -1;
    if (p.mask != nullptr)
      for (int64_t i = from * p.words + tid; i < to * p.words; i += kTreeThreads) p.mask[i] = 0;
  };
  const int b = blockIdx.x;
  if (b == p.batch) {  // the rows before the first sequence's and after the last one's
    const int64_t lo = in_range(p.tok_off[0]), hi = in_range(p.tok_off[p.batch]);
    none(0, lo);
    none(hi < lo ? lo : hi, p.tokens);
    return;
  }
  const int64_t t0 = in_range(p.tok_off[b]), t1 = in_range(p.tok_off[b + 1]);
  if (t1 <= t0) return;
  const int32_t first = p.first_pos[b];
  const int n = (int)(first < 0 ? 0 : (t1 - t0 < p.max_q ? t1 - t0 : p.max_q));
  none(t0 + n, t1);
  if (p.parent != nullptr) {
    for (int t = tid; t < n; t += kTreeThreads) {
      const int32_t a = p.parent[t0 + t];
      up[t] = a < 0 || a >= t ? -1 : a;
    }
    __syncthreads();
  }
  for (int t = tid; t < n; t += kTreeThreads) {
    int depth = 0;
    uint64_t* row = p.mask == nullptr ? nullptr : p.mask + (t0 + t) * p.words;
    int w = t >> 6;
    if (row != nullptr)
      for (int i = w + 1; i < p.words; ++i) row[i] = 0;
    if (p.parent == nullptr) {
      depth = t;
      if (row != nullptr) {
        for (int i = 0; i < w; ++i) row[i] = ~0ull;
        row[w] = ~0ull >> (63 - (t & 63));
      }
    } else {
      uint64_t bits = 1ull << (t & 63);
      for (int a = up[t]; a >= 0; a = up[a]) {
        ++depth;
        if (row != nullptr)
          for (; w > a >> 6; --w, bits = 0) row[w] = bits;
        bits |= 1ull << (a & 63);
      }
      if (row != nullptr)
        for (; w >= 0; --w, bits = 0) row[w] = bits;
    }
    p.pos[t0 + t] = first > INT32_MAX - 1 - depth ? INT32_MAX - 1 : first + depth;
  }
}

// One wave per segment.  Lane i finds pool rows of path token i (from where
// and to where); then 16 bytes of K or V per lane (and the two exponent bytes
// in one more) go row by row.  Token i goes to row i and path[i] >= i, so no row
// is written before all that read it have: a lane moves its own bytes of every
// row, and eight rows are read before they are written.  Latency bounds it.
__global__ __launch_bounds__(kTreeThreads) void paged_accept_kernel(AcceptParams p) {
  constexpr int kBatch = 8;
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t s = (int64_t)blockIdx.x * (kTreeThreads / kWave) + threadIdx.x / kWave;
  if (s >= (int64_t)p.units * p.Hkv) return;
  const int n = (int)(s / p.Hkv);
  const int b = n % p.batch;
  const int32_t first = p.first_pos[n];
  if (first < 0) return;
  const int32_t* table = p.table + s * p.pages_per_seg;
  const int64_t room = (int64_t)p.pages_per_seg << p.page_shift;
  const int32_t given = p.n_path[b];
  int32_t at = -1, before = -1;
  if (lane < p.max_path && lane < given) {
    at = p.path[(int64_t)b * p.max_path + lane];
    if (lane > 0) before = p.path[(int64_t)b * p.max_path + lane - 1];
  }
  const bool good = at > before && at >= 0 && (int64_t)first + at < room && first < INT32_MAX - at;
  const uint64_t bad = __builtin_amdgcn_ballot_w64(!good);
  const int count = bad == 0 ? kWave : __builtin_ctzll(bad);
  // -1: nothing to read or write
  int64_t from = -1, to = -1;
  if (lane < count && at != lane) {
    const int64_t x = (int64_t)first + at, y = (int64_t)first + lane;
    const int32_t px = table[x >> p.page_shift], py = table[y >> p.page_shift];
    const int64_t in = (1 << p.page_shift) - 1;
    if (px >= 0 && px < p.num_pages && py >= 0 && py < p.num_pages) {
      from = ((int64_t)px << p.page_shift) + (x & in);
      to = ((int64_t)py << p.page_shift) + (y & in);
    }
  }
  const int per = p.row_bytes / 16;
  char* const pool = lane < per ? p.k_pages : p.v_pages;
  const int64_t off = (int64_t)(lane < per ? lane : lane - per) * 16;
  for (int i0 = 0; i0 < count; i0 += kBatch) {
    u32x4 x[kBatch];
    uint16_t e[kBatch];
    int64_t f[kBatch], d[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      f[i] = __shfl(from, (i0 + i) & (kWave - 1), kWave);
      d[i] = __shfl(to, (i0 + i) & (kWave - 1), kWave);
      if (i0 + i >= count) f[i] = -1;
      if (f[i] < 0) continue;
      if (lane < 2 * per) x[i] = *reinterpret_cast<const u32x4*>(pool + f[i] * p.row_bytes + off);
      else if (lane == 2 * per && p.scales != nullptr) e[i] = *reinterpret_cast<const uint16_t*>(p.scales + 2 * f[i]);
    }
    wave_lds_fence();  // eight rows are read before one is written
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (f[i] < 0) continue;
      if (lane < 2 * per) *reinterpret_cast<u32x4*>(pool + d[i] * p.row_bytes + off) = x[i];
      else if (lane == 2 * per && p.scales != nullptr) *reinterpret_cast<uint16_t*>(p.scales + 2 * d[i]) = e[i];
    }
  }
  const int32_t len = first + count;
  if (lane == 0 && s == (int64_t)n * p.Hkv) p.new_len[n] = len;
  if (p.keep != nullptr) {
    const int64_t pages = ((int64_t)len + (1 << p.page_shift) - 1) >> p.page_shift;
    for (int i = lane; i < p.pages_per_seg; i += kWave) p.keep[s * p.pages_per_seg + i] = i < pages ? 1 : 0;
  }
}

}  // namespace

hipError_t launch_tree_plan(const TreePlanParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(tree_plan_kernel, dim3((unsigned)p.batch + 1), dim3(kTreeThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_paged_accept(const AcceptParams& p, hipStream_t stream) {
  constexpr int kPer = kTreeThreads / kWave;
  hipLaunchKernelGGL(paged_accept_kernel, dim3((unsigned)(((int64_t)p.units * p.Hkv + kPer - 1) / kPer)),
                     dim3(kTreeThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace dkv
