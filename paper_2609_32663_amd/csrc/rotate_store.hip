// Rotary positions, and rows of K and V written into a paged cache and read
// back, in bf16 or quantised (dkv_f8.hpp).
//
// Rotation.  Pair i of a head, at position t, turns by t f_i:
//   (a, b) -> m (a cos - b sin, a sin + b cos),
// with a, b elements i and i + n of the head (half layout, n pairs) or 2i and
// 2i + 1 (interleaved); the rest of the head stays.  Angles are taken in 64
// bits: at t = 10^6 an fp32 product is off by 0.06.  The products are in 64 bits
// too, so that a result is rounded once, to fp32 (and from there to the rows'
// type): fp32 products put one bf16 result of 10^5 on the other side of a
// border, which attention then shows (outputs off by 2.3e-5 of their norm).  They
// cost nothing beside the rows' way through memory.
//
// One wave per token (or `parts` waves where tokens are few, to fill the card):
// its lanes take the sine and cosine of a pair each and exchange them through
// LDS, then walk the token's rows, eight elements per lane; an element's
// partner comes from the lane that holds it, or from memory where the pairs do
// not line up with the lanes' eight.  A row's largest magnitude is a reduction
// over its 8 or 16 lanes.  Nothing meets beyond a wave.  Moving the rows bounds
// all of it.

#include <hip/hip_runtime.h>

#include <type_traits>

#include "dkv_f8.hpp"
#include "dkv_tree.hpp"

namespace dkv {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotWaves = kRotThreads / kWave;
constexpr int kMaxPairs = 128;  // heads of up to 256 elements
constexpr int kGroups = 4;      // row groups of a wave whose loads are in flight together

// Sine and cosine in 64 bits of x >= 0 below 2^32 (about 2 ulp): x - k pi/2 by two
// fused steps, the first of them exact as x and k (pi/2 rounded to 53 bits) are
// multiples of 2^-52 that nearly cancel, then the Taylor series up to pi/4.
__device__ __forceinline__ void sincos64(double x, double* s, double* c) {
  const double k = __builtin_rint(x * 0.63661977236758134308);
  double r = __builtin_fma(-k, 1.57079632679489655800, x);
  r = __builtin_fma(-k, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double ps = 1.0 / 355687428096000.0;  // 17!
  ps = __builtin_fma(ps, z, -1.0 / 1307674368000.0);
  ps = __builtin_fma(ps, z, 1.0 / 6227020800.0);
  ps = __builtin_fma(ps, z, -1.0 / 39916800.0);
  ps = __builtin_fma(ps, z, 1.0 / 362880.0);
  ps = __builtin_fma(ps, z, -1.0 / 5040.0);
  ps = __builtin_fma(ps, z, 1.0 / 120.0);
  ps = __builtin_fma(ps, z, -1.0 / 6.0);
  const double sn = __builtin_fma(r * z, ps, r);
  double pc = 1.0 / 20922789888000.0;  // 16!
  pc = __builtin_fma(pc, z, -1.0 / 87178291200.0);
  pc = __builtin_fma(pc, z, 1.0 / 479001600.0);
  pc = __builtin_fma(pc, z, -1.0 / 3628800.0);
  pc = __builtin_fma(pc, z, 1.0 / 40320.0);
  pc = __builtin_fma(pc, z, -1.0 / 720.0);
  pc = __builtin_fma(pc, z, 1.0 / 24.0);
  pc = __builtin_fma(pc, z, -0.5);
  const double cs = __builtin_fma(z, pc, 1.0);
  const int64_t q = (int64_t)k;
  const double u = (q & 1) ? cs : sn, w = (q & 1) ? sn : cs;
  *s = (q & 2) ? -u : u;
  *c = ((q + 1) & 2) ? -w : w;
}

// Eight elements of a row as they lie in memory.
template <typename T>
struct Raw;
template <>
struct Raw<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void zero() { w = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ float at(int e) const { return (e & 1) ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]); }
  __device__ __forceinline__ void put(int e, const uint16_t* x) {
    const uint32_t b = *x;
    w[e >> 1] = (e & 1) ? (w[e >> 1] & 0xFFFFu) | b << 16 : (w[e >> 1] & 0xFFFF0000u) | b;
  }
  __device__ __forceinline__ void shuffle(const Raw& from, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__shfl((int)from.w[i], lane, kWave);
  }
};
template <>
struct Raw<float> {
  f32x4 w[2];
  __device__ __forceinline__ void zero() { w[0] = w[1] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float at(int e) const { return w[e >> 2][e & 3]; }
  __device__ __forceinline__ void put(int e, const float* x) { w[e >> 2][e & 3] = *x; }
  __device__ __forceinline__ void shuffle(const Raw& from, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = __shfl(from.w[i >> 2][i & 3], lane, kWave);
  }
};

template <typename T>
__device__ __forceinline__ void load8(Raw<T>& r, const T* at) {  // at any element
  __builtin_memcpy(&r, at, sizeof(r));
}

__device__ __forceinline__ u32x4 pack_bf16(const float (&y)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16x2_t b;
    b[0] = (__bf16)y[2 * i];
    b[1] = (__bf16)y[2 * i + 1];
    w[i] = __builtin_bit_cast(uint32_t, b);
  }
  return w;
}

// x 2^-e for the conversion: within the largest code, and NaN for what has no
// finite value.  With the largest exponent 448 2^e lies beyond bf16; what
// passes 240 2^e rounds to that.
__device__ __forceinline__ float f8_scaled(float x, float inv, float most) {
  const float y = __builtin_amdgcn_fmed3f(x * inv, -most, most);
  return __builtin_isfinite(x) ? y : __builtin_nanf("");
}

enum RowKind { kRowX, kRowK, kRowV };
enum StoreMode { kRopeOnly, kStoreBf16, kStoreF8 };

// LPR: lanes per row, 0 for any (dim / 8, at most 32).  FAR: an element's partner
// is read from memory (half layout, pairs that do not line up with lanes).
template <typename T, int MODE, int LPR, bool FAR>
__global__ __launch_bounds__(kRotThreads, 4) void rotate_store_kernel(RotateParams p) {
  __shared__ double2 trig[kRotWaves][kMaxPairs];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int64_t id = (int64_t)blockIdx.x * kRotWaves + wave;
  const int32_t t = p.parts == 1 ? (int32_t)id : (int32_t)((uint32_t)id / (uint32_t)p.parts);
  const int part = (int)(id - (int64_t)t * p.parts);
  if (t >= p.tokens) return;
  const int lpr = LPR > 0 ? LPR : p.dim / 8;
  const int per = kWave / lpr;  // rows of a group
  const int row_in = lane / lpr, c = lane - row_in * lpr;
  const int rows = p.heads + (MODE == kRopeOnly ? 0 : 2 * p.Hkv);
  const int groups = (rows + per - 1) / per;
  const int n = p.pairs, i0 = 8 * c;
  const bool turns = p.pos != nullptr;
  const int32_t at = turns ? p.pos[t] : 0;
  const char* const xt = static_cast<const char*>(p.x) + t * p.x_stride;
  const char* const kt = static_cast<const char*>(p.k) + t * p.kv_stride;
  const char* const vt = static_cast<const char*>(p.v) + t * p.kv_stride;
  // the lane that holds the partners
  const int mate = lane + (i0 < n ? n / 8 : -(n / 8));
  double cs[8], sn[8];
  bool ready = false;

  for (int g0 = part; g0 < groups; g0 += kGroups * p.parts) {
    Raw<T> x[kGroups], y[FAR ? kGroups : 1];
    int row[kGroups];
    int64_t slot[kGroups];
#pragma unroll
    for (int b = 0; b < kGroups; ++b) {
      const int g = g0 + b * p.parts;
      row[b] = g * per + row_in;
      if (g >= groups || row[b] >= rows || row_in >= per) row[b] = -1;
      x[b].zero();
      if constexpr (FAR) y[b].zero();
      slot[b] = -1;
      if (row[b] < 0) continue;
      const int h = row[b] - p.heads;
      const char* base;
      if (MODE == kRopeOnly || h < 0) {
        base = xt + (int64_t)row[b] * p.dim * sizeof(T);
      } else {
        const int kv = h < p.Hkv ? h : h - p.Hkv;
        base = (h < p.Hkv ? kt : vt) + (int64_t)kv * p.dim * sizeof(T);
        slot[b] = p.slots[(int64_t)t * p.Hkv + kv];
      }
      const T* from = reinterpret_cast<const T*>(base);
      load8(x[b], from + i0);
      if constexpr (FAR) {
        if (h >= p.Hkv) continue;
        if (i0 + 8 <= n) {
          load8(y[b], from + i0 + n);
        } else if (i0 >= n && i0 + 8 <= 2 * n) {
          load8(y[b], from + i0 - n);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int i = i0 + e;
            if (i < 2 * n) y[b].put(e, from + (i < n ? i + n : i - n));
          }
        }
      }
    }
    if (turns && !ready) {
      ready = true;
      for (int i = lane; i < n; i += kWave) {
        double s, co;
        const float f = p.freq[i];
        sincos64((double)(at < 0 ? 0 : at) * __builtin_fabs((double)f), &s, &co);
        if (f < 0.f) s = -s;
        trig[wave][i] = double2{co * p.mscale, s * p.mscale};
      }
      wave_lds_fence();
      // cosine and signed sine of the lane's elements; 1 and 0 for those that stay
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = i0 + e;
        const int pair = p.interleaved ? i >> 1 : (i < n ? i : i - n);
        const bool stays = i >= 2 * n;
        const double2 w = trig[wave][stays ? 0 : pair];
        cs[e] = stays ? 1.0 : w.x;
        sn[e] = stays ? 0.0 : ((p.interleaved ? (i & 1) != 0 : i >= n) ? w.y : -w.y);
      }
    }
    if (at < 0) return;  // a row of no sequence
    // no lane writes before the wave's loads of these rows (rotation in place)
    wave_lds_fence();
#pragma unroll
    for (int b = 0; b < kGroups; ++b) {
      if (g0 + b * p.parts >= groups) break;
      const int h = row[b] - p.heads;
      const RowKind kind = MODE == kRopeOnly || h < 0 ? kRowX : (h < p.Hkv ? kRowK : kRowV);
      float out[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = x[b].at(e);
      if (turns) {
        Raw<T> m;
        if constexpr (FAR) m = y[b];
        else if (!p.interleaved) m.shuffle(x[b], mate);
        else m = x[b];
        if (__builtin_amdgcn_ballot_w64(row[b] >= 0 && kind != kRowV)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float w = !FAR && p.interleaved ? m.at(e ^ 1) : m.at(e);
            const float r = (float)__builtin_fma((double)out[e], cs[e], (double)w * sn[e]);
            // what stays keeps its bits
            if (kind != kRowV && i0 + e < 2 * n) out[e] = r;
          }
        }
      }
      if (MODE == kRopeOnly || kind == kRowX) {
        if (row[b] >= 0) {
          T* to = reinterpret_cast<T*>(static_cast<char*>(p.out) + t * p.out_stride) + (int64_t)row[b] * p.dim + i0;
          if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4*>(to) = f32x4{out[0], out[1], out[2], out[3]};
            *reinterpret_cast<f32x4*>(to + 4) = f32x4{out[4], out[5], out[6], out[7]};
          } else {
            *reinterpret_cast<u32x4*>(to) = pack_bf16(out);
          }
        }
      }
      if constexpr (MODE == kStoreBf16) {
        if (kind != kRowX && slot[b] >= 0 && slot[b] < p.pool_rows) {
          char* pool = static_cast<char*>(kind == kRowK ? p.k_pages : p.v_pages);
          *reinterpret_cast<u32x4*>(pool + (slot[b] * p.dim + i0) * 2) = pack_bf16(out);
        }
      }
      if constexpr (MODE == kStoreF8) {
        if (__builtin_amdgcn_ballot_w64(row[b] >= 0 && kind != kRowX)) {
          float most = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) most = fmaxf(most, __builtin_isfinite(out[e]) ? __builtin_fabsf(out[e]) : 0.f);
          // the largest of the row's 8 or 16 lanes
          most = fmaxf(most, dpp_mov<0xB1>(most));
          most = fmaxf(most, dpp_mov<0x4E>(most));
          most = fmaxf(most, dpp_mov<0x141>(most));
          if (LPR == 16) most = fmaxf(most, dpp_mov<0x140>(most));
          const int ex = f8_exponent(__float_as_uint(most));
          const float inv = __uint_as_float((uint32_t)(127 - ex) << 23), lim = ex == kF8MaxExp ? 240.f : 448.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) out[e] = f8_scaled(out[e], inv, lim);
          const uint2 codes = {f8_pack4(out[0], out[1], out[2], out[3]), f8_pack4(out[4], out[5], out[6], out[7])};
          if (kind != kRowX && slot[b] >= 0 && slot[b] < p.pool_rows) {
            char* pool = static_cast<char*>(kind == kRowK ? p.k_pages : p.v_pages);
            *reinterpret_cast<uint2*>(pool + slot[b] * p.dim + i0) = codes;
            if (c == 0) p.scales[2 * slot[b] + (kind == kRowV ? 1 : 0)] = (uint8_t)(ex + 127);
          }
        }
      }
    }
  }
}

// Waves per token: a whole token to a wave where tokens fill the card, else its
// row groups over several, up to 8 waves a compute unit where that gives a token
// three, else 16: with fewer, a token's rows wait for its few waves, more take a
// second round or the sines' work again (us, up to 8 / 16 waves, 32 + 8 + 8 heads
// quantised: 400 tokens 5.1 / 5.9, 500 5.6 / 6.6, 600 6.3 / 6.7, 682 6.5 / 6.9; 683
// 7.6 / 7.2, 760 7.8 / 7.4, 850 8.2 / 7.9, 1,001 8.5 / 8.3, 1,100 12.4 / 9.6, 1,365
// 12.8 / 10.2, 1,700 13.1 / 12.1, 2,047 13.4 / 12.4; in up to 32 waves 400 tokens 6.6,
// 1,001 11.5.  bf16 rows alike; 40 heads only rotated as well, but for 850 tokens, 6.2 /
// 6.4).
constexpr int64_t kRotFew = 2048, kRotFill = 4096;

template <typename T, int MODE>
hipError_t launch_rotate(RotateParams p, hipStream_t stream) {
  const int rows = p.heads + (MODE == kRopeOnly ? 0 : 2 * p.Hkv);
  const int per = kWave / (p.dim / 8);
  const int groups = (rows + per - 1) / per;
  const int64_t few = kRotFew / p.tokens, want = few >= 3 ? few : kRotFill / p.tokens;
  p.parts = (int32_t)(want < groups ? (want > 1 ? want : 1) : groups);
  const unsigned blocks = (unsigned)(((int64_t)p.tokens * p.parts + kRotWaves - 1) / kRotWaves);
  const bool far = p.pos != nullptr && !p.interleaved && p.pairs % 8 != 0;
  const auto launch = [&](auto lpr) {
    constexpr int L = decltype(lpr)::value;
    if (far) hipLaunchKernelGGL((rotate_store_kernel<T, MODE, L, true>), dim3(blocks), dim3(kRotThreads), 0, stream, p);
    else hipLaunchKernelGGL((rotate_store_kernel<T, MODE, L, false>), dim3(blocks), dim3(kRotThreads), 0, stream, p);
  };
  if (p.dim == 128) launch(std::integral_constant<int, 16>{});
  else if (p.dim == 64) launch(std::integral_constant<int, 8>{});
  else if constexpr (MODE == kRopeOnly) launch(std::integral_constant<int, 0>{});
  return hipGetLastError();
}

// ---------------------------------------------------------------- read back
// Eight elements of a K and of a V row per thread, so that a wave writes whole
// lines, rows of one token side by side.  Bound by moving the rows; results that
// the 256 MB last-level cache cannot hold for whoever reads them next are written
// past it (a context of 131,072 tokens, 8 heads, 816 MB moved: 146 us, 160 through it,
// 5.6 and 5.1 TB/s; 16 codes a thread, whose stores then leave lines in halves, 160
// and 239).
constexpr int64_t kLoadCachedBytes = 256 << 20;

template <bool F8, bool NT>
__global__ __launch_bounds__(kRotThreads) void paged_load_kernel(LoadParams p) {
  const int per_row = p.dim / 8;  // a power of two
  const int shift = 31 - __builtin_clz(per_row);
  const int64_t i = (int64_t)blockIdx.x * kRotThreads + threadIdx.x;
  const int64_t r = i >> shift;  // token * Hkv + head
  if (r >= (int64_t)p.tokens * p.Hkv) return;
  const int64_t slot = p.slots[r];
  if (slot < 0 || slot >= p.pool_rows) return;
  const int c = (int)(i & (per_row - 1));
  const uint32_t t = (uint32_t)r / (uint32_t)p.Hkv;
  const int64_t to = t * p.stride + ((r - (int64_t)t * p.Hkv) * p.dim + c * 8) * 2;
  const int64_t from = (slot * p.dim + c * 8) * (F8 ? 1 : 2);
  const char* const kp = static_cast<const char*>(p.k_pages) + from;
  const char* const vp = static_cast<const char*>(p.v_pages) + from;
  u32x4 k, v;
  if constexpr (F8) {
    const uint2 kc = *reinterpret_cast<const uint2*>(kp), vc = *reinterpret_cast<const uint2*>(vp);
    const uint32_t ex = *reinterpret_cast<const uint16_t*>(p.scales + 2 * slot);
    const float ke = f8_power(ex & 0xFF), ve = f8_power(ex >> 8);
    k = u32x4{f8_pair<false>(kc.x, ke), f8_pair<true>(kc.x, ke), f8_pair<false>(kc.y, ke), f8_pair<true>(kc.y, ke)};
    v = u32x4{f8_pair<false>(vc.x, ve), f8_pair<true>(vc.x, ve), f8_pair<false>(vc.y, ve), f8_pair<true>(vc.y, ve)};
  } else {
    k = *reinterpret_cast<const u32x4*>(kp);
    v = *reinterpret_cast<const u32x4*>(vp);
  }
  u32x4* const ko = reinterpret_cast<u32x4*>(static_cast<char*>(p.k_out) + to);
  u32x4* const vo = reinterpret_cast<u32x4*>(static_cast<char*>(p.v_out) + to);
  if constexpr (NT) {
    __builtin_nontemporal_store(k, ko);
    __builtin_nontemporal_store(v, vo);
  } else {
    *ko = k;
    *vo = v;
  }
}

}  // namespace

hipError_t launch_rope(const RotateParams& p, bool f32, hipStream_t stream) {
  return f32 ? launch_rotate<float, kRopeOnly>(p, stream) : launch_rotate<uint16_t, kRopeOnly>(p, stream);
}

hipError_t launch_paged_store(const RotateParams& p, bool f8, hipStream_t stream) {
  return f8 ? launch_rotate<uint16_t, kStoreF8>(p, stream) : launch_rotate<uint16_t, kStoreBf16>(p, stream);
}

hipError_t launch_paged_load(const LoadParams& p, bool f8, hipStream_t stream) {
  const int64_t n = (int64_t)p.tokens * p.Hkv * (p.dim / 8);
  const dim3 grid((unsigned)((n + kRotThreads - 1) / kRotThreads)), block(kRotThreads);
  const bool once = n * 32 > kLoadCachedBytes;
  if (f8 && once) hipLaunchKernelGGL((paged_load_kernel<true, true>), grid, block, 0, stream, p);
  else if (f8) hipLaunchKernelGGL((paged_load_kernel<true, false>), grid, block, 0, stream, p);
  else if (once) hipLaunchKernelGGL((paged_load_kernel<false, true>), grid, block, 0, stream, p);
  else hipLaunchKernelGGL((paged_load_kernel<false, false>), grid, block, 0, stream, p);
  return hipGetLastError();
}

}  // namespace dkv
