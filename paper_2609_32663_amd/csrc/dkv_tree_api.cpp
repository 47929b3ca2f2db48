// C-ABI entry points of rotary positions, quantised cache rows and drafted
// trees (see include/dkv.h).  Every argument is checked on the host before
// anything is enqueued.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "dkv_launch.hpp"
#include "dkv_query.hpp"
#include "dkv_tree.hpp"

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether [a, a + na) and [b, b + nb) share a byte.
bool overlap(const void* a, uint64_t na, const void* b, uint64_t nb) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a != nullptr && b != nullptr && (x <= y ? y - x < na : x - y < nb) && na > 0 && nb > 0;
}

dkv_status hip_status(hipError_t e) { return e == hipSuccess ? DKV_OK : DKV_ERR_HIP; }

bool page_rows_ok(int32_t pr) {
  return pr == 32 || pr == 64 || pr == 128 || pr == 256 || pr == 512 || pr == 1024;
}

bool format_ok(dkv_cache_format f) { return f == DKV_CACHE_BF16 || f == DKV_CACHE_F8; }

// Rows of `heads` x dim elements, tokens `stride` elements apart.
bool stride_ok(int64_t stride, int64_t heads, int32_t dim) { return stride >= heads * dim && stride <= INT32_MAX; }

dkv_status check_tree(int32_t batch, int32_t hq, int32_t hkv, int32_t d, int32_t num_tokens, int32_t max_q) {
  if (batch < 0 || hq <= 0 || hkv <= 0 || hq % hkv != 0 || num_tokens < 0 || max_q < 0) return DKV_ERR_INVALID_ARG;
  if (hq / hkv > DKV_MAX_GROUP || (d != 64 && d != 128)) return DKV_ERR_UNSUPPORTED;
  if ((int64_t)batch * hkv > DKV_MAX_SEGMENTS) return DKV_ERR_UNSUPPORTED;
  // query rows per segment must fit 31 bits, workgroups of 512 threads 32 bits of work-items
  const int64_t rows = (int64_t)(max_q < num_tokens ? max_q : num_tokens) * (hq / hkv);
  if (rows > INT32_MAX / 2) return DKV_ERR_UNSUPPORTED;
  if ((rows + dkv::kQueryRowsPerWG - 1) / dkv::kQueryRowsPerWG * batch * hkv > 0xFFFFFFFFLL / 512)
    return DKV_ERR_UNSUPPORTED;
  return DKV_OK;
}

}  // namespace

extern "C" {

dkv_status dkv_rope_freqs(dkv_rope_scaling kind, int32_t rot_dim, double base, double factor, double trained_len,
                          double low, double high, float* inv_freq, float* mscale) {
  if (rot_dim <= 0 || rot_dim % 2 != 0 || inv_freq == nullptr || mscale == nullptr) return DKV_ERR_INVALID_ARG;
  if (!std::isfinite(base) || base <= 1.0) return DKV_ERR_INVALID_ARG;
  if (kind != DKV_ROPE_PLAIN && kind != DKV_ROPE_LINEAR && kind != DKV_ROPE_BASE && kind != DKV_ROPE_WAVE &&
      kind != DKV_ROPE_RAMP)
    return DKV_ERR_INVALID_ARG;
  if (kind != DKV_ROPE_PLAIN && (!std::isfinite(factor) || factor < 1.0)) return DKV_ERR_INVALID_ARG;
  const bool bands = kind == DKV_ROPE_WAVE || kind == DKV_ROPE_RAMP;
  if (bands && (!std::isfinite(trained_len) || trained_len <= 0.0 || !std::isfinite(low) || !std::isfinite(high) ||
                low <= 0.0 || high <= low))
    return DKV_ERR_INVALID_ARG;
  if (kind == DKV_ROPE_BASE && rot_dim <= 2) return DKV_ERR_INVALID_ARG;
  const int32_t n = rot_dim / 2;
  const double pi = 3.14159265358979323846;
  // DKV_ROPE_BASE: the slowest pair turns `factor` times slower, the fastest as before
  const double b = kind == DKV_ROPE_BASE ? base * std::pow(factor, (double)rot_dim / (rot_dim - 2)) : base;
  double first = 0.0, last = 1.0;  // DKV_ROPE_RAMP: pairs between which the division sets in
  if (kind == DKV_ROPE_RAMP) {
    // the pair that turns t times over the trained length
    const auto pair = [&](double t) { return rot_dim * std::log(trained_len / (2 * pi * t)) / (2 * std::log(base)); };
    // Cut to a head's indexes before the slope is taken (a fastest pair that turns fewer than `high` times over a short
    // length stays as it was).
    first = std::fmax(std::floor(pair(high)), 0.0);
    last = std::fmin(std::ceil(pair(low)), rot_dim - 1.0);
  }
  for (int32_t i = 0; i < n; ++i) {
    const double f = std::pow(b, -(double)i / n);
    double g = f;
    if (kind == DKV_ROPE_LINEAR) g = f / factor;
    if (bands) {
      double keep;  // how much of the pair stays as trained
      if (kind == DKV_ROPE_WAVE) keep = (trained_len * f / (2 * pi) - low) / (high - low);  // by its turns
      else if (last > first) keep = 1.0 - (i - first) / (last - first);
      else keep = i <= last ? 1.0 : 0.0;  // the band lies beyond the indexes
      keep = std::fmin(std::fmax(keep, 0.0), 1.0);
      g = keep * f + (1.0 - keep) * f / factor;
    }
    inv_freq[i] = (float)g;
  }
  *mscale = kind == DKV_ROPE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return DKV_OK;
}

dkv_status dkv_rope(dkv_dtype dtype, int32_t num_tokens, int32_t num_heads, int32_t head_dim, const void* x,
                    int64_t x_stride, const int32_t* pos, const float* inv_freq, int32_t rot_dim, int32_t interleaved,
                    float mscale, void* out, int64_t out_stride, void* stream) {
  if (dtype != DKV_BF16 && dtype != DKV_F32) return DKV_ERR_INVALID_ARG;
  if (num_tokens < 0 || num_heads <= 0 || rot_dim <= 0 || rot_dim > head_dim || rot_dim % 2 != 0 || !std::isfinite(mscale))
    return DKV_ERR_INVALID_ARG;
  if (head_dim <= 0 || head_dim % 8 != 0 || head_dim > 256) return DKV_ERR_UNSUPPORTED;
  if (!stride_ok(x_stride, num_heads, head_dim) || !stride_ok(out_stride, num_heads, head_dim)) return DKV_ERR_INVALID_ARG;
  // four waves of 64 per workgroup, a wave per row at most
  if ((int64_t)num_tokens * num_heads > 0xFFFFFFFFLL / 256) return DKV_ERR_UNSUPPORTED;
  if (num_tokens == 0) return DKV_OK;
  if (x == nullptr || out == nullptr || pos == nullptr || inv_freq == nullptr) return DKV_ERR_INVALID_ARG;
  const int32_t elem = dtype == DKV_BF16 ? 2 : 4;
  if (!aligned16(x) || !aligned16(out) || x_stride * elem % 16 != 0 || out_stride * elem % 16 != 0)
    return DKV_ERR_MISALIGNED;
  dkv::RotateParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = x;
  p.out = out;
  p.pos = pos;
  p.freq = inv_freq;
  p.x_stride = x_stride * elem;
  p.out_stride = out_stride * elem;
  p.tokens = num_tokens;
  p.heads = num_heads;
  p.dim = head_dim;
  p.pairs = rot_dim / 2;
  p.interleaved = interleaved != 0;
  p.mscale = mscale;
  return hip_status(dkv::launch_rope(p, dtype == DKV_F32, (hipStream_t)stream));
}

dkv_status dkv_paged_store(dkv_cache_format format, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                           int32_t head_dim, const void* q, int64_t q_stride, const void* k_new, const void* v_new,
                           int64_t kv_stride, const int32_t* pos, const float* inv_freq, int32_t rot_dim,
                           int32_t interleaved, float mscale, void* q_out, int64_t q_out_stride, const int64_t* slots,
                           void* k_pages, void* v_pages, uint8_t* scales, int64_t num_pages, int32_t page_rows,
                           void* stream) {
  if (!format_ok(format)) return DKV_ERR_INVALID_ARG;
  if (num_tokens < 0 || num_q_heads < 0 || num_kv_heads <= 0 || num_pages < 0 || rot_dim < 0 || rot_dim > head_dim ||
      rot_dim % 2 != 0 || !std::isfinite(mscale))
    return DKV_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return DKV_ERR_UNSUPPORTED;
  if (!page_rows_ok(page_rows) || num_pages > INT32_MAX) return DKV_ERR_UNSUPPORTED;
  if (num_q_heads > 65536 || num_kv_heads > 65536) return DKV_ERR_UNSUPPORTED;
  if (!stride_ok(kv_stride, num_kv_heads, head_dim)) return DKV_ERR_INVALID_ARG;
  if (num_q_heads > 0 &&
      (!stride_ok(q_stride, num_q_heads, head_dim) || !stride_ok(q_out_stride, num_q_heads, head_dim)))
    return DKV_ERR_INVALID_ARG;
  if ((int64_t)num_tokens * ((int64_t)num_q_heads + 2 * (int64_t)num_kv_heads) > 0xFFFFFFFFLL / 256)
    return DKV_ERR_UNSUPPORTED;
  if (num_tokens == 0) return DKV_OK;
  if (k_new == nullptr || v_new == nullptr || slots == nullptr) return DKV_ERR_INVALID_ARG;
  if (num_pages > 0 && (k_pages == nullptr || v_pages == nullptr || (format == DKV_CACHE_F8 && scales == nullptr)))
    return DKV_ERR_INVALID_ARG;
  if (num_q_heads > 0 && (q == nullptr || q_out == nullptr)) return DKV_ERR_INVALID_ARG;
  if (rot_dim > 0 && (pos == nullptr || inv_freq == nullptr)) return DKV_ERR_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || kv_stride % 8 != 0 || !aligned16(k_pages) || !aligned16(v_pages) ||
      !aligned(slots, 8) || (format == DKV_CACHE_F8 && !aligned16(scales)))
    return DKV_ERR_MISALIGNED;
  if (num_q_heads > 0 && (!aligned16(q) || !aligned16(q_out) || q_stride % 8 != 0 || q_out_stride % 8 != 0))
    return DKV_ERR_MISALIGNED;
  dkv::RotateParams p;
  std::memset(&p, 0, sizeof(p));
  p.x = q;
  p.out = q_out;
  p.k = k_new;
  p.v = v_new;
  p.pos = rot_dim > 0 ? pos : nullptr;
  p.freq = inv_freq;
  p.slots = slots;
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.scales = scales;
  p.x_stride = q_stride * 2;
  p.out_stride = q_out_stride * 2;
  p.kv_stride = kv_stride * 2;
  p.pool_rows = num_pages * page_rows;
  p.tokens = num_tokens;
  p.heads = num_q_heads;
  p.Hkv = num_kv_heads;
  p.dim = head_dim;
  p.pairs = rot_dim / 2;
  p.interleaved = interleaved != 0;
  p.mscale = mscale;
  return hip_status(dkv::launch_paged_store(p, format == DKV_CACHE_F8, (hipStream_t)stream));
}

dkv_status dkv_paged_load(dkv_cache_format format, int32_t num_tokens, int32_t num_kv_heads, int32_t head_dim,
                          const void* k_pages, const void* v_pages, const uint8_t* scales, int64_t num_pages,
                          int32_t page_rows, const int64_t* slots, void* k_out, void* v_out, int64_t token_stride,
                          void* stream) {
  if (!format_ok(format)) return DKV_ERR_INVALID_ARG;
  if (num_tokens < 0 || num_kv_heads <= 0 || num_pages < 0) return DKV_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return DKV_ERR_UNSUPPORTED;
  if (!page_rows_ok(page_rows) || num_pages > INT32_MAX) return DKV_ERR_UNSUPPORTED;
  if (!stride_ok(token_stride, num_kv_heads, head_dim)) return DKV_ERR_INVALID_ARG;
  // one work-item per 16 bytes of a token's K rows, at most 16 a row
  if ((int64_t)num_tokens * num_kv_heads > (0xFFFFFFFFLL - 255) / 16) return DKV_ERR_UNSUPPORTED;
  if (num_tokens == 0 || num_pages == 0) return DKV_OK;
  if (k_pages == nullptr || v_pages == nullptr || slots == nullptr || k_out == nullptr || v_out == nullptr ||
      (format == DKV_CACHE_F8 && scales == nullptr))
    return DKV_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_out) || !aligned16(v_out) || token_stride % 8 != 0 ||
      !aligned(slots, 8) || (format == DKV_CACHE_F8 && !aligned16(scales)))
    return DKV_ERR_MISALIGNED;
  dkv::LoadParams p;
  std::memset(&p, 0, sizeof(p));
  p.k_pages = k_pages;
  p.v_pages = v_pages;
  p.scales = scales;
  p.slots = slots;
  p.k_out = k_out;
  p.v_out = v_out;
  p.pool_rows = num_pages * page_rows;
  p.stride = token_stride * 2;
  p.tokens = num_tokens;
  p.Hkv = num_kv_heads;
  p.dim = head_dim;
  return hip_status(dkv::launch_paged_load(p, format == DKV_CACHE_F8, (hipStream_t)stream));
}

dkv_status dkv_tree_plan(int32_t batch, int32_t num_tokens, int32_t max_q, const int32_t* tok_off,
                         const int32_t* first_pos, const int32_t* parent, int32_t* pos, uint64_t* mask,
                         int32_t mask_words, void* stream) {
  if (batch < 0 || num_tokens < 0 || max_q < 0 || mask_words < 0) return DKV_ERR_INVALID_ARG;
  const int32_t longest = max_q < num_tokens ? max_q : num_tokens;
  if (parent != nullptr && longest > DKV_MAX_TREE) return DKV_ERR_UNSUPPORTED;
  if (batch > DKV_MAX_SEGMENTS) return DKV_ERR_UNSUPPORTED;
  if (mask != nullptr && (int64_t)mask_words * 64 < longest) return DKV_ERR_INVALID_ARG;
  if (num_tokens == 0) return DKV_OK;
  if (tok_off == nullptr || pos == nullptr || (batch > 0 && first_pos == nullptr)) return DKV_ERR_INVALID_ARG;
  if (!aligned(mask, 8)) return DKV_ERR_MISALIGNED;
  // A sequence's workgroup writes its rows while others still read offsets and parents; its own parents it has read.
  const uint64_t tokens = 4 * (uint64_t)num_tokens, bits = 8 * (uint64_t)num_tokens * mask_words;
  const struct { const void* p; uint64_t n; } read[] = {
      {tok_off, 4 * ((uint64_t)batch + 1)}, {first_pos, 4 * (uint64_t)batch}, {parent, tokens}};
  for (const auto& in : read)
    if ((pos != in.p && overlap(pos, tokens, in.p, in.n)) || overlap(mask, bits, in.p, in.n)) return DKV_ERR_INVALID_ARG;
  if (pos == tok_off || pos == first_pos || overlap(pos, tokens, mask, bits)) return DKV_ERR_INVALID_ARG;
  dkv::TreePlanParams p;
  std::memset(&p, 0, sizeof(p));
  p.tok_off = tok_off;
  p.first_pos = first_pos;
  p.parent = parent;
  p.pos = pos;
  p.mask = mask;
  p.batch = batch;
  p.tokens = num_tokens;
  p.max_q = max_q;
  p.words = mask_words;
  return hip_status(dkv::launch_tree_plan(p, (hipStream_t)stream));
}

size_t dkv_paged_tree_workspace_bytes(dkv_cache_format format, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                      int32_t head_dim, int32_t num_tokens, int32_t max_q, int64_t rows_hint) {
  if (!format_ok(format) || check_tree(batch, num_q_heads, num_kv_heads, head_dim, num_tokens, max_q) != DKV_OK) return 0;
  if (batch == 0 || num_tokens == 0 || max_q == 0) return 0;
  const dkv::PagedPlanShape sh =
      dkv::paged_plan_shape(batch, num_kv_heads, num_q_heads / num_kv_heads, head_dim, num_tokens,
                            max_q < num_tokens ? max_q : num_tokens, rows_hint, format == DKV_CACHE_F8);
  return sh.plan_bytes + sh.rec_bytes;
}

dkv_status dkv_paged_tree_attn(dkv_cache_format format, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                               int32_t head_dim, int32_t num_tokens, int32_t max_q, const void* q, int64_t q_stride,
                               const int32_t* tok_off, const int32_t* first_pos, const uint64_t* mask, int32_t mask_words,
                               const void* k_pages, const void* v_pages, const uint8_t* scales, int64_t num_pages,
                               int32_t page_rows, const int32_t* entries, const int32_t* n_entries, int32_t max_entries,
                               float sm_scale, int64_t rows_hint, float* out, void* workspace, size_t workspace_bytes,
                               void* stream) {
  if (!format_ok(format)) return DKV_ERR_INVALID_ARG;
  const dkv_status st = check_tree(batch, num_q_heads, num_kv_heads, head_dim, num_tokens, max_q);
  if (st != DKV_OK) return st;
  if (!dkv::scale_in_range(sm_scale) || num_pages < 0 || max_entries < 0 || mask_words < 0) return DKV_ERR_INVALID_ARG;
  if (!page_rows_ok(page_rows)) return DKV_ERR_UNSUPPORTED;
  // the row space of a segment is walked with 32-bit rows, a mask row with 32-bit words
  if (num_pages > INT32_MAX || (int64_t)max_entries * page_rows > (int64_t)1 << 30 || mask_words > 1 << 20)
    return DKV_ERR_UNSUPPORTED;
  if (q_stride < (int64_t)num_q_heads * head_dim || q_stride > INT32_MAX) return DKV_ERR_INVALID_ARG;
  if (batch == 0 || num_tokens == 0 || max_q == 0) return DKV_OK;
  if (q == nullptr || tok_off == nullptr || first_pos == nullptr || n_entries == nullptr || out == nullptr ||
      (num_pages > 0 && (k_pages == nullptr || v_pages == nullptr)) || (max_entries > 0 && entries == nullptr) ||
      (format == DKV_CACHE_F8 && scales == nullptr))
    return DKV_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || !aligned16(entries) ||
      q_stride % 8 != 0 || !aligned(mask, 8) || (format == DKV_CACHE_F8 && !aligned16(scales)))
    return DKV_ERR_MISALIGNED;
  const dkv::PagedPlanShape sh =
      dkv::paged_plan_shape(batch, num_kv_heads, num_q_heads / num_kv_heads, head_dim, num_tokens,
                            max_q < num_tokens ? max_q : num_tokens, rows_hint, format == DKV_CACHE_F8);
  const size_t need = sh.plan_bytes + sh.rec_bytes;
  if (need > 0 && (workspace == nullptr || !aligned16(workspace) || workspace_bytes < need)) return DKV_ERR_WORKSPACE;

  dkv::QueryParams p;
  std::memset(&p, 0, sizeof(p));
  p.q = q;
  p.k = k_pages;
  p.v = v_pages;
  p.nseg = batch * num_kv_heads;
  p.Hkv = num_kv_heads;
  p.Hq = num_q_heads;
  p.G = num_q_heads / num_kv_heads;
  p.max_q = max_q < num_tokens ? max_q : num_tokens;
  p.rows = p.max_q * p.G;
  p.qtiles = (p.rows + dkv::kQueryRowsPerWG - 1) / dkv::kQueryRowsPerWG;
  p.scale_log2 = sm_scale * 1.4426950408889634f;
  p.out = out;
  p.tok_off = tok_off;
  p.first_pos = first_pos;
  p.entries = entries;
  p.n_entries = n_entries;
  p.num_pages = num_pages;
  p.q_stride = q_stride * 2;
  p.max_entries = max_entries;
  p.page_shift = __builtin_ctz((unsigned)page_rows);
  p.num_tokens = num_tokens;
  p.mask = mask;
  p.mask_words = mask_words;
  p.scales = format == DKV_CACHE_F8 ? scales : nullptr;
  if (sh.shorts) {
    const int64_t row_bytes = (int64_t)head_dim * (format == DKV_CACHE_F8 ? 2 : 4);  // of K and V
    p.stream_once = rows_hint <= 0 || rows_hint > dkv::kShortCachedBytes / row_bytes;
    p.P = sh.slices;
    p.rec_rows = sh.rec_rows;
    p.seg_meta = static_cast<int32_t*>(workspace);
    p.rec = reinterpret_cast<float*>(static_cast<char*>(workspace) + sh.plan_bytes);
    return hip_status(dkv::launch_paged_tree_short(p, head_dim, (hipStream_t)stream));
  }
  if (sh.slices > 0) {
    p.P = sh.slices;
    p.max_items = (int32_t)sh.units;
    p.plan = static_cast<int32_t*>(workspace);
    p.rec = reinterpret_cast<float*>(static_cast<char*>(workspace) + sh.plan_bytes);
  }
  return hip_status(dkv::launch_paged_tree_attn(p, head_dim, (hipStream_t)stream));
}

dkv_status dkv_paged_accept(dkv_cache_format format, int32_t num_units, int32_t batch, int32_t num_kv_heads,
                            int32_t head_dim, const int32_t* first_pos, const int32_t* path, const int32_t* n_path,
                            int32_t max_path, const int32_t* page_table, int32_t pages_per_seg, int32_t page_rows,
                            void* k_pages, void* v_pages, uint8_t* scales, int64_t num_pages, int32_t* new_len,
                            uint8_t* keep, void* stream) {
  if (!format_ok(format)) return DKV_ERR_INVALID_ARG;
  if (num_units < 0 || batch < 0 || num_kv_heads <= 0 || max_path < 0 || pages_per_seg < 0 || num_pages < 0)
    return DKV_ERR_INVALID_ARG;
  if (num_units > 0 && (batch == 0 || num_units % batch != 0)) return DKV_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return DKV_ERR_UNSUPPORTED;
  if (!page_rows_ok(page_rows) || num_pages > INT32_MAX) return DKV_ERR_UNSUPPORTED;
  if (max_path > DKV_MAX_PATH || (int64_t)num_units * num_kv_heads > 65535) return DKV_ERR_UNSUPPORTED;
  if (num_units == 0) return DKV_OK;
  if (first_pos == nullptr || n_path == nullptr || new_len == nullptr || (max_path > 0 && path == nullptr) ||
      (pages_per_seg > 0 && page_table == nullptr))
    return DKV_ERR_INVALID_ARG;
  if (num_pages > 0 && (k_pages == nullptr || v_pages == nullptr || (format == DKV_CACHE_F8 && scales == nullptr)))
    return DKV_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(v_pages) || (format == DKV_CACHE_F8 && !aligned16(scales)))
    return DKV_ERR_MISALIGNED;
  // A unit's first segment writes new_len, and every segment its own row of keep, while others still read the
  // lengths, paths and tables.
  const uint64_t units = 4 * (uint64_t)num_units, cells = (uint64_t)num_units * num_kv_heads * pages_per_seg;
  const struct { const void* p; uint64_t n; } read[] = {
      {first_pos, units}, {path, 4 * (uint64_t)batch * max_path}, {n_path, 4 * (uint64_t)batch}, {page_table, 4 * cells}};
  for (const auto& in : read)
    if (overlap(new_len, units, in.p, in.n) || overlap(keep, cells, in.p, in.n)) return DKV_ERR_INVALID_ARG;
  if (overlap(new_len, units, keep, cells)) return DKV_ERR_INVALID_ARG;
  dkv::AcceptParams p;
  std::memset(&p, 0, sizeof(p));
  p.first_pos = first_pos;
  p.path = path;
  p.n_path = n_path;
  p.table = page_table;
  p.k_pages = static_cast<char*>(k_pages);
  p.v_pages = static_cast<char*>(v_pages);
  p.scales = format == DKV_CACHE_F8 ? scales : nullptr;
  p.new_len = new_len;
  p.keep = keep;
  p.num_pages = num_pages;
  p.units = num_units;
  p.batch = batch;
  p.Hkv = num_kv_heads;
  p.max_path = max_path;
  p.pages_per_seg = pages_per_seg;
  p.page_shift = __builtin_ctz((unsigned)page_rows);
  p.row_bytes = head_dim * (format == DKV_CACHE_F8 ? 1 : 2);
  return hip_status(dkv::launch_paged_accept(p, (hipStream_t)stream));
}

}  // extern "C"
