/*
 * dkv.h -- C ABI of the Distance-KV inference hot path on MI355X (gfx950).
 *
 * Distance-KV keeps a static binary pattern M[layer][query head][distance bin]
 * (Sec. 3.2).  At inference the pattern is mapped to token positions measured
 * from the end of the context (Sec. 3.4, Eq. (4) and Eq. (5)), query heads that
 * share a KV head are combined by union (last paragraph of Sec. 3.4), the KV
 * cache is pruned and packed once in original token order, new tokens are
 * appended and always kept, and decode attends to the packed cache (Sec. 3.4).
 * This library runs those four steps on one GPU:
 *
 *   dkv_map_pattern   pattern -> per-KV-head keep masks and retained lengths
 *                     (dkv_map_pattern_ragged: contexts of different lengths)
 *   dkv_compact       dense K/V + keep mask -> packed K/V, offsets, lengths
 *                     (dkv_compact_bins: map and pack from the pattern in one
 *                     call, whole retained bins copied as blocks;
 *                     dkv_compact_bins_ragged: contexts of different lengths)
 *   dkv_append        new tokens -> free rows after each packed segment
 *   dkv_decode_attn   one decode step of attention over the packed segments
 *   dkv_query_attn    the query block after the context: attention over the
 *                     packed segments plus the block itself, causally
 *   dkv_page_select   zero-copy alternative to the pack: the retained runs
 *                     of a paged cache, listed in place
 *   dkv_paged_decode_attn  decode over a paged cache through those entries
 *   dkv_page_extend   page tables, slots and entries of growing requests, built
 *                     from their lengths (dkv_page_release: pages back)
 *   dkv_paged_append  new tokens -> their slots in the pages
 *   dkv_paged_query_attn  a chunk of new tokens of every sequence over a paged
 *                     cache, causally
 *   dkv_rope          rotary positions (dkv_rope_freqs: their frequencies)
 *   dkv_paged_store   new tokens into a paged cache of bf16 or 8-bit rows, with
 *                     their rotation (dkv_paged_load: rows back in bf16)
 *   dkv_tree_plan     positions and ancestors of drafted trees
 *   dkv_paged_tree_attn  trees, chunks and single tokens over a paged cache of
 *                     bf16 or 8-bit rows
 *   dkv_paged_accept  the accepted path of a tree kept in the cache
 *   dkv_topk_pattern  the exact-budget export of a pattern from retention
 *                     probabilities (K_rho largest entries)
 *
 * plus dkv_dense_decode_attn, the same attention kernel over an uncompressed
 * cache (the "Dense" comparator of Sec. 4.3).
 *
 * Conventions shared by every call
 * --------------------------------
 * - Pointers are DEVICE pointers unless marked (host).  The caller allocates
 *   and owns every buffer, including workspaces; the library allocates and
 *   frees nothing and keeps no state between calls.
 * - Every call only enqueues work on `stream` (a hipStream_t; NULL is the
 *   default stream) and returns without synchronising.  Buffers must stay
 *   alive until the stream has executed the work.  Calls are re-entrant;
 *   two calls that share an output or a workspace must be ordered by the
 *   caller.
 * - Arguments are checked on the host before anything is enqueued; on any
 *   error nothing is enqueued and the status says why.  DKV_ERR_HIP means the
 *   HIP runtime refused a launch.  Faults inside a kernel surface at the
 *   caller's next synchronisation.
 * - Positions are 0-indexed: position j of a context of length T has
 *   distance delta = T - 1 - j from the last context token.  (Eq. (4) is
 *   written for 1-indexed i = j + 1; with S = 128, R = 1024 and 128-token
 *   bins both give the paper's D = 1013 bins at T = 130,816.)
 * - Query head h belongs to KV head h / G, G = num_q_heads / num_kv_heads.
 * - Element types: DKV_BF16 (K, V, q as bfloat16) or DKV_F32.  Attention
 *   accumulates in fp32 and writes fp32.  head_dim is 64 or 128.  Row and
 *   base pointers of K, V, q, out and packed buffers must be 16-byte aligned.
 * - Sizes: N = num_units (independent (layer, sequence) units),
 *   Hq / Hkv heads, d = head_dim, T = context_len, D = num_bins.
 */
#ifndef DKV_H
#define DKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dkv_status {
  DKV_OK = 0,
  DKV_ERR_INVALID_ARG = 1, /* null pointer, negative or inconsistent size, bad bin edges */
  DKV_ERR_UNSUPPORTED = 2, /* head_dim, group size, bin count or segment count beyond limits */
  DKV_ERR_MISALIGNED = 3,  /* a K/V/q/out/packed pointer is not 16-byte aligned */
  DKV_ERR_CAPACITY = 4,    /* n_tail + n_new exceeds the free rows reserved per segment */
  DKV_ERR_WORKSPACE = 5,   /* workspace missing or smaller than the query function says */
  DKV_ERR_HIP = 6          /* the HIP runtime refused to launch a kernel */
} dkv_status;

typedef enum dkv_dtype { DKV_BF16 = 0, DKV_F32 = 1 } dkv_dtype;

/* Limits (checked; larger values return DKV_ERR_UNSUPPORTED). */
#define DKV_MAX_GROUP 16            /* Hq / Hkv */
#define DKV_MAX_GENERAL_BINS 512    /* bins with arbitrary edges */
#define DKV_MAX_UNIFORM_BINS 16384  /* bins with edges E[k] = W k */
#define DKV_MAX_SEGMENTS 2048       /* batch * num_kv_heads in one decode call */

/*
 * Shape of a pattern-mapping / compaction call (host struct).
 *
 * bin_edges (host) holds D + 1 offsets E[0] = 0 < E[1] < ... < E[D].  A
 * position that is neither sink (j < sink) nor recent (delta < recent) has
 * offset u = delta - recent past the recent window and lies in bin k when
 * E[k] <= u < E[k+1] (Eq. (4); the paper's layout is sink = 128,
 * recent = 1024, E[k] = 128 k).  Positions with u >= E[D] lie in no bin and
 * are pruned: only bins the context covers are instantiated (Sec. 3.4).
 */
typedef struct dkv_layout {
  int32_t num_units;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t context_len;
  int32_t sink;
  int32_t recent;
  int32_t num_bins;
  const int32_t *bin_edges;
} dkv_layout;

/*
 * dkv_map_pattern -- Eq. (5) of Sec. 3.4, then the GQA union.
 *
 * pattern  uint8 [N][Hq][D]; nonzero = bin retained for that query head.
 * kv_mask  out, uint8 [N][Hkv][T]; 1 where any query head of the group keeps
 *          the position (sink and recent positions are always 1), else 0.
 * kv_len   out, int32 [N][Hkv]; number of ones in each kv_mask row.
 * q_mask   out, optional (NULL to skip), uint8 [N][Hq][T]: the per-query-head
 *          logical decision m[l,h,j] of Eq. (5).
 * Limits: D <= DKV_MAX_GENERAL_BINS, or D <= DKV_MAX_UNIFORM_BINS when the
 * edges are uniform.  kv_mask and q_mask must be 16-byte aligned; with
 * context_len = 0 they are not written and may be NULL.
 */
dkv_status dkv_map_pattern(const dkv_layout *layout, const uint8_t *pattern,
                           uint8_t *kv_mask, int32_t *kv_len, uint8_t *q_mask,
                           void *stream);

/*
 * dkv_map_pattern_ragged -- dkv_map_pattern for a batch of contexts of
 * different lengths (e.g. sequences of a serving batch).
 *
 * unit_len  int32 [N] (device): unit n's context is the first unit_len[n]
 *           positions of its mask row (values are clamped to
 *           [0, context_len]).  Eq. (4) and Eq. (5) are applied with that
 *           length: distances count from the end of the unit's own context,
 *           so its sink, recent window and bins move with it, and positions
 *           at or past unit_len[n] are not retained.
 * layout->context_len is the row length of kv_mask, q_mask and the dense
 * cache handed to dkv_compact (the longest context).  Everything else as
 * dkv_map_pattern; packing, append and decode need no change, since they
 * follow the masks and lengths.
 */
dkv_status dkv_map_pattern_ragged(const dkv_layout *layout, const int32_t *unit_len,
                                  const uint8_t *pattern, uint8_t *kv_mask, int32_t *kv_len,
                                  uint8_t *q_mask, void *stream);

/* Workspace bytes dkv_compact needs for this layout (host, no GPU call). */
size_t dkv_compact_workspace_bytes(const dkv_layout *layout);

/*
 * dkv_compact -- the one-time prune and pack of Sec. 3.4 / Fig. 2(b).
 *
 * k, v       dense cache, [N][Hkv][T][d] rows of d elements of `dtype`.
 * kv_mask    uint8 [N][Hkv][T] (nonzero = retained), e.g. from dkv_map_pattern.
 * append_cap free rows reserved after every segment for dkv_append (>= 0).
 * k_out, v_out  packed output, out_rows rows of d elements.  Segment
 *            s = n * Hkv + g starts at seg_off[s] and holds its retained rows
 *            in original token order, followed by append_cap free rows that
 *            this call does not touch.
 * out_rows   capacity of k_out / v_out in rows.  The layout needs
 *            sum_s (kv_len[s] + append_cap) rows.  A segment whose retained
 *            rows and append room would not lie wholly below out_rows is not
 *            packed: nothing of it is written, its seg_len is set to -1 and
 *            its seg_off is clamped to out_rows, so no offset points past
 *            the buffer.  Every call that reads seg_len (dkv_append, the
 *            decode calls, dkv_query_attn) treats a negative length as a
 *            segment with no rows and no room: nothing is appended to it and
 *            its attention outputs are zeros.  *rows_needed reports the true
 *            requirement.
 * seg_off    out, int64 [N*Hkv], row offset of each segment (unit-major).
 * seg_len    out, int32 [N*Hkv], retained rows of each segment (-1: not
 *            packed, see out_rows).
 * src_pos    out, optional int32 [out_rows]: original position j of every
 *            packed row (free rows untouched).
 * rows_needed out, optional int64 [1]: sum_s (seg_len[s] + append_cap).
 * workspace  at least dkv_compact_workspace_bytes(layout) bytes (about
 *            4 * N * Hkv * T: a position list per segment, plus per-tile
 *            counts), no initial contents required.
 * DKV_ERR_UNSUPPORTED when N * Hkv > 65535 or T > 268,435,424 (the copy
 * dispatch, at most a K and a V workgroup of 256 work-items per 32 positions of
 * a segment, must hold fewer than 2^32 work-items).
 * The dense cache may be freed once the stream has executed this call: that
 * is what realises the memory reduction.
 */
dkv_status dkv_compact(const dkv_layout *layout, dkv_dtype dtype, const void *k,
                       const void *v, const uint8_t *kv_mask, int32_t append_cap,
                       void *k_out, void *v_out, int64_t out_rows, int64_t *seg_off,
                       int32_t *seg_len, int32_t *src_pos, int64_t *rows_needed,
                       void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes dkv_compact_bins needs for this layout (host, no GPU call);
 * 0 for a layout it does not accept. */
size_t dkv_compact_bins_workspace_bytes(const dkv_layout *layout);

/*
 * dkv_compact_bins -- map and pack in one call, straight from the pattern, as
 * a block gather.  Under Eq. (4)-(5) and the union of Sec. 3.4 a KV head keeps
 * its sink, its recent window and every bin that some query head of its group
 * keeps, and bin k is the contiguous range of positions
 * [T - recent - min(E[k+1], U), T - recent - E[k]) with U = T - sink - recent
 * the compressible span (empty when E[k] >= U).  The packed segment is those
 * ranges in token order, and each is copied as one block of rows (with the
 * paper's 128-token bins of Appendix A: 128 consecutive rows per kept bin).
 * No keep mask is read or written.
 *
 * pattern   uint8 [N][Hq][D] as for dkv_map_pattern.
 * Every other argument as dkv_compact, whose outputs this call reproduces
 * exactly for dkv_map_pattern's kv_mask of the same layout and pattern:
 * k_out, v_out (the retained rows; free rows untouched), seg_off, seg_len
 * (with the same -1 marker for segments that do not fit below out_rows),
 * src_pos and rows_needed.
 * workspace  at least dkv_compact_bins_workspace_bytes(layout) bytes, no
 *            initial contents required.
 * Limits: those of dkv_map_pattern and dkv_compact, N * Hkv <= 65,535 and
 * N * Hkv * (D + 3) <= 2^27 (the workspace's per-segment block tables);
 * beyond them DKV_ERR_UNSUPPORTED.  Other errors as dkv_compact's.
 */
dkv_status dkv_compact_bins(const dkv_layout *layout, dkv_dtype dtype, const void *k,
                            const void *v, const uint8_t *pattern, int32_t append_cap,
                            void *k_out, void *v_out, int64_t out_rows, int64_t *seg_off,
                            int32_t *seg_len, int32_t *src_pos, int64_t *rows_needed,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * dkv_compact_bins_ragged -- dkv_compact_bins for a batch of contexts of
 * different lengths (e.g. sequences of a serving batch).
 *
 * unit_len  int32 [N] (device), as for dkv_map_pattern_ragged: unit n's
 *           context is the first unit_len[n] positions of its dense rows
 *           (values are clamped to [0, context_len]); its sink, recent window
 *           and bins count from the end of that context, and positions at or
 *           past it are not retained.
 * The outputs equal dkv_compact's for dkv_map_pattern_ragged's kv_mask of the
 * same layout, lengths and pattern.  The dense rows keep layout->context_len
 * as their stride.  Everything else, limits and errors included, as
 * dkv_compact_bins; DKV_ERR_INVALID_ARG also for a null unit_len with N > 0.
 */
dkv_status dkv_compact_bins_ragged(const dkv_layout *layout, const int32_t *unit_len,
                                   dkv_dtype dtype, const void *k, const void *v,
                                   const uint8_t *pattern, int32_t append_cap, void *k_out,
                                   void *v_out, int64_t out_rows, int64_t *seg_off,
                                   int32_t *seg_len, int32_t *src_pos, int64_t *rows_needed,
                                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * dkv_append -- appended tokens are retained in full (Sec. 3.4).
 *
 * k_new, v_new  [num_segments][n_new][d]; token t of segment s is written to
 *               packed row seg_off[s] + seg_len[s] + n_tail + t.
 * n_tail        (host) tokens already appended to every segment.
 * append_cap    (host) free rows reserved per segment; n_tail + n_new must not
 *               exceed it (DKV_ERR_CAPACITY otherwise).
 * seg_off, seg_len  as returned by dkv_compact; pass seg_off + first segment
 *               to address a subset (e.g. one layer's B * Hkv segments).
 * K is stored already rotated (RoPE at the token's absolute position is the
 * caller's job); the library never re-rotates.
 */
dkv_status dkv_append(dkv_dtype dtype, int32_t num_segments, int32_t head_dim,
                      const void *k_new, const void *v_new, int32_t n_new, int32_t n_tail,
                      int32_t append_cap, void *k_c, void *v_c, const int64_t *seg_off,
                      const int32_t *seg_len, void *stream);

/* Workspace bytes for dkv_decode_attn / dkv_dense_decode_attn (host, no GPU call). */
size_t dkv_decode_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                  int32_t head_dim);

/*
 * dkv_decode_attn -- one decode step over the packed cache (Sec. 3.4).
 *
 * q        [B][Hq][d] queries of this step.
 * k_c, v_c packed cache (shared base pointers of a whole-stack compaction).
 * seg_off, seg_len  the B * Hkv segments of this call, batch-major
 *          (s = b * Hkv + g); for layer l of a stack compacted with units
 *          l * B + b, pass seg_off + l * B * Hkv and seg_len + l * B * Hkv.
 * n_tail   (host) appended tokens per segment; segment s attends rows
 *          [seg_off[s], seg_off[s] + seg_len[s] + n_tail).
 * Every query head of group g attends to all rows of segment (b, g): the
 * union of its group (Sec. 3.4).  out[b][h][:] = softmax(sm_scale * K q) V
 * over those rows, fp32 [B][Hq][d]; a segment with no rows (or seg_len < 0)
 * gives zeros.
 * sm_scale   any value with sm_scale * log2(e) finite in fp32 (negative and
 *          zero included); others return DKV_ERR_INVALID_ARG.  The same rule
 *          holds for every attention call of this library.
 * rows_hint (host) expected total rows of the call (0 = unknown); it only
 * sizes the split, never the result's correctness.
 * workspace  at least dkv_decode_workspace_bytes(...) bytes of scratch for
 *          the split partial results; no initial contents are required.  One
 *          workspace serves one call at a time (calls on one stream are
 *          ordered, so reusing it across a stream's calls is safe).
 * The call enqueues the split attention kernel and, when a segment is split
 * over several workgroups, a combine kernel.
 */
dkv_status dkv_decode_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                           int32_t num_kv_heads, int32_t head_dim, const void *q,
                           const void *k_c, const void *v_c, const int64_t *seg_off,
                           const int32_t *seg_len, int32_t n_tail, float sm_scale,
                           int64_t rows_hint, float *out, void *workspace,
                           size_t workspace_bytes, void *stream);

/*
 * dkv_append_decode_attn -- dkv_append followed by dkv_decode_attn, in one
 * launch: the decode step of a serving loop (Sec. 3.4: a new token's K/V is
 * appended and retained, then the step attends to the packed context plus
 * every appended token).
 *
 * k_new, v_new  [B * Hkv][n_new][d], written to packed rows
 *               seg_off[s] + seg_len[s] + n_tail + t exactly as dkv_append
 *               does; then every segment attends rows
 *               [seg_off[s], seg_off[s] + seg_len[s] + n_tail + n_new).
 * n_tail + n_new must not exceed append_cap (DKV_ERR_CAPACITY).  The result
 * equals the two separate calls with the same rows_hint, bit for bit.
 */
dkv_status dkv_append_decode_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                  int32_t num_kv_heads, int32_t head_dim, const void *q,
                                  const void *k_new, const void *v_new, int32_t n_new,
                                  int32_t n_tail, int32_t append_cap, void *k_c, void *v_c,
                                  const int64_t *seg_off, const int32_t *seg_len, float sm_scale,
                                  int64_t rows_hint, float *out, void *workspace,
                                  size_t workspace_bytes, void *stream);

/*
 * dkv_append_decode_attn_noalloc -- dkv_append_decode_attn for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): the same arguments without the
 * workspace, the same kernels and the same result bit for bit.
 *
 * The split's scratch is a static array of DKV_NOALLOC_SCRATCH_BYTES that
 * the library keeps on every GPU it runs on until the process ends; the call
 * itself allocates and frees nothing.  Shapes whose workspace
 * (dkv_decode_workspace_bytes) exceeds that size return DKV_ERR_UNSUPPORTED.
 * The first call on a device looks the array's address up (DKV_ERR_HIP if
 * that fails).  Every call on one GPU shares that GPU's array: two calls that
 * may overlap on one GPU (different streams, or different host threads)
 * race and must be ordered by the caller.  The array needs no initial
 * contents and keeps whatever the last call left.
 */
#define DKV_NOALLOC_SCRATCH_BYTES (16u << 20)
dkv_status dkv_append_decode_attn_noalloc(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                          int32_t num_kv_heads, int32_t head_dim, const void *q,
                                          const void *k_new, const void *v_new, int32_t n_new,
                                          int32_t n_tail, int32_t append_cap, void *k_c, void *v_c,
                                          const int64_t *seg_off, const int32_t *seg_len,
                                          float sm_scale, int64_t rows_hint, float *out,
                                          void *stream);

/*
 * dkv_dense_decode_attn -- the same attention over an uncompressed cache
 * k, v [B][Hkv][t_cap][d]; every segment attends rows [0, n_valid),
 * n_valid <= t_cap.  Same workspace rules as dkv_decode_attn.
 */
dkv_status dkv_dense_decode_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                 int32_t num_kv_heads, int32_t head_dim, const void *q,
                                 const void *k, const void *v, int64_t t_cap,
                                 int32_t n_valid, float sm_scale, float *out,
                                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * dkv_dense_append_decode_attn -- dense comparator of dkv_append_decode_attn:
 * writes k_new, v_new ([B * Hkv][n_new][d]) to rows n_valid .. n_valid+n_new-1
 * of every dense segment, then attends rows [0, n_valid + n_new).
 * n_valid + n_new must not exceed t_cap (DKV_ERR_CAPACITY).
 */
dkv_status dkv_dense_append_decode_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                        int32_t num_kv_heads, int32_t head_dim, const void *q,
                                        const void *k_new, const void *v_new, int32_t n_new,
                                        void *k, void *v, int64_t t_cap, int32_t n_valid,
                                        float sm_scale, float *out, void *workspace,
                                        size_t workspace_bytes, void *stream);

/* Workspace bytes for dkv_query_attn with the same shapes and rows_hint (host,
 * no GPU call); 0 when the call needs none (workspace may then be NULL). */
size_t dkv_query_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                 int32_t head_dim, int32_t n_q, int64_t rows_hint);

/*
 * dkv_query_attn -- attention of a block of n_q query tokens over the packed
 * cache (Sec. 3.4: after the one-time compaction the query tokens attend to
 * the compressed context, and their own K/V are appended and kept).
 *
 * q        [B][n_q][Hq][d] bf16, token-major (the layout of a model's
 *          activations).
 * The block's K/V must already be appended (dkv_append with n_new = n_q at
 * the same n_tail): segment s = b * Hkv + g then holds the packed context,
 * n_tail earlier appended tokens and the block, and query token i of
 * sequence b, head h (g = h / G) attends to rows
 * [seg_off[s], seg_off[s] + seg_len[s] + n_tail + i + 1): everything before
 * the block, and the block causally up to itself.
 * out      [B][n_q][Hq][d] fp32, softmax(sm_scale * K q) V over those rows.
 *          q, K, V and sm_scale must be finite: outputs for NaN or infinite
 *          inputs are unspecified (the kernels run without NaN semantics).
 * append_cap  free rows reserved per segment; n_tail + n_q <= append_cap.
 * rows_hint (host) total rows the call attends, sum over segments of
 *          seg_len + n_tail + n_q (0 = unknown); it sizes the split of the key
 *          ranges and must equal the value given to dkv_query_workspace_bytes.
 *          A wrong hint changes the split (and the speed), never the result.
 * workspace  dkv_query_workspace_bytes(...) bytes for the split's plan and
 *          per-range partial results (no initial contents required), or NULL
 *          when that is 0 (keys too few to split).
 * Only DKV_BF16 is supported (DKV_ERR_UNSUPPORTED otherwise); head_dim 64 or
 * 128; DKV_ERR_UNSUPPORTED also when a dispatch would exceed 2^32 work-items
 * (512 per workgroup).  When the keys are split the call enqueues the attention
 * kernel and a combine kernel, and before them a one-workgroup plan kernel
 * unless the block is short (at most 256 query rows n_q * G per segment; of
 * more than 64, where sizes and rows_hint say that the kernels for short blocks
 * are no slower); otherwise the attention kernel alone.
 */
dkv_status dkv_query_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                          int32_t num_kv_heads, int32_t head_dim, int32_t n_q, const void *q,
                          int32_t n_tail, int32_t append_cap, const void *k_c, const void *v_c,
                          const int64_t *seg_off, const int32_t *seg_len, float sm_scale,
                          int64_t rows_hint, float *out, void *workspace, size_t workspace_bytes,
                          void *stream);

/*
 * Exact-budget pattern export (Sec. 3.3, Eq. (topk-pattern); Appendix A,
 * exact-budget refinement).  The learned pattern keeps the K_rho entries of
 * the L x H x D tensor of retention probabilities with the largest
 * probability, K_rho = round(rho L H D) for a logical retention ratio rho.
 */

/* K_rho = round(rho * L * H * D), halves rounded up (the paper leaves them
 * open), computed in double (host).  Returns -1 unless 0 <= rho <= 1 and the
 * sizes are non-negative. */
int64_t dkv_budget_entries(double rho, int32_t num_layers, int32_t num_q_heads, int32_t num_bins);

/* Workspace bytes of dkv_topk_pattern (host, no GPU call); 0 for an empty or
 * too large tensor. */
size_t dkv_topk_workspace_bytes(int32_t num_layers, int32_t num_q_heads, int32_t num_bins);

/*
 * dkv_topk_pattern -- TopKMask(P, k): pattern[l][h][d] = 1 for the k largest
 * probs[l][h][d] over the whole tensor, 0 elsewhere.
 *
 * probs    float32 [L][Hq][D], 16-byte aligned (any values; NaN ranks below
 *          every number, -0 equals +0).
 * k        0 <= k <= L * Hq * D (DKV_ERR_INVALID_ARG otherwise), e.g.
 *          dkv_budget_entries(rho, L, Hq, D).
 * pattern  out, uint8 [L][Hq][D], 4-byte aligned, with exactly k ones: the
 *          pattern argument of dkv_map_pattern (one unit per layer).
 * workspace  dkv_topk_workspace_bytes(...) bytes, 4-byte aligned, no initial
 *          contents required (DKV_ERR_WORKSPACE otherwise).
 * Ties at the k-th value go to the lowest flat (layer, head, bin) indices, so
 * the result is unique and deterministic.  L * Hq * D < 2^31.  A radix
 * select of five small launches; nothing is read back to the host.
 */
dkv_status dkv_topk_pattern(int32_t num_layers, int32_t num_q_heads, int32_t num_bins,
                            const float *probs, int64_t k, uint8_t *pattern, void *workspace,
                            size_t workspace_bytes, void *stream);

/*
 * Zero-copy paged variant
 * -----------------------
 * The retained set of a segment is its sink, its recent window and a union
 * of whole distance bins (Eq. (4), Eq. (5) and the union of Sec. 3.4), i.e. a
 * few long runs of consecutive positions.  When the cache is kept in pages of
 * page_rows consecutive positions, those runs can be referenced where they
 * are instead of being packed (dkv_compact): with the paper's 128-token bins
 * (Appendix A) and 128-row pages every retained bin is a whole page.
 *
 * Paged cache: K and V pools [num_pages][page_rows][d]; page_table
 * [nseg][pages_per_seg] (int32) gives the physical page that holds positions
 * [p * page_rows, (p + 1) * page_rows) of segment s (logical page p).
 * page_rows is 32, 64, 128, 256, 512 or 1024.
 *
 * Entry: four int32 (physical page, logical page, lo, hi) naming slots
 * [lo, hi) of one page.  A segment's entries are listed in position order:
 * every maximal run of retained context positions within one page, then
 * the append region [T, T + append_cap) page by page.  Decode attends to the
 * slots of the entries whose positions are below T + (tokens appended).
 */
#define DKV_PAGE_ENTRY_INTS 4

/* Workspace bytes of dkv_page_select (host, no GPU call). */
size_t dkv_page_select_workspace_bytes(int32_t num_segments, int32_t context_len);

/*
 * Upper bound on the entries of one segment for keep masks made by
 * dkv_map_pattern with this layout (host): pages of the context, plus one
 * per bin, the sink and the recent window, plus the append region's pages.
 * Returns -1 for invalid arguments.
 */
int64_t dkv_page_entries_bound(const dkv_layout *layout, int32_t append_cap, int32_t page_rows);

/*
 * dkv_page_select -- the zero-copy alternative to dkv_compact: list the
 * retained rows of every segment in place (Sec. 3.4 keeps retained rows in
 * original order; here they keep their original pages too).
 *
 * kv_mask     uint8 [nseg][T], nonzero = retained (e.g. dkv_map_pattern's
 *             kv_mask with nseg = N * Hkv); 16-byte aligned.
 * page_table  int32 [nseg][pages_per_seg]; pages_per_seg * page_rows must be
 *             >= T + append_cap (DKV_ERR_INVALID_ARG otherwise).
 * entries     out, int32 [nseg][max_entries][4], 16-byte aligned.  Entries
 *             at index >= max_entries are not written.
 * n_entries   out, int32 [nseg]: the segment's entry count, even when it is
 *             larger than max_entries (the caller must then enlarge the
 *             array: decode reads at most max_entries entries and cannot
 *             append to a segment whose append entries are missing).
 * seg_len     out, int32 [nseg]: retained context positions (as kv_len).
 * page_used   out, optional uint8 [nseg][pages_per_seg]: 1 for every page an
 *             entry names; pages marked 0 hold no retained row and no append
 *             slot and may be returned to the pool -- that is where the
 *             memory reduction comes from.
 * workspace   dkv_page_select_workspace_bytes(nseg, T) bytes, no initial
 *             contents required.
 * Nothing is copied: the pools are neither read nor written.
 */
dkv_status dkv_page_select(int32_t num_segments, int32_t context_len, int32_t append_cap,
                           int32_t page_rows, const uint8_t *kv_mask, const int32_t *page_table,
                           int32_t pages_per_seg, int32_t max_entries, int32_t *entries,
                           int32_t *n_entries, int32_t *seg_len, uint8_t *page_used,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * dkv_paged_decode_attn -- one decode step over a paged cache (Sec. 3.4),
 * reading the retained rows in place through dkv_page_select's entries.
 *
 * q           [B][Hq][d]; segment s = b * Hkv + g.
 * k_pages, v_pages  the pools, num_pages pages of page_rows rows of d
 *             elements of `dtype`.
 * entries, n_entries, max_entries  as written by dkv_page_select for these
 *             segments (for a subset of a larger selection, offset entries
 *             by first * max_entries * 4 and n_entries by first).
 * context_len T of the selection; n_tail (host) tokens appended so far,
 *             at positions [T, T + n_tail).
 * Every query head of group g attends to the slots of segment (b, g)'s
 * entries whose positions lie below T + n_tail: the retained context and the
 * appended tokens (the union of Sec. 3.4).  An entry that names a page
 * outside [0, num_pages) or slots outside [0, page_rows) attends nothing.
 * The result is that of dkv_decode_attn over a packed cache of the same rows.
 * rows_hint (host) expected sum over segments of entries * page_rows (0 =
 * unknown); it only sizes the split.  out, workspace: as dkv_decode_attn,
 * with the same workspace size (dkv_decode_workspace_bytes).
 */
dkv_status dkv_paged_decode_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                 int32_t num_kv_heads, int32_t head_dim, const void *q,
                                 const void *k_pages, const void *v_pages, int64_t num_pages,
                                 int32_t page_rows, const int32_t *entries,
                                 const int32_t *n_entries, int32_t max_entries,
                                 int32_t context_len, int32_t n_tail, float sm_scale,
                                 int64_t rows_hint, float *out, void *workspace,
                                 size_t workspace_bytes, void *stream);

/*
 * dkv_paged_append_decode_attn -- the decode step of a serving loop over a
 * paged cache: token t of k_new, v_new ([B * Hkv][n_new][d]) is position
 * T + n_tail + t and is written to its slot of the page its append-region
 * entry names (Sec. 3.4: appended and retained), then the step attends as
 * dkv_paged_decode_attn with n_tail + n_new tokens appended, in one launch.
 * append_cap must be the value given to dkv_page_select, and n_tail + n_new
 * must not exceed it (DKV_ERR_CAPACITY).  A segment whose entry count
 * exceeded max_entries is not appended to.
 */
dkv_status dkv_paged_append_decode_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                        int32_t num_kv_heads, int32_t head_dim, const void *q,
                                        const void *k_new, const void *v_new, int32_t n_new,
                                        int32_t n_tail, int32_t append_cap, void *k_pages,
                                        void *v_pages, int64_t num_pages, int32_t page_rows,
                                        const int32_t *entries, const int32_t *n_entries,
                                        int32_t max_entries, int32_t context_len,
                                        float sm_scale, int64_t rows_hint, float *out,
                                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * Filling a paged cache
 * ---------------------
 * A server that admits and grows requests on the GPU needs no host copy of
 * its tables: dkv_page_extend gives every request the pages for its new
 * tokens and says where each token's rows go, dkv_paged_append writes them,
 * dkv_paged_query_attn lets the new tokens attend to what their request
 * holds, and dkv_page_release takes pages back (the ones a selection marks
 * unused, or all of a finished request).
 *
 * Units and segments are those of the other calls: unit n is one (layer,
 * sequence), segment s = n * Hkv + g, and every segment has pages of its own
 * (its KV head's rows of positions [p * page_rows, (p + 1) * page_rows)).
 * Tokens are token-major: row tok_off[n] + t of the batch's arrays is new
 * token t of unit n, as a model's activations lie.
 *
 * Free pages stand on a stack: free_pages[0 .. *n_free) (device), the top at
 * the end; *n_free is taken within [0, free_cap].  An output that has an
 * input's meaning (new_len and unit_len, n_free_out and n_free, table_out and
 * page_table) may be the same buffer, which updates it in place; otherwise
 * outputs and inputs must not overlap.
 */

/* Workspace bytes of dkv_page_extend (host, no GPU call). */
size_t dkv_page_extend_workspace_bytes(int32_t num_units);

/*
 * dkv_page_extend -- page tables, slots and entries from lengths.
 *
 * unit_new    int32 [N]: tokens to add to each unit.
 * unit_len    int32 [N]: positions that each unit holds (0 for a new request);
 *             its segments' pages for them are in page_table.
 * new_len     out, int32 [N]: unit_len + unit_new, or unit_len for a unit that
 *             is not served.
 * n_free_out  out, int32 [1]: the stack's height afterwards.
 * page_table  int32 [N * Hkv][pages_per_seg], in and out: the new pages' words
 *             are written, all others stay.  A unit needs
 *             Hkv * (ceil((len + new) / page_rows) - ceil(len / page_rows))
 *             pages; page i of the call, segment by segment and page by page,
 *             is the i-th from the top of the stack.
 * tok_off     out, int32 [N + 1]: exclusive sums of the new tokens (a negative
 *             unit_new counts as 0), at most max_tokens.
 * first_pos   out, int32 [N]: position of the unit's first new token (its
 *             unit_len), or -1 when it is not served.
 * slots       out, int64 [max_tokens][Hkv]: pool row (page * page_rows + slot)
 *             of every new token and head; -1 for tokens of units that are not
 *             served, for tokens whose page is negative, and for all rows at
 *             or past tok_off[N] (a padded batch writes nothing there).
 * entries     optional (NULL with max_entries = 0), int32
 *             [N * Hkv][max_entries][4], 16-byte aligned, in and out: entry p
 *             of a segment is (page, p, 0, slots filled) for its page p, the
 *             format of dkv_page_select for an unpruned cache; the entries of
 *             the pages that got tokens are written, below max_entries.
 *             This holds for every unit.  A selection's list (dkv_page_select
 *             of a mask with pruned positions: runs, not pages) is overwritten
 *             like the others and wrong from then on: after this call, and
 *             before the lists are read, dkv_page_select lists the segments
 *             of compressed units again, from the mask of their selection, with
 *             the positions past its context (new_len - T) as append_cap;
 *             page_table has their new pages by then.
 * n_entries   optional, int32 [N * Hkv], in and out: set to the pages of every
 *             served unit that got tokens (even above max_entries).
 * pages_needed optional out, int64 [1]: pages needed by all units that could
 *             be served with enough free pages.
 * A unit is not served when its length or new tokens are negative, its new
 * length passes pages_per_seg * page_rows (or 2^31 - 1), its rows do not lie
 * wholly below max_tokens, or the pages it needs, counted behind those of all
 * the units before it, pass the free ones.  Nothing of it changes; a unit that
 * needs no page is not held up by the ones before it.
 * DKV_ERR_UNSUPPORTED when N * Hkv > 65535, max_tokens > 2^31 - 128 or
 * max_tokens * Hkv > 2^32 - 256.
 * The call enqueues one kernel when max_tokens is at most 128, or at most 32,768
 * and neither new_len nor n_free_out is updated in place; otherwise one over
 * the units and one over the tokens.
 */
dkv_status dkv_page_extend(int32_t num_units, int32_t num_kv_heads, int32_t page_rows,
                           const int32_t *unit_new, const int32_t *unit_len, int32_t *new_len,
                           const int32_t *free_pages, int32_t free_cap, const int32_t *n_free,
                           int32_t *n_free_out, int32_t *page_table, int32_t pages_per_seg,
                           int32_t *tok_off, int32_t *first_pos, int64_t *slots,
                           int32_t max_tokens, int32_t *entries, int32_t *n_entries,
                           int32_t max_entries, int64_t *pages_needed, void *workspace,
                           size_t workspace_bytes, void *stream);

/* Workspace bytes of dkv_page_release (host, no GPU call). */
size_t dkv_page_release_workspace_bytes(int32_t num_segments, int32_t pages_per_seg);

/*
 * dkv_page_release -- pages back to the stack.
 *
 * page_table  int32 [nseg][pages_per_seg]; negative words name no page.
 * keep        optional uint8 [nseg][pages_per_seg]: a page goes when its byte
 *             is 0 (e.g. page_used of dkv_page_select); NULL: every page goes.
 * table_out   out, int32 [nseg][pages_per_seg]: -1 for the pages that went, the
 *             word of page_table otherwise.
 * free_pages  the pages that go are pushed on the stack in table order, below
 *             free_cap; a page that finds no room stays in the table.
 * n_free_out  out, int32 [1]: the stack's height afterwards.
 * A page that two words name is pushed twice: give every page one owner.
 * DKV_ERR_UNSUPPORTED when nseg * pages_per_seg > 2^31 - 1.
 */
dkv_status dkv_page_release(int32_t num_segments, int32_t pages_per_seg, const int32_t *page_table,
                            const uint8_t *keep, int32_t *table_out, int32_t *free_pages,
                            int32_t free_cap, const int32_t *n_free, int32_t *n_free_out,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * dkv_paged_append -- rows of new tokens into their slots (Sec. 3.4: appended
 * tokens are retained in full).
 *
 * k_new, v_new  [num_tokens][Hkv][d], tokens token_stride elements apart
 *               (>= Hkv * d, a multiple of 16 bytes; the K and V parts of a
 *               fused projection's rows can be passed where they are).
 * slots         int64 [num_tokens][Hkv] as dkv_page_extend writes them; a
 *               token and head with a slot outside [0, num_pages * page_rows)
 *               is skipped.  What rows with the same slot leave there is
 *               unspecified.
 * k_pages, v_pages  the pools, [num_pages][page_rows][d].
 */
dkv_status dkv_paged_append(dkv_dtype dtype, int32_t num_tokens, int32_t num_kv_heads,
                            int32_t head_dim, const void *k_new, const void *v_new,
                            int64_t token_stride, const int64_t *slots, void *k_pages,
                            void *v_pages, int64_t num_pages, int32_t page_rows, void *stream);

/* Workspace bytes for dkv_paged_query_attn with the same shapes and rows_hint
 * (host, no GPU call); 0 when the call needs none (workspace may be NULL). */
size_t dkv_paged_query_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                       int32_t head_dim, int32_t num_tokens, int32_t max_q,
                                       int64_t rows_hint);

/*
 * dkv_paged_query_attn -- attention of a chunk of new tokens of every sequence
 * over a paged cache (dkv_query_attn's counterpart for pages; chunks of
 * different lengths, single tokens included, in one call).
 *
 * q         [num_tokens][Hq][d] bf16, token-major, tokens q_stride elements
 *           apart (>= Hq * d, a multiple of 8: the Q part of a fused
 *           projection's rows can be passed where it is).
 * tok_off   int32 [B + 1]: sequence b's chunk is rows [tok_off[b],
 *           tok_off[b + 1]); taken within [0, num_tokens], and of a chunk
 *           longer than max_q only the first max_q tokens are attended.
 *           Chunks must not share rows.
 * first_pos int32 [B]: position of the chunk's first token; a negative one
 *           marks a sequence that attends nothing (its outputs are zeros).
 * entries, n_entries, max_entries  the pages of the B * Hkv segments, from
 *           dkv_page_extend (an unpruned cache) or dkv_page_select (the
 *           retained runs and the append region), in position order.
 *           Token i of the chunk, head h (g = h / G) attends to the slots of
 *           segment (b, g)'s entries whose position (logical page * page_rows
 *           + slot) is at most first_pos[b] + i: what the sequence holds, and
 *           the chunk causally up to itself.  The chunk's K/V must already be
 *           written (dkv_paged_append).  An entry that names a page outside
 *           [0, num_pages) or slots outside [0, page_rows) attends nothing;
 *           slots past the chunk's last position are never read.
 * out       [num_tokens][Hq][d] fp32, softmax(sm_scale * K q) V over those
 *           slots; zeros for a token that sees none.  Rows of no sequence
 *           (padding) are left as they were.
 *           q, the attended K and V and sm_scale must be finite; slots that no
 *           token of the chunk attends may hold anything.
 * max_q     (host) tokens of the longest chunk.
 * rows_hint (host) expected total rows of the call, sum over segments of
 *           entries * page_rows (0 = unknown, taken for a long cache); it
 *           sizes the split of the keys
 *           and must equal the value given to dkv_paged_query_workspace_bytes.
 * workspace dkv_paged_query_workspace_bytes(...) bytes, no initial contents
 *           required, or NULL when that is 0.
 * Scores, maxima and sums are fp32; a probability enters its product with V as
 * three bf16 parts (24 bits).
 * The call enqueues one kernel without a workspace; with one, an attention and
 * a combine kernel, and a plan kernel before them in chunks of more query rows
 * per KV head than the short-block kernels take (32 to 256, by the segments'
 * number and length).
 * Only DKV_BF16 is supported (DKV_ERR_UNSUPPORTED otherwise); head_dim 64 or
 * 128; DKV_ERR_UNSUPPORTED also when max_entries * page_rows > 2^30 or a
 * dispatch would exceed 2^32 work-items.
 */
dkv_status dkv_paged_query_attn(dkv_dtype dtype, int32_t batch, int32_t num_q_heads,
                                int32_t num_kv_heads, int32_t head_dim, int32_t num_tokens,
                                int32_t max_q, const void *q, int64_t q_stride,
                                const int32_t *tok_off, const int32_t *first_pos,
                                const void *k_pages, const void *v_pages, int64_t num_pages,
                                int32_t page_rows, const int32_t *entries,
                                const int32_t *n_entries, int32_t max_entries, float sm_scale,
                                int64_t rows_hint, float *out, void *workspace,
                                size_t workspace_bytes, void *stream);

/*
 * Rotary positions, a quantised cache and drafted trees
 * -----------------------------------------------------
 * A step of speculative decoding over a paged cache: dkv_page_extend gives the
 * drafted tokens pages and slots, dkv_tree_plan their ancestors and positions,
 * dkv_paged_store rotates q and K and writes K and V (in bf16, or quantised to
 * 8 bits), dkv_paged_tree_attn lets every token attend to its request and its
 * ancestors, and dkv_paged_accept keeps the accepted path.  Prompts in chunks
 * and single tokens take the same calls without a tree.
 *
 * Cache formats.  DKV_CACHE_BF16: pools of bf16 rows, as dkv_paged_append
 * fills them; `scales` is ignored.  DKV_CACHE_F8: a row of d values is d codes of
 * e4m3 (sign, 4 exponent bits, 3 mantissa bits, largest value 448, no
 * infinities) in a pool [num_pages][page_rows][d] of bytes, and an exponent
 * byte 127 + e; code c stands for c * 2^e.  scales is uint8
 * [num_pages][page_rows][2], 16-byte aligned, the bytes of the K and the V row.  e is the smallest
 * with the row's largest magnitude at most 448 * 2^e, within [-60, 120]; codes
 * are rounded to nearest, ties to even.  NaN and infinities become NaN, and do
 * not count for e.  A value is off by at most 2^-4 of itself, or 2^-10 * 2^e.
 * Pages, tables, slots and entries are the same for both formats.
 */
typedef enum dkv_cache_format { DKV_CACHE_BF16 = 0, DKV_CACHE_F8 = 1 } dkv_cache_format;

#define DKV_MAX_TREE 1024  /* tokens of a drafted tree (dkv_tree_plan with parents) */
#define DKV_MAX_PATH 64    /* tokens of an accepted path */

/* How rotary frequencies f_i = base^(-2i / rot_dim) are stretched by `factor`
 * for contexts longer than trained_len (dkv_rope_freqs). */
typedef enum dkv_rope_scaling {
  DKV_ROPE_PLAIN = 0,  /* not */
  DKV_ROPE_LINEAR = 1, /* all divided by factor */
  DKV_ROPE_BASE = 2,   /* base * factor^(rot_dim / (rot_dim - 2)): the slowest pair divided by factor */
  DKV_ROPE_WAVE = 3,   /* pairs with up to `low` turns over trained_len divided, from `high` on kept, linear between */
  DKV_ROPE_RAMP = 4    /* the same, linear in the pair's index between the pairs with `high` and `low` turns
                          (rounded outwards, cut to 0 .. rot_dim - 1); *mscale = 0.1 ln(factor) + 1 */
} dkv_rope_scaling;

/*
 * dkv_rope_freqs -- rotary frequencies (host, no GPU call): inv_freq[0 ..
 * rot_dim / 2) and the factor *mscale of the rotated elements (1 but for
 * DKV_ROPE_RAMP), computed in double.  base > 1, factor >= 1; 0 < low < high
 * turns and trained_len > 0 where the scaling uses them.
 */
dkv_status dkv_rope_freqs(dkv_rope_scaling kind, int32_t rot_dim, double base, double factor, double trained_len,
                          double low, double high, float *inv_freq, float *mscale);

/*
 * dkv_rope -- rotary positions of token-major rows.
 *
 * x, out    [num_tokens][num_heads][head_dim] of `dtype`, tokens x_stride and
 *           out_stride elements apart (multiples of 16 bytes); out == x with the
 *           same stride rotates in place, otherwise they must not overlap.
 * pos       int32 [num_tokens]; a token with a negative one is left out: its
 *           rows of `out` stay as they were.
 * inv_freq  float [rot_dim / 2] (device): pair i turns by pos * inv_freq[i],
 *           (a, b) -> mscale * (a cos - b sin, a sin + b cos); pos * |inv_freq[i]| below
 *           2^32.
 * rot_dim   even, at most head_dim: the rotated part of a head; the rest is copied.
 * interleaved  0: pair i is elements i and i + rot_dim / 2; otherwise 2i and 2i + 1.
 * head_dim a multiple of 8, at most 256 (DKV_ERR_UNSUPPORTED otherwise, as when
 * num_tokens * num_heads > 2^24 - 1).
 * Angles and products are computed in double; a result is rounded to fp32, and
 * from there to `dtype`.
 */
dkv_status dkv_rope(dkv_dtype dtype, int32_t num_tokens, int32_t num_heads, int32_t head_dim, const void *x,
                    int64_t x_stride, const int32_t *pos, const float *inv_freq, int32_t rot_dim, int32_t interleaved,
                    float mscale, void *out, int64_t out_stride, void *stream);

/*
 * dkv_tree_plan -- ancestors and positions of drafted tokens.
 *
 * tok_off, first_pos  int32 [batch + 1] (ascending) and [batch], as from
 *           dkv_page_extend: sequence b's new tokens are rows [tok_off[b],
 *           tok_off[b + 1]), the first max_q of them count.
 * parent    int32 [num_tokens] or NULL (every token follows the one before it):
 *           index among its sequence's new tokens of the one a token
 *           continues; one that is negative or does not come before the
 *           token makes it continue what the sequence held.
 * pos       out, int32 [num_tokens]: first_pos[b] + number of ancestors; -1 for
 *           rows of no sequence, of one with a negative first_pos, and past max_q.
 * mask      out, optional, uint64 [num_tokens][mask_words]: bit j of a row is
 *           set when new token j of the sequence is the token itself or an
 *           ancestor; zeros where pos is -1.  mask_words * 64 must be at least
 *           max_q (or num_tokens, if that is less).
 * pos may be parent itself; otherwise pos and mask share no byte with each other
 * or with tok_off, first_pos and parent (DKV_ERR_INVALID_ARG).
 * With parents max_q is at most DKV_MAX_TREE, batch at most DKV_MAX_SEGMENTS
 * (DKV_ERR_UNSUPPORTED otherwise).
 */
dkv_status dkv_tree_plan(int32_t batch, int32_t num_tokens, int32_t max_q, const int32_t *tok_off,
                         const int32_t *first_pos, const int32_t *parent, int32_t *pos, uint64_t *mask,
                         int32_t mask_words, void *stream);

/*
 * dkv_paged_store -- new tokens into a paged cache: q and K rotated, K and V
 * written to their slots in the cache's format, in one launch.
 *
 * q, q_out  [num_tokens][Hq][d] bf16, tokens q_stride and q_out_stride elements
 *           apart; q_out is q rotated as by dkv_rope (in place with q_out == q
 *           and the same stride).  With num_q_heads = 0 both may be NULL.
 * k_new, v_new  [num_tokens][Hkv][d] bf16, tokens kv_stride elements apart.
 * pos, inv_freq, rot_dim, interleaved, mscale  as for dkv_rope; rot_dim = 0: q
 *           and K are taken as they are and pos and inv_freq may be NULL.  With
 *           rotation a token with a negative pos is left out altogether.
 * slots     int64 [num_tokens][Hkv] as dkv_page_extend writes them; a row with a
 *           slot outside [0, num_pages * page_rows) is skipped.  What rows with
 *           the same slot leave there is unspecified.
 * K is rotated as by dkv_rope, but rounded from fp32 to the cache's format at
 * once.  head_dim 64 or 128; strides multiples
 * of 8 elements.
 */
dkv_status dkv_paged_store(dkv_cache_format format, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                           int32_t head_dim, const void *q, int64_t q_stride, const void *k_new, const void *v_new,
                           int64_t kv_stride, const int32_t *pos, const float *inv_freq, int32_t rot_dim,
                           int32_t interleaved, float mscale, void *q_out, int64_t q_out_stride, const int64_t *slots,
                           void *k_pages, void *v_pages, uint8_t *scales, int64_t num_pages, int32_t page_rows,
                           void *stream);

/*
 * dkv_paged_load -- rows of a paged cache back in bf16 (exact for both formats).
 *
 * slots     int64 [num_tokens][Hkv]: pool rows; k_out and v_out rows of a slot
 *           outside [0, num_pages * page_rows) stay as they were.
 * k_out, v_out  [num_tokens][Hkv][d] bf16, tokens token_stride elements apart (a
 *           multiple of 8).
 */
dkv_status dkv_paged_load(dkv_cache_format format, int32_t num_tokens, int32_t num_kv_heads, int32_t head_dim,
                          const void *k_pages, const void *v_pages, const uint8_t *scales, int64_t num_pages,
                          int32_t page_rows, const int64_t *slots, void *k_out, void *v_out, int64_t token_stride,
                          void *stream);

/* Workspace bytes for dkv_paged_tree_attn with the same shapes and rows_hint
 * (host, no GPU call); 0 when the call needs none (workspace may be NULL). */
size_t dkv_paged_tree_workspace_bytes(dkv_cache_format format, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                      int32_t head_dim, int32_t num_tokens, int32_t max_q, int64_t rows_hint);

/*
 * dkv_paged_tree_attn -- attention of every sequence's new tokens over a paged
 * cache, in bf16 or quantised, with a mask over the new tokens: trees of drafted
 * tokens, and without a mask chunks and single tokens (dkv_paged_query_attn).
 *
 * mask      uint64 [num_tokens][mask_words], 8-byte aligned (dkv_tree_plan writes
 *           it), or NULL.  A token of sequence b sees the slots of its segment's
 *           entries at positions below first_pos[b], and at first_pos[b] + j
 *           where bit j of its row is set, j within the sequence's new tokens
 *           (those that count: max_q).  Bits beyond mask_words * 64 count as 0.
 *           NULL: j up to the token itself.
 * k_pages, v_pages, scales  the pools in the cache's format; scales only for
 *           DKV_CACHE_F8, 16-byte aligned.
 * out       [num_tokens][Hq][d] fp32; zeros for a token that sees nothing.  Rows
 *           of no sequence are left as they were.
 * DKV_CACHE_F8: |sm_scale q k| below 2^23 and |V| below 2^25; the sum of the
 * probabilities is off beyond (a key's share of it counts down to 2^-41 of the
 * largest within).  The exponent bytes are those that dkv_paged_store writes, 67
 * to 247; one of a row of V below 67 counts as 67 (a row of zeros may have any).
 * q, sm_scale, and the K and V of all positions below first_pos[b] + (new tokens)
 * that entries name must be finite, also those of new tokens that a mask
 * hides; other slots may hold anything.
 * Every other argument as dkv_paged_query_attn's, with the workspace of
 * dkv_paged_tree_workspace_bytes and the same rules for the launches.
 * mask_words at most 2^20.
 * Quantised values enter the products exactly; scores, maxima and sums are
 * fp32; a probability enters its product with V as three bf16 parts (24 bits)
 * or, with a quantised cache, as two fp16 parts (22 bits).
 */
dkv_status dkv_paged_tree_attn(dkv_cache_format format, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                               int32_t head_dim, int32_t num_tokens, int32_t max_q, const void *q, int64_t q_stride,
                               const int32_t *tok_off, const int32_t *first_pos, const uint64_t *mask, int32_t mask_words,
                               const void *k_pages, const void *v_pages, const uint8_t *scales, int64_t num_pages,
                               int32_t page_rows, const int32_t *entries, const int32_t *n_entries, int32_t max_entries,
                               float sm_scale, int64_t rows_hint, float *out, void *workspace, size_t workspace_bytes,
                               void *stream);

/*
 * dkv_paged_accept -- keep an accepted path of the drafted tokens.
 *
 * Units are (layer, sequence) pairs, unit n = layer * batch + b, segments n *
 * Hkv + g, as for dkv_page_extend; all layers of a step go in one call.
 * first_pos int32 [num_units]: position of the unit's first new token; a unit
 *           with a negative one is left as it is (nothing of it is written).
 * path      int32 [batch][max_path]: indexes among sequence b's new tokens, from
 *           the root on, each larger than the one before; the first n_path[b]
 *           count, up to one that is not larger, is negative or lies past the
 *           page table.  max_path at most DKV_MAX_PATH.
 * The rows of token path[b][i] (position first_pos + path[b][i]) move to position
 * first_pos + i, in every segment's K and V; a row whose page (from or to) is
 * outside the pool does not move.
 * new_len   out, int32 [num_units]: first_pos + accepted tokens.
 * keep      optional out, uint8 [num_units * Hkv][pages_per_seg]: 1 for the pages
 *           of the first new_len positions, 0 for those behind them: the argument
 *           of dkv_page_release that takes the others back (set to 1
 *           before, so that units that are left out keep theirs).
 * new_len and keep share no byte with each other or with first_pos, path, n_path
 * and page_table (DKV_ERR_INVALID_ARG otherwise).
 * Entries need no change: what lies past a chunk's last position is not read,
 * and the next dkv_page_extend (with new_len as unit_len, after the pages
 * behind it have been released) writes those that change.
 * num_units * Hkv at most 65,535.
 */
dkv_status dkv_paged_accept(dkv_cache_format format, int32_t num_units, int32_t batch, int32_t num_kv_heads,
                            int32_t head_dim, const int32_t *first_pos, const int32_t *path, const int32_t *n_path,
                            int32_t max_path, const int32_t *page_table, int32_t pages_per_seg, int32_t page_rows,
                            void *k_pages, void *v_pages, uint8_t *scales, int64_t num_pages, int32_t *new_len,
                            uint8_t *keep, void *stream);

/* Static description of a status code. */
const char *dkv_status_string(dkv_status status);

#ifdef __cplusplus
}
#endif

#endif /* DKV_H */
