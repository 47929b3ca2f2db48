// Launch interface of rotary positions, quantised rows and drafted trees
// (argument checks live in the C-ABI layer).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace dkv {

// ------------------------------------------- rotation, store and read back
struct RotateParams {
  // Rows of a token: heads rows of x (rotated into out), then, in a store,
  // Hkv rows of k (rotated) and Hkv of v (as they are) into their slots.
  const void* x;       // [tokens][heads][dim], tokens x_stride bytes apart
  void* out;           // tokens out_stride bytes apart
  const void* k;       // [tokens][Hkv][dim], tokens kv_stride bytes apart
  const void* v;
  const int32_t* pos;  // [tokens]; null: nothing rotates
  const float* freq;   // [pairs]
  const int64_t* slots;  // [tokens][Hkv] pool rows
  void* k_pages;
  void* v_pages;
  uint8_t* scales;     // [pool_rows][2]: exponent bytes of the K and the V row
  int64_t x_stride, out_stride, kv_stride, pool_rows;
  int32_t tokens, heads, Hkv, dim;
  int32_t pairs;       // rotated pairs of a head
  int32_t interleaved;
  int32_t parts;       // waves that share a token's rows
  float mscale;
};
hipError_t launch_rope(const RotateParams& p, bool f32, hipStream_t stream);
hipError_t launch_paged_store(const RotateParams& p, bool f8, hipStream_t stream);

struct LoadParams {
  const void* k_pages;
  const void* v_pages;
  const uint8_t* scales;
  const int64_t* slots;  // [tokens][Hkv]
  void* k_out;           // [tokens][Hkv][dim] bf16, tokens `stride` bytes apart
  void* v_out;
  int64_t pool_rows, stride;
  int32_t tokens, Hkv, dim;
};
hipError_t launch_paged_load(const LoadParams& p, bool f8, hipStream_t stream);

// ------------------------------------------------------------- drafted trees
constexpr int kMaxTree = 1024;  // tokens of a drafted tree
constexpr int kMaxPath = 64;    // tokens of an accepted path

struct TreePlanParams {
  const int32_t* tok_off;    // [B + 1]
  const int32_t* first_pos;  // [B]
  const int32_t* parent;     // [tokens] or null (chains)
  int32_t* pos;              // [tokens]
  uint64_t* mask;            // [tokens][words] or null
  int32_t batch, tokens, max_q, words;
};
hipError_t launch_tree_plan(const TreePlanParams& p, hipStream_t stream);

struct AcceptParams {
  const int32_t* first_pos;  // [units]
  const int32_t* path;       // [batch][max_path]
  const int32_t* n_path;     // [batch]
  const int32_t* table;      // [units * Hkv][pages_per_seg]
  char* k_pages;
  char* v_pages;
  uint8_t* scales;           // null: rows without exponents
  int32_t* new_len;          // [units]
  uint8_t* keep;             // [units * Hkv][pages_per_seg] or null
  int64_t num_pages;
  int32_t units, batch, Hkv, max_path, pages_per_seg, page_shift, row_bytes;
};
hipError_t launch_paged_accept(const AcceptParams& p, hipStream_t stream);

}  // namespace dkv
