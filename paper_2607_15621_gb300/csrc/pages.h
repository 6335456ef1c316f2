// Launch interface of the operators over a cache in pages: rotary positions (rotary.cu), paged attention
// (paged_attention.cu), bounds and selection of pages (page_select.cu), page tables and copies (page_table.cu). Arguments have
// been checked by pages.cu.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fsx.h"
#include "kernels.h"
#include "llm.h"

namespace fsx {

constexpr int kMaxAxes = 4;          // of rotary positions
constexpr int kMaxPicked = 4096;     // pages that a selection takes
constexpr int kMaxPagesListed = 32768;  // pages of a request that a selection looks at
constexpr int kMaxPlanes = 512;      // of a copy of pages

struct RotaryArgs {
  const void* q;  // NULL: none
  long long q_stride;
  const void* k;
  const void* v;
  long long kv_stride;
  const int64_t* positions;  // [axes, rows]
  long long rows;
  int n_heads, n_kv_heads;
  void* q_out;
  long long q_out_stride;
  void* k_out;  // NULL: keys go to the cache only
  long long k_out_stride;
  const int64_t* dst_rows;
  void* k_cache;  // NULL: no cache
  void* v_cache;
  float* k_scale;
  float* v_scale;
  long long cache_rows;
  int* status;
  uint64_t turns[kHeadDim / 2];  // of pair j a position: 2^64 is a whole turn
  uint8_t axis[kHeadDim / 2];
};
cudaError_t launch_rotary(const RotaryArgs& a, int dtype, bool adjacent, bool cache8, cudaStream_t stream);

// What the operators over pages have in common: request b's row j is cache row table[b][j >> shift] << shift | j & (2^shift - 1)
struct PagedCache {
  const int32_t* table;  // [B, width]
  int width;
  int shift;
  int n_pages;
  const int64_t* lengths;
  int B;
};

struct PagedArgs {
  PagedCache pages;
  const void* q;
  long long q_stride;
  const void* k_cache;
  const void* v_cache;
  const float* k_scale;
  const float* v_scale;
  long long cache_rows;
  const int32_t* picked;  // [B, n_kv_heads, n_picked] or NULL
  int n_picked;
  int n_heads, n_kv_heads;
  void* out;
  float* lse;
  void* workspace;
  int* status;
};
size_t paged_attention_workspace_bytes(int B, int n_heads, int n_kv_heads);
cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, bool cache8, cudaStream_t stream);

struct BoundsArgs {
  PagedCache pages;
  const void* k_cache;
  const float* k_scale;
  long long cache_rows;
  const int64_t* start;  // NULL: 0
  int n_kv_heads;
  int8_t* bounds;      // [n_pages, n_kv_heads, 2, 128]
  float* bound_scale;  // [n_kv_heads, n_pages]
  int* status;
};
cudaError_t launch_page_bounds(const BoundsArgs& a, int cache_dtype, cudaStream_t stream);

struct SelectArgs {
  PagedCache pages;
  const void* q;
  long long q_stride;
  const int8_t* bounds;
  const float* bound_scale;
  int n_heads, n_kv_heads;
  int first, last;
  int32_t* picked;
  int n_picked;
  int* status;
};
cudaError_t launch_page_select(const SelectArgs& a, int dtype, cudaStream_t stream);

struct StepArgs {
  const int32_t* table;    // [B_in, width]
  const int64_t* lengths;  // [B_in]
  const int32_t* refs;     // [n_pages]
  int B_in;
  const int32_t* source;  // [B] or NULL: request i goes on from request i
  const int64_t* new_offsets;
  int B;
  long long new_rows;
  int width, shift, n_pages;
  int32_t* table_out;
  int64_t* lengths_out;
  int32_t* refs_out;
  int64_t* rows;
  int32_t* pairs;
  int32_t* n_pairs;
  int* status;
};
cudaError_t launch_pages_step(const StepArgs& a, cudaStream_t stream);

struct CompactArgs {
  const int32_t* table;
  const int64_t* lengths;
  const int32_t* refs;
  int B, width, shift, n_pages;
  int32_t* table_out;
  int32_t* refs_out;
  int32_t* pairs;
  int32_t* n_pairs;
  int* status;
};
cudaError_t launch_pages_compact(const CompactArgs& a, cudaStream_t stream);

cudaError_t launch_pages_copy(const fsx_page_plane* planes, int n_planes, int n_pages, const int32_t* pairs,
                              const int32_t* n_pairs, int max_pairs, int* status, cudaStream_t stream);

}  // namespace fsx
