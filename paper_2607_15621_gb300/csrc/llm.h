// Launch interface of the language-model operators: prompt attention (prompt_attention.cu), the
// 8-bit cache (cache8.cu) and the attention of drafted tokens (tree_attention.cu). Arguments have
// been checked by llm.cu.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fsx {

constexpr int kMaxSequences = 1024;  // B of prompt and tree attention
constexpr int kMaxGroup = 64;        // query heads per kv head
constexpr int kMaxDrafts = 64;       // new tokens of a request (one mask word)

// SMs of the current device (0: none); the most dynamic shared memory that launches of `fn` may ask for (launch.cu)
int sm_count();
cudaError_t allow_shared_memory(const void* fn, size_t bytes);

struct Cache8Args {
  const void* k;  // rows in or out, kv_stride elements apart
  const void* v;
  long long kv_stride;
  int dtype;  // fsx_dtype
  const int64_t* rows;
  long long n_rows;
  int n_kv_heads;
  void* k_cache;
  void* v_cache;
  float* k_scale;
  float* v_scale;
  long long cache_rows;
  int* status;
};
cudaError_t launch_cache_write(const Cache8Args& a, cudaStream_t stream);
cudaError_t launch_cache_read(const Cache8Args& a, cudaStream_t stream);

struct PromptArgs {
  const void* q;
  long long q_stride;
  const void* k;
  const void* v;
  long long kv_stride;
  const int64_t* q_offsets;
  const int64_t* kv_offsets;
  int B;
  long long q_rows, kv_rows;
  int n_heads, n_kv_heads;
  int causal;
  void* out;
  float* lse;
  int* status;
};
cudaError_t launch_prompt_attention(const PromptArgs& a, int dtype, cudaStream_t stream);

struct TreeArgs {
  const void* q;
  long long q_stride;
  const void* k_new;
  const void* v_new;
  long long new_stride;
  const int64_t* new_offsets;
  const uint64_t* mask;
  long long new_rows;
  const void* k_cache;
  const void* v_cache;
  const float* k_scale;
  const float* v_scale;
  long long cache_rows;
  const int64_t* starts;  // NULL: offsets
  const int64_t* offsets;
  int B;
  int n_heads, n_kv_heads;
  void* out;
  float* lse;
  void* workspace;
  int* status;
};
size_t tree_attention_workspace_bytes(int B, long long new_rows, int n_heads, int n_kv_heads);
// for many rows per request (tree_tc.cu)
size_t tree_tc_workspace_bytes(int B, long long new_rows, int n_heads, int n_kv_heads);
cudaError_t launch_tree_tc(const TreeArgs& a, int dtype, bool cache8, cudaStream_t stream);
cudaError_t launch_tree_attention(const TreeArgs& a, int dtype, bool cache8, cudaStream_t stream);

}  // namespace fsx
