// C-ABI entry points of the language-model operators: host checks, then the launch.
#include <cstdarg>
#include <cstdio>

#include "fsx.h"
#include "kernels.h"
#include "llm.h"

namespace fsx {
void set_error_message(const char* msg);
}

namespace {

fsx_status fail(fsx_status s, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  fsx::set_error_message(buf);
  return s;
}

fsx_status launched(cudaError_t e, const char* what) {
  return e == cudaSuccess ? FSX_OK : fail(FSX_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

constexpr long long kMaxRows = 0x7fffffffll;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

fsx_status check_heads(int n_heads, int n_kv_heads, int head_dim) {
  if (head_dim != fsx::kHeadDim) return fail(FSX_ERR_UNSUPPORTED, "head_dim must be 128");
  if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0)
    return fail(FSX_ERR_INVALID_ARG, "n_heads must be a positive multiple of n_kv_heads");
  if (n_heads / n_kv_heads > fsx::kMaxGroup || n_heads > 4096)
    return fail(FSX_ERR_UNSUPPORTED, "at most 64 heads per kv head and 4096 heads");
  return FSX_OK;
}

fsx_status check_stride(const char* what, const void* p, long long stride, int heads, int element) {
  if (stride < static_cast<long long>(heads) * fsx::kHeadDim || stride > (1ll << 32) || (stride * element) % 16 != 0)
    return fail(FSX_ERR_INVALID_ARG, "%s: the row stride must cover the heads and be a multiple of 16 bytes", what);
  if (!aligned16(p)) return fail(FSX_ERR_INVALID_ARG, "%s must be 16-byte aligned", what);
  return FSX_OK;
}

fsx_status check_cache8(const fsx::Cache8Args& a, int head_dim) {
  if (!a.status) return fail(FSX_ERR_INVALID_ARG, "d_status is NULL");
  if (a.dtype != FSX_F32 && a.dtype != FSX_BF16 && a.dtype != FSX_F16) return fail(FSX_ERR_INVALID_ARG, "bad dtype");
  if (a.n_rows < 0 || a.cache_rows < 0) return fail(FSX_ERR_INVALID_ARG, "n_rows and cache_rows must be >= 0");
  if (a.n_rows > kMaxRows || a.cache_rows > kMaxRows)
    return fail(FSX_ERR_UNSUPPORTED, "n_rows and cache_rows must be below 2^31");
  fsx_status s = check_heads(a.n_kv_heads, a.n_kv_heads, head_dim);
  if (s != FSX_OK) return s;
  if (a.n_rows == 0) return FSX_OK;
  if (!a.k || !a.v || !a.k_cache || !a.v_cache || !a.k_scale || !a.v_scale)
    return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (!a.rows && a.n_rows > a.cache_rows) return fail(FSX_ERR_INVALID_ARG, "n_rows exceeds cache_rows");
  const int element = a.dtype == FSX_F32 ? 4 : 2;
  if ((s = check_stride("d_k", a.k, a.kv_stride, a.n_kv_heads, element)) != FSX_OK) return s;
  if ((s = check_stride("d_v", a.v, a.kv_stride, a.n_kv_heads, element)) != FSX_OK) return s;
  if (!aligned16(a.k_cache) || !aligned16(a.v_cache)) return fail(FSX_ERR_INVALID_ARG, "caches must be 16-byte aligned");
  return FSX_OK;
}

}  // namespace

extern "C" {

fsx_status fsx_cache_write_e4m3(const void* d_k, const void* d_v, long long kv_stride, int dtype, const int64_t* d_rows,
                                long long n_rows, int n_kv_heads, int head_dim, void* d_k_cache, void* d_v_cache,
                                float* d_k_scale, float* d_v_scale, long long cache_rows, int* d_status, void* stream) {
  fsx::set_error_message("");
  const fsx::Cache8Args a{d_k,       d_v,       kv_stride, dtype,     d_rows,     n_rows,  n_kv_heads,
                          d_k_cache, d_v_cache, d_k_scale, d_v_scale, cache_rows, d_status};
  const fsx_status s = check_cache8(a, head_dim);
  if (s != FSX_OK || n_rows == 0) return s;
  return launched(fsx::launch_cache_write(a, static_cast<cudaStream_t>(stream)), "cache write");
}

fsx_status fsx_cache_read_e4m3(const void* d_k_cache, const void* d_v_cache, const float* d_k_scale,
                               const float* d_v_scale, long long cache_rows, const int64_t* d_rows, long long n_rows,
                               int n_kv_heads, int head_dim, void* d_k, void* d_v, long long kv_stride, int dtype,
                               int* d_status, void* stream) {
  fsx::set_error_message("");
  const fsx::Cache8Args a{d_k,
                          d_v,
                          kv_stride,
                          dtype,
                          d_rows,
                          n_rows,
                          n_kv_heads,
                          const_cast<void*>(d_k_cache),
                          const_cast<void*>(d_v_cache),
                          const_cast<float*>(d_k_scale),
                          const_cast<float*>(d_v_scale),
                          cache_rows,
                          d_status};
  const fsx_status s = check_cache8(a, head_dim);
  if (s != FSX_OK || n_rows == 0) return s;
  return launched(fsx::launch_cache_read(a, static_cast<cudaStream_t>(stream)), "cache read");
}

fsx_status fsx_prompt_attention(const void* d_q, long long q_stride, const void* d_k, const void* d_v,
                                long long kv_stride, int dtype, const int64_t* d_q_offsets,
                                const int64_t* d_kv_offsets, int B, long long q_rows, long long kv_rows, int n_heads,
                                int n_kv_heads, int head_dim, int causal, void* d_out, float* d_lse, int* d_status,
                                void* stream) {
  fsx::set_error_message("");
  if (!d_status || !d_q_offsets || !d_kv_offsets) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (dtype != FSX_BF16 && dtype != FSX_F16) return fail(FSX_ERR_INVALID_ARG, "dtype must be FSX_BF16 or FSX_F16");
  if (B < 1 || B > fsx::kMaxSequences) return fail(FSX_ERR_INVALID_ARG, "B must be in 1..1024");
  if (q_rows < 0 || kv_rows < 0) return fail(FSX_ERR_INVALID_ARG, "q_rows and kv_rows must be >= 0");
  if (q_rows > kMaxRows || kv_rows > kMaxRows) return fail(FSX_ERR_UNSUPPORTED, "rows must be below 2^31");
  if (causal != 0 && causal != 1) return fail(FSX_ERR_INVALID_ARG, "causal must be 0 or 1");
  fsx_status s = check_heads(n_heads, n_kv_heads, head_dim);
  if (s != FSX_OK || q_rows == 0) return s;
  if (!d_q || !d_out || (kv_rows > 0 && (!d_k || !d_v))) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if ((s = check_stride("d_q", d_q, q_stride, n_heads, 2)) != FSX_OK) return s;
  if (kv_rows > 0 && (s = check_stride("d_k", d_k, kv_stride, n_kv_heads, 2)) != FSX_OK) return s;
  if (kv_rows > 0 && (s = check_stride("d_v", d_v, kv_stride, n_kv_heads, 2)) != FSX_OK) return s;
  if (!aligned16(d_out)) return fail(FSX_ERR_INVALID_ARG, "d_out must be 16-byte aligned");
  const long long group_rows = q_rows * (n_heads / n_kv_heads);
  if (group_rows >= kMaxRows - 256 || (group_rows / 256 + B) * n_kv_heads >= kMaxRows - 65536)
    return fail(FSX_ERR_UNSUPPORTED, "q_rows times the heads per kv head must be below 2^31 - 257, and 256-row items below 2^31 - 65537");
  const fsx::PromptArgs a{d_q,    q_stride, d_k,     d_v,     kv_stride,  d_q_offsets, d_kv_offsets, B,
                          q_rows, kv_rows,  n_heads, n_kv_heads, causal, d_out,       d_lse,        d_status};
  return launched(fsx::launch_prompt_attention(a, dtype, static_cast<cudaStream_t>(stream)), "prompt attention");
}

size_t fsx_tree_attention_workspace_bytes(int B, long long new_rows, int n_heads, int n_kv_heads) {
  if (B < 1 || new_rows < 0 || n_kv_heads < 1 || n_heads < n_kv_heads) return 0;
  return fsx::tree_attention_workspace_bytes(B, new_rows, n_heads, n_kv_heads);
}

fsx_status fsx_tree_attention(const void* d_q, long long q_stride, const void* d_k_new, const void* d_v_new,
                              long long new_stride, int dtype, const int64_t* d_new_offsets, const uint64_t* d_mask,
                              long long new_rows, const void* d_k_cache, const void* d_v_cache, const float* d_k_scale,
                              const float* d_v_scale, int cache_dtype, long long cache_rows, const int64_t* d_starts,
                              const int64_t* d_offsets, int B, int n_heads, int n_kv_heads, int head_dim, void* d_out,
                              float* d_lse, void* d_workspace, size_t workspace_bytes, int* d_status, void* stream) {
  fsx::set_error_message("");
  if (!d_status || !d_new_offsets || !d_offsets) return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (dtype != FSX_BF16 && dtype != FSX_F16) return fail(FSX_ERR_INVALID_ARG, "dtype must be FSX_BF16 or FSX_F16");
  if (cache_dtype != dtype && cache_dtype != FSX_E4M3)
    return fail(FSX_ERR_INVALID_ARG, "cache_dtype must be dtype or FSX_E4M3");
  if (B < 1 || B > fsx::kMaxSequences) return fail(FSX_ERR_INVALID_ARG, "B must be in 1..1024");
  if (new_rows < 0 || cache_rows < 0) return fail(FSX_ERR_INVALID_ARG, "new_rows and cache_rows must be >= 0");
  if (new_rows > kMaxRows || cache_rows > kMaxRows) return fail(FSX_ERR_UNSUPPORTED, "rows must be below 2^31");
  fsx_status s = check_heads(n_heads, n_kv_heads, head_dim);
  if (s != FSX_OK || new_rows == 0) return s;
  if (new_rows * n_heads > 4 * kMaxRows) return fail(FSX_ERR_UNSUPPORTED, "new_rows times n_heads must be below 2^33");
  if (!d_q || !d_k_new || !d_v_new || !d_mask || !d_out || (cache_rows > 0 && (!d_k_cache || !d_v_cache)))
    return fail(FSX_ERR_INVALID_ARG, "NULL pointer argument");
  if (cache_dtype == FSX_E4M3 && cache_rows > 0 && (!d_k_scale || !d_v_scale))
    return fail(FSX_ERR_INVALID_ARG, "an e4m3 cache needs its scales");
  if ((s = check_stride("d_q", d_q, q_stride, n_heads, 2)) != FSX_OK) return s;
  if ((s = check_stride("d_k_new", d_k_new, new_stride, n_kv_heads, 2)) != FSX_OK) return s;
  if ((s = check_stride("d_v_new", d_v_new, new_stride, n_kv_heads, 2)) != FSX_OK) return s;
  if (!aligned16(d_out) || !aligned16(d_k_cache) || !aligned16(d_v_cache))
    return fail(FSX_ERR_INVALID_ARG, "d_out and the caches must be 16-byte aligned");
  const size_t need = fsx::tree_attention_workspace_bytes(B, new_rows, n_heads, n_kv_heads);
  if (!d_workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(d_workspace) & 255u) != 0)
    return fail(FSX_ERR_INVALID_ARG, "a 256-byte aligned workspace of %zu bytes is required", need);
  const fsx::TreeArgs a{d_q,       q_stride,  d_k_new,    d_v_new,  new_stride, d_new_offsets, d_mask,  new_rows,
                        d_k_cache, d_v_cache, d_k_scale,  d_v_scale, cache_rows, d_starts,     d_offsets, B,
                        n_heads,   n_kv_heads, d_out,     d_lse,    d_workspace, d_status};
  return launched(fsx::launch_tree_attention(a, dtype, cache_dtype == FSX_E4M3, static_cast<cudaStream_t>(stream)),
                  "tree attention");
}

}  // extern "C"
