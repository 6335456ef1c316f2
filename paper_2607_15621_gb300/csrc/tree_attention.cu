// Attention of a few new tokens of each request over its cache and over one another
// (fsx_tree_attention).
//
// A warp per (new token, head): lane l holds dims 4 l .. 4 l + 3 of the query and of the output; the
// cache rows, then the new tokens that the mask names, are taken one at a time with a running maximum and sum.
#include <type_traits>

#include "attention_rows.cuh"
#include "fsx.h"
#include "kernels.h"
#include "llm.h"

namespace fsx {

namespace {

template <typename T, bool C8>
__global__ void __launch_bounds__(128) tree_rows_kernel(const TreeArgs p) {
  using CT = typename std::conditional<C8, unsigned char, T>::type;
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31;
  const int kvh = h / (p.n_heads / p.n_kv_heads);
  const long long t0 = p.new_offsets[b], t1 = p.new_offsets[b + 1];
  const long long c0 = p.starts != nullptr ? p.starts[b] : p.offsets[b], len = p.offsets[b + 1] - p.offsets[b];
  if (t0 < 0 || t1 < t0 || t1 > p.new_rows || t1 - t0 > kMaxDrafts || c0 < 0 || len < 0 || c0 > p.cache_rows ||
      len > p.cache_rows - c0) {
    if (threadIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    return;
  }
  const int n = static_cast<int>(t1 - t0);
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 5); i < n; i += gridDim.x * 4) {
    RowState st;
    row_query(st, static_cast<const T*>(p.q) + (t0 + i) * p.q_stride + h * kHeadDim + lane * 4);
    for (long long j = 0; j < len; ++j) {
      const long long at = ((c0 + j) * p.n_kv_heads + kvh) * kHeadDim + lane * 4;
      float4 k = load4(static_cast<const CT*>(p.k_cache) + at), v = load4(static_cast<const CT*>(p.v_cache) + at);
      if (C8) {
        k = scaled(k, p.k_scale[kvh * p.cache_rows + c0 + j]);
        v = scaled(v, p.v_scale[kvh * p.cache_rows + c0 + j]);
      }
      row_key(st, k, v);
    }
    const uint64_t mask = p.mask[t0 + i];
    for (int j = 0; j < n; ++j)
      if ((mask >> j) & 1u) {
        const long long at = (t0 + j) * p.new_stride + kvh * kHeadDim + lane * 4;
        row_key(st, load4(static_cast<const T*>(p.k_new) + at), load4(static_cast<const T*>(p.v_new) + at));
      }
    row_finish(st, static_cast<T*>(p.out) + ((t0 + i) * p.n_heads + h) * kHeadDim + lane * 4,
               p.lse != nullptr ? p.lse + h * p.new_rows + t0 + i : nullptr, lane);
  }
}

}  // namespace

size_t tree_attention_workspace_bytes(int, long long, int, int) { return 256; }

cudaError_t launch_tree_attention(const TreeArgs& a, int dtype, bool cache8, cudaStream_t stream) {
  void* args[] = {const_cast<TreeArgs*>(&a)};
  const void* fn = dtype == FSX_BF16 ? (cache8 ? reinterpret_cast<const void*>(&tree_rows_kernel<__nv_bfloat16, true>)
                                               : reinterpret_cast<const void*>(&tree_rows_kernel<__nv_bfloat16, false>))
                                     : (cache8 ? reinterpret_cast<const void*>(&tree_rows_kernel<__half, true>)
                                               : reinterpret_cast<const void*>(&tree_rows_kernel<__half, false>));
  return launch_ex(fn, dim3(kMaxDrafts / 4, a.n_heads, a.B), dim3(128), 0, stream, false, args);
}

}  // namespace fsx
