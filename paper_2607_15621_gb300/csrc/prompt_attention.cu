// Attention of whole prompts, packed one after another (fsx_prompt_attention).
//
// A warp per (query row, head): lane l holds dims 4 l .. 4 l + 3 of the query and of the output; the
// keys that the row sees are taken one at a time with a running maximum and sum. Keys that it does not see are never read.
#include <math_constants.h>

#include "attention_rows.cuh"
#include "fsx.h"
#include "kernels.h"
#include "llm.h"

namespace fsx {

namespace {

template <typename T>
__global__ void __launch_bounds__(128) prompt_rows_kernel(const PromptArgs p) {
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31;
  const int kvh = h / (p.n_heads / p.n_kv_heads);
  const long long q0 = p.q_offsets[b], q1 = p.q_offsets[b + 1], k0 = p.kv_offsets[b], k1 = p.kv_offsets[b + 1];
  if (q0 < 0 || q1 < q0 || q1 > p.q_rows || k0 < 0 || k1 < k0 || k1 > p.kv_rows) {
    if (threadIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    return;
  }
  const long long nq = q1 - q0, nk = k1 - k0;
  for (long long i = blockIdx.x * 4 + (threadIdx.x >> 5); i < nq; i += gridDim.x * 4) {
    const long long see = p.causal ? min(nk, nk - nq + i + 1) : nk;
    RowState st;
    row_query(st, static_cast<const T*>(p.q) + (q0 + i) * p.q_stride + h * kHeadDim + lane * 4);
    for (long long j = 0; j < see; ++j) {
      const long long at = (k0 + j) * p.kv_stride + kvh * kHeadDim + lane * 4;
      row_key(st, load4(static_cast<const T*>(p.k) + at), load4(static_cast<const T*>(p.v) + at));
    }
    row_finish(st, static_cast<T*>(p.out) + ((q0 + i) * p.n_heads + h) * kHeadDim + lane * 4,
               p.lse != nullptr ? p.lse + h * p.q_rows + q0 + i : nullptr, lane);
  }
}

}  // namespace

cudaError_t launch_prompt_attention(const PromptArgs& a, int dtype, cudaStream_t stream) {
  const long long want = (a.q_rows + 3) / 4;
  const dim3 grid(static_cast<unsigned>(want < 256 ? want : 256), a.n_heads, a.B);
  void* args[] = {const_cast<PromptArgs*>(&a)};
  return launch_ex(dtype == FSX_BF16 ? reinterpret_cast<const void*>(&prompt_rows_kernel<__nv_bfloat16>)
                                     : reinterpret_cast<const void*>(&prompt_rows_kernel<__half>),
                   grid, dim3(128), 0, stream, false, args);
}

}  // namespace fsx
