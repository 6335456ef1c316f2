// How the attention of drafted tokens shares its work out: every (request, tile of its rows, kv head)
// is an item of ceil(cache rows / chunk) chunks and one more for the new tokens; the chunks of all items
// are one line, cut into equal ranges, one per CTA (the host knows no lengths, and one long request must
// fill the GPU as well as many short ones). An item that ranges cut is put together by whichever of
// its CTAs comes last, in the order of the ranges, so that results do not depend on the order of arrival.
// At most one cut item begins in a range and at most one ends in it: two slots of partial results and one counter a CTA.
#pragma once

#include "device_util.cuh"
#include "llm.h"

namespace fsx {

constexpr int kTreeMaxGrid = 1024;
constexpr size_t kTreeCounterBytes = kTreeMaxGrid * sizeof(int);

struct TreeRequest {
  long long c0;  // first cache row
  long long t0;  // first new token
  int len, n;    // cache rows, new tokens
};

// false: the offsets give no valid request
__device__ __forceinline__ bool tree_request(const TreeArgs& p, int b, TreeRequest& r) {
  const long long t1 = p.new_offsets[b + 1], o0 = p.offsets[b], len = p.offsets[b + 1] - o0;
  r.t0 = p.new_offsets[b];
  r.c0 = p.starts != nullptr ? p.starts[b] : o0;
  r.n = 0;
  r.len = 0;
  if (r.t0 < 0 || t1 < r.t0 || t1 > p.new_rows || t1 - r.t0 > kMaxDrafts || r.c0 < 0 || len < 0 || r.c0 > p.cache_rows ||
      len > p.cache_rows - r.c0)
    return false;
  r.n = static_cast<int>(t1 - r.t0);
  r.len = static_cast<int>(len);
  return true;
}

__device__ __forceinline__ int tree_chunks(int len, int chunk) { return (len + chunk - 1) / chunk + 1; }

// pre[b]: chunks of all items of the requests before b, pre[B] of all. THREADS threads of the CTA; `scratch`
// holds one value per warp.
template <int THREADS>
__device__ __forceinline__ void tree_prefix(const TreeArgs& p, int tile_rows, int chunk, long long* pre, long long* scratch) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = p.n_heads / p.n_kv_heads;
  const int per = (p.B + THREADS - 1) / THREADS;
  auto units = [&](int b) {
    TreeRequest r;
    if (!tree_request(p, b, r)) {
      if (blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
      return 0ll;
    }
    return static_cast<long long>((r.n * G + tile_rows - 1) / tile_rows) * p.n_kv_heads * tree_chunks(r.len, chunk);
  };
  long long mine = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < p.B) {
      pre[b] = mine;  // within this thread's requests
      mine += units(b);
    }
  }
  long long sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 31) scratch[warp] = sum;
  __syncthreads();
  long long before = sum - mine;
  for (int w = 0; w < warp; ++w) before += scratch[w];
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b < p.B) pre[b] += before;
  }
  if (tid == THREADS - 1) pre[p.B] = before + mine;
  __syncthreads();
}

// The part of an item that lies in this CTA's range [u, u1).
struct TreePiece {
  TreeRequest r;
  int kvh, row0;        // kv head, first row of the tile (row = token G + head of the group)
  int from, to, n;      // chunks from .. to - 1 of n; chunk n - 1 holds the new tokens
  int first_cta, last_cta;
};
__device__ __forceinline__ TreePiece tree_piece(const TreeArgs& p, const long long* pre, int tile_rows, int chunk, long long u,
                                                long long u1, long long per) {
  int lo = 0, hi = p.B;  // pre[lo] <= u < pre[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= u) lo = mid;
    else hi = mid;
  }
  TreePiece x;
  tree_request(p, lo, x.r);
  x.n = tree_chunks(x.r.len, chunk);
  const long long rel = u - pre[lo];
  const long long item = rel / x.n;
  x.from = static_cast<int>(rel - item * x.n);
  x.kvh = static_cast<int>(item % p.n_kv_heads);
  x.row0 = static_cast<int>(item / p.n_kv_heads) * tile_rows;
  const long long start = u - x.from, end = start + x.n;
  x.to = static_cast<int>(min(end, u1) - start);
  x.first_cta = static_cast<int>(start / per);
  x.last_cta = static_cast<int>((end - 1) / per);
  return x;
}

}  // namespace fsx
