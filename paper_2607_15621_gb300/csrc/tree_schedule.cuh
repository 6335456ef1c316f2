// How the attention of drafted tokens shares its work out. Every (request, tile of its rows, kv head)
// is an item of ceil(cache rows / chunk) chunks and one more for the new tokens. The kernel for many rows
// (tree_tc.cu) takes only the requests and the workspace's head from here; it plans, stores and joins its pieces itself.
//
// The kernel for few rows (tree_attention.cu): items of up to `few` chunks stay whole; longer ones are cut into near-equal pieces
// of `most` chunks at most, which follows from the number of all chunks (the host knows no lengths), so that one long request
// fills the GPU as well as many short ones. CTAs take pieces from one queue: equal shares fixed before left the SMs idle a
// quarter of the time (some read the caches faster than others, and a short cache costs more per row). The pieces of a cut
// item are put together by whichever comes last, in the order of its keys, so that results do not depend on the order of
// arrival.
//
// Workspace: the header, counters (one per cut item, at its first slot), one slot of partial results per piece of a cut
// item. Header and counters are zero between calls.
#pragma once

#include "device_util.cuh"
#include "llm.h"

namespace fsx {

constexpr int kTreeHeader = 64;      // ints: [0] pieces taken from the queue, beyond each CTA's first, [1] CTAs that are done
constexpr int kTreeCounters = 8192;  // as many for every kernel: what follows them may hold anything

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

// Geometry of a kernel's items
struct TreeShape {
  int tile_rows, chunk;  // rows of an item, keys of a chunk
  int few, many;         // an item of `few` chunks or less is not cut; a piece has `many` at most
  int slots;             // of the workspace
};

__device__ __forceinline__ int tree_chunks(const TreeShape& s, int len) { return static_cast<int>((static_cast<uint32_t>(len) + s.chunk - 1) / s.chunk) + 1; }
__device__ __forceinline__ int tree_pieces(const TreeShape& s, int n, int most) {
  return n <= s.few ? 1 : (n + most - 1) / most;
}

struct TreePlan {
  uint32_t* pieces;   // [B + 1] pieces of the requests before: at most 2^31 items and the slots of cut ones
  int* slots;         // [B + 1] slots of the requests before
  int most;           // chunks of a piece
};
__host__ __device__ constexpr size_t tree_plan_bytes(int B) { return (B + 1) * 2 * sizeof(int); }

// By all THREADS threads of the CTA; `at`: tree_plan_bytes(B) bytes; `scratch`: 2 values per warp.
template <int THREADS>
__device__ __forceinline__ TreePlan tree_plan(const TreeArgs& p, const TreeShape& shape, void* at, long long* scratch) {
  constexpr int kW = THREADS / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = p.n_heads / p.n_kv_heads;
  const int per = (p.B + THREADS - 1) / THREADS, b0 = tid * per, b1 = min(p.B, b0 + per);
  TreePlan plan;
  plan.pieces = static_cast<uint32_t*>(at);
  plan.slots = reinterpret_cast<int*>(plan.pieces + p.B + 1);
  auto items = [&](const TreeRequest& r) {
    return static_cast<long long>((r.n * G + shape.tile_rows - 1) / shape.tile_rows) * p.n_kv_heads;
  };
  // an even share, or a part of it; and cut items of n > most chunks take at most 2 n / most slots (in 32 bits where
  // it fits: a 64-bit division is a hundred instructions that every CTA waits for)
  auto most_of = [&](long long total) {
    const bool small = total < 0x3fffffff;
    const uint32_t even = small ? (static_cast<uint32_t>(total) + gridDim.x - 1) / gridDim.x : 0x7fffffffu;
    const uint32_t turns = (even + shape.many - 1) / shape.many;  // pieces that a CTA takes, if they were all alike
    const long long share = turns > 0 ? (even + turns - 1) / turns : 1;
    const long long room = small ? (2 * static_cast<uint32_t>(total) + shape.slots - 1) / shape.slots : (2 * total + shape.slots - 1) / shape.slots;
    return static_cast<int>(min(max(max(share, room), static_cast<long long>((shape.few + 1) / 2)), 0x7fffffffll));
  };
  if (p.B <= 32) {  // a lane a request, one barrier
    if (warp == 0) {
      TreeRequest r{};
      const bool mine = lane < p.B;
      if (mine && !tree_request(p, lane, r) && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
      const long long n_items = mine ? items(r) : 0;
      const int n = mine ? tree_chunks(shape, r.len) : 0;
      long long total = n_items * n;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      const int most = most_of(total);
      const int of = tree_pieces(shape, n, most);
      const uint32_t pieces = static_cast<uint32_t>(n_items) * of, slots = of > 1 ? pieces : 0;
      uint32_t sum = pieces, sum_slots = slots;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o), up_slots = __shfl_up_sync(0xffffffffu, sum_slots, o);
        if (lane >= o) {
          sum += up;
          sum_slots += up_slots;
        }
      }
      if (mine) {
        plan.pieces[lane] = sum - pieces;
        plan.slots[lane] = static_cast<int>(sum_slots - slots);
        if (lane == p.B - 1) plan.pieces[p.B] = sum;
      }
      if (lane == 0) scratch[0] = most;
    }
    __syncthreads();
    plan.most = static_cast<int>(scratch[0]);
    return plan;
  }
  long long total = 0;
  for (int b = b0; b < b1; ++b) {
    TreeRequest r;
    if (!tree_request(p, b, r) && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    total += items(r) * tree_chunks(shape, r.len);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) scratch[warp] = total;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kW; ++w) total += scratch[w];
  plan.most = most_of(total);
  long long mine = 0, mine_slots = 0;
  for (int b = b0; b < b1; ++b) {
    TreeRequest r;
    tree_request(p, b, r);
    const int n = tree_pieces(shape, tree_chunks(shape, r.len), plan.most);
    plan.pieces[b] = static_cast<uint32_t>(mine);  // within this thread's requests
    plan.slots[b] = static_cast<int>(mine_slots);
    mine += items(r) * n;
    mine_slots += n > 1 ? items(r) * n : 0;
  }
  long long sum = mine, sum_slots = mine_slots;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, sum, o), up_slots = __shfl_up_sync(0xffffffffu, sum_slots, o);
    if (lane >= o) {
      sum += up;
      sum_slots += up_slots;
    }
  }
  __syncthreads();
  if (lane == 31) {
    scratch[warp] = sum;
    scratch[kW + warp] = sum_slots;
  }
  __syncthreads();
  sum -= mine;
  sum_slots -= mine_slots;
  for (int w = 0; w < warp; ++w) {
    sum += scratch[w];
    sum_slots += scratch[kW + w];
  }
  for (int b = b0; b < b1; ++b) {
    plan.pieces[b] += static_cast<uint32_t>(sum);
    plan.slots[b] += static_cast<int>(sum_slots);
  }
  if (tid == THREADS - 1) plan.pieces[p.B] = static_cast<uint32_t>(sum + mine);
  __syncthreads();
  return plan;
}

struct TreePiece {
  TreeRequest r;
  int kvh, row0;    // kv head, first row of the tile (row = token G + head of the group)
  int from, to, n;  // chunks from .. to - 1 of n; chunk n - 1 holds the new tokens
  int slot, j, of;  // piece j of `of`; `slot` is that of piece 0
};
__device__ __forceinline__ TreePiece tree_piece(const TreeArgs& p, const TreeShape& shape, const TreePlan& plan, long long i) {
  int lo = 0, hi = p.B;  // pieces[lo] <= i < pieces[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (plan.pieces[mid] <= i) lo = mid;
    else hi = mid;
  }
  TreePiece x;
  tree_request(p, lo, x.r);
  x.n = tree_chunks(shape, x.r.len);
  x.of = tree_pieces(shape, x.n, plan.most);
  const uint32_t rel = static_cast<uint32_t>(i - plan.pieces[lo]);  // a request has less than 2^32 pieces
  const uint32_t item = rel / static_cast<uint32_t>(x.of);
  x.j = static_cast<int>(rel - item * x.of);
  x.slot = plan.slots[lo] + static_cast<int>(rel) - x.j;
  const uint32_t least = static_cast<uint32_t>(x.n) / static_cast<uint32_t>(x.of), more = x.n - least * x.of;
  x.from = static_cast<int>(x.j * least + min(static_cast<uint32_t>(x.j), more));
  x.to = static_cast<int>(x.from + least + (static_cast<uint32_t>(x.j) < more ? 1 : 0));
  const uint32_t tile = item / static_cast<uint32_t>(p.n_kv_heads);
  x.kvh = static_cast<int>(item - tile * p.n_kv_heads);
  x.row0 = static_cast<int>(tile) * shape.tile_rows;
  return x;
}

}  // namespace fsx
