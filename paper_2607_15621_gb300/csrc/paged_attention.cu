// Attention of one new token of each request over its cache in pages (fsx_paged_attention), all of them or those that a
// list picks for each kv head.
//
// The queries of a kv head's group are the rows, 8 NT of them an item, over the warps' steps of few_rows.cuh: 16 keys a step, keys
// as M of the matrix instructions. Bound by the cache's bytes. A page holds 16 rows or more, so the 16 keys of a step lie in one page and
// a warp needs one page number a step: at the start of a piece its lanes look up the pages of 32 steps at once, and a
// step's comes by a shuffle, so that no copy waits for the table.
//
// Items (request, tile of the group, kv head) are shared out in one of two ways:
//   line   few items. One CTA a SM with 8 warps and long rings; all steps of all items in one line, cut into as many equal ranges as there
//          are CTAs, so that every SM reads the same number of bytes; a cut less than 16 steps from an item's end moves there. Little work
//          goes in whole items or near-equal pieces of them, one a CTA. A CTA puts 8 warps together in shared memory, so an item that
//          is spread over the whole GPU has few partial results to join.
//   queue  many items. Four warps a CTA, three or four CTAs a SM, pieces of at most 14 chunks of 64 keys from one queue: SMs that
//          read faster take more, and one CTA's end overlaps with the others' loads.
// Keys and values are first to leave L2: the tables, queries and the kernel's own code, which a CTA fetches piece by piece as it comes to
// it, stay there (131,072 rows 58 -> 54 us).
// The pieces of a cut item are joined by the CTA that ends last, in the order of the keys. A piece that meets a page number
// outside the cache marks its result, and its item writes nothing.
//
// Measured: 128 requests of 64 to 2048 8-bit rows, 32 heads, 179 to 187 us (5.8 to 6.0 TB/s, 0.85 to 0.89 of a copy's rate; DRAM 73 %
// busy, issue slots 55 %; with weights in one part 173 to 183); one of 131,072 8-bit rows, 32 heads over 8, 49 to 52 us (5.3 to 5.6 TB/s: 4 us before the first products, 5
// after the last, SMs that differ by 12 %); 16 of 1000 to 8192 16-bit rows 44 us (5.2 TB/s); one of 224 rows 5.6 us.
#include <math_constants.h>

#include "few_rows.cuh"
#include "fsx.h"
#include "kernels.h"
#include "pages.h"

namespace fsx {

namespace {

// queue: chunks of an item that is not cut, and of a piece (64 requests of 500 to 4096 rows, 8 kv heads: 70 us, with 28 chunks 74)
constexpr int kFew = 8, kMany = 14;
// line, in steps: the least range; how near an item's end a cut moves there (32 requests of 500 to 4096 rows: 56 us, with 8 or 32 steps 61); the longest
// item that stays whole where there is little work (8 requests of 100 to 700 rows, 4 kv heads: 9.0 us, with 32 steps 10.5); how many a CTA that is
// (4 requests of 500 to 2000 rows, 32 kv heads: 18.5 us, 22.8 as a line)
constexpr int kLeast = 32, kSnap = 16, kWhole = 64, kShort = 128;
constexpr int kHeader = 64;          // ints of the workspace, queue: [0] pieces taken, [1] CTAs that are done
constexpr int kCounters = 8192;      // then one for each slot

struct Plan {
  int* len;          // [B] rows of the requests, -1: not in order
  uint32_t* pieces;  // [B + 1] pieces of the requests before
  int* slots;        // [B + 1] slots of the requests before
  int most;          // chunks of a piece
};
__host__ __device__ constexpr size_t plan_bytes(int B) { return (B + (B + 1) * 2) * sizeof(int); }

struct Request {
  int len;    // rows
  int pages;  // that hold them
  int steps;  // of 16 keys, over all pages or the picked ones
};
// -1: the length is negative or more than the table's pages hold; no items then
__device__ __forceinline__ int length_of(const PagedArgs& p, int b) {
  const long long len = p.pages.lengths[b];
  return len < 0 || len > static_cast<long long>(p.pages.width) << p.pages.shift || len > 0x7fffffffll - 64 ? -1 : static_cast<int>(len);
}
__device__ __forceinline__ Request request_of(const PagedArgs& p, int len) {
  Request r;
  r.len = len;
  r.pages = (len + (1 << p.pages.shift) - 1) >> p.pages.shift;
  r.steps = p.picked != nullptr ? min(r.pages, p.n_picked) << (p.pages.shift - 4) : (len + 15) >> 4;
  return r;
}
__device__ __forceinline__ int chunks_of(const Request& r) { return max(1, (r.steps + kWarps - 1) / kWarps); }
__device__ __forceinline__ int pieces_of(int n, int most) { return n <= kFew ? 1 : (n + most - 1) / most; }

// By all threads of the CTA; `scratch`: 2 values per warp. `items`: of a request that is in order.
__device__ __forceinline__ Plan make_plan(const PagedArgs& p, long long items, int slots, void* at, long long* scratch) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.pages.B;
  const int per = (B + kThreads - 1) / kThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  Plan plan;
  plan.len = static_cast<int*>(at);
  plan.pieces = reinterpret_cast<uint32_t*>(plan.len + B);
  plan.slots = reinterpret_cast<int*>(plan.pieces + B + 1);
  long long total = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = length_of(p, b);
    if (len < 0 && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    plan.len[b] = len;
    total += len < 0 ? 0 : chunks_of(request_of(p, len));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) scratch[warp] = total;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += scratch[w];
  total *= items;
  // an even share or a part of it; cut items of n > most chunks take at most 2 n / most slots
  if (total < 0x3fffffff) {
    const uint32_t even = (static_cast<uint32_t>(total) + gridDim.x - 1) / gridDim.x, turns = (even + kMany - 1) / kMany;
    const uint32_t share = turns > 0 ? (even + turns - 1) / turns : 1;
    plan.most = static_cast<int>(max(max(share, (2 * static_cast<uint32_t>(total) + slots - 1) / slots), (kFew + 1u) / 2));
  } else {
    plan.most = static_cast<int>(min((2 * total + slots - 1) / slots, 0x7fffffffll));
  }
  long long mine = 0, mine_slots = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = plan.len[b], of = len < 0 ? 0 : pieces_of(chunks_of(request_of(p, len)), plan.most);
    plan.pieces[b] = static_cast<uint32_t>(mine);  // within this thread's requests
    plan.slots[b] = static_cast<int>(mine_slots);
    mine += items * of;
    mine_slots += of > 1 ? items * of : 0;
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
    scratch[kWarps + warp] = sum_slots;
  }
  __syncthreads();
  sum -= mine;
  sum_slots -= mine_slots;
  for (int w = 0; w < warp; ++w) {
    sum += scratch[w];
    sum_slots += scratch[kWarps + w];
  }
  for (int b = b0; b < b1; ++b) {
    plan.pieces[b] += static_cast<uint32_t>(sum);
    plan.slots[b] += static_cast<int>(sum_slots);
  }
  if (tid == kThreads - 1) plan.pieces[B] = static_cast<uint32_t>(sum + mine);
  __syncthreads();
  return plan;
}

struct Piece {
  Request r;
  int b, kvh, row0;  // request, kv head, first row (head of the group) of the tile
  int from, to;      // steps
  int first, j, of;  // piece j of `of`; `first`: slot of piece 0 (line: its CTA)
};
__device__ __forceinline__ void set_item(const PagedArgs& p, Piece& x, uint32_t item, int tile_rows) {
  const uint32_t tile = item / static_cast<uint32_t>(p.n_kv_heads);
  x.kvh = static_cast<int>(item - tile * p.n_kv_heads);
  x.row0 = static_cast<int>(tile) * tile_rows;
}
// the last b with at[b] <= x, of at[0 .. n]
template <typename T>
__device__ __forceinline__ int find(const T* at, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ Piece piece_at(const PagedArgs& p, const Plan& plan, int tile_rows, uint32_t i) {
  Piece x;
  const int b = x.b = find(plan.pieces, p.pages.B, i);
  x.r = request_of(p, plan.len[b]);
  const int n = chunks_of(x.r);
  x.of = pieces_of(n, plan.most);
  const uint32_t rel = i - plan.pieces[b], item = rel / static_cast<uint32_t>(x.of);
  x.j = static_cast<int>(rel - item * x.of);
  x.first = plan.slots[b] + static_cast<int>(rel) - x.j;
  const uint32_t least = static_cast<uint32_t>(n) / static_cast<uint32_t>(x.of), more = n - least * x.of;
  x.from = static_cast<int>(x.j * least + min(static_cast<uint32_t>(x.j), more)) * kWarps;
  x.to = min(x.from + static_cast<int>(least + (static_cast<uint32_t>(x.j) < more ? 1 : 0)) * kWarps, x.r.steps);
  set_item(p, x, item, tile_rows);
  return x;
}

// The line of all steps: where each request's begin, and where the CTAs' ranges do. In 32 bits: the host sees to that.
struct Line {
  int* len;         // [B]
  uint32_t* start;  // [B + 1]
  uint32_t* cut;    // [CTAs + 1]
  uint32_t ranges;  // the rest of the CTAs have none
};
__host__ __device__ constexpr size_t line_bytes(int B, int ctas) { return (B + 2 * (B + 1) + ctas + 1) * sizeof(int); }
__device__ __forceinline__ uint32_t line_steps(const Request& r) { return max(1, r.steps); }

__device__ __forceinline__ uint32_t short_pieces(uint32_t n, uint32_t most) { return n <= kWhole ? 1u : (n + most - 1) / most; }

template <int W>
__device__ __forceinline__ Line make_line(const PagedArgs& p, uint32_t items, void* at, uint32_t* scratch) {
  constexpr int kThreadsLine = 32 * W;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.pages.B;
  Line line;
  line.len = static_cast<int*>(at);
  line.start = reinterpret_cast<uint32_t*>(line.len + B);
  line.cut = line.start + B + 1;
  uint32_t before = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < B; b0 += kThreadsLine) {  // a thread a request
    const int b = b0 + tid;
    uint32_t mine = 0;
    if (b < B) {
      const int len = length_of(p, b);
      line.len[b] = len;
      if (len >= 0) mine = items * line_steps(request_of(p, len));
      else if (blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    }
    uint32_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 31) scratch[warp] = sum;
    __syncthreads();
    uint32_t all = 0;
    const int warps = min(W, (B - b0 + 31) >> 5);
#pragma unroll 1
    for (int w = 0; w < warps; ++w) {
      if (w < warp) sum += scratch[w];
      all += scratch[w];
    }
    if (b < B) line.start[b] = before + sum - mine;
    before += all;
    if (b0 + kThreadsLine < B) __syncthreads();
  }
  if (tid == 0) line.start[B] = before;
  __syncthreads();
  const uint32_t ctas = gridDim.x, all_items = items * B;
  if (before < ctas * kShort && all_items <= ctas) {
    // little work: near-equal pieces of whole items, at most one a CTA, as many as there are CTAs for
    const uint32_t most = max(static_cast<uint32_t>(kLeast), (before + ctas - all_items) / max(1u, ctas - all_items));
    uint32_t* first = line.cut + ctas + 1;  // [B + 1] pieces of the requests before
    if (warp == 0) {
      uint32_t sum = 0;
#pragma unroll 1
      for (int b0 = 0; b0 < B; b0 += 32) {
        const int b = b0 + lane;
        const uint32_t mine = b < B && line.len[b] >= 0 ? items * short_pieces(line_steps(request_of(p, line.len[b])), most) : 0;
        uint32_t up_to = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t up = __shfl_up_sync(0xffffffffu, up_to, o);
          if (lane >= o) up_to += up;
        }
        if (b < B) first[b] = sum + up_to - mine;
        sum += __shfl_sync(0xffffffffu, up_to, 31);
      }
      if (lane == 0) first[B] = sum;
    }
    __syncthreads();
    line.ranges = max(1u, first[B]);
    for (uint32_t c = tid; c <= line.ranges; c += kThreadsLine) {
      uint32_t x = before;
      if (c < first[B]) {
        const int b = find(first, B, c);
        const uint32_t n = line_steps(request_of(p, line.len[b])), of = short_pieces(n, most), rel = c - first[b], item = rel / of;
        x = line.start[b] + item * n + (rel - item * of) * n / of;
      }
      line.cut[c] = x;
    }
    __syncthreads();
    return line;
  }
  // equal ranges; a cut less than 16 steps from an item's end moves there
  line.ranges = max(1u, min(ctas, before / kLeast));
  const uint32_t least = before / line.ranges, more = before - least * line.ranges;
  for (uint32_t c = tid; c <= line.ranges; c += kThreadsLine) {
    uint32_t x = c * least + c * more / line.ranges;
    if (c < line.ranges && c > 0) {
      const int b = find(line.start, B, x);
      const uint32_t n = line_steps(request_of(p, line.len[b])), off = (x - line.start[b]) % n;
      if (off < kSnap) x -= off;
      else if (n - off < kSnap) x += n - off;
    }
    line.cut[c] = x;
  }
  __syncthreads();
  return line;
}
// The part of the range that begins at step `at` of the line, up to its item's end; `at` moves on
__device__ __forceinline__ Piece segment_at(const PagedArgs& p, const Line& line, int tile_rows, uint32_t end, uint32_t& at) {
  Piece x;
  const int b = x.b = find(line.start, p.pages.B, at);
  x.r = request_of(p, line.len[b]);
  const uint32_t n = line_steps(x.r), rel = at - line.start[b], item = rel / n;
  x.from = static_cast<int>(rel - item * n);
  x.to = static_cast<int>(min(n, x.from + (end - at)));
  x.first = x.j = 0;
  x.of = 1;
  if (x.from > 0 || x.to < n) {
    const uint32_t s = at - x.from;
    x.first = find(line.cut, static_cast<int>(line.ranges), s);
    x.of = find(line.cut, static_cast<int>(line.ranges), s + n - 1) - x.first + 1;
    x.j = static_cast<int>(blockIdx.x) - x.first;
  }
  at += x.to - x.from;
  x.to = min(x.to, x.r.steps);  // a request without rows has a step of none
  set_item(p, x, item, tile_rows);
  return x;
}
// Slot of an item's piece: a CTA of a line has two, for the item that began before its range and for the one that goes on behind it
template <bool LINE>
__device__ __forceinline__ int slot_of(const Piece& x, int j) {
  return LINE ? 2 * (x.first + j) + (j == 0 ? 1 : 0) : x.first + j;
}

// First cache row of step `step` and how many of its 16 rows are keys of the request. False: no page of the cache.
__device__ __forceinline__ bool look_up(const PagedArgs& p, const Piece& it, int step, int& row, int& left) {
  row = left = 0;
  if (step >= it.r.steps) return true;
  const int shift = p.pages.shift, in_page = step & ((1 << (shift - 4)) - 1);
  int page = step >> (shift - 4);
  if (p.picked != nullptr) {
    page = p.picked[(static_cast<long long>(it.b) * p.n_kv_heads + it.kvh) * p.n_picked + page];
    if (page == -1) return true;
    if (page < 0 || page >= it.r.pages) return false;
  }
  left = min(16, it.r.len - ((page << shift) + in_page * 16));
  if (left <= 0) {
    left = 0;
    return true;
  }
  const int at = p.pages.table[static_cast<long long>(it.b) * p.pages.width + page];
  if (at < 0 || at >= p.pages.n_pages) {
    left = 0;
    return false;
  }
  row = (at << shift) + in_page * 16;
  return true;
}

// Rows of sums in shared memory: where dim d lies, and floats from row to row. A warp stores two dims of 8 lane groups g for 4 rows at
// once; turned by g within its 16 (8) dims and with this pitch they fall on different banks but for two (as they are, 16 at
// once on the same: 2 us for 7 rows of 16 warps).
template <bool C8>
constexpr int kPitch = C8 ? kD + 4 : kD + 2;
template <bool C8>
__device__ __forceinline__ int place_of(int d) {
  return C8 ? (d & ~15) | ((d + 2 * (d >> 5)) & 15) : (d & ~7) | ((d + 2 * ((d >> 5) & 1)) & 7);
}

// Warps of a CTA, rows that they put together at a time
template <bool C8, int NT, bool LINE>
struct Shape {
  static constexpr int kWarps = LINE ? 8 : fsx::kWarps;
  static constexpr int kStages = LINE ? (C8 ? 6 : 3) : Fit<C8, NT>::kStages;
  static constexpr int kCtas = LINE ? 1 : Fit<C8, NT>::kCtas;
  static constexpr int kPass = LINE ? 2 : Fit<C8, NT>::kPass;
};
template <bool C8, int NT, bool LINE>
struct Shared {  // and the plan behind it
  static constexpr int kW = Shape<C8, NT, LINE>::kWarps;
  long long scratch[2 * kW];
  __align__(128) unsigned char ring[kW][Shape<C8, NT, LINE>::kStages * Stage<C8>::kBytes];
  float m[kW][8 * NT], l[kW][8 * NT];  // of each warp
  float weight[kW][8 * NT], top[8 * NT], total[8 * NT];
  __align__(16) float o[kW][Shape<C8, NT, LINE>::kPass][kPitch<C8>];
  int left[kW][8];  // keys of the ring's stages
  int bad;          // of the piece
  uint32_t next;
  int last;
};

constexpr size_t slot_floats(int nt) { return static_cast<size_t>(8) * nt * (kD + 2); }
constexpr int slots_of(int nt) { return kCounters / nt; }  // 34 MB

template <int NT>
__device__ __forceinline__ float* slot_at(const PagedArgs& p, int slot) {
  return reinterpret_cast<float*>(static_cast<int*>(p.workspace) + kHeader + kCounters) +
         static_cast<size_t>(slot) * slot_floats(NT);
}

// Queries of the item's rows, as they lie
template <bool C8, int NT>
__device__ __forceinline__ void load_queries(uint32_t (&qf)[NT][8][2], const PagedArgs& p, const Piece& it, int G) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint16_t* q = static_cast<const uint16_t*>(p.q) + it.b * p.q_stride + static_cast<long long>(it.kvh) * G * kD;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = it.row0 + 8 * t + g;
    const bool there = row < G;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int d = C8 ? (k >> 2) * 64 + 16 * c + 4 * (k & 3) : 8 * (c + 4 * (k >> 1)) + 4 * (k & 1);
      const uint2 w = there ? *reinterpret_cast<const uint2*>(q + row * kD + d) : make_uint2(0u, 0u);
      qf[t][k][0] = w.x;
      qf[t][k][1] = w.y;
    }
  }
}

template <bool BF, bool C8, int NT, bool LINE>
__global__ void __launch_bounds__(32 * Shape<C8, NT, LINE>::kWarps, Shape<C8, NT, LINE>::kCtas) paged_kernel(const PagedArgs p) {
  using S = Stage<C8>;
  using Sm = Shared<C8, NT, LINE>;
  constexpr int kStages = Shape<C8, NT, LINE>::kStages, kPass = Shape<C8, NT, LINE>::kPass, kW = Sm::kW;
  constexpr int kPerRow = S::kRow / 16;
  constexpr int kTile = 8 * NT;
  extern __shared__ __align__(128) unsigned char raw_smem[];
  Sm& sm = *reinterpret_cast<Sm*>(raw_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const int G = p.n_heads / p.n_kv_heads;
  int* header = static_cast<int*>(p.workspace);
  const long long items = static_cast<long long>((G + kTile - 1) / kTile) * p.n_kv_heads;
  Plan plan;
  Line line;
  uint32_t total = 0, i = blockIdx.x;  // queue: pieces, this CTA's
  uint32_t at = 0, end = 0;            // line: where the next segment begins, and this CTA's range ends
  pdl_launch_dependents();
  pdl_wait();
  if (tid == 0) sm.bad = 0;  // the plan has barriers
  if constexpr (LINE) {
    line = make_line<kW>(p, static_cast<uint32_t>(items), raw_smem + sizeof(sm), reinterpret_cast<uint32_t*>(sm.scratch));
    if (blockIdx.x < line.ranges) {
      at = line.cut[blockIdx.x];
      end = line.cut[blockIdx.x + 1];
    }
  } else {
    plan = make_plan(p, items, slots_of(NT), raw_smem + sizeof(sm), sm.scratch);
    total = plan.pieces[p.pages.B];
  }
  const long long row_bytes = static_cast<long long>(p.n_kv_heads) * S::kRow;
  const uint32_t ring = smem_addr(sm.ring[warp]);
  const uint64_t policy = once_policy();

  // this warp's copies of a piece: steps from + warp, from + warp + kW, ...: `count`
  Piece it;
  const unsigned char *kc = nullptr, *vc = nullptr;
  const float* scales = nullptr;
  int staged = 0, count = 0, slot_in = 0, rows_of = 0, left_of = 0;
  bool bad = false;
  auto copy_next = [&](const Piece& x) {
    if (staged < count) {
      if ((staged & 31) == 0)  // a lane a step
        bad = !look_up(p, x, staged + lane < count ? x.from + (staged + lane) * kW + warp : 0x7fffffff, rows_of, left_of) || bad;
      const int row = __shfl_sync(0xffffffffu, rows_of, staged & 31), left = __shfl_sync(0xffffffffu, left_of, staged & 31);
      if (left > 0) {
        const uint32_t dst = ring + slot_in * S::kBytes;
        copy_rows<C8, false, true>(dst, kc + row * row_bytes, row_bytes, left, policy);
        copy_rows<C8, true, true>(dst, vc + row * row_bytes, row_bytes, left, policy);
        if (C8) copy4(dst + S::kOffScale + lane * 4, scales + row, (lane & 15) < left);
      }
      if (lane == 0) sm.left[warp][slot_in] = left;
    }
    cp_async_commit();
    ++staged;
    slot_in = slot_in + 1 == kStages ? 0 : slot_in + 1;
  };
  auto begin = [&](const Piece& x) {
    staged = 0;
    count = max(0, (x.to - x.from - warp + kW - 1) / kW);
    const long long off = static_cast<long long>(lane / kPerRow) * row_bytes + x.kvh * S::kRow + (lane % kPerRow) * 16;
    kc = static_cast<const unsigned char*>(p.k_cache) + off;
    vc = static_cast<const unsigned char*>(p.v_cache) + off;
    if (C8) scales = (lane < 16 ? p.k_scale : p.v_scale) + x.kvh * p.cache_rows + (lane & 15);
    slot_in = 0;
    bad = false;
#pragma unroll
    for (int n = 0; n < kStages - 1; ++n) copy_next(x);
  };

  bool more = LINE ? at < end : i < total;
  uint32_t qf[NT][8][2];
  if (more) {
    if constexpr (LINE) it = segment_at(p, line, kTile, end, at);
    else it = piece_at(p, plan, kTile, i);
    load_queries<C8, NT>(qf, p, it, G);  // in front of the cache's copies, which would keep them waiting
    begin(it);
  }
#pragma unroll 1
  while (more) {
    if (!LINE && tid == 0) sm.next = gridDim.x + atomicAdd(reinterpret_cast<unsigned*>(header), 1u);
    State<NT> st;
    float f[NT][2];
    make_queries<BF, C8, NT>(qf, f);
    // Weights go into the product in two parts of its type, bf16 over bf16 and fp16 otherwise, so that their rounding does not
    // show. An infinity among the values of a 16-bit cache times a second part of zero or less is none any more: sums that are not
    // finite are made again from the first parts alone.
    bool second = true;
#pragma unroll 1
    for (;;) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        st.m[t][0] = st.m[t][1] = -CUDART_INF_F;
        st.l[t][0] = st.l[t][1] = 0.f;
        st.k[t][0] = st.k[t][1] = power_of(kMostPower);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) st.o[j][t][e] = 0.f;
      }
      int slot_out = 0;
      const int steps = count;
#pragma unroll 1
      for (int n = 0; n < steps; ++n) {
        cp_async_wait<kStages - 2>();
        __syncwarp();  // every lane's copies of the stage; and the stage before is read
        const int left = sm.left[warp][slot_out];
        copy_next(it);
        if (left > 0) cache_step<BF, C8, NT, true>(st, sm.ring[warp] + slot_out * S::kBytes, qf, f, left, second);
        slot_out = slot_out + 1 == kStages ? 0 : slot_out + 1;
      }
      cp_async_wait<0>();
      if (C8 || !second) break;
      bool wild = false;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) wild = wild || !(fabsf(st.o[j][t][e]) < CUDART_INF_F);
      if (!__any_sync(0xffffffffu, wild)) break;
      second = false;
      begin(it);
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) sm.bad = 1;
    if (C8) {  // the sums without k
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float factor = power_of(-exponent_of(st.k[t][r]));
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            st.o[j][t][r] *= factor;
            st.o[j][t][2 + r] *= factor;
          }
        }
    }

    const int rows = min(kTile, G - it.row0);
    // ---- the next piece's first copies go out before this one's results are put together
    Piece next = it;
    bool goes_on = false;
    auto go_on = [&] {
      load_queries<C8, NT>(qf, p, next, G);
      begin(next);
    };
    if constexpr (LINE) {
      goes_on = at < end;
      if (goes_on) {
        next = segment_at(p, line, kTile, end, at);
        go_on();
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float l = st.l[t][r];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        if (g == 0) {
          sm.m[warp][8 * t + 2 * c + r] = st.m[t][r];
          sm.l[warp][8 * t + 2 * c + r] = l;
        }
      }
    __syncthreads();
    const bool wrong = sm.bad != 0;
    if constexpr (!LINE) {
      i = sm.next;
      goes_on = i < total;
      if (goes_on) {
        next = piece_at(p, plan, kTile, i);
        go_on();
      }
    }
    // ---- the warps' results: kPass rows at a time, or all of them where no copies are on their way into the rings
    auto lse_at = [&](int head) -> float& { return p.lse[static_cast<long long>(head) * p.pages.B + it.b]; };
    float* slot = slot_at<NT>(p, slot_of<LINE>(it, it.j));
    const bool all = LINE && !goes_on;
    const int pass = all ? kTile : kPass;
    float* const sums = all ? reinterpret_cast<float*>(&sm.ring[0][0]) : &sm.o[0][0][0];  // [kW][pass][kPitch]
    for (int row = tid >> 4; row < rows; row += 2 * kW) {  // 16 lanes a row, one a warp
      const int w = tid & 15;
      const float m = w < kW ? sm.m[w][row] : -CUDART_INF_F, l = w < kW ? sm.l[w][row] : 0.f;
      const uint32_t lanes = 0xffffu << (lane & 16);
      float top = m;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(lanes, top, o));
      const float a = weight_of(m, top);
      float total = a * l;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) total += __shfl_xor_sync(lanes, total, o);
      if (w < kW) sm.weight[w][row] = a;
      if (w == 0) {
        sm.top[row] = top;
        sm.total[row] = total;
      }
    }
#pragma unroll 1
    for (int base = 0; base < rows; base += pass) {
      const int here = min(rows, base + pass);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = 8 * t + 2 * c + r;
          if (row >= base && row < here) {
            float* to = sums + (warp * pass + row - base) * kPitch<C8>;
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<float2*>(to + place_of<C8>(out_dim<C8>(g, j, 0))) = make_float2(st.o[j][t][r], st.o[j][t][2 + r]);
          }
        }
      __syncthreads();
#pragma unroll 1
      for (int i = tid; i < (here - base) * kD; i += 32 * kW) {  // a thread a dim
        const int row = base + i / kD, dim = i & (kD - 1);
        const float* from = sums + (row - base) * kPitch<C8> + place_of<C8>(dim);
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < kW; ++w) o += sm.weight[w][row] * from[w * pass * kPitch<C8>];
        const float m = sm.top[row], l = sm.total[row];
        const int head = it.kvh * G + it.row0 + row;
        if (it.of > 1) {
          __stcg(slot + row * kD + dim, o);
          if (dim == 0) __stcg(reinterpret_cast<float2*>(slot + kTile * kD) + row, make_float2(m, wrong ? -1.f : l));
        } else if (!wrong) {
          const float y = l == 0.f ? 0.f : o / l;
          static_cast<uint16_t*>(p.out)[(static_cast<long long>(it.b) * p.n_heads + head) * kD + dim] = static_cast<uint16_t>(pack16<BF>(y, y));
          if (p.lse != nullptr && dim == 0) lse_at(head) = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
        }
      }
      __syncthreads();
    }
    if (tid == 0 && wrong) {
      sm.bad = 0;
      set_status(p.status, kStatusDeviceArg);
    }
    if (it.of > 1) {
      // the barrier behind the results, then one thread's fence for all of the CTA's
      if (tid == 0) {
        int* counter = header + kHeader + it.first;
        __threadfence();
        sm.last = atomicAdd(counter, 1) == it.of - 1;
        __threadfence();
        if (sm.last) *counter = 0;
      }
      __syncthreads();
      if (sm.last) {
        // `share` warps a row, each every share-th piece; 4 dims a lane
        const int share = max(1, kW / rows), at_once = kW / share;
#pragma unroll 1
        for (int row0 = 0; row0 < rows; row0 += at_once) {
          const int row = row0 + warp / share, part = warp % share;
          float m = -CUDART_INF_F, l = 0.f;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
          bool refused = false;
          if (row < rows && warp / share < at_once) {
#pragma unroll 1
            for (int j0 = part; j0 < it.of; j0 += kJoin * share) {  // in the order of the keys; the loads of kJoin pieces at once
              float2 x[kJoin];
              float4 v[kJoin];
#pragma unroll
              for (int j = 0; j < kJoin; ++j) {
                const float* other = slot_at<NT>(p, slot_of<LINE>(it, min(j0 + j * share, it.of - 1)));
                x[j] = load_l2(reinterpret_cast<const float2*>(other + kTile * kD) + row);
                v[j] = load_l2(reinterpret_cast<const float4*>(other + row * kD) + lane);
              }
              float top = m;
#pragma unroll
              for (int j = 0; j < kJoin; ++j) top = fmaxf(top, x[j].x);
              const float old = weight_of(m, top);
              m = top;
              l *= old;
              o = make_float4(o.x * old, o.y * old, o.z * old, o.w * old);
#pragma unroll
              for (int j = 0; j < kJoin; ++j) {
                const float a = weight_of(x[j].x, top);
                refused = refused || x[j].y < 0.f;
                if (j0 + j * share < it.of) {
                  l += a * x[j].y;
                  o.x += a * v[j].x;
                  o.y += a * v[j].y;
                  o.z += a * v[j].z;
                  o.w += a * v[j].w;
                }
              }
            }
          }
          if (share > 1) {  // the row's warps, by the first of them
            *reinterpret_cast<float4*>(&sm.o[warp][0][4 * lane]) = o;
            if (lane == 0) {
              sm.m[warp][0] = m;
              sm.l[warp][0] = refused ? -1.f : l;
            }
            __syncthreads();
            if (part == 0 && row < rows) {
              float top = m;
              for (int w = 1; w < share; ++w) top = fmaxf(top, sm.m[warp + w][0]);
              const float own = weight_of(m, top);
              l *= own;
              o = make_float4(o.x * own, o.y * own, o.z * own, o.w * own);
              for (int w = 1; w < share; ++w) {
                const float a = weight_of(sm.m[warp + w][0], top), lw = sm.l[warp + w][0];
                const float4 v = *reinterpret_cast<const float4*>(&sm.o[warp + w][0][4 * lane]);
                refused = refused || lw < 0.f;
                l += a * lw;
                o.x += a * v.x;
                o.y += a * v.y;
                o.z += a * v.z;
                o.w += a * v.w;
              }
              m = top;
            }
            __syncthreads();
          }
          if (row < rows && part == 0 && warp / share < at_once && !refused) {
            const int head = it.kvh * G + it.row0 + row;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            uint16_t* out = static_cast<uint16_t*>(p.out) + (static_cast<long long>(it.b) * p.n_heads + head) * kD + 4 * lane;
            *reinterpret_cast<uint2*>(out) = make_uint2(pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv));
            if (p.lse != nullptr && lane == 0) lse_at(head) = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
          }
        }
      }
    }
    __syncthreads();  // before the next piece writes what was read here
    it = next;
    more = goes_on;
  }
  if (!LINE && tid == 0 && atomicAdd(reinterpret_cast<unsigned*>(header) + 1, 1u) == gridDim.x - 1) {
    header[0] = 0;  // every CTA has taken its last piece
    header[1] = 0;
  }
}

struct Kernel {
  const void* fn;
  size_t smem;
  int ctas, threads;
};
template <bool BF, bool C8, int NT, bool LINE>
Kernel kernel_for() {
  using F = Shape<C8, NT, LINE>;
  return {reinterpret_cast<const void*>(&paged_kernel<BF, C8, NT, LINE>), sizeof(Shared<C8, NT, LINE>), F::kCtas, 32 * F::kWarps};
}
template <bool BF, bool C8>
Kernel kernel_of(int nt, bool line) {
  return nt == 1 ? (line ? kernel_for<BF, C8, 1, true>() : kernel_for<BF, C8, 1, false>())
                 : (line ? kernel_for<BF, C8, 2, true>() : kernel_for<BF, C8, 2, false>());
}

// 8-row tiles of an item: one where the group has no more rows; two hold its rows in twice the registers
int tile_count(int n_heads, int n_kv_heads) { return n_heads / n_kv_heads <= 8 ? 1 : 2; }

}  // namespace

size_t paged_attention_workspace_bytes(int B, int n_heads, int n_kv_heads) {
  const int nt = tile_count(n_heads, n_kv_heads);
  return (kHeader + kCounters) * sizeof(int) + slots_of(nt) * slot_floats(nt) * sizeof(float);
}

// Items a SM up to which the line is taken: 256 items of 500 to 4096 rows 56 us, in the queue 60; 512 of them 84 and 70.
constexpr int kLineItems = 2;

cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, bool cache8, cudaStream_t stream) {
  const int nt = tile_count(a.n_heads, a.n_kv_heads), G = a.n_heads / a.n_kv_heads;
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  const long long items = static_cast<long long>(a.pages.B) * a.n_kv_heads * ((G + 8 * nt - 1) / (8 * nt));
  const long long steps = ((static_cast<long long>(a.pages.width) << a.pages.shift) >> 4) * items;  // at most
  const bool line = items <= static_cast<long long>(kLineItems) * sms && steps < 0x7fffffffll && 2 * sms <= slots_of(nt);
  const Kernel k = dtype == FSX_BF16 ? (cache8 ? kernel_of<true, true>(nt, line) : kernel_of<true, false>(nt, line))
                                     : (cache8 ? kernel_of<false, true>(nt, line) : kernel_of<false, false>(nt, line));
  const size_t smem = k.smem + (line ? line_bytes(a.pages.B, sms) : plan_bytes(a.pages.B));
  const cudaError_t e = allow_shared_memory(k.fn, smem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<PagedArgs*>(&a)};
  return launch_ex(k.fn, dim3(static_cast<unsigned>(sms * k.ctas)), dim3(static_cast<unsigned>(k.threads)), smem, stream, true, args);
}

}  // namespace fsx
