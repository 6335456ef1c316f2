// Attention of drafted tokens (fsx_tree_attention) for items of many rows, on the 5th-generation tensor
// cores: up to 128 rows (token, head of the group) an item, or 256 (WIDE).
//
//   S = Q K^T     128 rows x 128 keys, A and B in shared memory, S in tensor memory
//   P = 2^(f S k_scale - m) v_scale k, rounded to the type of V, over its S; a thread holds a row; k: a power of two
//   O += P V      A in tensor memory, V read N-contiguous, O in tensor memory
// Two S / P / O sets and two groups of softmax warps: in an item of more than 128 rows each works on its
// own 128 rows and every chunk; else both on the same rows, one on the even and one on the odd chunks, so that
// the tensor core always has the other's work while one is at its exponentials; their two results meet at the end. Where a wait
// gives up, both groups leave together.
//
// Eight producer warps, four for K and four for V, copy the rows of a chunk by 16-byte asynchronous copies, each
// thread its own units, and wait for nobody: 16-bit rows straight into their slot, 8-bit rows into a private stage, from where the thread that copied
// them turns them into fp16 in the slot. A chunk whose scales are powers of two between 2^-15 and 2^7 (a cache as it is
// written, unless its values are extreme) becomes its values, exactly; any other keeps its codes, and the softmax
// multiplies scores and weights by the scales. bf16 queries and new tokens meet an 8-bit cache as fp16 times a power
// of two per row (their 8 bits fit; components 2^-22 below the row's largest may lose their last bits); the
// new tokens' powers stand where the cache rows' scales do. Rows past the range become zeros and are never read.
// Weights are fp16, whose range is narrow, and scales may have any size: where a chunk has scales, the weights are taken
// times a power of two `k` of each row's own, which brings the largest (weight times scale) that the row sees to 2^7 or, as
// long as k need not move, 2^15. What a row does not see, or sees with little weight, does not decide what is lost. Rows
// of zeros, whose scale says nothing, count as none. Where all of a chunk lies far below what k was chosen for, the sums
// themselves tell how far k may grow. Chunks without scales want k = 1.
// The values of new tokens are looked over on the way: a masked weight is 0, but 0 times an infinity or NaN is not,
// so these become 0 in the product and are added to the rows that see them at the end.
//
// Work: items are whole, or cut into pieces of at most `most` chunks that CTAs take from a queue, or the chunks of all
// items are one line, cut into equal ranges, one per CTA; whichever ends first by the count of rounds, chunks and
// of starts (a piece's queries and results take about as long as 5 chunks). Pieces keep items apart, which pays where they
// fill the GPU evenly; ranges leave no SM without work but may hold the end of one item and the start of the next. One
// warp finds the pieces and describes them in a ring for the other roles. Cut items are put together by a
// second kernel, a warp a row: 256 rows are too many for the one CTA that comes last.
//
// Measured (calls in a graph): one tree of 50 tokens, 32 heads over 8, behind 32768 8-bit rows: 49 to 50 us, of which the plan, the
// queries and the first keys take 10 us, 13.5 chunks of 256 rows 28 us (about 3,900 cycles each, of which MMAs 2,048 and
// exponentials 1,024: a tile's S, softmax and P V follow each other, and their instructions share the schedulers with
// the producers') and results and join 10 us. Eight requests of 24 tokens at most over 4096 to 8192 rows: 55 us with
// 8-bit, 52.5 us with 16-bit caches (3.9 TB/s). 16 requests of 6 to 11 tokens over 96 to 480 rows: 22 us, mostly the latency
// of the same steps: plan 2.5, first piece 1, queries 2.4, first keys 1, three chunks 6, results 4, join 2 us. k costs 2 %
// to 3 % of a call over an 8-bit cache.
//
// Registers: 640 threads at 96 from launch, which is what the compiler gives every role: a few words spill in all variants (24 to
// 28 bytes stored). Softmax warpgroups take 2 x 128, producers keep 2 x 80, MMA and scheduler 64 (with 104, 96 and 80, and with
// 128, 88 and 48, more spilled: the wide tree 52.4 and 50.2 us where this split took 48.9).
#include "chunk_line.h"
#include "fsx.h"
#include "kernels.h"
#include "llm.h"
#include "tc_attention.cuh"
#include "tree_schedule.cuh"

namespace fsx {

namespace {

constexpr int kD = kHeadDim;
constexpr int kTile = 128;                   // rows of a tile, keys of a chunk
constexpr int kSlotBytes = kTile * kD * 2;   // 32 KB
constexpr int kRawBytes = kTile * kD;        // 16 KB of codes
constexpr int kMmaWarp = 8, kSchedWarp = 9, kProdWarp = 12;
constexpr int kProds = 256;                  // producer threads
constexpr int kThreads = 384 + kProds;
constexpr int kPlans = 5;  // whole items; pieces of 1, 1.25, 1.5 and 2 ranges
constexpr int kWorkRing = 4;
constexpr int kWorkUsers = 17;               // warps that read a piece's description: MMA, producers, softmax
constexpr uint32_t kColS = 0, kColO = 256;
constexpr int kMaxGrid = 256;
constexpr int kPartials = 2 * kMaxGrid;      // slots of the workspace
constexpr int kStart = 5;                    // chunks that a piece's start and end cost

// A piece as every role sees it
struct Work {
  long long c0, t0;  // first cache row and first new token of the request
  int len, n;        // its cache rows and new tokens
  int kvh;           // -1: no more pieces
  int row0, rows;    // rows of the item
  int from, chunks;  // of this piece
  int pair;          // more than 128 rows: a softmax group per tile; else a group per chunk parity
  int has_new;       // its last chunk holds the new tokens
  int slot, first, j, of;  // piece j of `of`, its slot, and `first` for the join: ~slot of piece 0, or the CTA of its range
};

template <bool C8, bool WIDE>
struct Layout {
  static constexpr int kRows = WIDE ? 2 * kTile : kTile;
  static constexpr int kSlots = C8 ? (WIDE ? 3 : 4) : (WIDE ? 4 : 5);
  static constexpr int kRaw = C8 ? 3 : 0;
  static constexpr int kOffSlots = (WIDE ? 2 : 1) * kSlotBytes;
  static constexpr int kOffRaw = kOffSlots + kSlots * kSlotBytes;
  static constexpr int kOffScale = kOffRaw + kRaw * kRawBytes;  // C8: [ring][k, v][128]
  // The scales of chunk c are written while its K is made ready, so when the MMAs of K or V chunk c - 2 or before
  // are done: the weights of chunk c - 4 are behind.
  static constexpr int kScaleRing = C8 ? 4 : 0;
  static constexpr int kOffFactor = kOffScale + kScaleRing * 2 * kTile * 4;  // C8: [piece parity][row]
  static constexpr int kOffMl = kOffFactor + (C8 ? 2 * kRows * 4 : 0);       // [group][128] (m, l)
  static constexpr int kOffPower = kOffMl + 2 * kTile * 8;                   // C8: [group][128] log2 k
  static constexpr int kOffScratch = kOffPower + (C8 ? 2 * kTile * 4 : 0);
  static constexpr int kOffWork = kOffScratch + (2 * kPlans + 1 + kThreads / 32 + 1) / 2 * 8;
  static constexpr int kOffBar = kOffWork + kWorkRing * static_cast<int>(sizeof(Work));
  static constexpr int kMisc = kOffBar + 33 * 8;  // tmem, abort, wild[4], plain [4][2]
  static constexpr int kPlan = (kMisc + 14 * 4 + 7) / 8 * 8;
  static constexpr int kSmem = kPlan + (2 * kMaxSequences + 1) * 4;
};
static_assert(Layout<true, true>::kSmem <= 227 * 1024 && Layout<true, false>::kSmem <= 227 * 1024, "shared memory");
static_assert(Layout<false, true>::kSmem <= 227 * 1024 && Layout<false, false>::kSmem <= 227 * 1024, "shared memory");

__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  return h;
}
__device__ __forceinline__ float weight_of(float m, float top) { return m == -CUDART_INF_F ? 0.f : exp2_fast(m - top); }

// 2^e that brings `top`, a row's largest magnitude, to [2^7, 2^8) when it is divided by it; 1 for zeros, infinities
// and NaN
__device__ __forceinline__ float row_power(float top) {
  if (top == 0.f || !(top < CUDART_INF_F)) return 1.f;
  const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127 - 7;
  return __uint_as_float(static_cast<uint32_t>(127 + max(-126, min(e, 126))) << 23);
}
__device__ __forceinline__ float inverse_power(float p) {
  return __uint_as_float((254u << 23) - __float_as_uint(p));
}
template <bool BF>
__device__ __forceinline__ float top_of(uint4 x) {  // largest magnitude of 8 values
  float t = 0.f;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack16<BF>(w[i]);
    t = fmaxf(t, fmaxf(fabsf(y.x), fabsf(y.y)));
  }
  return t;
}
template <bool BF>
__device__ __forceinline__ uint4 times_to_half(uint4 x, float factor) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = unpack16<BF>(w[i]);
    w[i] = pack_half2(y.x * factor, y.y * factor);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool BF>
__device__ __forceinline__ uint4 take_out_wild(uint4 x, bool& wild) {  // values that are not finite become 0
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t bad = not_finite2<BF>(w[i]);
    wild = wild || bad != 0u;
    w[i] &= ~((bad >> 15) * 0xffffu);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float row_max16(float t) {  // over the 16 lanes that share a row
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
  return t;
}

// The line of work: pre[b] pieces (most > 0) or chunks (ranges) of the requests before b, pre[B] of all, in 32 bits: each 64-bit
// division is a hundred instructions that every CTA waits for. The chunks are counted first, in 64 bits (chunk_line.h); a line
// that is too long for places of 32 bits goes by whole items, of which there are below 2^23.
struct Line {
  uint32_t* pre;
  uint32_t most;  // chunks of a piece; 0: ranges
  uint32_t per;   // chunks of a range; 0: no ranges
};
__device__ __forceinline__ uint32_t chunks_of(int len) { return above(static_cast<uint32_t>(len), kTile) + 1; }  // the last one: new tokens
// By the whole CTA: a warp weighs a plan. `costs`: kPlans (cost, most), then the range and a value per warp
template <int ROWS>
__device__ __forceinline__ Line line_of(const TreeArgs& p, uint32_t* pre, uint32_t* chunks, uint32_t* costs) {
  constexpr int kW = kThreads / 32, kEach = (kMaxSequences + kThreads - 1) / kThreads;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t G = static_cast<uint32_t>(p.n_heads) / static_cast<uint32_t>(p.n_kv_heads);
#pragma unroll 1
  for (int b = tid; b < p.B; b += kThreads) {
    TreeRequest r;
    if (!tree_request(p, b, r) && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    pre[b] = above(r.n * G, ROWS) * p.n_kv_heads;  // items
    chunks[b] = r.n > 0 ? chunks_of(r.len) : 0;
  }
  __syncthreads();
  if (warp < kPlans) {
    ChunkCount mine;
    uint32_t longest = 0;
#pragma unroll 1
    for (int b = lane; b < p.B; b += 32) {
      mine.add(pre[b], chunks[b]);
      longest = max(longest, chunks[b]);
    }
    const uint64_t total = ChunkCount::sum(__reduce_add_sync(0xffffffffu, mine.low()), __reduce_add_sync(0xffffffffu, mine.high()));
    longest = __reduce_max_sync(0xffffffffu, longest);
    const uint32_t per = range_of(total, gridDim.x);
    // whole items, then pieces of 1, 1.25, 1.5 and 2 ranges
    const uint32_t most = warp == 0 ? longest : per * (warp < 4 ? 3 + warp : 8) / 4;
    float cost = CUDART_INF_F;
    if (most > 0 && (warp == 0 || most < longest)) {
      uint32_t pieces = 0;
#pragma unroll 1
      for (int b = lane; b < p.B; b += 32) pieces += pre[b] * above(chunks[b], most);
      pieces = __reduce_add_sync(0xffffffffu, pieces);
      const float rounds = ceilf(static_cast<float>(pieces) / static_cast<float>(gridDim.x));
      if (warp == 0 || pieces <= kPartials)
        cost = (rounds - 1.f) * (static_cast<float>(total) / static_cast<float>(pieces) + kStart) + most + kStart;
    }
    if (lane == 0) {
      costs[2 * warp] = __float_as_uint(cost);
      costs[2 * warp + 1] = most;
      if (warp == 0) costs[2 * kPlans] = per;
    }
  }
  __syncthreads();
  Line line{pre, 0, costs[2 * kPlans]};
  float best = line.per > 0 ? static_cast<float>(line.per + 2 * kStart) : CUDART_INF_F;
#pragma unroll
  for (int i = 0; i < kPlans; ++i) {
    const float cost = __uint_as_float(costs[2 * i]);
    if (cost < best) {
      best = cost;
      line.most = costs[2 * i + 1];
    }
  }
  // each thread's requests, then those of the threads before
  const int each = above(p.B, kThreads), b0 = min(p.B, tid * each);
  uint32_t mine[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = b0 + i;
    mine[i] = sum;
    if (i < each && b < p.B) sum += pre[b] * (line.most > 0 ? above(chunks[b], line.most) : chunks[b]);
  }
  uint32_t upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += up;
  }
  uint32_t* ends = costs + 2 * kPlans + 1;
  if (lane == 31) ends[warp] = upto;
  __syncthreads();
  const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? ends[lane] : 0u) + upto - sum;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (i < each && b0 + i < p.B) pre[b0 + i] = before + mine[i];
  }
  if (tid == kThreads - 1) pre[p.B] = before + sum;
  __syncthreads();
  return line;
}
static_assert(kThreads / 32 <= 32, "a lane a warp");

// The piece at `u` of the line; of a range that ends at u1
template <int ROWS>
__device__ __forceinline__ Work work_at(const TreeArgs& p, const Line& line, uint32_t u, uint32_t u1, uint32_t G) {
  int lo = 0, hi = p.B;  // pre[lo] <= u < pre[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (line.pre[mid] <= u) lo = mid;
    else hi = mid;
  }
  TreeRequest r;
  tree_request(p, lo, r);
  Work w{};
  w.c0 = r.c0;
  w.t0 = r.t0;
  w.len = r.len;
  w.n = r.n;
  const uint32_t n = chunks_of(r.len), rel = u - line.pre[lo];
  uint32_t item;
  if (line.most > 0) {
    const uint32_t of = above(n, line.most);
    item = rel / of;
    const uint32_t j = rel - item * of, least = n / of, more = n - least * of;
    w.of = static_cast<int>(of);
    w.j = static_cast<int>(j);
    w.from = static_cast<int>(j * least + min(j, more));
    w.chunks = static_cast<int>(least + (j < more ? 1 : 0));
    w.slot = static_cast<int>(min(u, static_cast<uint32_t>(kPartials - 1)));  // used if the item is cut: then u < kPartials
    w.first = ~(w.slot - w.j);
  } else {
    item = rel / n;
    w.from = static_cast<int>(rel - item * n);
    const uint32_t start = u - w.from, end = start + n;
    w.chunks = static_cast<int>(min(end, u1) - u);
    w.first = static_cast<int>(start / line.per);
    w.j = static_cast<int>(u / line.per) - w.first;
    w.of = static_cast<int>((end - 1) / line.per) - w.first + 1;
    w.slot = 2 * (w.first + w.j) + (w.j == 0 ? 1 : 0);
  }
  const uint32_t tile = item / static_cast<uint32_t>(p.n_kv_heads);
  w.kvh = static_cast<int>(item - tile * p.n_kv_heads);
  w.row0 = static_cast<int>(tile * ROWS);
  w.rows = min(ROWS, static_cast<int>(r.n * G) - w.row0);
  w.pair = w.rows > kTile;
  w.has_new = w.from + w.chunks == static_cast<int>(n);
  return w;
}
// slot of piece j of an item: at most one cut item begins in a range (slot 2 cta + 1) and one ends there (2 cta)
__device__ __forceinline__ int slot_of(int first, int j) { return first < 0 ? ~first + j : 2 * (first + j) + (j == 0 ? 1 : 0); }

// Workspace behind the header and counters: (Work::first, pieces) per (head, new token), then the slots:
// [rows][128] sums, [rows] (maximum, sum of weights)
__host__ __device__ constexpr size_t slot_floats(int rows) { return static_cast<size_t>(rows) * (kD + 2); }
__device__ __forceinline__ int2* table_of(const TreeArgs& p) {
  return reinterpret_cast<int2*>(static_cast<int*>(p.workspace) + kTreeHeader + kTreeCounters);
}
__host__ __device__ __forceinline__ size_t table_bytes(long long new_rows, int n_heads) {
  return (static_cast<size_t>(new_rows) * n_heads * sizeof(int2) + 255) / 256 * 256;
}
__device__ __forceinline__ float* slots_of(const TreeArgs& p) {
  return reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(table_of(p)) + table_bytes(p.new_rows, p.n_heads));
}

template <bool BF, bool C8, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const TreeArgs p) {
  using L = Layout<C8, WIDE>;
  constexpr bool kBf = BF && !C8;  // type of the operands
  // The largest weight is 2^kTopPower when the maximum moves, and 2^8 times that before it moves again: fp16 has room above,
  // and what lies far below the maximum keeps more of its bits
  constexpr float kTopPower = kBf ? 0.f : 7.f, kLag = 8.f + kTopPower;
  constexpr float kMostPower = 118.f;  // of log2 k
  constexpr int kSlots = L::kSlots;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t G = static_cast<uint32_t>(p.n_heads) / static_cast<uint32_t>(p.n_kv_heads);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
  // Per chunk, in rings of 4 (chunk n of the CTA: entry n mod 4, phase n / 4): every barrier is filled by one role and
  // waited for by each role that waits chunk after chunk, which is never 4 chunks behind.
  uint64_t* kfull = bars;         // K is there
  uint64_t* vfull = bars + 4;     // V is there
  uint64_t* sdone = bars + 8;     // S of both tiles done with K
  uint64_t* pdone = bars + 29;    // P V of both tiles done with V
  uint64_t* qfull = bars + 12;    // an item's queries are there
  uint64_t* qempty = bars + 13;   // the softmax warps are done with the piece and with their place
  uint64_t* sfull = bars + 14;    // [2] S of a chunk in tensor memory
  uint64_t* pfull = bars + 16;    // [2] P of a chunk over it
  uint64_t* odone = bars + 18;    // every P V of the piece done
  uint64_t* oread = bars + 19;    // its O read
  uint64_t* drain = bars + 20;    // every MMA done
  uint64_t* wfull = bars + 21;    // [4] a piece is described
  uint64_t* wempty = bars + 25;   // [4] and every role has read it
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* wild = reinterpret_cast<volatile int*>(tmem_slot + 2);  // [4]: piece ordinal + 1 with values taken out
  volatile int* plain_of = reinterpret_cast<volatile int*>(tmem_slot + 6);  // [4][k, v]: no scales left in the chunk
  Work* works = reinterpret_cast<Work*>(smem + L::kOffWork);
  float* scales = reinterpret_cast<float*>(smem + L::kOffScale);  // of keys; of values their logarithms, -infinity for a row of zeros
  float* row_factor = reinterpret_cast<float*>(smem + L::kOffFactor);
  float2* ml_of = reinterpret_cast<float2*>(smem + L::kOffMl);
  float* power_of = reinterpret_cast<float*>(smem + L::kOffPower);
  uint32_t* scratch = reinterpret_cast<uint32_t*>(smem + L::kOffScratch);
  constexpr int kScaleRing = L::kScaleRing > 0 ? L::kScaleRing : 1;
  if ((smem_addr(smem) & 1023u) != 0u) {  // the swizzled operands need a 1024-byte aligned base
    if (tid == 0) set_status(p.status, kStatusDeviceArg);
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) {
      mbar_init(kfull + i, kProds / 2);
      mbar_init(vfull + i, kProds / 2);
      mbar_init(sdone + i, 1);
      mbar_init(pdone + i, 1);
    }
    mbar_init(qfull, kProds);
    mbar_init(qempty, 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(sfull + i, 1);
      mbar_init(pfull + i, 4);
    }
    mbar_init(odone, 1);
    mbar_init(oread, 8);
    mbar_init(drain, 1);
    for (int i = 0; i < kWorkRing; ++i) {
      mbar_init(wfull + i, 1);
      mbar_init(wempty + i, kWorkUsers);
    }
    *abort = 0;
    for (int i = 0; i < 4; ++i) wild[i] = 0;
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  uint32_t* plan = reinterpret_cast<uint32_t*>(smem + L::kPlan);
  const Line line = line_of<L::kRows>(p, plan, plan + kMaxSequences + 1, scratch);
  fence_proxy_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
  // piece `ord` of the CTA: its description stays until every warp that uses it has given it back
  auto find_work = [&](int ord) {
    return wait_or_abort(wfull + ord % kWorkRing, (ord / kWorkRing) & 1, p.status, abort) && works[ord % kWorkRing].kvh >= 0;
  };
  auto give_back = [&](int ord) {
    __syncwarp();
    if (lane == 0) mbar_arrive(wempty + ord % kWorkRing);
  };
  // K of the CTA's chunk n lies in slot 2 n mod kSlots, V in slot 2 n + 1 mod kSlots
  auto wait_chunk = [&](uint64_t* ring, int n) { return wait_or_abort(ring + (n & 3), (n >> 2) & 1, p.status, abort); };

  if (warp >= kMmaWarp && warp < kProdWarp) {
  leave_registers<64>();
  if (warp == kSchedWarp) {
    // ---------------------------------------------------------------- pieces
    int* header = static_cast<int*>(p.workspace);
    const uint32_t total = line.pre[p.B];
    const bool queue = line.most > 0;
    uint32_t u = queue ? blockIdx.x : blockIdx.x * line.per;
    const uint32_t u1 = queue ? total : min(total, u + line.per);
#pragma unroll 1
    for (int ord = 0;; ++ord) {
      if (ord >= kWorkRing && !wait_or_abort(wempty + ord % kWorkRing, (ord / kWorkRing - 1) & 1, p.status, abort)) break;
      if (lane == 0) {
        Work w{};
        w.kvh = -1;
        if (u < u1) w = work_at<L::kRows>(p, line, u, u1, G);
        works[ord % kWorkRing] = w;
        mbar_arrive(wfull + ord % kWorkRing);
        if (w.kvh >= 0) u = queue ? gridDim.x + atomicAdd(reinterpret_cast<unsigned*>(header), 1u) : u + w.chunks;
        else u = 0xffffffffu;
      }
      u = __shfl_sync(0xffffffffu, u, 0);
      if (u == 0xffffffffu) break;
    }
    if (lane == 0 && atomicAdd(reinterpret_cast<unsigned*>(header) + 1, 1u) == gridDim.x - 1) {
      header[0] = 0;  // every CTA has taken its last piece
      header[1] = 0;
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs: the whole warp waits, one lane issues
    const bool leader = elect_lane();
    const uint32_t id_s = idesc_16(kBf, kTile, kTile, false), id_o = idesc_16(kBf, kTile, kD, true);
    const uint32_t slots = smem_addr(smem + L::kOffSlots);
    // descriptors: the low words change, the high ones are constants
    const uint32_t q_lo = static_cast<uint32_t>(sw128_desc(smem_addr(smem))), k_lo = static_cast<uint32_t>(sw128_desc(slots));
    const uint32_t v_lo = static_cast<uint32_t>(sw128_desc_mn(slots, 16384, 1024));
    auto k_desc = [](uint32_t lo) { return sw128_desc(0) >> 32 << 32 | lo; };
    auto v_desc = [](uint32_t lo) { return sw128_desc_mn(0, 16384, 1024) >> 32 << 32 | lo; };
    // What the loop needs of a piece stays in registers and slots are counted on: with a read of shared memory, a
    // division or a wait more per tile, this warp and not the tensor core was what a chunk took its time for.
    bool ok = true;
    int nk = 0, nv = 0;            // chunks whose S, whose P V has been issued
    uint32_t ks = 0, vs = 1;       // their slots
    uint32_t counts = 0;           // bits 0, 16: parity of the tiles' next P
#pragma unroll 1
    for (int ord = 0; ok; ++ord) {
      if (!find_work(ord)) break;
      const Work& w = works[ord % kWorkRing];
      const int chunks = w.chunks, has_new = w.has_new;
      const int lag = w.pair ? 1 : 2, tiles = w.pair ? 2 : 1;
      ok = wait_or_abort(qfull, ord & 1, p.status, abort);
#pragma unroll 1
      for (int j = 0; j < chunks + lag && ok; ++j) {
        const int jp = j - lag;  // per tile: P V of chunk jp, then S of chunk j
        if (jp >= 0) {
          ok = wait_chunk(vfull, nv);
          if (jp == 0 && ord > 0) ok = ok && wait_or_abort(oread, (ord - 1) & 1, p.status, abort);
        }
        if (!ok) break;
        const uint32_t vd = v_lo + vs * (kSlotBytes >> 4), kd = k_lo + ks * (kSlotBytes >> 4);
        uint32_t t = tiles == 2 ? 0u : j & 1;  // chunk by chunk, or both tiles
#pragma unroll 1
        for (int i = 0; i < tiles; ++i, ++t) {
          const uint32_t s_at = tmem + kColS + t * kTile, o_at = tmem + kColO + t * kTile;
          const bool last_tile = i + 1 == tiles;
          if (jp >= 0) {
            ok = wait_or_abort(pfull + t, (counts >> (16 * t)) & 1u, p.status, abort);
            if (!ok) break;
            counts ^= 1u << (16 * t);
            tc_fence_after();
            if (leader) {
              const uint32_t more = jp >= lag ? 1u : 0u;  // not the group's first chunk
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_f16_ta(o_at, s_at + k * 8, v_desc(vd + k * 128), id_o, k > 0 ? 1u : more);
              if (!(has_new && jp == chunks - 1)) {  // 64 keys more
#pragma unroll
                for (int k = 4; k < 8; ++k) umma_f16_ta(o_at, s_at + k * 8, v_desc(vd + k * 128), id_o, 1u);
              }
              if (last_tile) {
                umma_commit(pdone + (nv & 3));
                if (jp == chunks - 1) umma_commit(odone);
              }
            }
            __syncwarp();
          }
          if (j < chunks) {
            // behind P V, which may be what the chunk's slot waits for
            if (i == 0) ok = wait_chunk(kfull, nk);
            if (!ok) break;
            tc_fence_after();
            const uint32_t qd = q_lo + (tiles == 2 && t == 1 ? kSlotBytes >> 4 : 0);
            if (leader) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint32_t off = (k >> 2) * (16384 >> 4) + (k & 3) * 2;
                umma_f16(s_at, k_desc(qd + off), k_desc(kd + off), id_s, k > 0 ? 1u : 0u);
              }
              umma_commit(sfull + t);
              if (last_tile) umma_commit(sdone + (nk & 3));
            }
            __syncwarp();
          }
        }
        if (jp >= 0) {
          ++nv;
          vs = vs + 2 >= kSlots ? vs + 2 - kSlots : vs + 2;
        }
        if (j < chunks) {
          ++nk;
          ks = ks + 2 >= kSlots ? ks + 2 - kSlots : ks + 2;
        }
      }
      give_back(ord);
    }
    pdl_launch_dependents();  // the join's CTAs find their requests under the last results
    if (leader) umma_commit(drain);
    __syncwarp();
    mbar_wait(drain, 0, p.status);
  }
  } else if (warp >= kProdWarp) {
    leave_registers<80>();
    // ---------------------------------------------------------------- producers
    // Four warps make the K chunks ready, four the V chunks. A thread's units: of 16-bit rows, unit u of rows r0, r0 + 8,
    // ...; of codes, which are copied and converted 64 rows at a time, units u and u + 4 of rows r0 and r0 + 32: four
    // lanes a row, so that the 8 lanes whose fp16 units are stored together have rows of both parities and meet no
    // bank twice.
    const int is_v = (warp - kProdWarp) >> 2;
    const int pt = tid & 127;
    const int u = C8 ? pt & 3 : pt & 15, r0 = C8 ? pt >> 2 : pt >> 4;
    constexpr int kCopyRows = C8 ? 64 : kTile;  // rows of one copy
    constexpr int kAhead = C8 ? 2 : 1;          // copies under way beside the one that is made ready
    constexpr int kSteps = kTile / kCopyRows;
    const long long row_bytes = static_cast<long long>(p.n_kv_heads) * kD * (C8 ? 1 : 2);
    unsigned char* slots = smem + L::kOffSlots;
    unsigned char* raw = smem + L::kOffRaw + is_v * (3 * kRawBytes / 2) + pt * 16;  // three copies of 8 KB each
    const unsigned char* cache = static_cast<const unsigned char*>(is_v ? p.v_cache : p.k_cache) + u * 16;
    const float* scale_of = is_v ? p.v_scale : p.k_scale;
    const uint16_t* fresh = static_cast<const uint16_t*>(is_v ? p.v_new : p.k_new);
    bool ok = true;
    // Chunk n of this tensor takes the slot of the other tensor's or its own chunk kSlots before in the order K0 V0 K1 ...
    auto wait_slot = [&](int n) {
      const int before = 2 * n + is_v - kSlots;
      return before < 0 || wait_chunk(before & 1 ? pdone : sdone, before >> 1);
    };
    // the next copy: step `ci` of piece `iord`, which is up to two pieces ahead of the one made ready
    int iord = 0, ci = 0, cn = 0, left = 0;  // cn: steps of the cache rows; left: rows from this thread's first row on
    int in = 0, raw_in = 0;                  // chunks and raw stages copied
    const unsigned char* src = nullptr;
    bool more = false;
    auto begin_copies = [&] {
      more = find_work(iord);
      if (more) {
        const Work& x = works[iord % kWorkRing];
        const int key0 = x.from * kTile + r0;
        left = x.len - key0;
        src = cache + (x.c0 + key0) * row_bytes + x.kvh * (kD * (C8 ? 1 : 2));
        cn = (x.chunks - x.has_new) * kSteps;
      }
    };
    auto issue = [&] {
      if (more) {
        if (!C8) {
          const int c = 2 * in + is_v;
          ok = ok && wait_slot(in);
          if (ok) {
            const unsigned char* from = src;
            long long step = 8 * row_bytes;
            int rows = left;
            if (ci >= cn) {  // the new tokens
              const Work& x = works[iord % kWorkRing];
              step = 8 * p.new_stride * 2;
              rows = x.n - r0;
              from = reinterpret_cast<const unsigned char*>(fresh + (x.t0 + r0) * p.new_stride + x.kvh * kD + u * 8);
            }
            const uint32_t dst = smem_addr(slots + (c % kSlots) * kSlotBytes + tile_off(r0, u));  // rows 8 on lie 1024 bytes on
#pragma unroll 4
            for (int m = 0; m < 16; ++m, from += step) copy16(dst + m * 1024, from, 8 * m < rows);
          }
          ++in;
        } else if (ci < cn) {
          const uint32_t dst = smem_addr(raw) + raw_in * (kRawBytes / 2);
          const unsigned char* next = src + 32 * row_bytes;
          copy16(dst, src, left > 0);
          copy16(dst + 2048, src + 64, left > 0);
          copy16(dst + 4096, next, left > 32);
          copy16(dst + 6144, next + 64, left > 32);
        }
        raw_in = raw_in == 2 ? 0 : raw_in + 1;
        left -= kCopyRows;
        src += kCopyRows * row_bytes;
        if (++ci == works[iord % kWorkRing].chunks * kSteps) {
          ci = 0;
          ++iord;
          begin_copies();
        }
      }
      cp_async_commit();
    };
    // C8: this lane's scales of keys lane, lane + 32, ... of the next chunk that is made ready
    float sc_next[4];
    auto load_scales = [&](const Work& x, int j) {
      const int first = (x.from + j) * kTile + lane;
      const float* at = scale_of + x.kvh * p.cache_rows + x.c0 + first;
#pragma unroll
      for (int e = 0; e < 4; ++e) sc_next[e] = first + 32 * e < x.len ? __ldg(at + 32 * e) : 0.f;
    };
    begin_copies();
    if (C8 && more) load_scales(works[0], 0);
#pragma unroll 1
    for (int k = 0; k < kAhead; ++k) issue();
    int c = is_v, chunk_no = 0, raw_out = 0;
#pragma unroll 1
    for (int ord = 0; ok; ++ord) {
      if (!find_work(ord)) break;
      const Work& w = works[ord % kWorkRing];
      // ---- queries, by both groups
      if (ord > 0) ok = wait_or_abort(qempty, (ord - 1) & 1, p.status, abort);
      if (!ok) break;
      if (C8 && ord > 0) load_scales(w, 0);
      {
        const int qt = tid - kProdWarp * 32, qu = qt & 15;
        const uint16_t* q = static_cast<const uint16_t*>(p.q) + w.t0 * p.q_stride + w.kvh * G * kD + qu * 8;
        const int to = w.pair ? 2 * kTile : kTile;
        if (!C8) {  // all on their way at once
#pragma unroll 2
          for (int r = qt >> 4; r < to; r += 16) {
            const bool there = r < w.rows;
            const uint32_t row = w.row0 + (there ? r : 0), token = row / G;
            copy16(smem_addr(smem + (r >> 7) * kSlotBytes + tile_off(r & 127, qu)), q + token * p.q_stride + (row - token * G) * kD, there);
          }
          cp_async_commit();  // waited for with the piece's first chunk
        } else {
#pragma unroll 1
          for (int r1 = qt >> 4; r1 < to; r1 += 64) {  // four rows at a time
            // (token, head of the group) of row r1 + 16 qu by lane qu: a division for four rows
            const uint32_t row = w.row0 + r1 + 16 * (qu & 3), of = row / G, place = of << 16 | (row - of * G);
            uint4 x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t at = __shfl_sync(0xffffffffu, place, e, 16);
              x[e] = r1 + 16 * e < w.rows ? __ldg(reinterpret_cast<const uint4*>(q + (at >> 16) * p.q_stride + (at & 0xffffu) * kD))
                                          : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = r1 + 16 * e;
              float power = 1.f;
              if (BF) {
                power = row_power(row_max16(top_of<BF>(x[e])));
                x[e] = times_to_half<BF>(x[e], inverse_power(power));
              }
              if (qu == 0) row_factor[(ord & 1) * L::kRows + r] = power * kScaleLog2;
              *reinterpret_cast<uint4*>(smem + (r >> 7) * kSlotBytes + tile_off(r & 127, qu)) = x[e];
            }
          }
          fence_proxy_async();
          mbar_arrive(qfull);
        }
      }
      // ---- chunks
      const int chunks = w.chunks;
#pragma unroll 1
      for (int j = 0; j < chunks && ok; ++j, ++chunk_no, c += 2) {
        const bool is_new = w.has_new && j == chunks - 1;
        unsigned char* slot = slots + (c % kSlots) * kSlotBytes;
        if (C8) {
          ok = wait_slot(chunk_no);
          if (!ok) break;
          float* to_scales = scales + ((chunk_no % kScaleRing) * 2 + is_v) * kTile;
          if (!is_new) {
            // scales that leave every code exact in fp16: powers of two, 2^-15 <= s <= 2^7 (rows that are not there: 0)
            float sc[4];
            bool plain = true;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              sc[e] = sc_next[e];
              const uint32_t x = __float_as_uint(sc[e]);
              plain = plain && (x & 0x7fffffu) == 0u && (x == 0u || x - (112u << 23) <= 22u << 23);
            }
            plain = __all_sync(0xffffffffu, plain);
            if (j + 1 < chunks) load_scales(w, j + 1);
            if (pt < 32) {
              if (lane == 0) plain_of[(chunk_no & 3) * 2 + is_v] = plain ? 1 : 0;
              if (plain || !is_v) {
#pragma unroll
                for (int e = 0; e < 4; ++e) to_scales[lane + 32 * e] = plain ? (is_v ? 0.f : 1.f) : sc[e];
              }
            }
            unsigned char* to = slot + tile_off(r0, 2 * u);  // unit 2 u + 1 at the other place of its pair
            const int other = (r0 & 1) ? -16 : 16;
            // 64 rows; the copy issued first goes where those before were made ready from
            auto next_rows = [&](uint4 (&x)[4]) {
              issue();
              cp_async_wait<kAhead>();
              const unsigned char* mine = raw + raw_out * (kRawBytes / 2);
              raw_out = raw_out == 2 ? 0 : raw_out + 1;
#pragma unroll
              for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint4*>(mine + i * 2048);
            };
            // unit u + 4 (i & 1) of row r0 + 64 h + 32 (i >> 1)
            auto put_unit = [&](int h, int i, const uint32_t (&z)[8]) {
              unsigned char* at = to + h * 8192 + (i >> 1) * 4096 + (i & 1) * 16384;
              *reinterpret_cast<uint4*>(at) = make_uint4(z[0], z[1], z[2], z[3]);
              *reinterpret_cast<uint4*>(at + other) = make_uint4(z[4], z[5], z[6], z[7]);
            };
            if (plain) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint4 x[4];
                next_rows(x);
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // lane r0 has the scale
                  const __half2 f = __float2half2_rn(__shfl_sync(0xffffffffu, sc[2 * h + (i >> 1)], r0));
                  const uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                  uint32_t z[8];
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const uint32_t code = e4m3x2_to_half2(y[e >> 1] >> (16 * (e & 1)));
                    const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&code), f);
                    z[e] = *reinterpret_cast<const uint32_t*>(&v);
                  }
                  put_unit(h, i, z);
                }
              }
            } else {  // a loop of its own: with both in one, plain chunks took 2 % longer
#pragma unroll 1
              for (int h = 0; h < 2; ++h) {
                uint4 x[4];
                next_rows(x);
                if (is_v) {  // the four lanes of a row look whether it is zeros
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    uint32_t any = x[2 * i].x | x[2 * i].y | x[2 * i].z | x[2 * i].w | x[2 * i + 1].x | x[2 * i + 1].y |
                                   x[2 * i + 1].z | x[2 * i + 1].w;
                    any |= __shfl_xor_sync(0xffffffffu, any, 1);
                    any |= __shfl_xor_sync(0xffffffffu, any, 2);
                    const float s1 = __shfl_sync(0xffffffffu, h == 0 ? sc[i] : sc[2 + i], r0);
                    if (u == 0) to_scales[r0 + 64 * h + 32 * i] = (any & 0x7f7f7f7fu) == 0u ? -CUDART_INF_F : __log2f(s1);
                  }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                  uint32_t z[8];
#pragma unroll
                  for (int e = 0; e < 8; ++e) z[e] = e4m3x2_to_half2(y[e >> 1] >> (16 * (e & 1)));
                  put_unit(h, i, z);
                }
              }
            }
          } else {
            issue();
            issue();
            raw_out = raw_out == 0 ? 2 : raw_out - 1;  // two stages on
            if (pt == 0) plain_of[(chunk_no & 3) * 2 + is_v] = 0;
            bool found = false;
            const int nu = pt & 15;
            const uint16_t* from = fresh + w.t0 * p.new_stride + w.kvh * kD + nu * 8;
#pragma unroll 1
            for (int r1 = pt >> 4; r1 < kMaxDrafts; r1 += 32) {  // four rows at a time
              uint4 x[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                x[e] = r1 + 8 * e < w.n ? __ldg(reinterpret_cast<const uint4*>(from + (r1 + 8 * e) * p.new_stride)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int r = r1 + 8 * e;
                if (is_v) x[e] = take_out_wild<BF>(x[e], found);
                float power = 1.f;
                float top = 1.f;
                if (BF || is_v) {  // fp16 values only grow, which is exact
                  top = row_max16(top_of<BF>(x[e]));
                  power = BF ? row_power(top) : fminf(row_power(top), 1.f);
                  x[e] = times_to_half<BF>(x[e], inverse_power(power));
                }
                if (nu == 0) to_scales[r] = !is_v ? power : top == 0.f ? -CUDART_INF_F : __log2f(power);  // no row: zeros
                *reinterpret_cast<uint4*>(slot + tile_off(r, nu)) = x[e];
              }
            }
            if (found) wild[ord & 3] = ord + 1;
          }
        } else {
          // the piece's queries were committed behind the copies of its first kAhead chunks
          issue();
          if (j < kAhead) cp_async_wait<0>();
          else cp_async_wait<kAhead>();
          if (is_new && is_v) {
            bool found = false;
#pragma unroll 1
            for (int r = r0; r < kMaxDrafts; r += 8) {
              uint4* at = reinterpret_cast<uint4*>(slot + tile_off(r, u));
              bool here = false;
              const uint4 y = take_out_wild<BF>(*at, here);
              if (here) *at = y;
              found = found || here;
            }
            if (found) wild[ord & 3] = ord + 1;
          }
        }
        fence_proxy_async();
        if (!C8 && j == 0) mbar_arrive(qfull);
        mbar_arrive((is_v ? vfull : kfull) + (chunk_no & 3));
      }
      give_back(ord);
    }
    cp_async_wait<0>();
  } else {
    // ---------------------------------------------------------------- softmax of group t
    take_registers<128>();
    const int t = warp >> 2;
    const int r = tid & (kTile - 1);
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t scol = tmem + lanes + kColS + t * kTile, ocol = tmem + lanes + kColO;
    bool ok = true;
    int chunk0 = 0;
    uint32_t s_count = 0;
    // What all 256 threads of both groups say. No group may go on to a piece, or to its end, that the other has given up: it
    // would wait there for ever.
    auto both_groups = [](bool mine) {
      int all;
      asm volatile(
          "{\n .reg .pred p, q;\n setp.ne.s32 p, %1, 0;\n barrier.red.and.pred q, 1, 256, p;\n selp.s32 %0, 1, 0, q;\n}"
          : "=r"(all)
          : "r"(static_cast<int>(mine))
          : "memory");
      return all != 0;
    };
#pragma unroll 1
    for (int ord = 0;; ++ord) {
      if (!both_groups(find_work(ord))) break;  // (and the sums of the piece before are read)
      const Work& w = works[ord % kWorkRing];
      const int my_row = w.pair ? t * kTile + r : r;
      const bool mine = my_row < w.rows;
      const uint32_t at = w.row0 + (mine ? my_row : 0), token = at / G;
      const int head = w.kvh * G + (at - token * G);
      float m = -CUDART_INF_F, l = 0.f, f = kScaleLog2;
      float power = 0.f;  // C8: log2 k
      bool first = true;
      // O of this group times `alpha`
      auto rescale = [&](float alpha) {
#pragma unroll 1
        for (int c = 0; c < kD; c += 32) {
          uint32_t o[32];
          tmem_ld32_issue(ocol + t * kTile + c, o);
          tmem_wait_ld32(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
          tmem_st32(ocol + t * kTile + c, o);
        }
      };
#pragma unroll 1
      for (int j = w.pair ? 0 : t; j < w.chunks && ok; j += w.pair ? 1 : 2) {
        ok = wait_or_abort(sfull + t, s_count & 1, p.status, abort);
        ++s_count;
        // S is there, so K and its scales were; V's scales come with V
        if (C8) ok = ok && wait_chunk(vfull, chunk0 + j);
        if (!ok) break;
        tc_fence_after();
        const bool is_new = w.has_new && j == w.chunks - 1;
        const int left = w.len - (w.from + j) * kTile;  // cache rows of this chunk
        if (C8) f = row_factor[(ord & 1) * L::kRows + my_row];
        const bool plain = !C8 || (plain_of[((chunk0 + j) & 3) * 2] & plain_of[((chunk0 + j) & 3) * 2 + 1]) != 0;
        // (sums that k has made smaller by 2^40 or more might leave fp32 without it)
        if (!is_new && left >= kTile && plain && (!C8 || !__any_sync(0xffffffffu, power < -40.f))) {
          // ---- a whole chunk without scales
          float mx[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            uint32_t a[32], b[32];
            tmem_ld32_issue(scol + 32 * i, a);
            tmem_ld32_issue(scol + 32 * i + 32, b);
            tmem_wait_ld32(a);
            tmem_wait_ld32(b);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              mx[0] = max3(mx[0], __uint_as_float(a[e]), __uint_as_float(a[e + 1]));
              mx[1] = max3(mx[1], __uint_as_float(b[e]), __uint_as_float(b[e + 1]));
            }
          }
          const float top = fmaxf(mx[0], mx[1]) * f;
          if (__any_sync(0xffffffffu, top > m + kLag || (C8 && power != 0.f))) {
            const float m_new = top > m + kLag ? top - kTopPower : m;
            const float up = m_new == m ? 0.f : m_new - m;
            m = m_new;
            l *= exp2_fast(-up);
            if (!first) rescale(exp2_fast(-up - power));
            power = 0.f;
          }
          const float nm = m == -CUDART_INF_F ? 0.f : -m;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
          for (int i = 0; i < 2; ++i) {  // 64 keys: 32 columns of P over S columns that have been read
            uint32_t raw[2][32], pk[32];
            tmem_ld32_issue(scol + 64 * i, raw[0]);
            tmem_ld32_issue(scol + 64 * i + 32, raw[1]);
            tmem_wait_ld32(raw[0]);
            tmem_wait_ld32(raw[1]);
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float a = __uint_as_float(raw[e >> 4][2 * (e & 15)]), b = __uint_as_float(raw[e >> 4][2 * (e & 15) + 1]);
              fma2(a, b, f, nm);
              a = exp2_fast(a);
              b = exp2_fast(b);
              if (e & 1) add2(sum[2], sum[3], a, b);
              else add2(sum[0], sum[1], a, b);
              pk[e] = pack16<kBf>(a, b);
            }
            tmem_st32(scol + 32 * i, pk);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        } else {
          // ---- scales, the end of the cache or the new tokens: 32 keys at a time, twice
          const float4* ks = reinterpret_cast<const float4*>(scales + ((chunk0 + j) % kScaleRing) * 2 * kTile);
          const float4* lv = ks + kTile / 4;
          const uint64_t seen = is_new && mine ? p.mask[w.t0 + token] & (w.n < 64 ? (1ull << w.n) - 1 : ~0ull) : 0ull;
          auto scores = [&](int b, float (&s)[32]) {  // times the keys' scales; -infinity where the row does not see
            uint32_t raw[32];
            tmem_ld32_issue(scol + 32 * b, raw);
            tmem_wait_ld32(raw);
            const int here = left - 32 * b;
            const uint32_t bits = is_new ? (b < 2 ? static_cast<uint32_t>(seen >> (32 * b)) : 0u)
                                         : (here >= 32 ? 0xffffffffu : here <= 0 ? 0u : (1u << here) - 1u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 k = C8 ? ks[8 * b + e] : make_float4(1.f, 1.f, 1.f, 1.f);
              s[4 * e] = (bits >> (4 * e)) & 1u ? __uint_as_float(raw[4 * e]) * k.x : -CUDART_INF_F;
              s[4 * e + 1] = (bits >> (4 * e + 1)) & 1u ? __uint_as_float(raw[4 * e + 1]) * k.y : -CUDART_INF_F;
              s[4 * e + 2] = (bits >> (4 * e + 2)) & 1u ? __uint_as_float(raw[4 * e + 2]) * k.z : -CUDART_INF_F;
              s[4 * e + 3] = (bits >> (4 * e + 3)) & 1u ? __uint_as_float(raw[4 * e + 3]) * k.w : -CUDART_INF_F;
            }
          };
          const int blocks = is_new ? 2 : 4;
          float top = -CUDART_INF_F, top_v = -CUDART_INF_F;  // of the scores, and of them with the values' scales
#pragma unroll 1
          for (int b = 0; b < blocks; ++b) {
            float s[32];
            scores(b, s);
#pragma unroll
            for (int e = 0; e < 32; e += 2) top = max3(top, s[e], s[e + 1]);
            if (C8) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float4 v = lv[8 * b + e];
                top_v = max3(top_v, fmaf(s[4 * e], f, v.x), fmaf(s[4 * e + 1], f, v.y));
                top_v = max3(top_v, fmaf(s[4 * e + 2], f, v.z), fmaf(s[4 * e + 3], f, v.w));
              }
            }
          }
          top *= f;
          const float above = C8 ? top_v - m + power : 0.f;  // of the largest weight times scale times k
          // (fp16 keeps 11 bits down to 2^-14, so 4 bits of range for what lies below the largest)
          const bool far_below = C8 && !first && !plain && above < -10.f && top_v > -CUDART_INF_F;
          if (__any_sync(0xffffffffu, top > m + kLag || (C8 && above > 8.f + kTopPower) || far_below)) {
            const float m_new = top > m + kLag ? top - kTopPower : m;
            const float up = m_new == m ? 0.f : m_new - m;
            m = m_new;
            l *= exp2_fast(-up);
            float alpha = exp2_fast(-up);
            if (C8) {
              const float held = floorf(power + up);  // the sums as large as they are
              float most = first ? kMostPower : held;
              if (__any_sync(0xffffffffu, far_below)) {
                float a = 0.f;
#pragma unroll 1
                for (int c = 0; c < kD; c += 32) {
                  uint32_t o[32];
                  tmem_ld32_issue(ocol + t * kTile + c, o);
                  tmem_wait_ld32(o);
#pragma unroll
                  for (int e = 0; e < 32; ++e) a = fmaxf(a, fabsf(__uint_as_float(o[e])));
                }
                const int room = a < CUDART_INF_F ? min(max(142 - static_cast<int>(__float_as_uint(a) >> 23), 0), 120) : 0;
                if (far_below) most = held + static_cast<float>(room);  // they grow to 2^16 at most
              }
              if (top_v > -CUDART_INF_F) most = fminf(most, floorf(kTopPower - (top_v - m)));
              most = fminf(most, kMostPower);
              alpha = exp2_fast(most - power - up);
              power = most;
            }
            if (!first) rescale(alpha);
          }
          const float nm = m == -CUDART_INF_F ? 0.f : -m;
          const float nv = nm + power;
#pragma unroll 1
          for (int b = 0; b < blocks; ++b) {
            float s[32];
            scores(b, s);
            uint32_t pk[16];
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x = exp2_fast(fmaf(s[2 * e], f, nm)), y = exp2_fast(fmaf(s[2 * e + 1], f, nm));
              sum += x + y;
              if (C8) {
                const float2 v = reinterpret_cast<const float2*>(lv)[16 * b + e];
                x = exp2_fast(fmaf(s[2 * e], f, v.x) + nv);
                y = exp2_fast(fmaf(s[2 * e + 1], f, v.y) + nv);
              }
              pk[e] = pack16<kBf>(x, y);
            }
            l += sum;
            // 16 columns of P over S columns 16 b .. 16 b + 15: read before by this thread's block b / 2
            asm volatile(
                "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
                    scol + 16 * b),
                "r"(pk[0]), "r"(pk[1]), "r"(pk[2]), "r"(pk[3]), "r"(pk[4]), "r"(pk[5]), "r"(pk[6]), "r"(pk[7]), "r"(pk[8]),
                "r"(pk[9]), "r"(pk[10]), "r"(pk[11]), "r"(pk[12]), "r"(pk[13]), "r"(pk[14]), "r"(pk[15])
                : "memory");
          }
        }
        first = false;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pfull + t);
      }
      // ---- the piece's result
      ok = ok && wait_or_abort(odone, ord & 1, p.status, abort);
      tc_fence_after();
      if (!w.pair) {
        ml_of[t * kTile + r] = make_float2(m, l);
        if (C8) power_of[t * kTile + r] = power;
      }
      if (!both_groups(ok)) break;
      float w0 = 1.f, w1 = 0.f;  // of the two accumulators, for `pair` of this group's own
      if (!w.pair) {
        const float2 a = ml_of[r], b = ml_of[kTile + r];
        m = fmaxf(a.x, b.x);
        w0 = weight_of(a.x, m);
        w1 = weight_of(b.x, m);
        l = a.y * w0 + b.y * w1;
        if (C8) {
          w0 = weight_of(a.x - power_of[r], m);
          w1 = weight_of(b.x - power_of[kTile + r], m);
        }
      } else if (C8) {
        w0 = exp2_fast(-power);
      }
      const bool whole = w.of == 1;
      const bool two = !w.pair && w.chunks > 1;
      const bool any_wild = w.has_new && wild[ord & 3] == ord + 1;
      const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
      w0 *= inv;
      w1 *= inv;
      // 32 columns at a time through this warp's 4 KB of the queries' place (all S are done), so that rows are
      // written in 128-byte or, as sums, 64-byte pieces by neighbouring lanes; unit u of row r lies at u ^ (r mod 8)
      float* place = reinterpret_cast<float*>(smem + warp * 4096);
      float* slot = slots_of(p) + static_cast<size_t>(w.slot) * slot_floats(L::kRows);
      uint16_t* out = static_cast<uint16_t*>(p.out) + w.t0 * p.n_heads * kD;
      const int d_from = w.pair ? 0 : t * (kD / 2), d_to = w.pair ? kD : d_from + kD / 2;
      const uint32_t own = ocol + (w.pair ? t * kTile : 0);
      const int row_base = (w.pair ? t * kTile : 0) + (warp & 3) * 32;
      const uint32_t line_at = token * p.n_heads + head;  // of this lane's row, from the request's first on
      if (row_base < w.rows) {
#pragma unroll 1
        for (int d = d_from; d < d_to; d += 32) {
          uint32_t o[32];
          float x[32];
          tmem_ld32_issue(own + d, o);
          tmem_wait_ld32(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]) * w0;
          if (two) {
            tmem_ld32_issue(own + kTile + d, o);
            tmem_wait_ld32(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] += __uint_as_float(o[e]) * w1;
          }
          if (mine && any_wild) {
            const uint64_t seen = p.mask[w.t0 + token];
#pragma unroll 1
            for (int k = 0; k < w.n; ++k)
              if ((seen >> k) & 1u) {
                const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v_new) + (w.t0 + k) * p.new_stride + w.kvh * kD + d);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const uint32_t bad = not_finite2<BF>(v[e]);
                  const float2 y = unpack16<BF>(v[e]);
                  if (bad & 0x8000u) x[2 * e] += y.x;
                  if (bad & 0x80000000u) x[2 * e + 1] += y.y;
                }
              }
          }
          __syncwarp();  // the columns before are read
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<float4*>(place + lane * 32 + ((e ^ (lane & 7)) << 2)) = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
          __syncwarp();
          const int e = lane & 7;
#pragma unroll 4
          for (int k = lane >> 3; k < 32; k += 4) {
            const int row = row_base + k;
            const uint32_t row_line = __shfl_sync(0xffffffffu, line_at, k);
            if (row < w.rows) {
              const float4 y = *reinterpret_cast<const float4*>(place + k * 32 + ((e ^ (k & 7)) << 2));
              if (whole) {
                *reinterpret_cast<uint2*>(out + row_line * kD + d + 4 * e) =
                    make_uint2(pack16<BF>(y.x, y.y), pack16<BF>(y.z, y.w));
              } else {
                __stcg(reinterpret_cast<float4*>(slot + row * kD + d) + e, y);
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(oread);
      if (mine && (w.pair || t == 0)) {
        if (whole) {
          if (p.lse != nullptr) p.lse[head * p.new_rows + w.t0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
        } else {
          __stcg(reinterpret_cast<float2*>(slot + L::kRows * kD) + my_row, make_float2(m, l));
        }
        if (w.j == 0) table_of(p)[head * p.new_rows + w.t0 + token] = make_int2(w.first, w.of);
      }
      chunk0 += w.chunks;
      give_back(ord);
      fence_proxy_async();  // the queries' place goes back to the tensor core
      __syncwarp();
      if (lane == 0) mbar_arrive(qempty);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// The rows of cut items: a warp a row, 4 dims a lane, the pieces in the order of their keys, kJoin of them loaded at
// once. ROWS: rows of a slot. What does not hang on the pieces is done before they are waited for.
constexpr int kJoin = 10;
template <bool BF, int ROWS>
__global__ void __launch_bounds__(128) tree_join_kernel(const TreeArgs p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long at = static_cast<long long>(blockIdx.x) * 4 + warp;  // token * n_heads + head
  const long long token = at / p.n_heads;
  const int head = static_cast<int>(at - token * p.n_heads);
  long long t0 = -1;  // first token of its request
  if (token < p.new_rows) {
    for (int b0 = 0; b0 < p.B && t0 < 0; b0 += 32) {
      TreeRequest r;
      const bool mine = b0 + lane < p.B && tree_request(p, b0 + lane, r) && token >= r.t0 && token < r.t0 + r.n;
      const uint32_t found = __ballot_sync(0xffffffffu, mine);
      if (found != 0u) t0 = __shfl_sync(0xffffffffu, r.t0, __ffs(found) - 1);
    }
  }
  const int G = p.n_heads / p.n_kv_heads;
  const int row = static_cast<int>(token - t0) * G % ROWS;
  pdl_wait();
  if (t0 < 0) return;
  const int2 entry = table_of(p)[head * p.new_rows + token];
  const int of = entry.y;
  if (of <= 1 || of > kPartials || slot_of(entry.x, 0) < 0 || slot_of(entry.x, of - 1) >= kPartials) return;
  const int my_row = (row + head % G) % ROWS;
  const float* slots = slots_of(p);
  auto slot = [&](int j) { return slots + slot_of(entry.x, j) * slot_floats(ROWS); };
  float4 v[kJoin];
  auto load = [&](int j0) {
#pragma unroll
    for (int e = 0; e < kJoin; ++e)
      v[e] = j0 + e < of ? __ldcg(reinterpret_cast<const float4*>(slot(j0 + e) + my_row * kD) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  load(0);
  float m = -CUDART_INF_F;
  for (int j = lane; j < of; j += 32) m = fmaxf(m, __ldcg(slot(j) + ROWS * kD + 2 * my_row));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int j0 = 0; j0 < of; j0 += kJoin) {
    if (j0 > 0) load(j0);
    float w = 0.f;
    if (lane < min(kJoin, of - j0)) {
      const float2 x = __ldcg(reinterpret_cast<const float2*>(slot(j0 + lane) + ROWS * kD) + my_row);
      w = weight_of(x.x, m);
      l += w * x.y;
    }
#pragma unroll
    for (int e = 0; e < kJoin; ++e) {
      const float a = __shfl_sync(0xffffffffu, w, e);
      o.x += a * v[e].x;
      o.y += a * v[e].y;
      o.z += a * v[e].z;
      o.w += a * v[e].w;
    }
  }
  l = warp_sum(l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at * kD + 4 * lane) =
      make_uint2(pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv));
  if (p.lse != nullptr && lane == 0) p.lse[head * p.new_rows + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
}

struct Kernels {
  const void* main;
  const void* join;
  size_t smem;
};
template <bool BF, bool C8, bool WIDE>
Kernels kernels_for() {
  return {reinterpret_cast<const void*>(&tree_tc_kernel<BF, C8, WIDE>),
          reinterpret_cast<const void*>(&tree_join_kernel<BF, Layout<C8, WIDE>::kRows>), Layout<C8, WIDE>::kSmem};
}
template <bool BF>
Kernels kernels_of(bool cache8, bool wide) {
  return cache8 ? (wide ? kernels_for<BF, true, true>() : kernels_for<BF, true, false>())
                : (wide ? kernels_for<BF, false, true>() : kernels_for<BF, false, false>());
}

// Items of 256 rows read the cache once for twice the rows; those of 128 keep one more chunk in shared memory and have
// both groups at work on any item. By the rows that a request has on average: 8-bit caches with about 24 rows a request
// 53.0 us, 62.5 with wide items; 72 rows 57.4 and 66.7 (16-bit 53.8 and 50.6); 200 rows 64.9, and 52.5 with wide items (all
// before the softmax had more registers).
bool is_wide(int B, long long new_rows, int group) { return new_rows * group > static_cast<long long>(B) * kTile; }

}  // namespace

size_t tree_tc_workspace_bytes(int B, long long new_rows, int n_heads, int n_kv_heads) {
  return (kTreeHeader + kTreeCounters) * sizeof(int) + table_bytes(new_rows, n_heads) +
         kPartials * slot_floats(is_wide(B, new_rows, n_heads / n_kv_heads) ? 2 * kTile : kTile) * sizeof(float);
}

cudaError_t launch_tree_tc(const TreeArgs& a, int dtype, bool cache8, cudaStream_t stream) {
  const bool wide = is_wide(a.B, a.new_rows, a.n_heads / a.n_kv_heads);
  const Kernels k = dtype == FSX_BF16 ? kernels_of<true>(cache8, wide) : kernels_of<false>(cache8, wide);
  const long long join_blocks = (a.new_rows * a.n_heads + 3) / 4;  // below 2^31: the caller sees to it
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  cudaError_t e = allow_shared_memory(k.main, k.smem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<TreeArgs*>(&a)};
  e = launch_ex(k.main, dim3(static_cast<unsigned>(sms < kMaxGrid ? sms : kMaxGrid)), dim3(kThreads), k.smem, stream, false, args);
  if (e != cudaSuccess) return e;
  return launch_ex(k.join, dim3(static_cast<unsigned>(join_blocks)), dim3(128), 0, stream, true, args);
}

}  // namespace fsx
