// Page tables: a step of them (requests forked, freed and grown), compaction, and the copies of pages that both ask for
// (fsx_pages_step, fsx_pages_compact, fsx_pages_copy).
//
// A page is free when nobody holds it (refs 0). The free pages that a step hands out are the lowest ones, in the order of the requests, so
// that equal states give equal tables: counts of holders are sums of atomics, which do not depend on their order, and every place is a
// count of what lies before it.
//
// A step and a compaction are one launch each, of one cluster of 8 CTAs: their phases follow one another by cluster barriers (0.5 us each),
// each CTA takes an eighth of the pages, and the CTAs tell each other their counts through distributed shared memory.
// Bound by latency: a handful of dependent trips to memory; the holders' counts are read twice.
// The copies are bound by memory: both ends of every page move once, all layers in one launch.
//
// Measured: a step of 64 requests over 8192 pages 7.9 us; a compaction of 48 over 4096 pages 7.7 us; 803 pages of 32 KB in 8 planes
// 68 us (6.2 TB/s, 0.91 of a copy's rate); 39 of them 4.1 us.
#include <cooperative_groups.h>

#include "device_util.cuh"
#include "fsx.h"
#include "kernels.h"
#include "pages.h"

namespace cg = cooperative_groups;

namespace fsx {

namespace {

constexpr int kCtas = 8;
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kPerThread = kMaxSequences / kThreads;  // requests
constexpr int kAtOnce = 8;                           // entries of a table's row that a lane loads at once

enum : int { kStatusOom = 3 };

struct TableShared {
  __align__(16) int last[kMaxSequences];  // a request's last page, if new tokens go into it, else -1
  int n[kMaxSequences];                   // its rows before its new tokens
  int add[kMaxSequences];                 // new tokens, 0: none or not possible
  long long end[kMaxSequences];           // pages that it and the requests before it need
  unsigned char copies[kMaxSequences];
  short leaves[kMaxSequences];  // the last of the others that write into the page that it keeps, if any, else -1
  int nth[kMaxSequences];       // copies of the requests before
  long long scan[kWarps];
  int scan2[kWarps];
  int counts[2][kCtas];
};

// sum over the threads before this one; `total`: of all
__device__ __forceinline__ int scan_before(int x, int* warps, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  __syncthreads();
  if (lane == 31) warps[warp] = sum;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) sum += warps[w];
    total += warps[w];
  }
  return sum - x;
}

// The pages first .. end - 1 of this CTA
__device__ __forceinline__ void part_of(int n_pages, int rank, int& first, int& end) {
  const int part = ((n_pages + kCtas - 1) / kCtas + 3) & ~3;
  first = static_cast<int>(min(static_cast<long long>(n_pages), static_cast<long long>(rank) * part));
  end = static_cast<int>(min(static_cast<long long>(n_pages), static_cast<long long>(first) + part));
}

// Every CTA's `mine`, where every CTA can read it. All of them run already.
__device__ __forceinline__ void tell(cg::cluster_group& cluster, int (&counts)[kCtas], int rank, int mine) {
  if (threadIdx.x < kCtas) *cluster.map_shared_rank(&counts[rank], threadIdx.x) = mine;
  cluster.sync();
}

// Rows of request `i` of a table of lengths; -1: more than its pages hold, or negative
__device__ __forceinline__ int rows_at(const int64_t* lengths, int i, int width, int shift) {
  const long long n = lengths[i];
  return n < 0 || n > static_cast<long long>(width) << shift || n > 0x7fffffffll - 64 ? -1 : static_cast<int>(n);
}
__device__ __forceinline__ int pages_for(long long n, int shift) { return static_cast<int>((n + (1 << shift) - 1) >> shift); }

__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads) step_kernel(const StepArgs a) {
  extern __shared__ __align__(16) unsigned char raw_smem[];
  TableShared& sm = *reinterpret_cast<TableShared*>(raw_smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank()), tid = threadIdx.x, lane = tid & 31;
  const int thread = rank * kThreads + tid, warp = thread >> 5;
  constexpr int kAllThreads = kCtas * kThreads, kAllWarps = kAllThreads / 32;
  const bool moved = a.table_out != a.table;
  pdl_launch_dependents();
  pdl_wait();
  if (a.refs_out != a.refs) {
    for (int i = thread; i < a.n_pages; i += kAllThreads) a.refs_out[i] = a.refs[i];
  }
  // ---- every request's rows, new tokens and last page; every CTA for itself
  auto source = [&](int i) { return a.source != nullptr ? a.source[i] : i; };
  for (int i = tid; i < a.B; i += kThreads) {
    const int src = source(i);
    const long long t0 = a.new_offsets[i], t1 = a.new_offsets[i + 1];
    const bool known = src >= -1 && src < a.B_in;
    int n = known && src >= 0 ? rows_at(a.lengths, src, a.width, a.shift) : 0;
    bool fine = t0 >= 0 && t1 >= t0 && t1 <= a.new_rows;
    long long add = fine ? t1 - t0 : 0;
    if (!known || n < 0) {  // comes out empty
      n = 0;
      add = 0;
      fine = false;
    }
    if (n + add > static_cast<long long>(a.width) << a.shift || n + add > 0x7fffffffll - 64) {
      add = 0;
      fine = false;
    }
    int last = -1;
    if (add > 0 && (n & ((1 << a.shift) - 1)) != 0) {
      last = a.table[static_cast<long long>(src) * a.width + (n >> a.shift)];
      if (last < 0 || last >= a.n_pages) {
        add = 0;
        last = -1;
        fine = false;
      }
    }
    if (!fine && rank == 0) set_status(a.status, kStatusDeviceArg);
    sm.n[i] = n;
    sm.add[i] = static_cast<int>(add);
    sm.last[i] = last;
  }
  for (int i = a.B + tid; i < ((a.B + 3) & ~3); i += kThreads) sm.last[i] = -1;
  cluster.sync();
  // ---- rows of the table, and the holders of their pages: a warp a new or an old row; a request that goes on from itself changes none
  for (int w = warp; w < a.B + a.B_in; w += kAllWarps) {
    if (w < a.B) {
      const int src = source(w);
      if (!moved && src == w) continue;
      const int had = pages_for(sm.n[w], a.shift);
      const int32_t* from = a.table + static_cast<long long>(src) * a.width;  // not read where had is 0
      int32_t* to = a.table_out + static_cast<long long>(w) * a.width;
      for (int j0 = lane; j0 < a.width; j0 += 32 * kAtOnce) {
        int page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) page[u] = j0 + 32 * u < had ? from[j0 + 32 * u] : -1;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const int j = j0 + 32 * u;
          if (j < a.width) to[j] = page[u];
          if (src != w && j < had) {
            if (page[u] >= 0 && page[u] < a.n_pages) atomicAdd(a.refs_out + page[u], 1);
            else set_status(a.status, kStatusDeviceArg);
          }
        }
      }
    } else {
      const int i = w - a.B;
      if (i < a.B && source(i) == i) continue;
      const int n = rows_at(a.lengths, i, a.width, a.shift);
      if (n < 0 && lane == 0) set_status(a.status, kStatusDeviceArg);
      const int had = n > 0 ? pages_for(n, a.shift) : 0;
      const int32_t* from = a.table + static_cast<long long>(i) * a.width;
      for (int j0 = lane; j0 < had; j0 += 32 * kAtOnce) {
        int page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) page[u] = j0 + 32 * u < had ? from[j0 + 32 * u] : 0;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
          if (j0 + 32 * u < had) {
            if (page[u] >= 0 && page[u] < a.n_pages) atomicSub(a.refs_out + page[u], 1);
            else set_status(a.status, kStatusDeviceArg);
          }
      }
    }
  }
  cluster.sync();
  // ---- what each request needs, and the free pages of this CTA's part
  int first, last_page;
  part_of(a.n_pages, rank, first, last_page);
  int free_pages = 0;
  for (int i = first + 4 * tid; i < last_page; i += 4 * kThreads)  // parts begin at multiples of 4
#pragma unroll
    for (int j = 0; j < 4; ++j) free_pages += i + j < last_page && load_l2(a.refs_out + i + j) <= 0;
  long long need[kPerThread], mine = 0;
  int copy[kPerThread], leaves[kPerThread], my_copies = 0;
  const int per = (a.B + kThreads - 1) / kThreads;  // requests of a thread, one behind another
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    const int i = tid * per + u;
    need[u] = 0;
    copy[u] = 0;
    leaves[u] = -1;
    if (u < per && i < a.B) {
      const int last = sm.last[i], held = last >= 0 ? load_l2(a.refs_out + last) : 0;
      if (held > 1) {  // of all that write into it the last one keeps it, if nobody else holds it
        int writers = 0, behind = -1, next = -1;  // the last one, and the one before it
        auto see = [&](int page, int x) {
          if (page == last) {
            ++writers;
            next = behind;
            behind = x;
          }
        };
        for (int x = 0; x < a.B; x += 4) {
          const int4 other = *reinterpret_cast<const int4*>(&sm.last[x]);
          see(other.x, x);
          see(other.y, x + 1);
          see(other.z, x + 2);
          see(other.w, x + 3);
        }
        copy[u] = !(held == writers && i == behind);
        if (!copy[u]) leaves[u] = next;
      }
      if (sm.add[i] > 0) need[u] = pages_for(static_cast<long long>(sm.n[i]) + sm.add[i], a.shift) - (pages_for(sm.n[i], a.shift) - copy[u]);
      mine += need[u];
      my_copies += copy[u];
    }
  }
  // sums over the threads before: pages in the upper bits, at most 1024 copies below
  long long packed = mine << 11 | my_copies;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, packed, o);
    if (lane >= o) packed += up;
  }
  free_pages = __reduce_add_sync(0xffffffffu, free_pages);
  if (lane == 31) {
    sm.scan[tid >> 5] = packed;
    sm.scan2[tid >> 5] = free_pages;
  }
  __syncthreads();
  long long all = 0;
  int in_part = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < (tid >> 5)) packed += sm.scan[w];
    all += sm.scan[w];
    in_part += sm.scan2[w];
  }
  const long long total = all >> 11;
  const int total_copies = static_cast<int>(all & 2047);
  long long before = (packed >> 11) - mine;
  int copies_before = static_cast<int>(packed & 2047) - my_copies;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    const int i = tid * per + u;
    if (u < per && i < a.B) {
      before += need[u];
      sm.end[i] = before;
      sm.copies[i] = static_cast<unsigned char>(copy[u]);
      sm.leaves[i] = static_cast<short>(leaves[u]);
      sm.nth[i] = copies_before;
      copies_before += copy[u];
    }
  }
  tell(cluster, sm.counts[0], rank, in_part);
  long long all_free = 0, nth_free = 0;
  for (int r = 0; r < kCtas; ++r) {
    if (r < rank) nth_free += sm.counts[0][r];
    all_free += sm.counts[0][r];
  }
  // A request grows if the pages last for it and all before it, or if it needs none. One that keeps a page which others write into grows only if
  // they leave it: where the last of them gets a page for its copy, those before it have theirs.
  auto start_of = [&](int i) { return i > 0 ? sm.end[i - 1] : 0ll; };
  auto grows = [&](int i) {
    return (sm.end[i] <= all_free || sm.end[i] == start_of(i)) && (sm.leaves[i] < 0 || sm.end[sm.leaves[i]] <= all_free);
  };
  const long long wanted = min(total, all_free);
  for (int base = first; base < last_page && nth_free < wanted; base += kThreads) {
    const int page = base + tid;
    const bool is_free = page < last_page && load_l2(a.refs_out + page) <= 0;
    int in_tile;
    const long long nth = nth_free + scan_before(is_free ? 1 : 0, sm.scan2, in_tile);
    nth_free += in_tile;
    if (!is_free || nth >= wanted) continue;
    int lo = 0, hi = a.B - 1;  // the first request whose end lies above nth
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sm.end[mid] > nth) hi = mid;
      else lo = mid + 1;
    }
    if (!grows(lo)) continue;
    const int n = sm.n[lo], kept = pages_for(n, a.shift) - sm.copies[lo], col = kept + static_cast<int>(nth - start_of(lo));
    a.table_out[static_cast<long long>(lo) * a.width + col] = page;
    a.refs_out[page] = 1;
    const long long t0 = a.new_offsets[lo], end = static_cast<long long>(n) + sm.add[lo];
    for (long long x = max(static_cast<long long>(n), static_cast<long long>(col) << a.shift); x < min(end, static_cast<long long>(col + 1) << a.shift); ++x)
      a.rows[t0 + x - n] = (static_cast<long long>(page) << a.shift) + (x - (static_cast<long long>(col) << a.shift));
    if (sm.copies[lo] && col == kept) {
      a.pairs[2 * sm.nth[lo]] = sm.last[lo];
      a.pairs[2 * sm.nth[lo] + 1] = page;
    }
  }
  // ---- lengths, rows in pages that are there already; one CTA
  if (rank != kCtas - 1) return;
  int copied = 0;
  for (int i = tid; i < a.B; i += kThreads) {
    const bool grown = grows(i);
    const int n = sm.n[i], add = sm.add[i];
    const long long t0 = a.new_offsets[i], t1 = a.new_offsets[i + 1];
    a.lengths_out[i] = n + (grown ? add : 0);
    if (!grown) set_status(a.status, kStatusOom);
    if (!grown || add == 0) {
      for (long long t = max(t0, 0ll); t < min(t1, a.new_rows); ++t) a.rows[t] = -1;
    } else if (sm.last[i] >= 0) {
      if (sm.copies[i]) {
        atomicSub(a.refs_out + sm.last[i], 1);
        ++copied;
      } else {
        const int col = n >> a.shift;
        const long long end = min(static_cast<long long>(n) + add, static_cast<long long>(col + 1) << a.shift);
        for (long long x = n; x < end; ++x)
          a.rows[t0 + x - n] = (static_cast<long long>(sm.last[i]) << a.shift) + (x - (static_cast<long long>(col) << a.shift));
      }
    }
  }
  if (total > all_free) {  // not all of them
    scan_before(copied, sm.scan2, copied);
  } else {
    copied = total_copies;
  }
  if (tid == 0) *a.n_pairs = copied;
}

__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreads) compact_kernel(const CompactArgs a) {
  __shared__ int scan[kWarps];
  __shared__ int counts[3][kCtas];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = static_cast<int>(cluster.block_rank()), tid = threadIdx.x;
  const int thread = rank * kThreads + tid;
  constexpr int kAllThreads = kCtas * kThreads;
  int first, end;
  part_of(a.n_pages, rank, first, end);
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // this CTA runs
  pdl_launch_dependents();
  pdl_wait();
  int mine = 0;
  for (int i = first + tid; i < end; i += kThreads) {
    const int r = a.refs[i];
    mine += r > 0;
    if (r < 0 || a.refs_out != a.refs) a.refs_out[i] = max(r, 0);
  }
  int in_part;
  scan_before(mine, scan, in_part);
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // every CTA of the cluster runs
  tell(cluster, counts[0], rank, in_part);
  int used = 0;
  for (int r = 0; r < kCtas; ++r) used += counts[0][r];
  // ---- the i-th page in use at `used` or above goes to the i-th free one below: as many as those
  int moves = 0, room = 0;
  for (int i = first + tid; i < end; i += kThreads) {
    const bool in_use = load_l2(a.refs_out + i) > 0;
    moves += in_use && i >= used;
    room += !in_use && i < used;
  }
  int all_moves, all_room;
  scan_before(moves, scan, all_moves);
  scan_before(room, scan, all_room);
  if (tid < kCtas) *cluster.map_shared_rank(&counts[2][rank], tid) = all_room;
  tell(cluster, counts[1], rank, all_moves);
  int nth_move = 0, nth_room = 0, m = 0;
  for (int r = 0; r < kCtas; ++r) {
    if (r < rank) {
      nth_move += counts[1][r];
      nth_room += counts[2][r];
    }
    m += counts[1][r];
  }
  for (int base = first; base < end; base += kThreads) {
    const int i = base + tid;
    const bool there = i < end, in_use = there && load_l2(a.refs_out + i) > 0;
    const bool goes = in_use && i >= used, takes = there && !in_use && i < used;
    int in_tile;
    // a tile may hold both, in two runs: one scan for both, halves of a word
    const int at = scan_before((goes ? 1 : 0) + (takes ? 1 << 16 : 0), scan, in_tile);
    if (goes) a.pairs[2 * (nth_move + (at & 0xffff))] = i;
    if (takes) a.pairs[2 * (nth_room + (at >> 16)) + 1] = i;
    nth_move += in_tile & 0xffff;
    nth_room += in_tile >> 16;
  }
  cluster.sync();
  // ---- holders move; the old place keeps the new one for the tables, as -1 - page
  for (int i = thread; i < m; i += kAllThreads) {
    const int src = load_l2(a.pairs + 2 * i), dst = load_l2(a.pairs + 2 * i + 1);
    a.refs_out[dst] = load_l2(a.refs_out + src);
    a.refs_out[src] = -1 - dst;
  }
  cluster.sync();
  const long long entries = static_cast<long long>(a.B) * a.width;
  for (long long e = thread; e < entries; e += kAllThreads) {
    const int b = static_cast<int>(e / a.width), j = static_cast<int>(e - static_cast<long long>(b) * a.width);
    const int n = rows_at(a.lengths, b, a.width, a.shift);
    int page = a.table[e];
    bool changed = a.table_out != a.table;
    if (n < 0) {
      if (j == 0) set_status(a.status, kStatusDeviceArg);
    } else if (j < pages_for(n, a.shift)) {
      if (page < 0 || page >= a.n_pages) {
        set_status(a.status, kStatusDeviceArg);
      } else if (page >= used) {
        const int r = load_l2(a.refs_out + page);
        if (r < 0) {
          page = -1 - r;
          changed = true;
        }
      }
    }
    if (changed) a.table_out[e] = page;
  }
  cluster.sync();
  for (int i = thread; i < m; i += kAllThreads) a.refs_out[load_l2(a.pairs + 2 * i)] = 0;
  if (thread == 0) *a.n_pairs = m;
}

// ---------------------------------------------------------------- copies

constexpr int kCopyThreads = 256;
constexpr int kUnit = 16384;  // bytes that a CTA moves at a time
constexpr int kSmall = 2048;  // bytes of a page in a plane, all segments, up to which a warp moves them, eight planes a CTA: 800 pages of
// 8-bit rows of 8 heads with scales over 4 layers take 37 us, with a CTA a segment 151

struct CopyPlane {
  unsigned char* base;
  long long page_bytes, stride;
  int segments, units;  // units of a segment; with `together` > 1 of all of them
  int together;         // segments of a unit: short ones go many at a time
  int first;            // units of the planes before, of one page
};
// `segs` segments of `bytes` each, `stride` apart, from one page to another, by THREADS threads
template <int THREADS, typename T>
__device__ __forceinline__ void copy_segments(unsigned char* base, long long stride, long long from, long long to, int segs, int bytes) {
  const uint32_t each = static_cast<uint32_t>(bytes) / sizeof(T), all = each * segs;
#pragma unroll 1
  for (uint32_t i = threadIdx.x % THREADS; i < all; i += 2 * THREADS) {  // two at once: few registers, which the long copies need
    const uint32_t j = i + THREADS, seg_i = i / each, seg_j = j / each;
    unsigned char* const at_i = base + seg_i * stride + static_cast<long long>(i - seg_i * each) * sizeof(T);
    unsigned char* const at_j = base + seg_j * stride + static_cast<long long>(j - seg_j * each) * sizeof(T);
    const T x = *reinterpret_cast<const T*>(at_i + from);
    T y;
    if (j < all) y = *reinterpret_cast<const T*>(at_j + from);
    *reinterpret_cast<T*>(at_i + to) = x;
    if (j < all) *reinterpret_cast<T*>(at_j + to) = y;
  }
}

template <int THREADS>
__device__ __forceinline__ void copy_some(const CopyPlane& p, int seg0, int segs, int src, int dst) {
  unsigned char* const base = p.base + seg0 * p.stride;
  const long long from = src * p.page_bytes, to = dst * p.page_bytes;
  const int bytes = static_cast<int>(p.page_bytes);
  if (((reinterpret_cast<uintptr_t>(p.base) | static_cast<uintptr_t>(p.segments > 1 ? p.stride : 0) | static_cast<uintptr_t>(bytes)) & 15u) == 0)
    copy_segments<THREADS, uint4>(base, p.stride, from, to, segs, bytes);
  else
    copy_segments<THREADS, uint32_t>(base, p.stride, from, to, segs, bytes);
}

// PLANES: room in the kernel's parameters, 2.6 or 20 KB (2.4 or 2.9 us of the caller's time)
template <int PLANES>
struct CopyArgs {
  const int32_t* pairs;
  const int32_t* n_pairs;
  int max_pairs, n_pages, n_planes, units;  // units of one page over all planes
  int n_large, large_units;                 // the planes whose pages are more than kSmall bytes come first
  int* status;
  CopyPlane planes[PLANES];
};

template <int PLANES>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ CopyArgs<PLANES> a) {
  const int tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  // the first pair is read beside the count: there are max_pairs of them in memory
  const long long most = static_cast<long long>(a.max_pairs) * a.units;
  long long w = blockIdx.x;
  int pair = static_cast<int>(w / a.units);
  int2 ends = w < most ? *(reinterpret_cast<const int2*>(a.pairs) + pair) : make_int2(0, 0);
  int n = *a.n_pairs;
  if (n < 0 || n > a.max_pairs) {
    if (blockIdx.x == 0 && tid == 0) set_status(a.status, kStatusDeviceArg);
    n = 0;
  }
  const long long total = static_cast<long long>(n) * a.units;
  for (; w < total; w += gridDim.x) {
    const int unit = static_cast<int>(w - static_cast<long long>(pair) * a.units), src = ends.x, dst = ends.y;
    if (w + gridDim.x < total) {
      pair = static_cast<int>((w + gridDim.x) / a.units);
      ends = *(reinterpret_cast<const int2*>(a.pairs) + pair);
    }
    if (src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages) {
      if (tid == 0) set_status(a.status, kStatusDeviceArg);
      continue;
    }
    if (unit >= a.large_units) {
      const int small = a.n_large + (unit - a.large_units) * (kCopyThreads / 32) + (tid >> 5);
      if (small < a.n_planes) copy_some<32>(a.planes[small], 0, a.planes[small].segments, src, dst);
      continue;
    }
    int lo = 0, hi = a.n_large - 1;  // the last plane that begins at `unit` or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.planes[mid].first <= unit) lo = mid;
      else hi = mid - 1;
    }
    const CopyPlane& p = a.planes[lo];
    const int in_plane = unit - p.first;
    if (p.together > 1) {
      const int seg0 = in_plane * p.together;
      copy_some<kCopyThreads>(p, seg0, min(p.together, p.segments - seg0), src, dst);
      continue;
    }
    const int segment = in_plane / p.units;
    const long long at = static_cast<long long>(in_plane - segment * p.units) * kUnit;
    const long long bytes = min(static_cast<long long>(kUnit), p.page_bytes - at);
    const unsigned char* from = p.base + segment * p.stride + src * p.page_bytes + at;
    unsigned char* to = p.base + segment * p.stride + dst * p.page_bytes + at;
    if (((reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(to) | static_cast<uintptr_t>(bytes)) & 15u) == 0) {
      constexpr int kEach = kUnit / 16 / kCopyThreads;
      const int n16 = static_cast<int>(bytes >> 4);
      uint4 x[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (tid + i * kCopyThreads < n16) x[i] = reinterpret_cast<const uint4*>(from)[tid + i * kCopyThreads];
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (tid + i * kCopyThreads < n16) reinterpret_cast<uint4*>(to)[tid + i * kCopyThreads] = x[i];
    } else {
      for (int i = tid; i < static_cast<int>(bytes >> 2); i += kCopyThreads)
        reinterpret_cast<uint32_t*>(to)[i] = reinterpret_cast<const uint32_t*>(from)[i];
    }
  }
}

}  // namespace

cudaError_t launch_pages_step(const StepArgs& a, cudaStream_t stream) {
  const void* fn = reinterpret_cast<const void*>(&step_kernel);
  const cudaError_t e = allow_shared_memory(fn, sizeof(TableShared));
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<StepArgs*>(&a)};
  return launch_ex(fn, dim3(kCtas), dim3(kThreads), sizeof(TableShared), stream, true, args);
}

cudaError_t launch_pages_compact(const CompactArgs& a, cudaStream_t stream) {
  void* args[] = {const_cast<CompactArgs*>(&a)};
  return launch_ex(reinterpret_cast<const void*>(&compact_kernel), dim3(kCtas), dim3(kThreads), 0, stream, true, args);
}

template <int PLANES>
static cudaError_t copy_with(const fsx_page_plane* planes, int n_planes, int n_pages, const int32_t* pairs, const int32_t* n_pairs, int max_pairs,
                             int* status, cudaStream_t stream) {
  CopyArgs<PLANES> a;
  a.pairs = pairs;
  a.n_pairs = n_pairs;
  a.max_pairs = max_pairs;
  a.n_pages = n_pages;
  a.n_planes = n_planes;
  a.status = status;
  long long units = 0;
  int large = 0, small = n_planes;
  for (int i = 0; i < n_planes; ++i) {
    const long long bytes = planes[i].page_bytes, segments = planes[i].segments;
    const bool is_small = bytes * segments <= kSmall;
    const long long together = bytes * 2 <= kUnit && segments > 1 ? (kUnit / bytes < segments ? kUnit / bytes : segments) : 1;
    const long long each = together > 1 ? (segments + together - 1) / together : (bytes + kUnit - 1) / kUnit;
    a.planes[is_small ? --small : large++] =
        CopyPlane{static_cast<unsigned char*>(planes[i].base), bytes, planes[i].segment_stride, static_cast<int>(segments),
                  static_cast<int>(each), static_cast<int>(together), static_cast<int>(units)};
    if (!is_small) units += together > 1 ? each : each * segments;
    if (units > 0x3fffffffll) return cudaErrorInvalidValue;
  }
  a.n_large = large;
  a.large_units = static_cast<int>(units);
  units += (n_planes - large + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  a.units = static_cast<int>(units);
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  const long long most = units * max_pairs, want = static_cast<long long>(sms) * 8;
  void* args[] = {&a};
  return launch_ex(reinterpret_cast<const void*>(&copy_kernel<PLANES>), dim3(static_cast<unsigned>(most < want ? most : want)), dim3(kCopyThreads), 0,
                   stream, true, args);
}

cudaError_t launch_pages_copy(const fsx_page_plane* planes, int n_planes, int n_pages, const int32_t* pairs,
                              const int32_t* n_pairs, int max_pairs, int* status, cudaStream_t stream) {
  return n_planes <= 64 ? copy_with<64>(planes, n_planes, n_pages, pairs, n_pairs, max_pairs, status, stream)
                        : copy_with<kMaxPlanes>(planes, n_planes, n_pages, pairs, n_pairs, max_pairs, status, stream);
}

}  // namespace fsx
