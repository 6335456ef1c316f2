// Bounds of the keys of a page, and the pages that a query's score selects (fsx_page_bounds, fsx_page_select).
//
// Bounds: per page, kv head and dimension the least and the largest key, as int8 codes times a power of two per page and head, the
// smallest that brings the largest magnitude to 127 or below. A power of two makes key / scale exact; the codes are
// rounded outwards, so that they bound the keys. 260 bytes stand for a page's keys of a head: 1/16 of a page of 16 rows of bf16.
//
// Score of a page for a query head: 2^(e_q + e_p) sum_d max(c_d lo_d, c_d hi_d), c the query's codes (int8, a power of two a head):
// what the largest product of the query with a key inside the bounds could be, but for the rounding of the query. max(c lo, c hi) is
// c hi where c > 0 and c lo elsewhere: two dot products of int8 with the positive and the negative part of c, in whole numbers
// below 2^22, times a power of two: exact in fp32, and so is the largest over the heads of a group. The pages that are
// chosen depend on no order of summation.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "fsx.h"
#include "kernels.h"
#include "pages.h"
#include "rows8.cuh"
#include "tc_attention.cuh"

namespace cg = cooperative_groups;

namespace fsx {

namespace {

// the smallest power of two s >= 2^-126 with top / s <= 127, top >= 0 and finite; 1 for 0
__device__ __forceinline__ float scale_of(float top) {
  const uint32_t b = __float_as_uint(top);  // f 2^E, 1 <= f < 2: 2^(E - 6) holds f <= 127 / 64
  const int e = max(static_cast<int>(b >> 23) - 127 - 6 + ((b & 0x7fffffu) > 0x7e0000u ? 1 : 0), -126);
  return b == 0u ? 1.f : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
__device__ __forceinline__ float inverse(float power) { return __uint_as_float(0x7f000000u - __float_as_uint(power)); }

// false: the length is negative or more than the table's pages hold
__device__ __forceinline__ bool rows_of(const PagedCache& p, int b, int& len, int& pages) {
  const long long n = p.lengths[b];
  len = pages = 0;
  if (n < 0 || n > static_cast<long long>(p.width) << p.shift || n > 0x7fffffffll - 64) return false;
  len = static_cast<int>(n);
  pages = static_cast<int>((n + (1 << p.shift) - 1) >> p.shift);
  return true;
}

// ---------------------------------------------------------------- bounds

constexpr int kBoundsWarps = 8;

// A warp a page and kv head: 16 lanes a row of 16-bit keys (two rows at once), 8 lanes a row of codes (four).
template <int TYPE>
__global__ void __launch_bounds__(32 * kBoundsWarps) bounds_kernel(const BoundsArgs a) {
  constexpr bool kC8 = TYPE == FSX_E4M3, kBf = TYPE == FSX_BF16;
  constexpr int kLanes = kC8 ? 8 : 16, kValues = kHeadDim / kLanes, kAtOnce = 32 / kLanes;
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes, sub = lane / kLanes;
  const int b = blockIdx.y;
  int len, pages;
  const bool fine = rows_of(a.pages, b, len, pages);
  const long long start = a.start != nullptr ? a.start[b] : 0;
  if (!fine || start < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) set_status(a.status, kStatusDeviceArg);
    return;
  }
  const int shift = a.pages.shift;
  const int first = start >= len ? pages : static_cast<int>(start >> shift);
  const long long units = static_cast<long long>(pages - first) * a.n_kv_heads;
  const long long row_bytes = static_cast<long long>(a.n_kv_heads) * kHeadDim * (kC8 ? 1 : 2);
  bool wild = false, lost = false;
  for (long long u = static_cast<long long>(blockIdx.x) * kBoundsWarps + warp; u < units; u += static_cast<long long>(gridDim.x) * kBoundsWarps) {
    const int page = first + static_cast<int>(u / a.n_kv_heads), kvh = static_cast<int>(u % a.n_kv_heads);
    const int at = __ldg(a.pages.table + static_cast<long long>(b) * a.pages.width + page);
    if (at < 0 || at >= a.pages.n_pages) {
      lost = true;
      continue;
    }
    const int filled = min(len - (page << shift), 1 << shift);
    const long long row0 = static_cast<long long>(at) << shift;
    const unsigned char* src = static_cast<const unsigned char*>(a.k_cache) + (row0 + sub) * row_bytes + kvh * (kHeadDim * (kC8 ? 1 : 2)) + l * 16;
    const float* scales = kC8 ? a.k_scale + kvh * a.cache_rows + row0 + sub : nullptr;
    float lo[kValues], hi[kValues];
#pragma unroll
    for (int j = 0; j < kValues; ++j) {
      lo[j] = CUDART_INF_F;
      hi[j] = -CUDART_INF_F;
    }
    for (int r0 = 0; r0 < filled; r0 += kAhead * kAtOnce) {
      uint4 x[kAhead];
      float s[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int r = r0 + i * kAtOnce;  // rows behind the last: the page's first, once more
        const int take = r + sub < filled ? r : -sub;
        x[i] = __ldg(reinterpret_cast<const uint4*>(src + take * row_bytes));
        s[i] = kC8 ? __ldg(scales + take) : 1.f;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int j = 0; j < kValues / 2; ++j) {
          float2 y;
          if (kC8) {
            y = unpack_e4m3x2(w[j >> 1] >> ((j & 1) * 16));
            y.x *= s[i];
            y.y *= s[i];
          } else {
            y = unpack16<kBf>(w[j & 3]);
          }
          if (!(fabsf(y.x) < CUDART_INF_F && fabsf(y.y) < CUDART_INF_F)) {  // left out
            wild = true;
            if (fabsf(y.x) < CUDART_INF_F) {
              lo[2 * j] = fminf(lo[2 * j], y.x);
              hi[2 * j] = fmaxf(hi[2 * j], y.x);
            }
            if (fabsf(y.y) < CUDART_INF_F) {
              lo[2 * j + 1] = fminf(lo[2 * j + 1], y.y);
              hi[2 * j + 1] = fmaxf(hi[2 * j + 1], y.y);
            }
            continue;
          }
          lo[2 * j] = fminf(lo[2 * j], y.x);
          hi[2 * j] = fmaxf(hi[2 * j], y.x);
          lo[2 * j + 1] = fminf(lo[2 * j + 1], y.y);
          hi[2 * j + 1] = fmaxf(hi[2 * j + 1], y.y);
        }
      }
    }
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < kValues; ++j) {
#pragma unroll
      for (int o = kLanes; o < 32; o <<= 1) {
        lo[j] = fminf(lo[j], __shfl_xor_sync(0xffffffffu, lo[j], o));
        hi[j] = fmaxf(hi[j], __shfl_xor_sync(0xffffffffu, hi[j], o));
      }
      if (lo[j] > hi[j]) lo[j] = hi[j] = 0.f;  // no finite key
      top = fmaxf(top, fmaxf(fabsf(lo[j]), fabsf(hi[j])));
    }
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float scale = scale_of(top), inv = inverse(scale);
    if (sub < 2) {  // 0: the least, 1: the largest
      uint32_t c[kValues / 4];
#pragma unroll
      for (int j = 0; j < kValues / 4; ++j) {
        c[j] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = sub == 0 ? lo[4 * j + i] : hi[4 * j + i];  // outwards, also where the quotient is below fp32
          const float y = sub == 0 ? fminf(floorf(x * inv), x < 0.f ? -1.f : 127.f) : fmaxf(ceilf(x * inv), x > 0.f ? 1.f : -127.f);
          c[j] |= (static_cast<uint32_t>(static_cast<int>(y)) & 0xffu) << (8 * i);
        }
      }
      int8_t* out = a.bounds + ((static_cast<long long>(at) * a.n_kv_heads + kvh) * 2 + sub) * kHeadDim + l * kValues;
      if constexpr (kC8) *reinterpret_cast<uint4*>(out) = make_uint4(c[0], c[1], c[kValues / 4 - 2], c[kValues / 4 - 1]);
      else *reinterpret_cast<uint2*>(out) = make_uint2(c[0], c[1]);
    }
    if (lane == 0) a.bound_scale[static_cast<long long>(kvh) * a.pages.n_pages + at] = scale;
  }
  if (wild) set_status(a.status, kStatusRange);
  if (lost) set_status(a.status, kStatusDeviceArg);
}

// ---------------------------------------------------------------- selection

constexpr int kSelectThreads = 256;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kMaxSplit = 8;                              // CTAs of a cluster
constexpr int kMaxKeys = kMaxPagesListed / kMaxSplit;     // pages of a CTA
constexpr int kHeadTile = 4;

struct __align__(16) SelectShared {
  uint32_t hist[256];
  uint32_t sum[256];
  uint32_t counts[2][kMaxSplit];  // above the border, at it, of each CTA
  uint32_t warps[2][kSelectWarps];
  uint32_t border, above;  // of this pass: digit, keys above it
};

// order of floats as order of unsigned numbers
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A cluster a request and kv head; CTA r scores the r-th part of the pages and keeps their keys, the border is found by digits of 8
// bits over all of them, and every CTA writes what it chose behind the choices of those before it.
template <bool BF>
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const SelectArgs a) {
  extern __shared__ __align__(16) unsigned char raw_smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int split = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = a.n_heads / a.n_kv_heads;
  const int item = blockIdx.x / split, b = item / a.n_kv_heads, kvh = item - b * a.n_kv_heads;
  SelectShared& sm = *reinterpret_cast<SelectShared*>(raw_smem);
  float* q_scale = reinterpret_cast<float*>(raw_smem + sizeof(SelectShared));  // [G]
  const int tiles = (G + kHeadTile - 1) / kHeadTile;
  int8_t* q_code = reinterpret_cast<int8_t*>(q_scale + tiles * kHeadTile);  // [G][2][128]: negative part, positive part
  uint32_t* keys = reinterpret_cast<uint32_t*>(q_code + tiles * kHeadTile * 256);
  int32_t* out = a.picked + static_cast<long long>(item) * a.n_picked;
  int len, pages;
  const bool fine = rows_of(a.pages, b, len, pages);
  if (!fine && rank == 0 && tid == 0) set_status(a.status, kStatusDeviceArg);
  if (pages <= a.n_picked) {  // all of them
    if (rank == 0)
      for (int i = tid; i < a.n_picked; i += kSelectThreads) out[i] = i < pages ? i : -1;
    return;  // the whole cluster
  }
  // ---- the queries' codes; what is not finite counts as 0
  for (int h = warp; h < tiles * kHeadTile; h += kSelectWarps) {
    float x[4] = {0.f, 0.f, 0.f, 0.f}, top = 0.f;
    if (h < G) {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.q) + b * a.q_stride + (kvh * G + h) * kHeadDim) + lane);
      const float2 u = unpack16<BF>(w.x), v = unpack16<BF>(w.y);
      x[0] = u.x, x[1] = u.y, x[2] = v.x, x[3] = v.y;
    }
    bool wild = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!(fabsf(x[i]) < CUDART_INF_F)) {
        x[i] = 0.f;
        wild = true;
      }
      top = fmaxf(top, fabsf(x[i]));
    }
    if (wild && rank == 0) set_status(a.status, kStatusRange);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float scale = scale_of(top), inv = inverse(scale);
    uint32_t neg = 0, pos = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = static_cast<int>(rintf(x[i] * inv));
      neg |= (static_cast<uint32_t>(min(c, 0)) & 0xffu) << (8 * i);
      pos |= (static_cast<uint32_t>(max(c, 0)) & 0xffu) << (8 * i);
    }
    reinterpret_cast<uint32_t*>(q_code + h * 256)[lane] = neg;
    reinterpret_cast<uint32_t*>(q_code + h * 256 + 128)[lane] = pos;
    if (lane == 0) q_scale[h] = scale;
  }
  __syncthreads();
  // ---- scores: 4 lanes a page, 8 pages a warp; unit 4 i + sub of a page's 16 units of 16 bytes
  const int part = (pages + split - 1) / split, p0 = min(pages, rank * part), n = min(pages, p0 + part) - p0;
  const int sub = lane & 3;
  bool lost = false;
  for (int base = warp * 8; base < n; base += kSelectWarps * 8) {
    const int i = base + (lane >> 2), page = p0 + i;
    int at = i < n ? __ldg(a.pages.table + static_cast<long long>(b) * a.pages.width + page) : 0;
    if (at < 0 || at >= a.pages.n_pages) {
      lost = true;
      at = -1;
    }
    const long long where = static_cast<long long>(max(at, 0)) * a.n_kv_heads + kvh;
    const int4* src = reinterpret_cast<const int4*>(a.bounds + where * 256) + sub;
    int4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = __ldg(src + 4 * u);
    const float scale = __ldg(a.bound_scale + static_cast<long long>(kvh) * a.pages.n_pages + max(at, 0));
    float best = -CUDART_INF_F;
    for (int t = 0; t < tiles; ++t) {
      int acc[kHeadTile];
#pragma unroll
      for (int h = 0; h < kHeadTile; ++h) {
        acc[h] = 0;
        const int4* q = reinterpret_cast<const int4*>(q_code + (t * kHeadTile + h) * 256) + sub;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int4 y = q[4 * u];
          acc[h] = __dp4a(x[u].x, y.x, acc[h]);
          acc[h] = __dp4a(x[u].y, y.y, acc[h]);
          acc[h] = __dp4a(x[u].z, y.z, acc[h]);
          acc[h] = __dp4a(x[u].w, y.w, acc[h]);
        }
        acc[h] += __shfl_xor_sync(0xffffffffu, acc[h], 1);
        acc[h] += __shfl_xor_sync(0xffffffffu, acc[h], 2);
        if (t * kHeadTile + h < G) {
          const int e = static_cast<int>(__float_as_uint(scale) >> 23) + static_cast<int>(__float_as_uint(q_scale[t * kHeadTile + h]) >> 23) - 254;
          best = fmaxf(best, static_cast<float>(acc[h]) * __uint_as_float(static_cast<uint32_t>(127 + max(-100, min(100, e))) << 23));
        }
      }
    }
    if (i < n && sub == 0)
      keys[i] = page < a.first || page >= pages - a.last ? 0xffffffffu : at < 0 ? 0u : key_of(best);
  }
  if (lost) set_status(a.status, kStatusDeviceArg);
  // ---- the border: the n_picked-th largest key, digit by digit
  uint32_t prefix = 0, want = static_cast<uint32_t>(a.n_picked);  // digits found; keys still to take among those that share them
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    sm.hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSelectThreads) {
      const uint32_t k = keys[i];
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&sm.hist[(k >> shift) & 255u], 1u);
    }
    if (split > 1) cluster.sync();
    else __syncthreads();
    uint32_t mine = 0;
    for (int r = 0; r < split; ++r) mine += split > 1 ? *cluster.map_shared_rank(&sm.hist[tid], r) : sm.hist[tid];
    // keys in this digit and above, from the highest digit down
    uint32_t sum = mine;
    const int rev = 255 - tid;  // thread t sums digits t and above: lanes in reversed order
    sm.sum[rev] = mine;
    __syncthreads();
    sum = sm.sum[tid];
    const uint32_t own = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 31) sm.warps[0][warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += sm.warps[0][w];
    if (sum >= want && sum - own < want) {  // one thread: its digit is 255 - tid
      sm.border = 255u - tid;
      sm.above = sum - own;
    }
    if (split > 1) cluster.sync();  // and every CTA has read the others' counts
    else __syncthreads();
    prefix = prefix << 8 | sm.border;
    want -= sm.above;
  }
  // ---- every thread a run of keys; how many lie above the border and at it
  const int per = (n + kSelectThreads - 1) / kSelectThreads, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  uint32_t above = 0, at_it = 0;
  for (int i = i0; i < i1; ++i) {
    above += keys[i] > prefix;
    at_it += keys[i] == prefix;
  }
  uint32_t sa = above, sb = at_it;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t ua = __shfl_up_sync(0xffffffffu, sa, o), ub = __shfl_up_sync(0xffffffffu, sb, o);
    if (lane >= o) {
      sa += ua;
      sb += ub;
    }
  }
  if (lane == 31) {
    sm.warps[0][warp] = sa;
    sm.warps[1][warp] = sb;
  }
  __syncthreads();
  for (int w = 0; w < warp; ++w) {
    sa += sm.warps[0][w];
    sb += sm.warps[1][w];
  }
  if (split > 1) {
    if (tid == kSelectThreads - 1)
      for (int r = 0; r < split; ++r) {
        *cluster.map_shared_rank(&sm.counts[0][rank], r) = sa;
        *cluster.map_shared_rank(&sm.counts[1][rank], r) = sb;
      }
    cluster.sync();
    for (int r = 0; r < rank; ++r) {
      sa += sm.counts[0][r];
      sb += sm.counts[1][r];
    }
  }
  uint32_t before = sa - above, equal = sb - at_it;
  for (int i = i0; i < i1; ++i) {
    if (keys[i] > prefix) {
      out[before + min(equal, want)] = p0 + i;
      ++before;
    } else if (keys[i] == prefix) {
      if (equal < want) out[before + equal] = p0 + i;
      ++equal;
    }
  }
}

}  // namespace

cudaError_t launch_page_bounds(const BoundsArgs& a, int cache_dtype, cudaStream_t stream) {
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  // warps for the whole GPU over all requests, and no more than a request's pages can have
  const long long most = (static_cast<long long>(a.pages.width) * a.n_kv_heads + kBoundsWarps - 1) / kBoundsWarps;
  const long long want = (static_cast<long long>(sms) * 8 + a.pages.B - 1) / a.pages.B;
  const unsigned x = static_cast<unsigned>(want < most ? want : most);
  if (x == 0) return cudaSuccess;
  void* args[] = {const_cast<BoundsArgs*>(&a)};
  const void* fn = cache_dtype == FSX_E4M3   ? reinterpret_cast<const void*>(&bounds_kernel<FSX_E4M3>)
                   : cache_dtype == FSX_BF16 ? reinterpret_cast<const void*>(&bounds_kernel<FSX_BF16>)
                                             : reinterpret_cast<const void*>(&bounds_kernel<FSX_F16>);
  return launch_ex(fn, dim3(x, static_cast<unsigned>(a.pages.B)), dim3(32 * kBoundsWarps), 0, stream, false, args);
}

cudaError_t launch_page_select(const SelectArgs& a, int dtype, cudaStream_t stream) {
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  const long long items = static_cast<long long>(a.pages.B) * a.n_kv_heads;
  int split = 1;  // CTAs an item: while they leave SMs idle and have 64 pages and more each; no more pages a CTA than it keeps
  while (split < kMaxSplit && ((items * split < sms && a.pages.width > 64 * split) || a.pages.width > kMaxKeys * split)) split *= 2;
  const int G = a.n_heads / a.n_kv_heads, tiles = (G + kHeadTile - 1) / kHeadTile;
  const size_t smem = sizeof(SelectShared) + static_cast<size_t>(tiles) * kHeadTile * (256 + sizeof(float)) +
                      static_cast<size_t>((a.pages.width + split - 1) / split) * sizeof(uint32_t);
  const void* fn = dtype == FSX_BF16 ? reinterpret_cast<const void*>(&select_kernel<true>) : reinterpret_cast<const void*>(&select_kernel<false>);
  const cudaError_t e = allow_shared_memory(fn, smem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<SelectArgs*>(&a)};
  return launch_ex(fn, dim3(static_cast<unsigned>(items * split)), dim3(kSelectThreads), smem, stream, false, args, 1, split);
}

}  // namespace fsx
