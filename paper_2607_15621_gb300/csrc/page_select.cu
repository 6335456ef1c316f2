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
//
// Measured: bounds of 3,117 pages of 32 rows, 8 heads, bf16, 36 us (5.9 TB/s, 0.86 of a copy's rate; DRAM 70 % busy), of codes 37 us,
// the newest page of 16 requests 3.5 us; 64 of up to 1024 pages for 16 requests and 8 kv heads 11.1 us, 96 of 2047 for one request 8.5 us.
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

// Least and largest of packed 16-bit values; a NaN stays
template <bool BF>
__device__ __forceinline__ void bound2(uint32_t& lo, uint32_t& hi, uint32_t low, uint32_t high) {
  if (BF) {
    asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(lo) : "r"(low));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(hi) : "r"(high));
  } else {
    asm("min.NaN.f16x2 %0, %0, %1;" : "+r"(lo) : "r"(low));
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(hi) : "r"(high));
  }
}

// Ends of a lane's values over rows from, from + step, ... below `filled` of a page, kAhead of them loaded at once; `src`, `scales`: at the
// lane's own row `sub` of the first. CAREFUL: values that are not finite change neither end, and are reported; else they
// show in the ends (16 bits: NaN and infinities; codes: infinities, and NaN codes by `wild`).
template <int TYPE, int AHEAD, bool CAREFUL>
struct Ends {
  static constexpr bool kC8 = TYPE == FSX_E4M3, kBf = TYPE == FSX_BF16;
  static constexpr int kLanes = kC8 ? 8 : 16, kValues = kHeadDim / kLanes, kAtOnce = 32 / kLanes;
  static __device__ __forceinline__ void scan(const unsigned char* src, const float* scales, long long row_bytes, int sub, int from, int step, int filled,
                                              float (&lo)[kValues], float (&hi)[kValues], bool& wild) {
    constexpr uint32_t kInf = kBf ? 0x7f807f80u : 0x7c007c00u;
    uint32_t lo2[4], hi2[4];
    if constexpr (kC8) {
#pragma unroll
      for (int j = 0; j < kValues; ++j) {
        lo[j] = CUDART_INF_F;
        hi[j] = -CUDART_INF_F;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo2[j] = kInf;
        hi2[j] = kInf | 0x80008000u;
      }
    }
#pragma unroll 1
    for (int r0 = from; r0 < filled; r0 += AHEAD * step) {
      uint4 x[AHEAD];
      float s[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int r = r0 + i * step;  // rows behind the last: the page's first, once more
        const int take = r + sub < filled ? r : -sub;
        x[i] = *reinterpret_cast<const uint4*>(src + take * row_bytes);
        s[i] = kC8 ? scales[take] : 1.f;
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        if constexpr (!kC8) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t low = w[j], high = w[j];
            if (CAREFUL) {
              const uint32_t bad = not_finite2<kBf>(w[j]), mask = (bad >> 15) * 0xffffu;
              wild = wild || bad != 0u;
              low = (w[j] & ~mask) | (kInf & mask);
              high = (w[j] & ~mask) | ((kInf | 0x80008000u) & mask);
            }
            bound2<kBf>(lo2[j], hi2[j], low, high);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            wild = wild || (((w[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0u;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              float2 y = unpack_e4m3x2(w[j] >> (t * 16));
              y.x *= s[i];
              y.y *= s[i];
              float2 z = y;
              if (CAREFUL) {
                const bool bad_x = !(fabsf(y.x) < CUDART_INF_F), bad_y = !(fabsf(y.y) < CUDART_INF_F);
                wild = wild || bad_x || bad_y;
                if (bad_x) y.x = CUDART_INF_F, z.x = -CUDART_INF_F;
                if (bad_y) y.y = CUDART_INF_F, z.y = -CUDART_INF_F;
              }
              const int v = 4 * j + 2 * t;
              lo[v] = fminf(lo[v], y.x);
              hi[v] = fmaxf(hi[v], z.x);
              lo[v + 1] = fminf(lo[v + 1], y.y);
              hi[v + 1] = fmaxf(hi[v + 1], z.y);
            }
          }
        }
      }
    }
    if constexpr (!kC8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bound2<kBf>(lo2[j], hi2[j], __shfl_xor_sync(0xffffffffu, lo2[j], 16), __shfl_xor_sync(0xffffffffu, hi2[j], 16));
        const float2 x = unpack16<kBf>(lo2[j]), y = unpack16<kBf>(hi2[j]);
        lo[2 * j] = x.x, lo[2 * j + 1] = x.y, hi[2 * j] = y.x, hi[2 * j + 1] = y.y;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kValues; ++j)
#pragma unroll
        for (int o = kLanes; o < 32; o <<= 1) {
          lo[j] = fminf(lo[j], __shfl_xor_sync(0xffffffffu, lo[j], o));
          hi[j] = fmaxf(hi[j], __shfl_xor_sync(0xffffffffu, hi[j], o));
        }
    }
  }
};

// The same of rows of codes whose scales are powers of two within 2^14 of one another: a code times its scale over the largest so far is
// exact in fp16 (a code's last bit is 2^-9, fp16's 2^-24), so that two values are scaled and compared at once. In fp32 it takes
// 2.5 times the instructions (131,000 rows of 8 heads 57 us, of which all but 17 for them). A NaN code shows in the ends. False:
// the scales are not like that.
template <int AHEAD>
__device__ __forceinline__ bool scan_plain(const unsigned char* src, const float* scales, long long row_bytes, int sub, int from, int step, int filled,
                                           float (&lo)[16], float (&hi)[16]) {
  uint32_t lo2[8], hi2[8], top = 0, low = 0xffffffffu, all = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo2[j] = 0x7c007c00u;
    hi2[j] = 0xfc00fc00u;
  }
#pragma unroll 1
  for (int r0 = from; r0 < filled; r0 += AHEAD * step) {
    uint4 x[AHEAD];
    uint32_t s[AHEAD], most = 0, least = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int r = r0 + i * step;  // rows behind the last: the page's first, once more
      const int take = r + sub < filled ? r : -sub;
      x[i] = *reinterpret_cast<const uint4*>(src + take * row_bytes);
      s[i] = __float_as_uint(scales[take]);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      most = max(most, s[i]);
      least = min(least, s[i]);
      all |= s[i];
    }
    most = __reduce_max_sync(0xffffffffu, most);
    low = min(low, __reduce_min_sync(0xffffffffu, least));
    if (most > top) {  // the ends so far, in the new unit
      const uint32_t d = top == 0 ? 0u : (most - top) >> 23, q = d < 15u ? (15u - d) << 10 : 0u, q2 = q | q << 16;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (top != 0) {
          const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&lo2[j]), *reinterpret_cast<const __half2*>(&q2));
          const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&hi2[j]), *reinterpret_cast<const __half2*>(&q2));
          lo2[j] = *reinterpret_cast<const uint32_t*>(&y);
          hi2[j] = *reinterpret_cast<const uint32_t*>(&z);
        }
      top = most;
    }
    if (top - low > 14u << 23) return false;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      const uint32_t q = (15u - ((top - s[i]) >> 23)) << 10, q2 = q | q << 16;  // the quotient, 2^0 to 2^-14
      const __half2 f = *reinterpret_cast<const __half2*>(&q2);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t y;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(static_cast<uint16_t>(w[j >> 1] >> ((j & 1) * 16))));
        const __half2 z = __hmul2(*reinterpret_cast<const __half2*>(&y), f);
        y = *reinterpret_cast<const uint32_t*>(&z);
        bound2<false>(lo2[j], hi2[j], y, y);
      }
    }
  }
  if (__any_sync(0xffffffffu, (all & 0x807fffffu) != 0u) || top >= 0x7f800000u || low == 0u) return false;
  const float unit = __uint_as_float(top);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int o = 8; o < 32; o <<= 1)
      bound2<false>(lo2[j], hi2[j], __shfl_xor_sync(0xffffffffu, lo2[j], o), __shfl_xor_sync(0xffffffffu, hi2[j], o));
    const float2 x = unpack16<false>(lo2[j]), y = unpack16<false>(hi2[j]);
    lo[2 * j] = x.x * unit, lo[2 * j + 1] = x.y * unit, hi[2 * j] = y.x * unit, hi[2 * j + 1] = y.y * unit;
  }
  return true;
}

// `share` warps a page and kv head, 1 or 8: 8 where pages are few (those that new rows went into), for a shorter chain.
// 16 lanes a row of 16-bit keys (two rows at once), 8 lanes a row of codes (four).
template <int TYPE, int SHARE>
__global__ void __launch_bounds__(32 * kBoundsWarps, TYPE == FSX_E4M3 ? 3 : 4) bounds_kernel(const BoundsArgs a) {
  constexpr bool kC8 = TYPE == FSX_E4M3, kBf = TYPE == FSX_BF16;
  constexpr int kLanes = kC8 ? 8 : 16, kValues = kHeadDim / kLanes, kAtOnce = 32 / kLanes;
  constexpr int kAhead = SHARE > 1 ? 2 : 8;
  __shared__ float part[SHARE > 1 ? kBoundsWarps : 1][2][kHeadDim];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % kLanes, sub = lane / kLanes;
  const int b = blockIdx.y;
  pdl_launch_dependents();
  pdl_wait();
  int len, pages;
  const long long start = a.start != nullptr ? a.start[b] : 0;
  const bool fine = rows_of(a.pages, b, len, pages);
  if (!fine || start < 0) {
    if (blockIdx.x == 0 && threadIdx.x == 0) set_status(a.status, kStatusDeviceArg);
    return;
  }
  const int shift = a.pages.shift;
  const int first = start >= len ? pages : static_cast<int>(start >> shift);
  const uint32_t units = static_cast<uint32_t>(pages - first) * a.n_kv_heads;  // below 2^31: see the host
  const long long row_bytes = static_cast<long long>(a.n_kv_heads) * kHeadDim * (kC8 ? 1 : 2);
  const uint32_t stride = gridDim.x * (kBoundsWarps / SHARE);
  bool wild = false, lost = false;
  const int32_t* const table = a.pages.table + static_cast<long long>(b) * a.pages.width + first;
  uint32_t u = blockIdx.x * (kBoundsWarps / SHARE) + (SHARE > 1 ? 0 : warp);
  int ahead = u < units ? table[u / a.n_kv_heads] : 0;
  for (; u < units; u += stride) {
    const uint32_t nth = u / a.n_kv_heads;
    const int page = first + static_cast<int>(nth), kvh = static_cast<int>(u - nth * a.n_kv_heads), at = ahead;
    if (u + stride < units) ahead = table[(u + stride) / a.n_kv_heads];
    if (at < 0 || at >= a.pages.n_pages) {
      lost = true;
      continue;  // the same for all of the unit's warps
    }
    const int filled = min(len - (page << shift), 1 << shift);
    const long long row0 = static_cast<long long>(at) << shift;
    const unsigned char* src = static_cast<const unsigned char*>(a.k_cache) + (row0 + sub) * row_bytes + kvh * (kHeadDim * (kC8 ? 1 : 2)) + l * 16;
    const float* scales = kC8 ? a.k_scale + kvh * a.cache_rows + row0 + sub : nullptr;
    float lo[kValues], hi[kValues];
    const int from = SHARE > 1 ? warp * kAtOnce : 0;
    bool plain = false;
    if constexpr (kC8) plain = scan_plain<kAhead>(src, scales, row_bytes, sub, from, kAtOnce * SHARE, filled, lo, hi);
    if (!plain) Ends<TYPE, kC8 ? 1 : kAhead, kC8>::scan(src, scales, row_bytes, sub, from, kAtOnce * SHARE, filled, lo, hi, wild);
    bool bad = false;  // an end that is not finite; of a warp without rows both are infinite
#pragma unroll
    for (int j = 0; j < kValues; ++j) bad = bad || !(fabsf(lo[j]) < CUDART_INF_F) || !(fabsf(hi[j]) < CUDART_INF_F);
    if (__any_sync(0xffffffffu, bad) && from < filled) Ends<TYPE, 1, true>::scan(src, scales, row_bytes, sub, from, kAtOnce * SHARE, filled, lo, hi, wild);
    if constexpr (SHARE > 1) {  // the warps' ends, by the first warp
      if (sub == 0) {
#pragma unroll
        for (int j = 0; j < kValues / 4; ++j) {
          reinterpret_cast<float4*>(&part[warp][0][l * kValues])[j] = make_float4(lo[4 * j], lo[4 * j + 1], lo[4 * j + 2], lo[4 * j + 3]);
          reinterpret_cast<float4*>(&part[warp][1][l * kValues])[j] = make_float4(hi[4 * j], hi[4 * j + 1], hi[4 * j + 2], hi[4 * j + 3]);
        }
      }
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int w = 1; w < kBoundsWarps; ++w)
#pragma unroll
          for (int j = 0; j < kValues / 4; ++j) {
            const float4 x = reinterpret_cast<const float4*>(&part[w][0][l * kValues])[j], y = reinterpret_cast<const float4*>(&part[w][1][l * kValues])[j];
            lo[4 * j] = fminf(lo[4 * j], x.x), lo[4 * j + 1] = fminf(lo[4 * j + 1], x.y);
            lo[4 * j + 2] = fminf(lo[4 * j + 2], x.z), lo[4 * j + 3] = fminf(lo[4 * j + 3], x.w);
            hi[4 * j] = fmaxf(hi[4 * j], y.x), hi[4 * j + 1] = fmaxf(hi[4 * j + 1], y.y);
            hi[4 * j + 2] = fmaxf(hi[4 * j + 2], y.z), hi[4 * j + 3] = fmaxf(hi[4 * j + 3], y.w);
          }
      }
      __syncthreads();
      if (warp != 0) continue;
    }
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < kValues; ++j) {
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

constexpr int kSelectThreads = 512;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kMaxSplit = 8;  // CTAs of a cluster
constexpr int kHeadTile = 4;
// CTAs a SM, and pages of a CTA, from which on an item is not split further (128 items of up to 1024 pages: 11.4 us, split for 2 CTAs a SM 15.1)
constexpr int kIdle = 1, kFewPages = 128;
constexpr int kAtOnce = 2;  // times 8 pages of a warp
constexpr int kDigit = 11, kBins = 1 << kDigit, kPerThread = kBins / kSelectThreads;

constexpr uint32_t kFewKeys = 256;  // at the border, which are compared with one another

struct __align__(16) SelectShared {
  uint32_t hist[kBins];  // and the keys at the border
  uint32_t least[kMaxSplit * kSelectWarps], most[kMaxSplit * kSelectWarps];  // keys that the warps of all CTAs have found
  uint32_t warps[2][kSelectWarps];
  uint32_t border, above, at_it;  // of a pass: digit, keys above it, keys at it
  uint32_t gathered;
};

// order of floats as order of unsigned numbers
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A cluster a request and kv head: its CTAs score a part of the pages each and store the keys in the first CTA's shared
// memory, which then finds the border alone, by digits of 11 bits counted from the lowest key, and writes the pages above it.
template <bool BF>
__global__ void __launch_bounds__(kSelectThreads, 2) select_kernel(const SelectArgs a) {
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
  pdl_launch_dependents();
  pdl_wait();
  int len, pages;
  const bool fine = rows_of(a.pages, b, len, pages);
  if (!fine && rank == 0 && tid == 0) set_status(a.status, kStatusDeviceArg);
  if (pages <= a.n_picked) {  // all of them
    if (rank == 0)
      for (int i = tid; i < a.n_picked; i += kSelectThreads) out[i] = i < pages ? i : -1;
    return;  // the whole cluster
  }
  if (split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // this CTA runs
  const int part = (pages + split - 1) / split, p0 = min(pages, rank * part), n = min(pages, p0 + part) - p0;
  bool lost = false;
  for (int i = tid; i < n; i += kSelectThreads) {  // where the pages are, in the keys' place
    const int at = a.pages.table[static_cast<long long>(b) * a.pages.width + p0 + i];
    const bool there = at >= 0 && at < a.pages.n_pages;
    lost = lost || !there;
    keys[i] = there ? static_cast<uint32_t>(at) : 0xffffffffu;
  }
  if (rank == 0) {
    for (int i = tid; i < kBins; i += kSelectThreads) sm.hist[i] = 0;
    if (tid == 0) sm.gathered = 0;
  }
  if (lost) set_status(a.status, kStatusDeviceArg);
  // ---- the queries' codes; what is not finite counts as 0
  for (int h = warp; h < tiles * kHeadTile; h += kSelectWarps) {
    float x[4] = {0.f, 0.f, 0.f, 0.f}, top = 0.f;
    if (h < G) {
      const uint2 w = *(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.q) + b * a.q_stride + (kvh * G + h) * kHeadDim) + lane);
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
  if (split > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // every CTA of the cluster runs
  uint32_t* const all_keys = split > 1 ? cluster.map_shared_rank(keys, 0) : keys;
  // ---- scores: 4 lanes a page, 8 pages a warp, kAtOnce times; unit 4 u + sub of a page's 16 units of 16 bytes
  const int sub = lane & 3;
  const int p_first = a.first, p_last = pages - a.last;  // the pages that are not taken anyway
  uint32_t least = 0xffffffffu, most = 0;                // keys of theirs
  for (int base = warp * (8 * kAtOnce); base < n; base += kSelectWarps * (8 * kAtOnce)) {
    int4 x[kAtOnce][4];
    float scale[kAtOnce], best[kAtOnce];
#pragma unroll
    for (int t = 0; t < kAtOnce; ++t) {
      const int i = base + 8 * t + (lane >> 2);
      const uint32_t at = i < n ? keys[i] : 0u;
      const long long page = at == 0xffffffffu ? 0 : at;
      const int4* src = reinterpret_cast<const int4*>(a.bounds + (page * a.n_kv_heads + kvh) * 256) + sub;
#pragma unroll
      for (int u = 0; u < 4; ++u) x[t][u] = src[4 * u];
      scale[t] = a.bound_scale[static_cast<long long>(kvh) * a.pages.n_pages + page];
      best[t] = -CUDART_INF_F;
    }
    for (int head = 0; head < tiles * kHeadTile; head += kHeadTile) {
      int acc[kAtOnce][kHeadTile];
#pragma unroll
      for (int h = 0; h < kHeadTile; ++h) {
        const int4* q = reinterpret_cast<const int4*>(q_code + (head + h) * 256) + sub;
#pragma unroll
        for (int t = 0; t < kAtOnce; ++t) acc[t][h] = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int4 y = q[4 * u];
#pragma unroll
          for (int t = 0; t < kAtOnce; ++t) {
            acc[t][h] = __dp4a(x[t][u].x, y.x, acc[t][h]);
            acc[t][h] = __dp4a(x[t][u].y, y.y, acc[t][h]);
            acc[t][h] = __dp4a(x[t][u].z, y.z, acc[t][h]);
            acc[t][h] = __dp4a(x[t][u].w, y.w, acc[t][h]);
          }
        }
      }
      // sums over the 4 lanes; lane `sub` ends with that of head `sub`
      const int e_q = static_cast<int>(__float_as_uint(q_scale[head + sub]) >> 23) - 254;
#pragma unroll
      for (int t = 0; t < kAtOnce; ++t) {
        const bool up = sub & 1, high = sub & 2;
        int s0 = up ? acc[t][1] : acc[t][0], s1 = up ? acc[t][3] : acc[t][2];
        s0 += __shfl_xor_sync(0xffffffffu, up ? acc[t][0] : acc[t][1], 1);
        s1 += __shfl_xor_sync(0xffffffffu, up ? acc[t][2] : acc[t][3], 1);
        const int sum = (high ? s1 : s0) + __shfl_xor_sync(0xffffffffu, high ? s0 : s1, 2);
        const int e = max(-100, min(100, e_q + static_cast<int>(__float_as_uint(scale[t]) >> 23)));
        if (head + sub < G) best[t] = fmaxf(best[t], static_cast<float>(sum) * __uint_as_float(static_cast<uint32_t>(127 + e) << 23));
      }
    }
#pragma unroll
    for (int t = 0; t < kAtOnce; ++t) {
      best[t] = fmaxf(best[t], __shfl_xor_sync(0xffffffffu, best[t], 1));
      best[t] = fmaxf(best[t], __shfl_xor_sync(0xffffffffu, best[t], 2));
      const int i = base + 8 * t + (lane >> 2);
      if (i < n && sub == 0) {
        const uint32_t key = keys[i] == 0xffffffffu ? 0u : key_of(best[t]);
        all_keys[p0 + i] = key;
        if (p0 + i >= p_first && p0 + i < p_last) {
          least = min(least, key);
          most = max(most, key);
        }
      }
    }
  }
  least = __reduce_min_sync(0xffffffffu, least);
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) {
    SelectShared* const to = split > 1 ? cluster.map_shared_rank(&sm, 0) : &sm;
    to->least[rank * kSelectWarps + warp] = least;
    to->most[rank * kSelectWarps + warp] = most;
  }
  if (split > 1) cluster.sync();  // the keys are in the first CTA; nothing is read from the others
  else __syncthreads();
  if (rank != 0) return;
  // ---- the border among the pages that are not taken anyway: the want-th largest key
  uint32_t want = static_cast<uint32_t>(a.n_picked - a.first - a.last);
  for (int w = lane; w < split * kSelectWarps; w += 32) {
    least = min(least, sm.least[w]);
    most = max(most, sm.most[w]);
  }
  least = __reduce_min_sync(0xffffffffu, least);
  most = __reduce_max_sync(0xffffffffu, most);
  // (key - least) >> shift: above `border` taken, at it the first `want` ones
  uint32_t border = 0;
  int shift = 32 - __clz(most - least);
  bool whole = want == 0;
  if (whole) border = 0xffffffffu, shift = 0;  // no key - least is as large: scores are finite
  for (bool first = true; !whole && shift > 0; first = false) {
    const int width = min(kDigit, shift), below = shift;
    shift -= width;
    if (!first) {
      for (int i = tid; i < kBins; i += kSelectThreads) sm.hist[i] = 0;
      __syncthreads();
    }
    for (int i = p_first + tid; i < p_last; i += kSelectThreads) {
      const uint32_t k = keys[i] - least;
      if (first || (k >> below) == border) atomicAdd(&sm.hist[(k >> shift) & ((1u << width) - 1)], 1u);
    }
    __syncthreads();
    uint32_t mine[kPerThread], own = 0;  // thread t counts kPerThread digits, from the highest down
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) own += mine[i] = sm.hist[kBins - 1 - (tid * kPerThread + i)];
    uint32_t sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += up;
    }
    if (lane == 31) sm.warps[0][warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += sm.warps[0][w];
    uint32_t above = sum - own;
    if (sum >= want && above < want) {  // one thread
#pragma unroll
      for (int i = 0; i < kPerThread; ++i) {
        if (above < want && above + mine[i] >= want) {
          sm.border = static_cast<uint32_t>(kBins - 1 - (tid * kPerThread + i));
          sm.above = above;
          sm.at_it = mine[i];
          above = want;
        } else {
          above += mine[i];
        }
      }
    }
    __syncthreads();
    border = (first ? 0u : border << width) | sm.border;
    want -= sm.above;
    const uint32_t at_border = sm.at_it;
    whole = at_border == want;
    if (!whole && shift > 0 && at_border <= kFewKeys) {  // a handful as a rule: each is compared with all
      for (int i = p_first + tid; i < p_last; i += kSelectThreads) {
        const uint32_t k = keys[i] - least;
        if ((k >> shift) == border) sm.hist[atomicAdd(&sm.gathered, 1u)] = k;
      }
      __syncthreads();
      if (tid < at_border) {
        const uint32_t own_key = sm.hist[tid];
        uint32_t larger = 0, equal_too = 0;
        for (uint32_t i = 0; i < at_border; ++i) {
          larger += sm.hist[i] > own_key;
          equal_too += sm.hist[i] >= own_key;
        }
        if (larger < want && equal_too >= want) {  // equal keys write the same
          sm.border = own_key;
          sm.above = larger;
        }
      }
      __syncthreads();
      border = sm.border;
      want -= sm.above;
      shift = 0;
    }
  }
  // ---- every thread a run of pages; how many lie above the border and at it
  const int per = (pages + kSelectThreads - 1) / kSelectThreads, i0 = min(pages, tid * per), i1 = min(pages, i0 + per);
  auto rank_of = [&](int i) {  // 2: above, 1: at the border
    if (i < p_first || i >= p_last) return 2;
    const uint32_t k = (keys[i] - least) >> shift;
    return k > border ? 2 : k == border ? 1 : 0;
  };
  uint32_t above = 0, at_it = 0;
  for (int i = i0; i < i1; ++i) {
    const int r = rank_of(i);
    above += r == 2;
    at_it += r == 1;
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
  uint32_t before = sa - above, equal = sb - at_it;
  for (int i = i0; i < i1; ++i) {
    const int r = rank_of(i);
    if (r == 2) {
      out[before + min(equal, want)] = i;
      ++before;
    } else if (r == 1) {
      if (equal < want) out[before + equal] = i;
      ++equal;
    }
  }
}

}  // namespace

template <int SHARE>
static const void* bounds_of(int cache_dtype) {
  return cache_dtype == FSX_E4M3   ? reinterpret_cast<const void*>(&bounds_kernel<FSX_E4M3, SHARE>)
         : cache_dtype == FSX_BF16 ? reinterpret_cast<const void*>(&bounds_kernel<FSX_BF16, SHARE>)
                                   : reinterpret_cast<const void*>(&bounds_kernel<FSX_F16, SHARE>);
}

cudaError_t launch_page_bounds(const BoundsArgs& a, int cache_dtype, cudaStream_t stream) {
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  // With a start, pages are few: the ones that new rows went into (16 of 32 rows, 8 heads: 3.5 us, with a warp a page 5.6). Without, twice as many warps as run at once over all requests, and no
  // more than a request's pages can have.
  const bool few = a.start != nullptr;
  const int each = few ? 1 : kBoundsWarps;
  const long long most = (static_cast<long long>(a.pages.width) * a.n_kv_heads + each - 1) / each;
  const long long want = (static_cast<long long>(sms) * (few ? 8 : 16) + a.pages.B - 1) / a.pages.B;
  const unsigned x = static_cast<unsigned>(want < most ? want : most);
  void* args[] = {const_cast<BoundsArgs*>(&a)};
  return launch_ex(few ? bounds_of<kBoundsWarps>(cache_dtype) : bounds_of<1>(cache_dtype), dim3(x, static_cast<unsigned>(a.pages.B)), dim3(32 * kBoundsWarps),
                   0, stream, true, args);
}

cudaError_t launch_page_select(const SelectArgs& a, int dtype, cudaStream_t stream) {
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  const long long items = static_cast<long long>(a.pages.B) * a.n_kv_heads;
  int split = 1;  // CTAs an item: while SMs are left and each has 128 pages and more
  while (split < kMaxSplit && items * split < sms * kIdle && a.pages.width > kFewPages * split) split *= 2;
  const int G = a.n_heads / a.n_kv_heads, tiles = (G + kHeadTile - 1) / kHeadTile;
  const size_t smem = sizeof(SelectShared) + static_cast<size_t>(tiles) * kHeadTile * (256 + sizeof(float)) +
                      static_cast<size_t>(a.pages.width) * sizeof(uint32_t);
  const void* fn = dtype == FSX_BF16 ? reinterpret_cast<const void*>(&select_kernel<true>) : reinterpret_cast<const void*>(&select_kernel<false>);
  const cudaError_t e = allow_shared_memory(fn, smem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<SelectArgs*>(&a)};
  return launch_ex(fn, dim3(static_cast<unsigned>(items * split)), dim3(kSelectThreads), smem, stream, true, args, 1, split);
}

}  // namespace fsx
