// The 8-bit cache: rows of keys and values quantised to e4m3 as they are written, and read back.
//
// Per row and kv head: s = 2^e, the smallest power of two with max|x| / s <= 448 (e >= -126), code =
// e4m3(x / s), value = s code. A power of two makes x / s exact, so the code is x rounded once; against
// the scale max|x| / 448 it costs nothing in precision, since e4m3 keeps its relative step over the
// range (only values 2^-14 of the maximum meet subnormals a bit earlier).
// Scales lie as [head, row]: the attention of one head reads them along the rows.
// Codes and scales of a row are stored by several lanes, and the rows of a call by warps in no order, so that destinations have
// to be distinct: to order writers of one row would take a pass over the row numbers ahead of this one, as long as a small
// write itself.
//
// Both kernels are bound by memory: 16 lanes hold a row of a head (8 values each, 16-byte loads or
// stores of the 16-bit side, 8 bytes of codes), a warp takes 8 consecutive rows, all loads issued
// before the first use, so that a resident SM has 64 KB or more in flight. Measured: 28,001 rows of 32 heads from fp32
// 189 us (6.1 TB/s, 0.90 of a copy's rate; DRAM 75 % busy), 50,000 rows back to bf16 199 us (6.25 TB/s, 0.92); 4 rows
// 2.5 us, a launch.
#include <cuda_fp8.h>

#include "device_util.cuh"
#include "fsx.h"
#include "kernels.h"
#include "llm.h"

namespace fsx {

namespace {

constexpr int kWarpRows = 8;      // rows of one head a warp works on
constexpr int kThreads = 128;
constexpr int kPerLane = kWarpRows / 2;  // rows per half-warp

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&x)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void load8<__half>(const __half* p, float (&x)[8]) {
  const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(__half* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_half2(x[0], x[1]), pack_half2(x[2], x[3]), pack_half2(x[4], x[5]), pack_half2(x[6], x[7]));
}

__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack_e4m3x2(uint32_t v) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(v)));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// Warp w of the grid: unit w of (row group, tensor, head), heads fastest, so that neighbouring warps
// touch neighbouring bytes of a row.
struct Unit {
  long long row0;
  int head;
  bool is_v, any;
};
__device__ __forceinline__ Unit unit_of(const Cache8Args& a) {
  const long long w = static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
  const int per_group = 2 * a.n_kv_heads;
  const long long group = w / per_group;
  const int rest = static_cast<int>(w - group * per_group);
  return Unit{group * kWarpRows, rest % a.n_kv_heads, rest >= a.n_kv_heads, group * kWarpRows < a.n_rows};
}

// the cache row of each of this half-warp's rows, -1: none
__device__ __forceinline__ void cache_rows_of(const Cache8Args& a, long long row0, int half, long long (&at)[kPerLane]) {
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const long long r = row0 + 2 * i + half;
    at[i] = -1;
    if (r < a.n_rows) {
      const long long c = a.rows != nullptr ? __ldg(reinterpret_cast<const long long*>(a.rows) + r) : r;
      if (c >= 0 && c < a.cache_rows) at[i] = c;
      else set_status(a.status, kStatusDeviceArg);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const Cache8Args a) {
  const Unit u = unit_of(a);
  if (!u.any) return;  // the whole warp
  const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15;
  const T* src = static_cast<const T*>(u.is_v ? a.v : a.k) + u.head * kHeadDim + l * 8;
  long long at[kPerLane];
  cache_rows_of(a, u.row0, half, at);
  float x[kPerLane][8];
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    if (at[i] >= 0) {
      load8<T>(src + (u.row0 + 2 * i + half) * a.kv_stride, x[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    }
  }
  unsigned char* codes = static_cast<unsigned char*>(u.is_v ? a.v_cache : a.k_cache);
  float* scales = (u.is_v ? a.v_scale : a.k_scale) + u.head * a.cache_rows;
  bool wild = false;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    uint32_t top = 0;  // bits of the largest finite magnitude
    bool mine = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t m = __float_as_uint(x[i][j]) & 0x7fffffffu;
      if (m < 0x7f800000u) top = max(top, m);
      else mine = true;
    }
    wild = wild || mine;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    // top = f 2^E, 1 <= f < 2 (below: E = -127, a subnormal): 2^(E - 8) holds f <= 1.75
    int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = max(e, -126);
    const bool zero = top == 0;
    const float scale = zero ? 1.f : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
    const float inv = zero ? 1.f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = pack_e4m3x2(x[i][2 * j] * inv, x[i][2 * j + 1] * inv);
    if (mine) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if ((__float_as_uint(x[i][j]) & 0x7fffffffu) >= 0x7f800000u) c[j >> 1] |= 0x7fu << ((j & 1) * 8);
    }
    if (at[i] >= 0) {
      *reinterpret_cast<uint2*>(codes + (at[i] * a.n_kv_heads + u.head) * kHeadDim + l * 8) =
          make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
      if (l == 0) scales[at[i]] = scale;
    }
  }
  if (wild) set_status(a.status, kStatusRange);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const Cache8Args a) {
  const Unit u = unit_of(a);
  if (!u.any) return;
  const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15;
  T* dst = static_cast<T*>(const_cast<void*>(u.is_v ? a.v : a.k)) + u.head * kHeadDim + l * 8;
  const unsigned char* codes = static_cast<const unsigned char*>(u.is_v ? a.v_cache : a.k_cache);
  const float* scales = (u.is_v ? a.v_scale : a.k_scale) + u.head * a.cache_rows;
  long long at[kPerLane];
  cache_rows_of(a, u.row0, half, at);
  uint2 c[kPerLane];
  float s[kPerLane];
#pragma unroll
  for (int i = 0; i < kPerLane; ++i)
    if (at[i] >= 0) {
      c[i] = __ldg(reinterpret_cast<const uint2*>(codes + (at[i] * a.n_kv_heads + u.head) * kHeadDim + l * 8));
      s[i] = __ldg(scales + at[i]);
    }
#pragma unroll
  for (int i = 0; i < kPerLane; ++i)
    if (at[i] >= 0) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = unpack_e4m3x2((j < 2 ? c[i].x : c[i].y) >> ((j & 1) * 16));
        x[2 * j] = f.x * s[i];
        x[2 * j + 1] = f.y * s[i];
      }
      store8(dst + (u.row0 + 2 * i + half) * a.kv_stride, x);
    }
}

unsigned blocks_of(const Cache8Args& a) {  // n_rows < 2^31 and at most 4096 heads: below 2^42 / 2^5 units
  const long long warps = (a.n_rows + kWarpRows - 1) / kWarpRows * 2 * a.n_kv_heads;
  const long long blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
  return blocks > 0x7fffffffll ? 0u : static_cast<unsigned>(blocks);
}

}  // namespace

cudaError_t launch_cache_write(const Cache8Args& a, cudaStream_t stream) {
  const unsigned blocks = blocks_of(a);
  if (blocks == 0) return cudaErrorInvalidConfiguration;
  void* args[] = {const_cast<Cache8Args*>(&a)};
  const void* fn = a.dtype == FSX_F32    ? reinterpret_cast<const void*>(&cache_write_kernel<float>)
                   : a.dtype == FSX_BF16 ? reinterpret_cast<const void*>(&cache_write_kernel<__nv_bfloat16>)
                                         : reinterpret_cast<const void*>(&cache_write_kernel<__half>);
  return launch_ex(fn, dim3(blocks), dim3(kThreads), 0, stream, false, args);
}

cudaError_t launch_cache_read(const Cache8Args& a, cudaStream_t stream) {
  const unsigned blocks = blocks_of(a);
  if (blocks == 0) return cudaErrorInvalidConfiguration;
  void* args[] = {const_cast<Cache8Args*>(&a)};
  const void* fn = a.dtype == FSX_F32    ? reinterpret_cast<const void*>(&cache_read_kernel<float>)
                   : a.dtype == FSX_BF16 ? reinterpret_cast<const void*>(&cache_read_kernel<__nv_bfloat16>)
                                         : reinterpret_cast<const void*>(&cache_read_kernel<__half>);
  return launch_ex(fn, dim3(blocks), dim3(kThreads), 0, stream, false, args);
}

}  // namespace fsx
