// One query row of an attention, held by a warp: lane l has dims 4 l .. 4 l + 3.
#pragma once

#include <cuda_fp8.h>
#include <math_constants.h>

#include "device_util.cuh"

namespace fsx {

__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xffff0000u));
}
__device__ __forceinline__ float4 load4(const __half* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&w.x));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&w.y));
  return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ float4 load4(const unsigned char* p) {  // e4m3
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  uint32_t a, b;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"(static_cast<uint16_t>(w)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"(static_cast<uint16_t>(w >> 16)));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a));
  const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&b));
  return make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ float4 scaled(float4 x, float s) { return make_float4(x.x * s, x.y * s, x.z * s, x.w * s); }

struct RowState {
  float4 q, o;
  float m, l;  // running maximum of the scaled scores, sum of exp(score - m)
};
template <typename T>
__device__ __forceinline__ void row_query(RowState& st, const T* q) {
  st.q = scaled(load4(q), 0.08838834764831845f);  // 1 / sqrt(128)
  st.o = make_float4(0.f, 0.f, 0.f, 0.f);
  st.m = -CUDART_INF_F;
  st.l = 0.f;
}
__device__ __forceinline__ void row_key(RowState& st, float4 k, float4 v) {
  const float s = warp_sum(st.q.x * k.x + st.q.y * k.y + st.q.z * k.z + st.q.w * k.w);
  const float m = fmaxf(st.m, s);
  const float base = m == -CUDART_INF_F ? 0.f : m;
  const float a = expf(st.m - base), w = expf(s - base);
  st.l = st.l * a + w;
  st.o.x = st.o.x * a + w * v.x;
  st.o.y = st.o.y * a + w * v.y;
  st.o.z = st.o.z * a + w * v.z;
  st.o.w = st.o.w * a + w * v.w;
  st.m = m;
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void store4(__half* p, float4 x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_half2(x.x, x.y), pack_half2(x.z, x.w));
}
template <typename T>
__device__ __forceinline__ void row_finish(const RowState& st, T* out, float* lse, int lane) {
  store4(out, st.l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : scaled(st.o, 1.f / st.l));
  if (lse != nullptr && lane == 0) *lse = st.l == 0.f ? -CUDART_INF_F : st.m + logf(st.l);
}

}  // namespace fsx
