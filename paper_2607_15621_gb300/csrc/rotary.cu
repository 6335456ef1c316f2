// Rotary positions of one or several axes for queries and keys, and the keys' and values' rows written into a cache in the
// same pass (fsx_rotary).
//
// Pair j of a head turns by pos[axis_j] rate_j: (a, b) -> (a cos - b sin, a sin + b cos). The angle is taken in whole turns as
// 64-bit fixed point: turns_j = rate_j / (2 pi) in units of 2^-64, rounded down, and pos * turns_j modulo 2^64 is the fraction of a turn,
// exactly as far as turns_j is (2^-33 at a position of 2^31); its upper 32 bits, less than 2^-32 below it, give the quarter turn and the
// rest, whose sine and cosine are Taylor's series. An
// angle in fp32 would be off by 2^-24 of itself, at position 100,000 by half a percent of a turn.
// Products in fp32, rounded once to the type; keys go into an 8-bit cache from their rounded values, so that a cache written
// here has the bits of one written from the rotated keys by fsx_cache_write_e4m3.
//
// Bound by memory (no product to speak of): 8 lanes hold a head of a row, 16 values each, the two halves of 8 pairs; a warp
// takes 4 heads at a time, 16 in flight. Its lanes compute the row's 64 sines and cosines, two each, and share them through
// shared memory: each is used by all heads of the row. Where rows are few they are shared out by heads over several warps.
// Measured: 28,001 rows of 48 heads in 16 bits, with keys and cache, 111 to 113 us (6.7 TB/s, 0.98 of a copy's rate; DRAM 76 % busy), into
// 8-bit pages 104 us (0.97); 128 rows into 8-bit pages 3.4 us; one row 1.6 us, where the launch is all.
#include "fsx.h"
#include "kernels.h"
#include "pages.h"
#include "rows8.cuh"
#include "tc_attention.cuh"

namespace fsx {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kFewGroups = 2;  // of 4 heads: a row's

template <bool BF>
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack16<BF>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <bool BF>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack16<BF>(x[0], x[1]), pack16<BF>(x[2], x[3]), pack16<BF>(x[4], x[5]), pack16<BF>(x[6], x[7]));
}

// Cosine and sine of `t` 2^-32 turns. |x| <= pi / 4 behind the nearest quarter: Taylor's series to x^8 and x^9 leave 2.5e-8 and 2e-9 out,
// about fp32's rounding of the result (28,001 rows of 5 heads 19.4 us, with sincospif, which takes arguments of any size, 19.7).
__device__ __forceinline__ float2 turned_by(uint32_t t) {
  const uint32_t q = (t + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(t - (q << 30))) * (6.28318530718f / 4294967296.f);
  const float y = x * x;
  const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const uint32_t cosine = __float_as_uint(q & 1u ? s : c) ^ ((q + 1u) & 2u) << 30, sine = __float_as_uint(q & 1u ? c : s) ^ (q & 2u) << 30;
  return make_float2(__uint_as_float(cosine), __uint_as_float(sine));
}

// 16 values of a head's row, 8 lanes a row: codes and the row's scale as fsx_cache_write_e4m3 makes them. False: values
// that are not finite. The largest magnitude is found two values at a time, of their 16 bits without the sign; only rows with
// values that are not finite look at each.
template <bool BF>
__device__ __forceinline__ bool quantise(const uint4 (&y)[2], uint2 (&code)[2], float& scale) {
  constexpr uint32_t kInf = BF ? 0x7f80u : 0x7c00u;
  const uint32_t w[8] = {y[0].x, y[0].y, y[0].z, y[0].w, y[1].x, y[1].y, y[1].z, y[1].w};
  uint32_t two = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(two) : "r"(w[i] & 0x7fff7fffu));
  uint32_t most = max(two & 0xffffu, two >> 16);
  const bool wild = most >= kInf;  // this lane's
  if (__any_sync(0xffffffffu, wild)) {
    most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t lo = w[i] & 0x7fffu, hi = w[i] >> 16 & 0x7fffu;
      if (lo < kInf) most = max(most, lo);
      if (hi < kInf) most = max(most, hi);
    }
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  const float2 tops = unpack16<BF>(most);
  const uint32_t top = __float_as_uint(tops.x);
  int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = max(e, -126);
  const bool zero = top == 0;
  scale = zero ? 1.f : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
  const float inv = zero ? 1.f : __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 x = unpack16<BF>(w[4 * h + j]);
      c[j] = pack_e4m3x2(x.x * inv, x.y * inv);
      if (wild) {
        if ((w[4 * h + j] & 0x7fffu) >= kInf) c[j] |= 0x7fu;
        if ((w[4 * h + j] >> 16 & 0x7fffu) >= kInf) c[j] |= 0x7f00u;
      }
    }
    code[h] = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
  }
  return !wild;
}

enum { kNoCache = 0, kCache16 = 1, kCache8 = 2 };

// `parts` warps a row, `per` groups of 4 heads each, AHEAD of them loaded at once. ROWS: a warp takes `rows_each` rows one after another, the next
// one's loads ahead, so that the pairs' axes and rates, which lanes read at different places of the parameters, are read once.
template <bool BF, bool ADJACENT, int CACHE, int AHEAD, bool ROWS>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const __grid_constant__ RotaryArgs a, int parts, int per, int rows_each) {
  __shared__ __align__(16) float2 turn[kWarps][kHeadDim / 2];  // cosine, sine
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & 7;
  uint64_t turns[2];
  const int64_t* positions[2];
  // Lanes read the parameters at different places, one after another. Few rows: ahead of the wait for the kernel before. Many: behind the loads
  // of the heads (1000 rows of 48 heads: 6.3 us, ahead of them 6.7).
  auto read_pairs = [&] {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      turns[h] = a.turns[lane + 32 * h];
      positions[h] = a.positions + a.axis[lane + 32 * h] * a.rows;
    }
  };
  if (AHEAD == 2) read_pairs();
  const long long w = static_cast<long long>(blockIdx.x) * kWarps + warp, block = w / parts;
  const int part = static_cast<int>(w - block * parts);
  long long row = ROWS ? block * rows_each : block;
  const long long row_end = ROWS ? min(a.rows, row + rows_each) : min(a.rows, row + 1);
  if (row >= row_end) return;  // the whole warp
  pdl_wait();
  const int nq = a.q != nullptr ? a.n_heads : 0, nk = a.k != nullptr ? a.n_kv_heads : 0;
  const int slots = nq + nk + (CACHE != kNoCache ? nk : 0);
  const int group0 = part * per, group_end = min(group0 + per, (slots + 3) >> 2);
  constexpr int kSecond = ADJACENT ? 8 : kHeadDim / 2;  // from a lane's first 8 values to its others
  const int dim = ADJACENT ? 16 * l : 8 * l;
  uint4 x[AHEAD][2];
  long long pos[2], at = -1;
  auto load = [&](long long r, int group, uint4 (&to)[2]) {  // plain loads: a result may replace its input
    const int s = group * 4 + (lane >> 3);
    if (group < group_end && s < slots) {
      const uint16_t* src = s < nq        ? static_cast<const uint16_t*>(a.q) + r * a.q_stride + s * kHeadDim
                            : s < nq + nk ? static_cast<const uint16_t*>(a.k) + r * a.kv_stride + (s - nq) * kHeadDim
                                          : static_cast<const uint16_t*>(a.v) + r * a.kv_stride + (s - nq - nk) * kHeadDim;
      to[0] = *reinterpret_cast<const uint4*>(src + dim);
      to[1] = *reinterpret_cast<const uint4*>(src + dim + kSecond);
    } else {
      to[0] = to[1] = make_uint4(0u, 0u, 0u, 0u);
    }
  };
  auto load_row = [&](long long r) {  // what a row needs besides its heads
    pos[0] = positions[0][r];
    pos[1] = positions[1][r];
    if (CACHE != kNoCache) at = a.dst_rows != nullptr ? a.dst_rows[r] : r;
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(row, group0 + i, x[i]);
  if (AHEAD != 2) read_pairs();
  load_row(row);
  bool wild = false, lost = false;
#pragma unroll 1
  for (; row < row_end; ++row) {
    const bool more = ROWS && row + 1 < row_end;
#pragma unroll
    for (int h = 0; h < 2; ++h) turn[warp][lane + 32 * h] = turned_by(static_cast<uint32_t>((static_cast<uint64_t>(pos[h]) * turns[h]) >> 32));
    const bool kept = CACHE != kNoCache && at >= 0 && at < a.cache_rows;
    lost = lost || (CACHE != kNoCache && !kept);
    const long long to_row = at;
    if (more) load_row(row + 1);
    __syncwarp();
    float2 t[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 y = reinterpret_cast<const float4*>(&turn[warp][8 * l])[i];
      t[2 * i] = make_float2(y.x, y.y);
      t[2 * i + 1] = make_float2(y.z, y.w);
    }
    __syncwarp();  // before the next row's are written
#pragma unroll 1
    for (int base = group0; base < group_end; base += AHEAD) {
      const bool last = base + AHEAD >= group_end;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int s = (base + i) * 4 + (lane >> 3);
        const bool there = base + i < group_end && s < slots;
        uint4 y[2] = {x[i][0], x[i][1]};
        if (!last) load(row, base + AHEAD + i, x[i]);
        else if (more) load(row + 1, group0 + i, x[i]);
        const bool is_v = s >= nq + nk;
        if (!is_v) {
          float f[2][8];
          unpack8<BF>(y[0], f[0]);
          unpack8<BF>(y[1], f[1]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float& p0 = ADJACENT ? f[j >> 2][2 * (j & 3)] : f[0][j];
            float& p1 = ADJACENT ? f[j >> 2][2 * (j & 3) + 1] : f[1][j];
            const float c = t[j].x, z = t[j].y, u = p0, o = p1;
            p0 = u * c - o * z;
            p1 = u * z + o * c;
          }
          y[0] = pack8<BF>(f[0]);
          y[1] = pack8<BF>(f[1]);
        }
        const int kv = s - (is_v ? nq + nk : nq);
        if (there && !is_v) {
          uint16_t* out = s < nq ? static_cast<uint16_t*>(a.q_out) + row * a.q_out_stride + s * kHeadDim
                                 : static_cast<uint16_t*>(a.k_out) + row * a.k_out_stride + kv * kHeadDim;
          if (s < nq || a.k_out != nullptr) {
            *reinterpret_cast<uint4*>(out + dim) = y[0];
            *reinterpret_cast<uint4*>(out + dim + kSecond) = y[1];
          }
        }
        if (CACHE == kCache16) {
          if (there && s >= nq && kept) {
            uint16_t* out = static_cast<uint16_t*>(is_v ? a.v_cache : a.k_cache) + (to_row * nk + kv) * kHeadDim + dim;
            *reinterpret_cast<uint4*>(out) = y[0];
            *reinterpret_cast<uint4*>(out + kSecond) = y[1];
          }
        } else if (CACHE == kCache8) {
          if (__any_sync(0xffffffffu, there && s >= nq)) {
            uint2 code[2];
            float scale;
            const bool fine = quantise<BF>(y, code, scale);
            if (there && s >= nq) {
              wild = wild || !fine;
              if (kept) {
                unsigned char* out = static_cast<unsigned char*>(is_v ? a.v_cache : a.k_cache) + (to_row * nk + kv) * kHeadDim + dim;
                if (ADJACENT) {
                  *reinterpret_cast<uint4*>(out) = make_uint4(code[0].x, code[0].y, code[1].x, code[1].y);
                } else {
                  *reinterpret_cast<uint2*>(out) = code[0];
                  *reinterpret_cast<uint2*>(out + kSecond) = code[1];
                }
                if (l == 0) (is_v ? a.v_scale : a.k_scale)[kv * a.cache_rows + to_row] = scale;
              }
            }
          }
        }
      }
    }
  }
  if (lost && lane == 0) set_status(a.status, kStatusDeviceArg);
  if (CACHE == kCache8 && wild) set_status(a.status, kStatusRange);
}

template <int AHEAD, bool ROWS, bool BF, bool ADJACENT>
const void* kernel_for(int cache) {
  return cache == kNoCache  ? reinterpret_cast<const void*>(&rotary_kernel<BF, ADJACENT, kNoCache, AHEAD, ROWS>)
         : cache == kCache16 ? reinterpret_cast<const void*>(&rotary_kernel<BF, ADJACENT, kCache16, AHEAD, ROWS>)
                             : reinterpret_cast<const void*>(&rotary_kernel<BF, ADJACENT, kCache8, AHEAD, ROWS>);
}
template <int AHEAD, bool ROWS>
const void* kernel_of(bool bf, bool adjacent, int cache) {
  return bf ? (adjacent ? kernel_for<AHEAD, ROWS, true, true>(cache) : kernel_for<AHEAD, ROWS, true, false>(cache))
            : (adjacent ? kernel_for<AHEAD, ROWS, false, true>(cache) : kernel_for<AHEAD, ROWS, false, false>(cache));
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, int dtype, bool adjacent, bool cache8, cudaStream_t stream) {
  const int cache = a.k_cache == nullptr ? kNoCache : cache8 ? kCache8 : kCache16;
  const int nk = a.k != nullptr ? a.n_kv_heads : 0;
  const int slots = (a.q != nullptr ? a.n_heads : 0) + (cache != kNoCache ? 2 : 1) * nk;
  if (slots == 0) return cudaSuccess;
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  // 8 warps a SM and more where rows are few; and no warp has more than 4 groups of heads as long as all warps run at once
  // (128 rows of 48 heads: 4.4 us, with 32 warps a SM 5.1; 1000 rows 5.6, with whole rows 6.8)
  const int groups = (slots + 3) / 4, least = (groups + 3) / 4;
  long long want = (static_cast<long long>(sms) * 8 + a.rows - 1) / a.rows;
  if (want < least && a.rows * least <= static_cast<long long>(sms) * 20) want = least;
  const int split = static_cast<int>(want < groups ? want : groups);
  int per = (groups + split - 1) / split;
  int parts = (groups + per - 1) / per;
  // Rows of few heads, several to a warp while there are twice as many warps as run at once: 28,001 rows of 5 heads 19.4 us for 28.6; of 48 heads
  // 119 for 111, by the registers that the next row's loads take
  const long long each = a.rows * parts / (static_cast<long long>(sms) * 40);
  int rows_each = static_cast<int>(groups > kFewGroups || each < 1 ? 1 : each < 8 ? each : 8);
  const long long blocks = ((a.rows + rows_each - 1) / rows_each * parts + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  // two groups at once where a warp has no more (one row of 96 heads 2.0 us, with four 2.4: instructions for heads that are not there)
  const bool bf = dtype == FSX_BF16;
  const void* fn = rows_each > 1 ? kernel_of<2, true>(bf, adjacent, cache)
                   : per <= 2    ? kernel_of<2, false>(bf, adjacent, cache)
                                 : kernel_of<4, false>(bf, adjacent, cache);
  void* args[] = {const_cast<RotaryArgs*>(&a), &parts, &per, &rows_each};
  return launch_ex(fn, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, true, args);
}

}  // namespace fsx
