// What the attention of a few rows over a cache shares between drafted tokens (tree_attention.cu) and single tokens over
// pages (paged_attention.cu): a warp's ring of 16-key stages, the online softmax over 8 NT rows, and its matrix products.
// The layouts and roundings are explained in tree_attention.cu.
#pragma once

#include <math_constants.h>

#include "kernels.h"
#include "tc_attention.cuh"

namespace fsx {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kChunk = 16 * kWarps;
constexpr int kD = kHeadDim;
constexpr int kJoin = 12;  // pieces whose partial results are loaded at once

// 4 bytes to shared memory, 0 if not `there` (then nothing is read)
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  return h;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {  // 8 x 8 16-bit tile, packed pairs along a row
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <bool BF>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (BF)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    mma_f16_16816(d, a0, a1, a2, a3, b0, b1);
}
__device__ __forceinline__ uint32_t word(const uint4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }

// 16 keys of a warp's ring stage: K rows, V rows, then (C8) the 16 scales of each. 16-byte unit u of row r lies
// at u ^ (r & 1) * 4 (K) or u ^ (r & 6) (V): the 8 lanes that are served together read 8 different units.
template <bool C8>
struct Stage {
  static constexpr int kRow = C8 ? kD : 2 * kD;
  static constexpr int kK = C8 ? 2 : 4, kV = C8 ? 1 : 2;  // 16-byte units per row and lane
  static constexpr int kOffV = 16 * kRow, kOffScale = 32 * kRow;
  static constexpr int kBytes = 32 * kRow + (C8 ? 128 : 0);
};

constexpr int kMostPower = 118;  // k is 2^118 at most, also where the sums are zero: k times a weight of 2^8 is finite
constexpr int kTopPower = 7;     // where the largest product goes when k moves

template <int NT>
struct State {
  float o[8][NT][4];  // [dim pair][8 rows]: (dim 0; row 2 c, 2 c + 1), (dim 1; the same)
  float m[NT][2], l[NT][2];
  float k[NT][2];     // C8: o is the sums times k, a power of two
};
__device__ __forceinline__ float power_of(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }
__device__ __forceinline__ int exponent_of(float x) { return static_cast<int>(__float_as_uint(x) >> 23) - 127; }  // x >= 0

// largest over the 8 lanes that hold a row pair's other keys or dims
__device__ __forceinline__ float max_over_g(float x) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

// Bits g and g + 8 of the warp's 16 value rows: all codes are zeros. A lane looks at half a row; `v`: the stage's V rows.
__device__ __forceinline__ uint2 zero_rows(const unsigned char* v) {
  const int lane = threadIdx.x & 31, g = lane >> 2;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 x = reinterpret_cast<const uint4*>(v + (lane >> 1) * kD + (lane & 1) * (kD / 2))[i];
    any |= x.x | x.y | x.z | x.w;
  }
  const uint32_t none = __ballot_sync(0xffffffffu, (any & 0x7f7f7f7fu) == 0u), rows = none & none >> 1;
  return make_uint2((rows >> (2 * g)) & 1u, (rows >> (2 * g + 16)) & 1u);
}

// Scores s[nt][key half * 2 + row] of 16 keys -> weights into the state, P^T packed for O^T. BF: type of the weights.
// C8: vs are the scales of values of keys g, g + 8, `v` their rows. SPLIT: pt[nt][2 ..] is what rounding took off the weights,
// itself in that type, for a second product (cache_step: if `second`).
template <bool BF, bool C8, int NT, bool SPLIT = false>
__device__ __forceinline__ void softmax_step(State<NT>& st, float (&s)[NT][4], float (&vs)[2], const unsigned char* v, uint32_t (&pt)[NT][SPLIT ? 4 : 2]) {
  float w[NT][4], p[NT][4];
  auto weigh = [&](int t, int e) {
    const int r = e & 1;
    w[t][e] = exp2_fast(s[t][e] - (st.m[t][r] == -CUDART_INF_F ? 0.f : st.m[t][r]));
    p[t][e] = C8 ? w[t][e] * st.k[t][r] * vs[e >> 1] : w[t][e];
  };
  bool move = false;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      move = move || fmaxf(s[t][r], s[t][2 + r]) > st.m[t][r] + 8.f;
      if (C8) {
        weigh(t, r);
        weigh(t, 2 + r);
        move = move || fmaxf(p[t][r], p[t][2 + r]) > 32768.f;
      }
    }
  if (__any_sync(0xffffffffu, move)) {
    if (C8) {
      const uint2 zero = zero_rows(v);
      if (zero.x) vs[0] = 0.f;
      if (zero.y) vs[1] = 0.f;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float m = fmaxf(st.m[t][r], max_over_g(fmaxf(s[t][r], s[t][2 + r])));
        const float up = m == st.m[t][r] ? 0.f : m - st.m[t][r];
        float alpha = exp2_fast(-up);
        st.m[t][r] = m;
        st.l[t][r] *= alpha;
        if (C8) {  // the sums do not grow, and no product leaves its range
          weigh(t, r);
          weigh(t, 2 + r);
          const float top = max_over_g(fmaxf(w[t][r] * vs[0], w[t][2 + r] * vs[1]));
          const float is = static_cast<float>(exponent_of(st.k[t][r]));
          const float will = fminf(fminf(floorf(is + up), static_cast<float>(kTopPower - exponent_of(top))), static_cast<float>(kMostPower));
          st.k[t][r] = power_of(static_cast<int>(will));
          alpha = exp2_fast(will - is - up);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          st.o[j][t][r] *= alpha;
          st.o[j][t][2 + r] *= alpha;
        }
      }
    if (C8) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) weigh(t, e);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!C8) weigh(t, e);
      st.l[t][e & 1] += w[t][e];
    }
    const uint32_t first = pack16<BF>(p[t][0], p[t][1]), second = pack16<BF>(p[t][2], p[t][3]);
    pt[t][0] = transpose8x8(first);
    pt[t][1] = transpose8x8(second);
    if (SPLIT) {
      const float2 x = unpack16<BF>(first), y = unpack16<BF>(second);
      float rest[4] = {p[t][0] - x.x, p[t][1] - x.y, p[t][2] - y.x, p[t][3] - y.y};
      if (C8) {  // weights are 2^15 at most, second parts 8; an infinite scale's weight is infinite in its first part, and has a second one too
#pragma unroll
        for (int e = 0; e < 4; ++e) rest[e] = fminf(rest[e], 32.f);
      }
      pt[t][SPLIT ? 2 : 0] = transpose8x8(pack16<BF>(rest[0], rest[1]));
      pt[t][SPLIT ? 3 : 1] = transpose8x8(pack16<BF>(rest[2], rest[3]));
    }
  }
}

template <bool BF, bool C8, int NT, bool SPLIT = false>
__device__ __forceinline__ void cache_step(State<NT>& st, const unsigned char* x, const uint32_t (&q)[NT][8][2],
                                           const float (&f)[NT][2], int left, bool second = true) {
  using S = Stage<C8>;
  constexpr bool kBf = BF && !C8;
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  uint4 xk[2][S::kK];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int u = 0; u < S::kK; ++u)
      xk[h][u] = *reinterpret_cast<const uint4*>(x + (g + 8 * h) * S::kRow + (((c + 4 * u) ^ ((g & 1) << 2)) << 4));
  float s[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[t][e] = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    uint32_t a[4];
    if (C8) {
      const uint32_t w0 = word(xk[0][k >> 2], k & 3), w1 = word(xk[1][k >> 2], k & 3);
      a[0] = e4m3x2_to_half2(w0);
      a[1] = e4m3x2_to_half2(w1);
      a[2] = e4m3x2_to_half2(w0 >> 16);
      a[3] = e4m3x2_to_half2(w1 >> 16);
    } else {
      a[0] = word(xk[0][k >> 1], 2 * (k & 1));
      a[1] = word(xk[1][k >> 1], 2 * (k & 1));
      a[2] = word(xk[0][k >> 1], 2 * (k & 1) + 1);
      a[3] = word(xk[1][k >> 1], 2 * (k & 1) + 1);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) mma<kBf>(s[t], a[0], a[1], a[2], a[3], q[t][k][0], q[t][k][1]);
  }
  float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
  if (C8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ks[h] = reinterpret_cast<const float*>(x + S::kOffScale)[g + 8 * h];
      vs[h] = reinterpret_cast<const float*>(x + S::kOffScale)[16 + g + 8 * h];
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float y = s[t][2 * h + r] * (C8 ? f[t][r] * ks[h] : kScaleLog2);
        s[t][2 * h + r] = g + 8 * h < left ? y : -CUDART_INF_F;
      }
  uint32_t pt[NT][SPLIT ? 4 : 2];
  softmax_step<kBf, C8, NT, SPLIT>(st, s, vs, x + S::kOffV, pt);
  uint4 xv[4][S::kV];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 2 * c + (i & 1) + 8 * (i >> 1);
#pragma unroll
    for (int u = 0; u < S::kV; ++u)
      xv[i][u] = *reinterpret_cast<const uint4*>(x + S::kOffV + r * S::kRow + (((g ^ (r & 6)) + 8 * u) << 4));
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      h[i] = C8 ? e4m3x2_to_half2(word(xv[i][0], j >> 1) >> ((j & 1) * 16)) : word(xv[i][C8 ? 0 : j >> 2], j & 3);
    const uint32_t a0 = __byte_perm(h[0], h[1], 0x5410), a1 = __byte_perm(h[0], h[1], 0x7632);
    const uint32_t a2 = __byte_perm(h[2], h[3], 0x5410), a3 = __byte_perm(h[2], h[3], 0x7632);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      mma<kBf>(st.o[j][t], a0, a1, a2, a3, pt[t][0], pt[t][1]);
      if (SPLIT && second) mma<kBf>(st.o[j][t], a0, a1, a2, a3, pt[t][SPLIT ? 2 : 0], pt[t][SPLIT ? 3 : 1]);
    }
  }
}

// What is read once: first to leave L2, so that tables, queries, partial results and the kernel's own code stay there
__device__ __forceinline__ uint64_t once_policy() {
  uint64_t policy;
  asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ void copy16_once(uint32_t dst, const void* src, bool there, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(policy) : "memory");
}

// One tensor's 16 keys into a stage. `src`: this lane's unit of its first row of them; rows past `left` become zeros. ONCE: by
// `policy`.
template <bool C8, bool V, bool ONCE = false>
__device__ __forceinline__ void copy_rows(uint32_t dst, const unsigned char* src, long long row_bytes, int left, uint64_t policy = 0) {
  using S = Stage<C8>;
  constexpr int kPerRow = S::kRow / 16, kStep = 32 / kPerRow;  // lanes a row, rows a warp copies at once
  const int lane = threadIdx.x & 31, u = lane % kPerRow, r0 = lane / kPerRow;
#pragma unroll
  for (int i = 0; i < 16 / kStep; ++i) {
    const int r = r0 + i * kStep;
    const int at = V ? u ^ (r & 6) : u ^ ((r & 1) << 2);
    const uint32_t to = dst + (V ? S::kOffV : 0) + r * S::kRow + at * 16;
    if (ONCE) copy16_once(to, src + i * kStep * row_bytes, r < left, policy);
    else copy16(to, src + i * kStep * row_bytes, r < left);
  }
}

// The dim of output (j, e) of lane row group g
template <bool C8>
__device__ __forceinline__ int out_dim(int g, int j, int e) {
  return C8 ? 16 * g + 2 * j + e : (j >> 2) * 64 + 8 * g + 2 * (j & 3) + e;
}

// The same as B operands; C8: bf16 as fp16 times 2^-e, f the factor that undoes it
template <bool BF, bool C8, int NT>
__device__ __forceinline__ void make_queries(uint32_t (&qf)[NT][8][2], float (&f)[NT][2]) {
  const int c = threadIdx.x & 3;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (C8 && !BF) {
      f[t][0] = f[t][1] = kScaleLog2;  // fp16 as it is
    } else if (C8) {
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 x = unpack16<BF>(qf[t][k][i]);
          top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // the largest magnitude goes to [2^7, 2^8); a row of zeros, infinities or NaN is taken as it is
      const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127 - 7;
      const bool plain = top == 0.f || !(top < CUDART_INF_F);
      const int ec = plain ? 0 : max(-126, min(e, 126));
      const float up = __uint_as_float(static_cast<uint32_t>(127 - ec) << 23);
      const float back = __uint_as_float(static_cast<uint32_t>(127 + ec) << 23);
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 x = unpack16<BF>(qf[t][k][i]);
          qf[t][k][i] = pack_half2(x.x * up, x.y * up);
        }
      f[t][0] = __shfl_sync(0xffffffffu, back, 8 * c) * kScaleLog2;
      f[t][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4) * kScaleLog2;
    }
  }
}

// CTAs an SM holds, stages of 16 keys in each warp's ring, rows that the warps put together at a time
template <bool C8, int NT>
struct Fit {
  static constexpr int kCtas = NT == 1 && C8 ? 4 : 3;
  static constexpr int kStages = C8 ? 3 : 2;
  static constexpr int kPass = 2 * NT;
};
__device__ __forceinline__ float weight_of(float m, float top) { return m == -CUDART_INF_F ? 0.f : exp2_fast(m - top); }

}  // namespace

}  // namespace fsx
