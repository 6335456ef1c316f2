// Attention of a few new tokens of each request over its cache and over one another
// (fsx_tree_attention), for up to 8 NT rows (token, head of the group) an item.
//
// Bound by the cache's bytes. Each warp copies its own keys into a ring of its own (no barrier between
// warps), 16 at a time, two and more stages ahead: loads straight into registers, one step ahead, kept only
// 48 KB a SM on their way and read 128 single tokens' 8-bit caches at 3.6 TB/s. Per 16 keys:
//   S^T = K Q^T      m16n8k16, keys as M, 8 rows as N: with one row the other form (rows as M) spends twice
//                    the instructions and registers on rows that are not there
//   O^T += V^T P^T   dims as M: P^T comes out of S^T by a transposing move of its packed 8 x 8 tiles
// Which 4 dims a lane holds of a K = 16 step, and which 2 of an M = 16 tile, is free as long as both
// operands agree: a lane takes whole 16-byte units of a row, so a warp's loads cover 64 to 128 bytes a row.
//   lane (g, c) = (lane / 4, lane % 4): K of keys g, g + 8; V of keys 2 c, 2 c + 1, 2 c + 8, 2 c + 9;
//   scores and weights of keys g, g + 8 for rows 2 c, 2 c + 1; outputs of rows 2 c, 2 c + 1 for 16 dims.
// 8-bit caches: codes become fp16 exactly, bf16 queries fp16 times a power of two per row (their 8 bits fit;
// components 2^-22 below the row's largest may lose their last bits), a key's scale multiplies its
// score, a value's scale its weight. Weights are then fp16, also for bf16 queries; fp16 has a narrow range, and value scales
// may have any size, so the product's weights are taken times a power of two `k` of each row's own, which brings the
// largest (weight times scale) so far, for codes the largest contribution to the output up to a factor of two, to
// 2^7 .. 2^15. So neither a large value of little weight nor the new tokens decide what is lost: k of what the
// new tokens leave follows from their sums, and rows of zeros, whose scale says nothing, are left out of it.
// 16-bit caches and the new tokens use their own type, weights rounded to it.
// The running maximum moves only when a score exceeds it by more than 2^8, and k only when a weight exceeds 2^15, both
// seen by one vote a step.
//
// The 4 warps of a CTA take every fourth 16 keys of a chunk of 64 and are put together in shared memory. Items are cut
// into pieces that CTAs take from a queue (tree_schedule.cuh); the last one to end joins the pieces of its item.
//
// Measured: single tokens of 128 requests, 1.08 GB of 8-bit cache, 170 to 175 us (6.2 TB/s, 0.91 of a copy's rate; DRAM
// 81 % busy, issue slots 53 %). One token over 224 rows of a 16-bit cache 6.5 us, which is one launch and three
// dependent trips to memory: offsets, keys, results.
#include <math_constants.h>

#include <type_traits>

#include "fsx.h"
#include "kernels.h"
#include "llm.h"
#include "tc_attention.cuh"
#include "tree_schedule.cuh"

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
// C8: vs are the scales of values of keys g, g + 8, `v` their rows.
template <bool BF, bool C8, int NT>
__device__ __forceinline__ void softmax_step(State<NT>& st, float (&s)[NT][4], float (&vs)[2], const unsigned char* v, uint32_t (&pt)[NT][2]) {
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
    pt[t][0] = transpose8x8(pack16<BF>(p[t][0], p[t][1]));
    pt[t][1] = transpose8x8(pack16<BF>(p[t][2], p[t][3]));
  }
}

template <bool BF, bool C8, int NT>
__device__ __forceinline__ void cache_step(State<NT>& st, const unsigned char* x, const uint32_t (&q)[NT][8][2],
                                           const float (&f)[NT][2], int left) {
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
  uint32_t pt[NT][2];
  softmax_step<kBf, C8, NT>(st, s, vs, x + S::kOffV, pt);
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
    for (int t = 0; t < NT; ++t) mma<kBf>(st.o[j][t], a0, a1, a2, a3, pt[t][0], pt[t][1]);
  }
}

// One tensor's 16 keys into a stage. `src`: this lane's unit of its first row of them; rows past `left` become zeros.
template <bool C8, bool V>
__device__ __forceinline__ void copy_rows(uint32_t dst, const unsigned char* src, long long row_bytes, int left) {
  using S = Stage<C8>;
  constexpr int kPerRow = S::kRow / 16, kStep = 32 / kPerRow;  // lanes a row, rows a warp copies at once
  const int lane = threadIdx.x & 31, u = lane % kPerRow, r0 = lane / kPerRow;
#pragma unroll
  for (int i = 0; i < 16 / kStep; ++i) {
    const int r = r0 + i * kStep;
    const int at = V ? u ^ (r & 6) : u ^ ((r & 1) << 2);
    copy16(dst + (V ? S::kOffV : 0) + r * S::kRow + at * 16, src + i * kStep * row_bytes, r < left);
  }
}

// The dim of output (j, e) of lane row group g
template <bool C8>
__device__ __forceinline__ int out_dim(int g, int j, int e) {
  return C8 ? 16 * g + 2 * j + e : (j >> 2) * 64 + 8 * g + 2 * (j & 3) + e;
}

// New tokens key .. key + 15 of the request: their own type, one mask bit per row and token. A masked
// weight is 0 but 0 times an infinity or NaN is not: such values go into the product as 0. True: there are some, for
// add_wild. Comes before the cache's steps.
template <bool BF, bool C8, int NT>
__device__ __forceinline__ bool new_step(State<NT>& st, const TreeArgs& p, const TreePiece& it, uint32_t G, int key) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int left = it.r.n - key;
  const uint16_t* kn = static_cast<const uint16_t*>(p.k_new) + (it.r.t0 + key) * p.new_stride + it.kvh * kD;
  const uint16_t* vn = static_cast<const uint16_t*>(p.v_new) + (it.r.t0 + key) * p.new_stride + it.kvh * kD;
  const uint16_t* q = static_cast<const uint16_t*>(p.q);
  const uint32_t rows = it.r.n * G;
  float s[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[t][e] = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int d = 16 * k + 4 * c;
    uint2 a[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      a[h] = g + 8 * h < left ? __ldg(reinterpret_cast<const uint2*>(kn + (g + 8 * h) * p.new_stride + d)) : make_uint2(0u, 0u);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t row = it.row0 + 8 * t + g, token = row / G;
      const uint2 b = row < rows ? __ldg(reinterpret_cast<const uint2*>(q + (it.r.t0 + token) * p.q_stride +
                                                                         (it.kvh * G + row - token * G) * kD + d))
                                 : make_uint2(0u, 0u);
      mma<BF>(s[t], a[0].x, a[1].x, a[0].y, a[1].y, b.x, b.y);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint32_t row = it.row0 + 8 * t + 2 * c + r;
      const uint64_t mask = row < rows ? p.mask[it.r.t0 + row / G] >> key : 0ull;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool sees = g + 8 * h < left && ((mask >> (g + 8 * h)) & 1u);
        s[t][2 * h + r] = sees ? s[t][2 * h + r] * kScaleLog2 : -CUDART_INF_F;
      }
    }
  float ones[2] = {1.f, 1.f};
  uint32_t pt[NT][2];
  softmax_step<BF, false, NT>(st, s, ones, nullptr, pt);
  uint32_t wild = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = 2 * c + (i & 1) + 8 * (i >> 1);
      h[i] = at < left ? __ldg(reinterpret_cast<const uint32_t*>(vn + at * p.new_stride + out_dim<C8>(g, j, 0))) : 0u;
      const uint32_t bad = not_finite2<BF>(h[i]);
      wild |= bad;
      h[i] &= ~((bad >> 15) * 0xffffu);
    }
    const uint32_t a0 = __byte_perm(h[0], h[1], 0x5410), a1 = __byte_perm(h[0], h[1], 0x7632);
    const uint32_t a2 = __byte_perm(h[2], h[3], 0x5410), a3 = __byte_perm(h[2], h[3], 0x7632);
#pragma unroll
    for (int t = 0; t < NT; ++t) mma<BF>(st.o[j][t], a0, a1, a2, a3, pt[t][0], pt[t][1]);
  }
  if (C8) {  // the sums' largest magnitude goes to [2^15, 2^16)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fmaxf(fabsf(st.o[j][t][r]), fabsf(st.o[j][t][2 + r])));
        top = max_over_g(top);
        st.k[t][r] = top < CUDART_INF_F ? power_of(min(15 - exponent_of(top), kMostPower)) : 1.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          st.o[j][t][r] *= st.k[t][r];
          st.o[j][t][2 + r] *= st.k[t][r];
        }
      }
  }
  return __any_sync(0xffffffffu, wild != 0);
}

// The values that new_step took out, for the rows that see them; k is 1
template <bool BF, bool C8, int NT>
__device__ __forceinline__ void add_wild(State<NT>& st, const TreeArgs& p, const TreePiece& it, uint32_t G, int key) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint16_t* vn = static_cast<const uint16_t*>(p.v_new) + (it.r.t0 + key) * p.new_stride + it.kvh * kD;
  const uint32_t rows = it.r.n * G;
#pragma unroll 1
  for (int i = 0; i < min(it.r.n - key, 16); ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t v = __ldg(reinterpret_cast<const uint32_t*>(vn + i * p.new_stride + out_dim<C8>(g, j, 0)));
      const uint32_t bad = not_finite2<BF>(v);
      if (bad == 0u) continue;
      const float2 y = unpack16<BF>(v);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t row = it.row0 + 8 * t + 2 * c + r;
          if (row < rows && (p.mask[it.r.t0 + row / G] >> (key + i)) & 1u) {
            if (bad & 0x8000u) st.o[j][t][r] += y.x;
            if (bad & 0x80000000u) st.o[j][t][2 + r] += y.y;
          }
        }
    }
}

// Queries of the item's rows, as they lie
template <bool C8, int NT>
__device__ __forceinline__ void load_queries(uint32_t (&qf)[NT][8][2], const TreeArgs& p, const TreePiece& it, uint32_t G) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint16_t* q = static_cast<const uint16_t*>(p.q) + it.r.t0 * p.q_stride + it.kvh * G * kD;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint32_t row = it.row0 + 8 * t + g, token = row / G;
    const bool there = row < it.r.n * G;
    const uint16_t* src = q + (there ? token * p.q_stride + (row - token * G) * kD : 0ll);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int d = C8 ? (k >> 2) * 64 + 16 * c + 4 * (k & 3) : 8 * (c + 4 * (k >> 1)) + 4 * (k & 1);
      const uint2 w = there ? __ldg(reinterpret_cast<const uint2*>(src + d)) : make_uint2(0u, 0u);
      qf[t][k][0] = w.x;
      qf[t][k][1] = w.y;
    }
  }
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
template <bool C8, int NT>
struct Shared {  // and the plan behind it
  long long scratch[2 * kWarps];
  __align__(128) unsigned char ring[kWarps][Fit<C8, NT>::kStages * Stage<C8>::kBytes];
  float m[kWarps][8 * NT], l[kWarps][8 * NT];
  float o[kWarps][Fit<C8, NT>::kPass][kD];
  long long next;
  int last;
};

__device__ __forceinline__ float weight_of(float m, float top) { return m == -CUDART_INF_F ? 0.f : exp2_fast(m - top); }

// Workspace behind the header: a counter per slot, then the slots: [rows][128] sums, [rows] (maximum, sum of weights)
constexpr size_t slot_floats(int nt) { return static_cast<size_t>(8) * nt * (kD + 2); }
constexpr int slots_of(int nt) { return kTreeCounters / nt; }  // 34 MB

template <int NT>
__device__ __forceinline__ float* slot_at(const TreeArgs& p, int slot) {
  return reinterpret_cast<float*>(static_cast<int*>(p.workspace) + kTreeHeader + kTreeCounters) +
         static_cast<size_t>(slot) * slot_floats(NT);
}

template <bool BF, bool C8, int NT>
__global__ void __launch_bounds__(kThreads, Fit<C8, NT>::kCtas) tree_kernel(const TreeArgs p) {
  using S = Stage<C8>;
  constexpr int kStages = Fit<C8, NT>::kStages, kPass = Fit<C8, NT>::kPass;
  constexpr int kPerRow = S::kRow / 16;
  constexpr TreeShape kShape{8 * NT, kChunk, 8, 28, slots_of(NT)};
  extern __shared__ __align__(128) unsigned char raw_smem[];
  Shared<C8, NT>& sm = *reinterpret_cast<Shared<C8, NT>*>(raw_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const uint32_t G = static_cast<uint32_t>(p.n_heads) / static_cast<uint32_t>(p.n_kv_heads);
  int* header = static_cast<int*>(p.workspace);
  const TreePlan plan = tree_plan<kThreads>(p, kShape, raw_smem + sizeof(sm), sm.scratch);
  const long long total = plan.pieces[p.B];
  const long long row_bytes = static_cast<long long>(p.n_kv_heads) * S::kRow;
  const uint32_t ring = smem_addr(sm.ring[warp]);

  // this warp's copies of a piece: keys staged, staged + 64, ... < end
  const unsigned char *kc = nullptr, *vc = nullptr;
  const float* scales = nullptr;
  int staged = 0, end = 0, slot_in = 0;
  auto copy_next = [&] {
    const int left = end - staged;
    if (left > 0) {
      const uint32_t dst = ring + slot_in * S::kBytes;
      copy_rows<C8, false>(dst, kc, row_bytes, left);
      copy_rows<C8, true>(dst, vc, row_bytes, left);
      if (C8) copy4(dst + S::kOffScale + lane * 4, scales, (lane & 15) < left);
    }
    cp_async_commit();
    staged += kChunk;
    kc += kChunk * row_bytes;
    vc += kChunk * row_bytes;
    scales += C8 ? kChunk : 0;
    slot_in = slot_in + 1 == kStages ? 0 : slot_in + 1;
  };
  auto begin = [&](const TreePiece& x) {
    staged = x.from * kChunk + 16 * warp;
    end = min(x.r.len, min(x.to, x.n - 1) * kChunk);
    const long long at = (x.r.c0 + staged + lane / kPerRow) * row_bytes + x.kvh * S::kRow + (lane % kPerRow) * 16;
    kc = static_cast<const unsigned char*>(p.k_cache) + at;
    vc = static_cast<const unsigned char*>(p.v_cache) + at;
    if (C8) scales = (lane < 16 ? p.k_scale : p.v_scale) + x.kvh * p.cache_rows + x.r.c0 + staged + (lane & 15);
    slot_in = 0;
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) copy_next();
  };

  long long i = blockIdx.x;
  TreePiece it;
  uint32_t qf[NT][8][2];
  if (i < total) {
    it = tree_piece(p, kShape, plan, i);
    load_queries<C8, NT>(qf, p, it, G);  // in front of the cache's copies
    begin(it);
  }
#pragma unroll 1
  while (i < total) {
    if (tid == 0) sm.next = gridDim.x + static_cast<long long>(atomicAdd(reinterpret_cast<unsigned*>(header), 1u));
    State<NT> st;
    float f[NT][2];
    make_queries<BF, C8, NT>(qf, f);
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
    // the new tokens first, while the cache's first rows are on their way
    bool wild = false;
    if (it.to == it.n && 16 * warp < it.r.n) wild = new_step<BF, C8, NT>(st, p, it, G, 16 * warp);
    int slot_out = 0;
#pragma unroll 1
    for (int key = it.from * kChunk + 16 * warp; key < end; key += kChunk) {
      cp_async_wait<kStages - 2>();
      __syncwarp();  // every lane's copies of the stage; and the stage before is read
      copy_next();
      cache_step<BF, C8, NT>(st, sm.ring[warp] + slot_out * S::kBytes, qf, f, end - key);
      slot_out = slot_out + 1 == kStages ? 0 : slot_out + 1;
    }
    cp_async_wait<0>();
    __syncwarp();
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
    if (wild) add_wild<BF, C8, NT>(st, p, it, G, 16 * warp);

    const int rows = min(8 * NT, static_cast<int>(it.r.n * G - it.row0));
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
    // ---- the next piece's first copies go out before this one's results are put together
    const long long i_next = sm.next;
    TreePiece next = it;
    if (i_next < total) {
      next = tree_piece(p, kShape, plan, i_next);
      load_queries<C8, NT>(qf, p, next, G);
      begin(next);
    }
    // ---- the four warps' results, kPass rows at a time; a thread a dim
    auto finish = [&](int row, float m, float l, float o) {
      const uint32_t at = it.row0 + row, token = at / G, head = it.kvh * G + at - token * G;
      const float y = l == 0.f ? 0.f : o / l;
      static_cast<uint16_t*>(p.out)[((it.r.t0 + token) * p.n_heads + head) * kD + tid] = static_cast<uint16_t>(pack16<BF>(y, y));
      if (p.lse != nullptr && tid == 0)
        p.lse[head * p.new_rows + it.r.t0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
    };
    float* slot = slot_at<NT>(p, it.slot + it.j);
#pragma unroll
    for (int base = 0; base < 8 * NT; base += kPass) {
      if (base >= rows) break;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = 8 * t + 2 * c + r;
          if (row >= base && row < base + kPass && row < rows) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              *reinterpret_cast<float2*>(&sm.o[warp][row - base][out_dim<C8>(g, j, 0)]) = make_float2(st.o[j][t][r], st.o[j][t][2 + r]);
            }
          }
        }
      __syncthreads();
#pragma unroll 1
      for (int row = base; row < min(rows, base + kPass); ++row) {
        const float m = fmaxf(fmaxf(sm.m[0][row], sm.m[1][row]), fmaxf(sm.m[2][row], sm.m[3][row]));
        float l = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float a = weight_of(sm.m[w][row], m);
          l += a * sm.l[w][row];
          o += a * sm.o[w][row - base][tid];
        }
        if (it.of == 1) {
          finish(row, m, l, o);
        } else {
          __stcg(slot + row * kD + tid, o);
          if (tid == 0) __stcg(reinterpret_cast<float2*>(slot + 8 * NT * kD) + row, make_float2(m, l));
        }
      }
      __syncthreads();
    }
    if (it.of > 1) {
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        int* counter = header + kTreeHeader + it.slot;
        sm.last = atomicAdd(counter, 1) == it.of - 1;
        if (sm.last) *counter = 0;
      }
      __syncthreads();
      if (sm.last) {
        __threadfence();
        const float* first = slot_at<NT>(p, it.slot);
#pragma unroll 1
        for (int row = warp; row < rows; row += kWarps) {  // a warp a row, 4 dims a lane
          float m = -CUDART_INF_F, l = 0.f;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int j0 = 0; j0 < it.of; j0 += kJoin) {  // in the order of the keys; the loads of kJoin pieces at once
            float2 x[kJoin];
            float4 v[kJoin];
#pragma unroll
            for (int j = 0; j < kJoin; ++j) {
              const float* other = first + min(j0 + j, it.of - 1) * slot_floats(NT);
              x[j] = __ldcg(reinterpret_cast<const float2*>(other + 8 * NT * kD) + row);
              v[j] = __ldcg(reinterpret_cast<const float4*>(other + row * kD) + lane);
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
              if (j0 + j < it.of) {
                l += a * x[j].y;
                o.x += a * v[j].x;
                o.y += a * v[j].y;
                o.z += a * v[j].z;
                o.w += a * v[j].w;
              }
            }
          }
          const uint32_t at = it.row0 + row, token = at / G, head = it.kvh * G + at - token * G;
          const float inv = l == 0.f ? 0.f : 1.f / l;
          uint16_t* out = static_cast<uint16_t*>(p.out) + ((it.r.t0 + token) * p.n_heads + head) * kD + 4 * lane;
          *reinterpret_cast<uint2*>(out) = make_uint2(pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv));
          if (p.lse != nullptr && lane == 0)
            p.lse[head * p.new_rows + it.r.t0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
        }
      }
    }
    __syncthreads();  // before the next piece writes what was read here
    it = next;
    i = i_next;
  }
  if (tid == 0 && atomicAdd(reinterpret_cast<unsigned*>(header) + 1, 1u) == gridDim.x - 1) {
    header[0] = 0;  // every CTA has taken its last piece
    header[1] = 0;
  }
}

struct Kernel {
  const void* fn;
  size_t smem;
  int ctas;  // per SM
};
template <bool BF, bool C8, int NT>
Kernel kernel_for() {
  return {reinterpret_cast<const void*>(&tree_kernel<BF, C8, NT>), sizeof(Shared<C8, NT>), Fit<C8, NT>::kCtas};
}
template <bool BF, bool C8>
Kernel kernel_of(int nt) {
  return nt == 1 ? kernel_for<BF, C8, 1>() : kernel_for<BF, C8, 2>();
}

// 8-row tiles of an item, by the rows that a request has on average; 0: the kernel of tree_tc.cu. Measured over eight
// 8-bit caches of 4096 to 8192 rows: 8 to 16 rows a request 42 to 44 us here, 51.8 there; 16 to 32 rows 51.5 us there,
// 57.0 here, in items of 16 that read the cache twice. Two tiles where one will do: 7.6 for 6.5 us (one token over 224
// rows), 205 for 168 us (128 tokens).
int tile_count(int B, long long new_rows, int n_heads, int n_kv_heads) {
  const long long rows = (new_rows * (n_heads / n_kv_heads) + B - 1) / B;
  return rows <= 8 ? 1 : rows <= 16 ? 2 : 0;
}

}  // namespace

size_t tree_attention_workspace_bytes(int B, long long new_rows, int n_heads, int n_kv_heads) {
  const int nt = tile_count(B, new_rows, n_heads, n_kv_heads);
  if (nt == 0) return tree_tc_workspace_bytes(B, new_rows, n_heads, n_kv_heads);
  return (kTreeHeader + kTreeCounters) * sizeof(int) + slots_of(nt) * slot_floats(nt) * sizeof(float);
}

cudaError_t launch_tree_attention(const TreeArgs& a, int dtype, bool cache8, cudaStream_t stream) {
  const int nt = tile_count(a.B, a.new_rows, a.n_heads, a.n_kv_heads);
  if (nt == 0) return launch_tree_tc(a, dtype, cache8, stream);
  const Kernel k = dtype == FSX_BF16 ? (cache8 ? kernel_of<true, true>(nt) : kernel_of<true, false>(nt))
                                     : (cache8 ? kernel_of<false, true>(nt) : kernel_of<false, false>(nt));
  const size_t smem = k.smem + tree_plan_bytes(a.B);
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  const cudaError_t e = allow_shared_memory(k.fn, smem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<TreeArgs*>(&a)};
  return launch_ex(k.fn, dim3(static_cast<unsigned>(sms * k.ctas)), dim3(kThreads), smem, stream, false, args);
}

}  // namespace fsx
