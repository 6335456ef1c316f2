// Attention of whole prompts, packed one after another (fsx_prompt_attention), on the 5th-generation
// tensor cores.
//
// A sequence's queries that share a kv head, token-major with the group's heads inside (row = token G +
// head), are cut into items of two 128-row tiles; a CTA works on one item of one kv head. Keys come in
// chunks of 128 up to the last that a row of the item sees. Per tile and chunk
//   S = Q K^T            A, B in shared memory, S in tensor memory (128 fp32 columns)
//   P = 2^(c S - m)      a thread holds a whole row: no exchange between lanes; P is rounded to the
//                        type of V and written over its S (64 columns)
//   O += P V             A in tensor memory, V read N-contiguous, O in tensor memory (128 columns)
// The two tiles alternate: while the softmax of one runs, the tensor core works on the other
// (P V of its last chunk, then S of its next). An MMA thread's MMAs run in order, so S of chunk j
// being there means that P V of chunk j - 1 is done: the running maximum may then be moved and O
// rescaled (by the softmax threads, only when a maximum grew by more than 2^8) without another wait.
//
// Warps 0-3, 4-7: softmax of tile 0, 1 (they also load the queries and write the outputs); warp 8 issues
// MMAs; warp 9 loads K and V chunks by TMA into a ring of five 32 KB stages (K0 V0 K1 V1 ...); warps
// 10-11 guard the V chunks that some row of the item sees only in part (the diagonal, the end of the
// sequence): a masked weight is 0, but 0 times an infinity or NaN is not, so rows past the sequence become
// zeros, and values that are not finite too; such a value is added to the rows that do see it at the end.
//
// Items are taken longest first: block i works on the i-th item in the order of its number of
// chunks, found by counting (the host knows no lengths).
#include "fsx.h"
#include "gemm_tc.h"
#include "kernels.h"
#include "llm.h"
#include "tc_attention.cuh"

namespace fsx {

namespace {

constexpr int kD = kHeadDim;
constexpr int kTile = 128;              // query rows of a tile, keys of a chunk
constexpr int kItemRows = 2 * kTile;
constexpr int kStages = 5;
constexpr int kStageBytes = kTile * kD * 2;  // 32 KB
constexpr int kMmaWarp = 8, kLoadWarp = 9;  // the last two guard
constexpr int kThreads = 384;           // three warpgroups: 168 registers a thread at launch
constexpr int kMaxGuarded = 3;          // 256 rows are at most 256 tokens: their diagonals and the end
constexpr uint32_t kColS = 0, kColO = 256;
constexpr int kOffRing = 2 * kStageBytes;  // the two Q tiles lie in front
constexpr int kOffBar = kOffRing + kStages * kStageBytes;
// full[5], empty[5], gfull[3], gdone[3], qfull[2], sfull[2], pfull[2][2], odone[2], drain
constexpr int kNumBars = 27;
constexpr int kSmem = kOffBar + kNumBars * 8 + 64;
static_assert(kSmem <= 227 * 1024, "shared memory");
static_assert(kMaxSequences * 16 <= kStages * kStageBytes, "the lengths lie in the ring before it is used");

struct Maps {
  CUtensorMap k, v;
};

struct Item {
  int b;            // sequence, -1: none
  long long row0;   // first packed row of the item
  long long q0, k0; // first query row, first key row
  int nq, nk;
};

// keys that query token i of (nq, nk) sees
__device__ __forceinline__ int sees(int causal, int nq, int nk, long long i) {
  if (!causal) return nk;
  const long long n = i + 1 + nk - nq;
  return static_cast<int>(n < 0 ? 0 : (n > nk ? nk : n));
}

// items of a sequence with at least c chunks (c = 0: all of them); they are its last ones
__device__ __forceinline__ int items_from(int causal, int G, int nq, int nk, int c) {
  const long long rows = static_cast<long long>(nq) * G;
  const int n = static_cast<int>((rows + kItemRows - 1) / kItemRows);
  if (c == 0) return n;
  const long long key = static_cast<long long>(c - 1) * kTile;  // the first key of chunk c - 1 must be seen
  if (key >= nk) return 0;
  if (!causal) return n;
  const long long token = key - (nk - nq);  // the first token that sees it
  return token <= 0 ? n : n - static_cast<int>((token * G) / kItemRows);
}

// The item of rank `rank` in the order of decreasing chunks, by one warp. lens: (nq, nk) per sequence.
__device__ __forceinline__ Item find_item(const PromptArgs& p, const int2* lens, int G, int rank) {
  const int lane = threadIdx.x & 31;
  auto count = [&](int c) {
    int n = 0;
    for (int b = lane; b < p.B; b += 32) n += items_from(p.causal, G, lens[b].x, lens[b].y, c);
    return static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(n)));
  };
  Item it;
  it.b = -1;
  if (rank >= count(0)) return it;
  int lo = 0, hi = static_cast<int>((p.kv_rows + kTile - 1) / kTile) + 1;  // count(lo) > rank >= count(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (count(mid) > rank) lo = mid;
    else hi = mid;
  }
  int left = rank - count(lo + 1);  // among the items with exactly lo chunks, by sequence
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int b = b0 + lane;
    int from = 0, n = 0;
    if (b < p.B) {
      const int all = items_from(p.causal, G, lens[b].x, lens[b].y, 0);
      const int ge = items_from(p.causal, G, lens[b].x, lens[b].y, lo);
      from = all - ge;
      n = ge - items_from(p.causal, G, lens[b].x, lens[b].y, lo + 1);
      if (!p.causal) from = 0;
    }
    int before = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += up;
    }
    const int total = __shfl_sync(0xffffffffu, before, 31);
    before -= n;
    if (left < total) {
      const uint32_t mine = __ballot_sync(0xffffffffu, left >= before && left < before + n);
      const int src = __ffs(mine) - 1;
      const int t = from + left - before;
      it.b = b0 + src;
      it.row0 = static_cast<long long>(__shfl_sync(0xffffffffu, t, src)) * kItemRows;
      it.nq = lens[it.b].x;
      it.nk = lens[it.b].y;
      it.q0 = p.q_offsets[it.b];
      it.k0 = p.kv_offsets[it.b];
      return it;
    }
    left -= total;
  }
  return it;
}

template <bool BF>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const PromptArgs p, const __grid_constant__ Maps maps) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = p.n_heads / p.n_kv_heads;
  const int kvh = static_cast<int>(blockIdx.x % static_cast<unsigned>(p.n_kv_heads));
  const int rank = static_cast<int>(blockIdx.x / static_cast<unsigned>(p.n_kv_heads));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBar);
  uint64_t* full = bars;         // [5] a stage's chunk is there
  uint64_t* empty = bars + 5;    // [5] the MMAs that read it are done
  uint64_t* gfull = bars + 10;   // [3] a V chunk to be guarded has landed
  uint64_t* gdone = bars + 13;   // [3] and is guarded (waited for in place of `full`)
  uint64_t* qfull = bars + 16;   // [2] a tile's queries are there
  uint64_t* sfull = bars + 18;   // [2] S of a chunk in tensor memory
  uint64_t* pfull = bars + 20;   // [2][2] P of half a chunk written over it
  uint64_t* odone = bars + 24;   // [2] every P V of the tile done
  uint64_t* drain = bars + 26;   // every MMA done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* wild = reinterpret_cast<volatile int*>(tmem_slot + 2);  // a guarded value was not finite
  Item* item_slot = reinterpret_cast<Item*>(smem);  // before the queries
  if ((smem_addr(smem) & 1023u) != 0u) {  // the swizzled operands need a 1024-byte aligned base
    if (tid == 0) set_status(p.status, kStatusDeviceArg);
    return;
  }

  // ---- which item
  int2* lens = reinterpret_cast<int2*>(smem + kOffRing);
  for (int b = tid; b < p.B; b += kThreads) {
    const long long q0 = p.q_offsets[b], q1 = p.q_offsets[b + 1], k0 = p.kv_offsets[b], k1 = p.kv_offsets[b + 1];
    const bool good = q0 >= 0 && q1 >= q0 && q1 <= p.q_rows && k0 >= 0 && k1 >= k0 && k1 <= p.kv_rows;
    if (!good && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    lens[b] = good ? make_int2(static_cast<int>(q1 - q0), static_cast<int>(k1 - k0)) : make_int2(0, 0);
  }
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < kMaxGuarded; ++i) {
      mbar_init(gfull + i, 1);
      mbar_init(gdone + i, 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(qfull + i, 4);
      mbar_init(sfull + i, 1);
      mbar_init(pfull + 2 * i, 4);
      mbar_init(pfull + 2 * i + 1, 4);
      mbar_init(odone + i, 1);
    }
    mbar_init(drain, 1);
    *abort = 0;
    *wild = 0;
  }
  __syncthreads();
  if (warp == 0) {
    const Item found = find_item(p, lens, G, rank);
    if (lane == 0) *item_slot = found;
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_proxy_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const Item it = *item_slot;
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
  __syncthreads();  // the queries go where the item lies
  const long long rows = static_cast<long long>(it.nq) * G;
  int n[2] = {0, 0};  // chunks of each tile
  if (it.b >= 0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const long long first = it.row0 + t * kTile;
      if (first < rows) {
        const long long last = min(first + kTile, rows) - 1;
        n[t] = (sees(p.causal, it.nq, it.nk, last / G) + kTile - 1) / kTile;
      }
    }
  }
  const int n_all = max(n[0], n[1]);
  // chunks from here on are seen in part by some row of the item
  const int guard0 = it.b >= 0 ? sees(p.causal, it.nq, it.nk, it.row0 / G) / kTile : 0;

  if (it.b < 0) {
    // nothing: more blocks than items
  } else if (warp >= kMmaWarp) {
  leave_registers<88>();  // of 3 x 168 a lane at launch; the softmax warpgroups take 2 x 208
  if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs
    if (lane == 0) {
      const uint32_t id_s = idesc_16(BF, kTile, kTile, false), id_o = idesc_16(BF, kTile, kD, true);
      const uint32_t ring = smem_addr(smem + kOffRing), q = smem_addr(smem);
      bool ok = true;
      // the guarded chunks are the last three V chunks at most: no later chunk takes their stages
      auto stage_bar = [&](int c, uint32_t& parity) {
        const bool guarded = (c & 1) && (c >> 1) >= guard0;
        parity = guarded ? 0 : (c / kStages) & 1;
        return guarded ? gdone + ((c >> 1) - guard0) : full + c % kStages;
      };
      auto test_stage = [&](int c) {
        uint32_t parity;
        uint64_t* bar = stage_bar(c, parity);
        return test_bar(bar, parity);
      };
      auto need_stage = [&](int c, uint32_t there) {
        uint32_t parity;
        uint64_t* bar = stage_bar(c, parity);
        ok = ok && (there || wait_or_abort(bar, parity, p.status, abort));
      };
      uint32_t k_there = 0, v_there = 0, p_there[2][2] = {{0, 0}, {0, 0}};  // tested already
#pragma unroll 1
      for (int j = 0; j <= n_all && ok; ++j) {  // per tile: P V of chunk j - 1, then S of chunk j
        const uint32_t vb = ring + ((2 * j + 2 * kStages - 1) % kStages) * kStageBytes, kb = ring + ((2 * j) % kStages) * kStageBytes;
        if (j > 0) need_stage(2 * j - 1, v_there);
        if (j < n_all) need_stage(2 * j, k_there);
        v_there = k_there = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t s_at = tmem + kColS + t * kTile, o_at = tmem + kColO + t * kTile;
          if (!ok) break;
          if (j > 0 && j <= n[t]) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {  // the keys' first 64, whose weights are there first
              ok = p_there[t][half] || wait_or_abort(pfull + 2 * t + half, (j - 1) & 1, p.status, abort);
              if (!ok) break;
              tc_fence_after();
              if (half == 0 && !p_there[t][1]) p_there[t][1] = test_bar(pfull + 2 * t + 1, (j - 1) & 1);
#pragma unroll
              for (int k = 4 * half; k < 4 * half + 4; ++k)
                umma_f16_ta(o_at, s_at + k * 8, sw128_desc_mn(vb + k * 2048, 16384, 1024), id_o, j > 1 || k > 0 ? 1u : 0u);
            }
            if (!ok) break;
            p_there[t][0] = p_there[t][1] = 0;
            if (j == n[t]) umma_commit(odone + t);
          }
          if (j < n[t]) {
            if (j == 0) ok = wait_or_abort(qfull + t, 0, p.status, abort);
            if (!ok) break;
            tc_fence_after();
            // the other tile's weights: of chunk j - 1 for tile 1, of chunk j for tile 0 (there after its S)
            const int pj = t == 0 ? j - 1 : j;
            if (pj >= 0 && pj < n[t ^ 1]) {
              p_there[t ^ 1][0] = test_bar(pfull + 2 * (t ^ 1), pj & 1);
              p_there[t ^ 1][1] = test_bar(pfull + 2 * (t ^ 1) + 1, pj & 1);
            }
            if (t == 1 && j < n_all) {
              v_there = test_stage(2 * j + 1);
              if (j + 1 < n_all) k_there = test_stage(2 * j + 2);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t off = (k >> 2) * 16384 + (k & 3) * 32;
              umma_f16(s_at, sw128_desc(q + t * kStageBytes + off), sw128_desc(kb + off), id_s, k > 0 ? 1u : 0u);
            }
            umma_commit(sfull + t);
          }
        }
        if (!ok) break;
        if (j > 0) umma_commit(empty + (2 * j - 1) % kStages);
        if (j < n_all) umma_commit(empty + (2 * j) % kStages);
      }
      umma_commit(drain);
      mbar_wait(drain, 0, p.status);
    }
    __syncwarp();
  } else if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- loads
    if (lane == 0) {
      int c = 0;
      bool ok = true;
#pragma unroll 1
      for (; c < 2 * n_all; ++c) {
        const int s = c % kStages, j = c >> 1;
        if (c >= kStages) ok = wait_or_abort(empty + s, (c / kStages - 1) & 1, p.status, abort);
        if (!ok) break;
        uint64_t* bar = (c & 1) && j >= guard0 ? gfull + (j - guard0) : full + s;
        unsigned char* dst = smem + kOffRing + s * kStageBytes;
        const int row = static_cast<int>(it.k0 + static_cast<long long>(j) * kTile);
        mbar_arrive_expect_tx(bar, kStageBytes);
        tma_load_head(dst, (c & 1) ? &maps.v : &maps.k, 0, kvh, row, bar);
        tma_load_head(dst + kStageBytes / 2, (c & 1) ? &maps.v : &maps.k, 64, kvh, row, bar);
      }
      if (!ok)  // what is on its way lands before the CTA leaves
        for (int d = max(0, c - kStages); d < c; ++d) {
          const int j = d >> 1;
          if ((d & 1) && j >= guard0) mbar_wait(gfull + (j - guard0), 0, p.status);
          else mbar_wait(full + d % kStages, (d / kStages) & 1, p.status);
        }
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- guard
#pragma unroll 1
    for (int j = guard0; j < n_all; ++j) {
      if (!wait_or_abort(gfull + (j - guard0), 0, p.status, abort)) break;
      const int s = (2 * j + 1) % kStages;
      unsigned char* v = smem + kOffRing + s * kStageBytes;
      const int in_range = it.nk - j * kTile;  // rows of the sequence in this chunk
      uint32_t bad = 0;
#pragma unroll 4
      for (int r = (warp & 1) * 2 + (lane >> 4); r < kTile; r += 4) {
        uint4* u = reinterpret_cast<uint4*>(v + tile_off(r, lane & 15));
        if (r >= in_range) {
          *u = make_uint4(0u, 0u, 0u, 0u);
        } else {
          uint4 x = *u;
          const uint32_t f[4] = {not_finite2<BF>(x.x), not_finite2<BF>(x.y), not_finite2<BF>(x.z), not_finite2<BF>(x.w)};
          if ((f[0] | f[1] | f[2] | f[3]) != 0u) {
            bad = 1u;
            uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] &= ~((f[i] >> 15) * 0xffffu);  // 16-bit lanes of ones where flagged
            *u = make_uint4(y[0], y[1], y[2], y[3]);
          }
        }
      }
      if (bad) *wild = 1;
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(gdone + (j - guard0));
    }
  }
  } else {
    // ---------------------------------------------------------------- softmax of tile t
    take_registers<208>();
    const int t = warp >> 2;
    const int r = tid & (kTile - 1);  // this thread's row: tensor-memory lane r
    const long long first = it.row0 + t * kTile;
    const int valid = static_cast<int>(max(0ll, min(static_cast<long long>(kTile), rows - first)));
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    unsigned char* qt = smem + t * kStageBytes;
    const long long token0 = first / G;
    const uint32_t head0 = static_cast<uint32_t>(first - token0 * G);  // row i of the tile: (head0 + i) / G tokens on
    {
      const uint16_t* q = static_cast<const uint16_t*>(p.q);
      const int u = tid & 15;
#pragma unroll
      for (int i = 0; i < kTile / 8; ++i) {  // all on their way at once
        const int at = ((tid & (kTile - 1)) >> 4) + 8 * i;
        const bool there = at < valid;
        const uint32_t g = head0 + (there ? at : 0), on = g / static_cast<uint32_t>(G);
        copy16(smem_addr(qt + tile_off(at, u)), q + (it.q0 + token0 + on) * p.q_stride + (kvh * G + g - on * G) * kD + u * 8, there);
      }
      cp_async_commit();
      cp_async_wait<0>();
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(qfull + t);
    }
    const bool mine = r < valid;
    const uint32_t my_g = head0 + (mine ? r : 0), my_on = my_g / static_cast<uint32_t>(G);
    const long long token = token0 + my_on;
    const int head = kvh * G + static_cast<int>(my_g - my_on * G);
    const int see = mine ? sees(p.causal, it.nq, it.nk, token) : 0;
    const int see_all = valid > 0 ? sees(p.causal, it.nq, it.nk, token0) : 0;  // every row of the tile sees these
    const uint32_t scol = tmem + lanes + kColS + t * kTile, ocol = tmem + lanes + kColO + t * kTile;
    float m = -CUDART_INF_F, l = 0.f;  // in units of log2; m may lag behind the maximum by up to 8
    bool ok = true;
#pragma unroll 1
    for (int j = 0; j < n[t]; ++j) {
      ok = wait_or_abort(sfull + t, j & 1, p.status, abort);
      if (!ok) break;
      tc_fence_after();
      uint32_t raw[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32_issue(scol + 32 * i, raw[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_wait_ld32(raw[i]);
      if ((j + 1) * kTile > see_all) {
        const int left = see - j * kTile;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (32 * i + e >= left) raw[i][e] = 0xff800000u;  // -infinity
      }
      float mx[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mx[i] = __uint_as_float(raw[i][0]);
#pragma unroll
        for (int e = 1; e < 31; e += 2) mx[i] = max3(mx[i], __uint_as_float(raw[i][e]), __uint_as_float(raw[i][e + 1]));
        mx[i] = fmaxf(mx[i], __uint_as_float(raw[i][31]));
      }
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * kScaleLog2;
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float m_new = fmaxf(m, top);
        const float alpha = m_new == m ? 1.f : exp2_fast(m - m_new);
        m = m_new;
        l *= alpha;
        if (j > 0) {
#pragma unroll 1
          for (int c = 0; c < kD; c += 32) {
            uint32_t o[32];
            tmem_ld32_issue(ocol + c, o);
            tmem_wait_ld32(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st32(ocol + c, o);
          }
        }
      }
      const float nm = m == -CUDART_INF_F ? 0.f : -m;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // 64 keys: 32 columns of P
        uint32_t pk[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          float a = __uint_as_float(raw[2 * i + (e >> 4)][2 * (e & 15)]), b = __uint_as_float(raw[2 * i + (e >> 4)][2 * (e & 15) + 1]);
          fma2(a, b, kScaleLog2, nm);
          a = exp2_fast(a);
          b = exp2_fast(b);
          if (e & 1) add2(sum[2], sum[3], a, b);
          else add2(sum[0], sum[1], a, b);
          pk[e] = pack16<BF>(a, b);
        }
        tmem_st32(scol + 32 * i, pk);
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pfull + 2 * t + i);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    // ---- output
    if (ok && n[t] > 0) ok = wait_or_abort(odone + t, 0, p.status, abort);
    if (ok) {
      tc_fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      uint16_t* out = static_cast<uint16_t*>(p.out) + ((it.q0 + token) * p.n_heads + head) * kD;
#pragma unroll 1
      for (int c = 0; c < kD; c += 32) {
        uint32_t o[32];
        if (n[t] > 0) {
          tmem_ld32_issue(ocol + c, o);
          tmem_wait_ld32(o);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;
        }
        if (mine) {
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = l == 0.f ? 0.f : __uint_as_float(o[e]) * inv;
          if (*wild) {  // values that the guards took out, for the rows that see them
            for (int k = guard0 * kTile; k < see; ++k) {
              const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v) + (it.k0 + k) * p.kv_stride + kvh * kD + c);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const uint32_t f = not_finite2<BF>(v[e]);
                const float2 y = unpack16<BF>(v[e]);
                if (f & 0x8000u) x[2 * e] += y.x;
                if (f & 0x80000000u) x[2 * e + 1] += y.y;
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(out + c + 8 * e) =
                make_uint4(pack16<BF>(x[8 * e], x[8 * e + 1]), pack16<BF>(x[8 * e + 2], x[8 * e + 3]),
                           pack16<BF>(x[8 * e + 4], x[8 * e + 5]), pack16<BF>(x[8 * e + 6], x[8 * e + 7]));
        }
      }
      if (mine && p.lse != nullptr)
        p.lse[head * p.q_rows + it.q0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

}  // namespace

cudaError_t launch_prompt_attention(const PromptArgs& a, int dtype, cudaStream_t stream) {
  const long long G = a.n_heads / a.n_kv_heads;
  // at most this many items: every sequence rounds up once
  const long long blocks = (a.q_rows * G / kItemRows + a.B) * a.n_kv_heads;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  Maps maps{};
  if (a.kv_rows > 0 && (!encode_kv_map(&maps.k, a.k, a.kv_rows, a.n_kv_heads, a.kv_stride * 2, 2, kTile) ||
                        !encode_kv_map(&maps.v, a.v, a.kv_rows, a.n_kv_heads, a.kv_stride * 2, 2, kTile)))
    return cudaErrorInvalidValue;
  const void* fn = dtype == FSX_BF16 ? reinterpret_cast<const void*>(&prompt_kernel<true>)
                                     : reinterpret_cast<const void*>(&prompt_kernel<false>);
  const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<PromptArgs*>(&a), &maps};
  return launch_ex(fn, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), kSmem, stream, false, args);
}

}  // namespace fsx
