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
// Warps 0-3, 4-7: softmax of tile 0, 1 (they also write the outputs); warp 8 issues
// MMAs; warp 9 loads K and V chunks by TMA into a ring of five 32 KB stages (K0 V0 K1 V1 ...); warps
// 10-11 load the queries and guard the V chunks that some row of the item sees only in part (the diagonal, the end of the
// sequence): a masked weight is 0, but 0 times an infinity or NaN is not, so rows past the sequence become
// zeros, and values that are not finite too; such a value is added to the rows that do see it at the end.
//
// A CTA works through up to 36 items, one CTA per SM: the next item's first loads and scores run under
// the last one's outputs (an item of its own CTA spent 13,000 cycles before its first chunk and 4,000 after
// the last; a chunk takes about 2,600). Items go longest first, mirrored from round to round; the rank of an item
// in the order of chunks is found by counting (the host knows no lengths).
//
// Measured: 8192 tokens, 32 heads over 8, causal: 323 to 326 us in a graph, 1690 TFLOP/s (0.89 of the library's matrix product), 368 us
// call by call on changing inputs.
// A chunk of two tiles takes 2,600 cycles, of which its MMAs need 2,048 (tensor pipe 74 % active over the kernel) and its
// exponentials 1,024. 16 prompts of 139 to 452 tokens: 32 us, where items of one to four chunks pay 5,000 cycles each for
// their start and outputs. Four chunks of 123 to 511 tokens behind 1277 to 1936 rows: 48 us; 160 items for 152 SMs, so
// eight CTAs do two.
// Outputs leave by bulk copies, a warp's 32 rows each: 16-byte stores of the same rows held a warp for 1,900 cycles.
//
// Stages are released by the softmax threads (S of chunk j there: K of j and V of j - 1 are free).
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
constexpr int kMmaWarp = 8, kLoadWarp = 9, kAuxWarp = 10;  // two of them
constexpr int kThreads = 384;           // three warpgroups: 168 registers a thread at launch
constexpr int kWarps = kThreads / 32;
constexpr int kMaxRounds = 36;          // items of a CTA
constexpr int kGuarded = 4;             // ring of guarded chunks: no more than 3 V chunks lie in the stages
constexpr uint32_t kColS = 0, kColO = 256;
constexpr int kOffRing = 2 * kStageBytes;  // the two Q tiles lie in front
constexpr int kOffBar = kOffRing + kStages * kStageBytes;
// full[5], empty[5], gfull[4], qfull[2], qempty[2], sfull[2], pfull[2][2], odone[2], oread[2], drain
constexpr int kNumBars = 29;
constexpr int kOffItems = kOffBar + kNumBars * 8 + 32;

struct Maps {
  CUtensorMap k, v;
  CUtensorMap q;    // if G divides a tile: [64 columns, heads, rows, 2 blocks], a box is a tile
  CUtensorMap out;  // if G divides a warp's 32 rows: the same, a box is 32 rows
};

// Rows (token G + head) are counted in 32 bits: 2^31 rows of queries would be 550 GB. Each 64-bit division is some
// hundred instructions, and the code of all roles has to stay near.
struct Item {
  long long q0, k0;  // first query row, first key row of the sequence
  uint32_t row0;     // first packed row of the item
  int nq, nk;
  int n[2];          // chunks of each tile
  int guard0;        // chunks from here on are seen in part by some row of the item
  int kvh;           // -1: none
  int pad;
};
constexpr int kSmem = kOffItems + kMaxRounds * static_cast<int>(sizeof(Item));
static_assert(kSmem <= 227 * 1024, "shared memory");
struct Sequence {
  long long q0, k0;
  int nq, nk;
};
static_assert(kMaxSequences * sizeof(Sequence) <= kStages * kStageBytes, "the sequences lie in the ring before it is used");

// keys that query token i of (nq, nk) sees
__device__ __forceinline__ int sees(int causal, int nq, int nk, int i) {
  return causal ? max(0, min(nk, i + 1 + nk - nq)) : nk;
}

// Byte offset of 16-byte unit u of row r of a warp's 32 output rows: two swizzled blocks of 64 columns, 4 KB apart
__device__ __forceinline__ uint32_t out_off(int r, int u) {
  return static_cast<uint32_t>((u >> 3) * 4096 + r * 128 + (((u & 7) ^ (r & 7)) << 4));
}

// items of a sequence with at least c chunks (c = 0: all of them); they are its last ones
__device__ __forceinline__ int items_from(int causal, uint32_t G, int nq, int nk, int c) {
  const int n = static_cast<int>((nq * G + kItemRows - 1) / kItemRows);
  if (c == 0) return n;
  const int key = (c - 1) * kTile;  // the first key of chunk c - 1 must be seen
  if (key >= nk) return 0;
  const int token = key - (nk - nq);  // the first token that sees it
  return !causal || token <= 0 ? n : n - static_cast<int>(token * G / kItemRows);
}

// The item of rank `rank` by one warp; in the order of decreasing chunks if `ordered`, else by sequence.
// False: there are not so many.
__device__ __forceinline__ bool find_item(const PromptArgs& p, const Sequence* seqs, uint32_t G, int rank, bool ordered, Item& it) {
  const int lane = threadIdx.x & 31;
  if (p.B == 1 && ordered) {  // the last items have the most chunks
    const int n = items_from(p.causal, G, seqs[0].nq, seqs[0].nk, 0);
    if (rank >= n) return false;
    rank = n - 1 - rank;
    ordered = false;
  }
  int level = 0, left = rank;  // among the items with exactly `level` chunks (all of them if not ordered), by sequence
  if (ordered) {
    auto count = [&](int c) {
      int n = 0;
      for (int b = lane; b < p.B; b += 32) n += items_from(p.causal, G, seqs[b].nq, seqs[b].nk, c);
      return static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(n)));
    };
    if (rank >= count(0)) return false;
    int most = 0;
    for (int b = lane; b < p.B; b += 32) most = max(most, seqs[b].nk);
    int hi = (__reduce_max_sync(0xffffffffu, most) + kTile - 1) / kTile + 1;  // count(level) > rank >= count(hi)
    while (hi - level > 1) {
      const int mid = (level + hi) >> 1;
      if (count(mid) > rank) level = mid;
      else hi = mid;
    }
    left -= count(level + 1);
  }
  for (int b0 = 0; b0 < p.B; b0 += 32) {
    const int b = b0 + lane;
    int from = 0, n = 0;
    if (b < p.B) {
      n = items_from(p.causal, G, seqs[b].nq, seqs[b].nk, 0);
      if (ordered) {
        const int ge = items_from(p.causal, G, seqs[b].nq, seqs[b].nk, level);
        from = p.causal ? n - ge : 0;
        n = ge - items_from(p.causal, G, seqs[b].nq, seqs[b].nk, level + 1);
      }
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
      const int src = __ffs(__ballot_sync(0xffffffffu, left >= before && left < before + n)) - 1;
      const int t = from + left - before;
      const int found = b0 + src;
      it.row0 = static_cast<uint32_t>(__shfl_sync(0xffffffffu, t, src)) * kItemRows;
      it.nq = seqs[found].nq;
      it.nk = seqs[found].nk;
      it.q0 = seqs[found].q0;
      it.k0 = seqs[found].k0;
      const uint32_t rows = it.nq * G;
      for (int i = 0; i < 2; ++i) {
        const uint32_t first = it.row0 + i * kTile;
        it.n[i] = first < rows ? (sees(p.causal, it.nq, it.nk, (min(first + kTile, rows) - 1) / G) + kTile - 1) / kTile : 0;
      }
      it.guard0 = sees(p.causal, it.nq, it.nk, it.row0 / G) / kTile;
      return true;
    }
    left -= total;
  }
  return false;
}

// two stages on in the ring
__device__ __forceinline__ void two_on(uint32_t& stage, uint32_t& phase) {
  stage += 2;
  if (stage >= kStages) {
    stage -= kStages;
    phase ^= 1u;
  }
}

// token and head of the group of a packed row, two rows on at a time; `two`: 2 / G and 2 % G
struct RowWalk {
  uint32_t token, head;
  __device__ __forceinline__ RowWalk(uint32_t row, uint32_t G, uint2) : token(row / G), head(row - token * G) {}
  __device__ __forceinline__ void next(uint32_t G, uint2 two) {
    token += two.x;
    head += two.y;
    if (head >= G) {
      head -= G;
      ++token;
    }
  }
};

template <bool BF>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const PromptArgs p, const int rounds, const __grid_constant__ Maps maps) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t G = static_cast<uint32_t>(p.n_heads) / static_cast<uint32_t>(p.n_kv_heads);
  const uint2 two = make_uint2(2 / G, 2 % G);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBar);
  uint64_t* full = bars;         // [5] a stage's chunk is there (and guarded)
  uint64_t* empty = bars + 5;    // [5] the MMAs that read it are done
  uint64_t* gfull = bars + 10;   // [4] a V chunk to be guarded has landed
  uint64_t* qfull = bars + 14;   // [2] a tile's queries are there
  uint64_t* qempty = bars + 16;  // [2] every S of the tile's item is done
  uint64_t* sfull = bars + 18;   // [2] S of a chunk in tensor memory
  uint64_t* pfull = bars + 20;   // [2][2] P of half a chunk written over it
  uint64_t* odone = bars + 24;   // [2] every P V of the tile's item done
  uint64_t* oread = bars + 26;   // [2] and its O read
  uint64_t* drain = bars + 28;   // every MMA done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* wild = reinterpret_cast<volatile int*>(tmem_slot + 2);  // [4]: item + 1 with a guarded value that is not finite
  Item* items = reinterpret_cast<Item*>(smem + kOffItems);
  if ((smem_addr(smem) & 1023u) != 0u) {  // the swizzled operands need a 1024-byte aligned base
    if (tid == 0) set_status(p.status, kStatusDeviceArg);
    return;
  }

  // ---- the CTA's items
  Sequence* seqs = reinterpret_cast<Sequence*>(smem + kOffRing);
  for (int b = tid; b < p.B; b += kThreads) {
    const long long q0 = p.q_offsets[b], q1 = p.q_offsets[b + 1], k0 = p.kv_offsets[b], k1 = p.kv_offsets[b + 1];
    const bool good = q0 >= 0 && q1 >= q0 && q1 <= p.q_rows && k0 >= 0 && k1 >= k0 && k1 <= p.kv_rows;
    if (!good && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    seqs[b] = good ? Sequence{q0, k0, static_cast<int>(q1 - q0), static_cast<int>(k1 - k0)} : Sequence{0, 0, 0, 0};
  }
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full + i, 2);
      mbar_init(empty + i, 4);
    }
    for (int i = 0; i < kGuarded; ++i) mbar_init(gfull + i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(qfull + i, 2);
      mbar_init(qempty + i, 1);
      mbar_init(sfull + i, 1);
      mbar_init(pfull + 2 * i, 4);
      mbar_init(pfull + 2 * i + 1, 4);
      mbar_init(odone + i, 1);
      mbar_init(oread + i, 4);
    }
    mbar_init(drain, 1);
    *abort = 0;
    for (int i = 0; i < 4; ++i) wild[i] = 0;
  }
  __syncthreads();
#pragma unroll 1
  for (int k = warp; k < rounds; k += kWarps) {
    const unsigned slot = k * gridDim.x + ((k & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    Item it{};
    const int rank = static_cast<int>(slot / static_cast<unsigned>(p.n_kv_heads));
    it.kvh = find_item(p, seqs, G, rank, rounds > 1, it) ? static_cast<int>(slot - rank * static_cast<unsigned>(p.n_kv_heads)) : -1;
    if (lane == 0) items[k] = it;
  }
  if (warp == kMmaWarp) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_proxy_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
  // Counts that run through the CTA's items: c-th chunk of the ring (K0 V0 K1 ...), g-th guarded chunk, and per
  // tile the chunks and the items with chunks. A barrier's phase is the count of its uses.

  if (warp >= kMmaWarp) {
  leave_registers<88>();  // of 3 x 168 a lane at launch; the softmax warpgroups take 2 x 208
  if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs: the whole warp waits, one lane issues
    const bool leader = elect_lane();
    const uint32_t id_s = idesc_16(BF, kTile, kTile, false), id_o = idesc_16(BF, kTile, kD, true);
    const uint32_t ring = smem_addr(smem + kOffRing);
    // descriptors change by their addresses alone
    const uint64_t q_desc = sw128_desc(smem_addr(smem)), k_desc = sw128_desc(ring), v_desc = sw128_desc_mn(ring, 16384, 1024);
    bool ok = true;
    uint32_t sk = 0, pk = 0, sv = 1, pv = 0;              // stage and phase of the next K and V
    uint32_t done0 = 0, done1 = 0, uses0 = 0, uses1 = 0;  // chunks and items of the tiles before this item
#pragma unroll 1
    for (int i = 0; i < rounds && ok; ++i) {
      const Item it = items[i];
      if (it.kvh < 0) continue;
      const int n_all = max(it.n[0], it.n[1]);
#pragma unroll 1
      for (int j = 0; j <= n_all && ok; ++j) {  // per tile: P V of chunk j - 1, then S of chunk j
        const uint64_t kd = k_desc + sk * (kStageBytes >> 4), vd = v_desc + sv * (kStageBytes >> 4);
        if (j > 0) ok = wait_or_abort(full + sv, pv, p.status, abort);
        if (ok && j < n_all) ok = wait_or_abort(full + sk, pk, p.status, abort);
        if (!ok) break;
#pragma unroll 1
        for (int t = 0; t < 2; ++t) {
          const int n = t ? it.n[1] : it.n[0];
          const uint32_t done = t ? done1 : done0, uses = t ? uses1 : uses0;
          const uint32_t s_at = tmem + kColS + t * kTile, o_at = tmem + kColO + t * kTile;
          if (j > 0 && j <= n) {
            const uint32_t parity = (done + j - 1) & 1;
            if (j == 1 && uses > 0) ok = wait_or_abort(oread + t, (uses - 1) & 1, p.status, abort);
            if (!ok) break;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {  // the keys' first 64, whose weights are there first
              ok = wait_or_abort(pfull + 2 * t + half, parity, p.status, abort);
              if (!ok) break;
              tc_fence_after();
              if (leader) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  umma_f16_ta(o_at, s_at + half * 32 + k * 8, vd + (half * 4 + k) * 128, id_o, j > 1 || half > 0 || k > 0 ? 1u : 0u);
              }
              __syncwarp();
            }
            if (!ok) break;
            if (leader && j == n) umma_commit(odone + t);
          }
          if (j < n) {
            if (j == 0) ok = wait_or_abort(qfull + t, uses & 1, p.status, abort);
            if (!ok) break;
            tc_fence_after();
            const uint64_t qd = q_desc + t * (kStageBytes >> 4);
            if (leader) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint32_t off = (k >> 2) * (16384 >> 4) + (k & 3) * 2;
                umma_f16(s_at, qd + off, kd + off, id_s, k > 0 ? 1u : 0u);
              }
              umma_commit(sfull + t);
            }
            __syncwarp();
          }
        }
        if (j > 0) two_on(sv, pv);
        if (j < n_all) two_on(sk, pk);
      }
      done0 += it.n[0];
      done1 += it.n[1];
      uses0 += it.n[0] > 0 ? 1 : 0;
      uses1 += it.n[1] > 0 ? 1 : 0;
    }
    if (leader) umma_commit(drain);
    __syncwarp();
    mbar_wait(drain, 0, p.status);
  } else if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- loads of K and V
    if (lane == 0) {
      int c = 0, g = 0;
      uint32_t guarded = 0;  // bit 0: the last chunk, bit 1: the one before, ...
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < rounds && ok; ++i) {
        const Item it = items[i];
        if (it.kvh < 0) continue;
        const int n_all = max(it.n[0], it.n[1]);
#pragma unroll 1
        for (int k = 0; k < 2 * n_all; ++k) {
          const int s = c % kStages, j = k >> 1;
          if (c >= kStages) ok = wait_or_abort(empty + s, (c / kStages - 1) & 1, p.status, abort);
          if (!ok) break;
          const bool guard = (k & 1) && j >= it.guard0;
          uint64_t* bar = guard ? gfull + g % kGuarded : full + s;
          mbar_arrive_expect_tx(bar, kStageBytes);
          if (!guard) mbar_arrive(bar);  // for the two guard warps
          tma_load_chunk(smem + kOffRing + s * kStageBytes, (k & 1) ? &maps.v : &maps.k,
                         static_cast<int>(it.k0 + static_cast<long long>(j) * kTile), 0, it.kvh, bar);
          guarded = guarded << 1 | (guard ? 1u : 0u);
          g += guard ? 1 : 0;
          ++c;
        }
      }
      // What is on its way lands before the CTA leaves, also where all loads were issued before another role gave up
      for (int d = c - 1; d >= 0 && d >= c - kStages; --d, guarded >>= 1) {
        if (guarded & 1u) {
          --g;
          mbar_wait(gfull + g % kGuarded, (g / kGuarded) & 1, p.status);
        } else {
          mbar_wait(full + d % kStages, (d / kStages) & 1, p.status);
        }
      }
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- queries and guarded chunks, half of the rows a warp
    const int side = warp - kAuxWarp;
    const bool by_tma = kTile % G == 0;
    uint32_t uses[2] = {0, 0};
    int c0 = 0, g = 0;
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < rounds && ok; ++i) {
      const Item it = items[i];
      if (it.kvh < 0) continue;
      const int n_all = max(it.n[0], it.n[1]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (it.n[t] > 0 && ok) {
          if (uses[t] > 0) ok = wait_or_abort(qempty + t, (uses[t] - 1) & 1, p.status, abort);
          if (ok && by_tma) {
            ++uses[t];
            if (lane == 0) {
              if (side == 0) {
                mbar_arrive_expect_tx(qfull + t, kStageBytes);
                tma_load_chunk(smem + t * kStageBytes, &maps.q, it.kvh * G, static_cast<int>(it.q0) + (it.row0 + t * kTile) / G, 0, qfull + t);
              } else {
                mbar_arrive(qfull + t);
              }
            }
          } else if (ok) {
            const int half = side * (kTile / 2), u = lane & 15;
            const uint16_t* q = static_cast<const uint16_t*>(p.q) + it.q0 * p.q_stride + it.kvh * G * kD + u * 8;
            const uint32_t rows = it.nq * G;
            uint32_t row = it.row0 + t * kTile + half + (lane >> 4);
            RowWalk at(row, G, two);
            const uint32_t dst = smem_addr(smem + t * kStageBytes);
#pragma unroll 2
            for (int r = half + (lane >> 4); r < half + kTile / 2; r += 2, row += 2, at.next(G, two)) {
              const bool there = row < rows;
              copy16(dst + tile_off(r, u), q + (there ? at.token * p.q_stride + at.head * kD : 0ll), there);
            }
          }
        }
        cp_async_commit();
      }
      if (!by_tma) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (t == 0) cp_async_wait<1>();
          else cp_async_wait<0>();
          if (it.n[t] > 0 && ok) {
            ++uses[t];
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(qfull + t);
          }
        }
      }
#pragma unroll 1
      for (int j = it.guard0; j < n_all && ok; ++j, ++g) {
        ok = wait_or_abort(gfull + g % kGuarded, (g / kGuarded) & 1, p.status, abort);
        if (!ok) break;
        const int s = (c0 + 2 * j + 1) % kStages;
        unsigned char* v = smem + kOffRing + s * kStageBytes;
        const int in_range = it.nk - j * kTile;  // rows of the sequence in this chunk
        // rows r, r + 8, ... lie 1024 bytes apart; a lane takes unit u of two such columns of rows
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          const int r = side * 4 + c * 2 + (lane >> 4);
          uint4* at = reinterpret_cast<uint4*>(v + tile_off(r, lane & 15));
          if (in_range < kTile) {  // the end of the sequence
#pragma unroll 1
            for (int k = 0; k < kTile / 8; ++k)
              if (r + 8 * k >= in_range) at[k * 64] = make_uint4(0u, 0u, 0u, 0u);
          }
          uint32_t bad = 0;
#pragma unroll 8
          for (int k = 0; k < kTile / 8; ++k) {
            const uint4 x = at[k * 64];
            bad |= not_finite2<BF>(x.x) | not_finite2<BF>(x.y) | not_finite2<BF>(x.z) | not_finite2<BF>(x.w);
          }
          if (bad != 0u) {
            wild[i & 3] = i + 1;
#pragma unroll 1
            for (int k = 0; k < kTile / 8; ++k) {
              uint32_t* w = reinterpret_cast<uint32_t*>(at + k * 64);
#pragma unroll 1
              for (int e = 0; e < 4; ++e) w[e] &= ~((not_finite2<BF>(w[e]) >> 15) * 0xffffu);  // 16-bit lanes of ones where flagged
            }
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(full + s);
      }
      c0 += 2 * n_all;
    }
    cp_async_wait<0>();
    if (by_tma && lane == 0)  // queries on their way land before the CTA leaves
      for (int t = 0; t < 2; ++t)
        if (uses[t] > 0) mbar_wait(qfull + t, (uses[t] - 1) & 1, p.status);
  }
  } else {
    // ---------------------------------------------------------------- softmax of tile t
    take_registers<208>();
    const int t = warp >> 2;
    const int r = tid & (kTile - 1);  // this thread's row: tensor-memory lane r
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t scol = tmem + lanes + kColS + t * kTile, ocol = tmem + lanes + kColO + t * kTile;
    bool ok = true;
    int c0 = 0;
    uint32_t done = 0, uses = 0;
#pragma unroll 1
    for (int i = 0; i < rounds && ok; ++i) {
    const Item it = items[i];
    if (it.kvh < 0) continue;
    const int n_all = max(it.n[0], it.n[1]);
    const int n = t == 0 ? it.n[0] : it.n[1];
    const uint32_t first = it.row0 + t * kTile;
    const bool mine = first + r < it.nq * G;
    const uint32_t row = first + (mine ? r : 0), token = row / G;
    const int head = it.kvh * G + (row - token * G);
    const int see = mine ? sees(p.causal, it.nq, it.nk, token) : 0;
    const int see_all = sees(p.causal, it.nq, it.nk, first / G);  // every row of the tile sees these
    float m = -CUDART_INF_F, l = 0.f;  // in units of log2; m may lag behind the maximum by up to 8
    uint32_t at_k = c0 % kStages;      // stage of the chunk's K
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
      ok = wait_or_abort(sfull + t, (done + j) & 1, p.status, abort);
      if (!ok) break;
      tc_fence_after();
      uint32_t raw[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32_issue(scol + 32 * i, raw[i]);
      if (lane == 0) {
        if (t == 1 || j >= it.n[1]) {  // S of both tiles: K of chunk j and V of j - 1 are free
          if (j > 0) mbar_arrive(empty + (at_k == 0 ? kStages - 1 : at_k - 1));
          if (j + 1 != it.n[0]) mbar_arrive(empty + at_k);  // tile 0 writes its output through its last one
        }
        if (warp == 4 * t && j == n - 1) mbar_arrive(qempty + t);
      }
      at_k = at_k + 2 >= kStages ? at_k + 2 - kStages : at_k + 2;
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
    // ---- output: through the stage of the tile's last K (tile 0) or V (tile 1) chunk, so that rows are written whole
    if (ok && n > 0) ok = wait_or_abort(odone + t, uses & 1, p.status, abort);
    if (ok) {
      tc_fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int stage = (c0 + (t == 0 ? 2 * n - 2 : 2 * n - 1)) % kStages;
      unsigned char* staged = smem + kOffRing + (n > 0 ? stage : 0) * kStageBytes + (warp & 3) * 8192;  // this warp's 32 rows
      const bool found = wild[i & 3] == i + 1;
      uint16_t* out = static_cast<uint16_t*>(p.out) + (it.q0 * p.n_heads + it.kvh * G) * kD + (lane & 15) * 8;
      if (n > 0) {
#pragma unroll 1
        for (int c = 0; c < kD; c += 32) {
          uint32_t o[32];
          tmem_ld32_issue(ocol + c, o);
          tmem_wait_ld32(o);
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]) * inv;  // zeros where no weight is
          if (found) {  // values that the guard took out, for the rows that see them
#pragma unroll 1
            for (int k = it.guard0 * kTile; k < see; ++k) {
              const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v) + (it.k0 + k) * p.kv_stride + it.kvh * kD + c);
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
            *reinterpret_cast<uint4*>(staged + out_off(lane, c / 8 + e)) =
                make_uint4(pack16<BF>(x[8 * e], x[8 * e + 1]), pack16<BF>(x[8 * e + 2], x[8 * e + 3]),
                           pack16<BF>(x[8 * e + 4], x[8 * e + 5]), pack16<BF>(x[8 * e + 6], x[8 * e + 7]));
        }
        tc_fence_before();
        fence_proxy_async();  // the next copy into the stage comes behind these writes
        __syncwarp();
        if (lane == 0) mbar_arrive(oread + t);
      }
      const int rows = static_cast<int>(it.nq * G - first);
      int r2 = (r & ~31) + (lane >> 4);  // this warp's 32 rows, two at a time
      const bool by_tma = n > 0 && 32 % G == 0 && (r & ~31) + 32 <= rows;
      if (by_tma) {
        if (lane == 0) {
          tma_store_chunk(&maps.out, staged, it.kvh * G, static_cast<int>(it.q0) + (first + (r & ~31)) / G, 0);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
      } else {
        RowWalk at(first + r2, G, two);
        out += (static_cast<long long>(at.token) * p.n_heads + at.head) * kD;
        const int step = (two.x * p.n_heads + two.y) * kD, wrap = (p.n_heads - static_cast<int>(G)) * kD;
#pragma unroll 1
        for (int k = 0; k < 16; k += 8) {  // eight rows are read, then written: a store may not be passed by a read
          uint4 x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            x[e] = n > 0 ? *reinterpret_cast<const uint4*>(staged + out_off((r2 + 2 * e) & 31, lane & 15)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int e = 0; e < 8; ++e, r2 += 2) {
            if (r2 < rows) *reinterpret_cast<uint4*>(out) = x[e];
            out += step;
            at.head += two.y;
            if (at.head >= G) {
              at.head -= G;
              out += wrap;
            }
          }
        }
      }
      if (mine && p.lse != nullptr)
        p.lse[head * p.q_rows + it.q0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
      if (n > 0) {
        __syncwarp();
        if (lane == 0) {
          if (by_tma) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          mbar_arrive(empty + stage);
          if (t == 0 && it.n[1] < n_all) mbar_arrive(empty + (c0 + 2 * n_all - 1) % kStages);  // there is no tile 1
        }
        __syncwarp();
      }
    }
    c0 += 2 * n_all;
    done += n;
    uses += n > 0 ? 1 : 0;
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
  // at most this many items, which the caller keeps below 2^31: every sequence rounds up once
  const long long items = (a.q_rows * G / kItemRows + a.B) * a.n_kv_heads;
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  // one CTA per SM; beyond kMaxRounds items each, further waves of CTAs
  const long long waves = (items + static_cast<long long>(sms) * kMaxRounds - 1) / (static_cast<long long>(sms) * kMaxRounds);
  const long long grid = items < waves * sms ? items : waves * sms;
  int rounds = static_cast<int>((items + grid - 1) / grid);
  Maps maps{};
  if (kTile % G == 0 && !encode_q_map(&maps.q, a.q, a.q_rows, a.n_heads, a.q_stride * 2, static_cast<int>(G), kTile))
    return cudaErrorInvalidValue;
  if (32 % G == 0 && !encode_q_map(&maps.out, a.out, a.q_rows, a.n_heads, static_cast<long long>(a.n_heads) * kD * 2, static_cast<int>(G), 32))
    return cudaErrorInvalidValue;
  if (a.kv_rows > 0 && (!encode_kv_map(&maps.k, a.k, a.kv_rows, a.n_kv_heads, a.kv_stride * 2, kTile) ||
                        !encode_kv_map(&maps.v, a.v, a.kv_rows, a.n_kv_heads, a.kv_stride * 2, kTile)))
    return cudaErrorInvalidValue;
  const void* fn = dtype == FSX_BF16 ? reinterpret_cast<const void*>(&prompt_kernel<true>)
                                     : reinterpret_cast<const void*>(&prompt_kernel<false>);
  const cudaError_t e = allow_shared_memory(fn, kSmem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<PromptArgs*>(&a), &rounds, &maps};
  return launch_ex(fn, dim3(static_cast<unsigned>(grid)), dim3(kThreads), kSmem, stream, false, args);
}

}  // namespace fsx
