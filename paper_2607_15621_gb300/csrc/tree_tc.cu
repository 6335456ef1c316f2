// Attention of drafted tokens (fsx_tree_attention) for items of many rows, on the 5th-generation tensor
// cores: up to 128 rows (token, head of the group) an item, or 256 (WIDE).
//
//   S = Q K^T     128 rows x 128 keys, A and B in shared memory, S in tensor memory
//   P = 2^(f S k_scale - m) v_scale / vs, rounded to the type of V, over its S; a thread holds a row
//   O += P V      A in tensor memory, V read N-contiguous, O in tensor memory
// Two S / P / O sets and two groups of softmax warps: in an item of more than 128 rows each works on its
// own 128 rows and every chunk; else both on the same rows, one on the even and one on the odd chunks, so that
// the tensor core always has the other's work while one is at its exponentials; their two results meet at the end.
//
// Four producer warps copy the rows of a chunk by 16-byte asynchronous copies, each thread its own units, and wait
// for nobody: 16-bit rows straight into their slot, 8-bit rows into a private stage, from where the thread that copied
// them turns them into fp16 in the slot. A chunk whose scales are powers of two between 2^-15 and 2^7 (a cache as it is
// written, unless its values are extreme) becomes its values, exactly; any other keeps its codes, and the softmax
// multiplies scores and weights by the scales. bf16 queries and new tokens meet an 8-bit cache as fp16 times a power
// of two per row (their 8 bits fit; components 2^-22 below the row's largest may lose their last bits); the
// new tokens' powers stand where the cache rows' scales do. Rows past the range become zeros and are never read.
// The values of new tokens are looked over on the way: a masked weight is 0, but 0 times an infinity or NaN is not,
// so these become 0 in the product and are added to the rows that see them at the end.
//
// Work is shared out as in tree_schedule.cuh: one warp takes pieces from the queue and describes them in a
// ring for the other roles; cut items are put together by a second kernel, a warp a row: 256 rows
// are too many for the one CTA that comes last.
//
// Registers: 512 threads at 128 from launch; softmax warpgroups take 2 x 184, MMA and scheduler 56, producers 88.
#include "fsx.h"
#include "kernels.h"
#include "llm.h"
#include "tc_attention.cuh"
#include "tree_schedule.cuh"

namespace fsx {

namespace {

constexpr int kD = kHeadDim;
constexpr int kTile = 128;                   // rows of a tile, keys of a chunk
constexpr int kSlotBytes = kTile * kD * 2;   // 32 KB
constexpr int kRawBytes = kTile * kD;        // 16 KB of codes
constexpr int kMmaWarp = 8, kSchedWarp = 9, kProdWarp = 12;
constexpr int kThreads = 512;
constexpr int kWorkRing = 4;
constexpr int kWorkUsers = 13;               // warps that read a piece's description: MMA, producers, softmax
constexpr uint32_t kColS = 0, kColO = 256;
constexpr int kPartials = 512;               // slots of the workspace

// A piece as every role sees it
struct Work {
  long long c0, t0;  // first cache row and first new token of the request
  int len, n;        // its cache rows and new tokens
  int kvh;           // -1: no more pieces
  int row0, rows;    // rows of the item
  int from, chunks;  // of this piece
  int pair;          // more than 128 rows: a softmax group per tile; else a group per chunk parity
  int has_new;       // its last chunk holds the new tokens
  int slot, j, of;
};

template <bool C8, bool WIDE>
struct Layout {
  static constexpr int kRows = WIDE ? 2 * kTile : kTile;
  static constexpr int kSlots = C8 ? (WIDE ? 3 : 4) : (WIDE ? 4 : 5);
  static constexpr int kRaw = C8 ? 3 : 0;
  static constexpr int kOffSlots = (WIDE ? 2 : 1) * kSlotBytes;
  static constexpr int kOffRaw = kOffSlots + kSlots * kSlotBytes;
  static constexpr int kOffScale = kOffRaw + kRaw * kRawBytes;  // C8: [ring][k, v][128]
  // The scales of chunk c are written while its K is made ready, so when the MMAs of K or V chunk c - 2 or before
  // are done: the weights of chunk c - 4 are behind.
  static constexpr int kScaleRing = C8 ? 4 : 0;
  static constexpr int kOffFactor = kOffScale + kScaleRing * 2 * kTile * 4;  // C8: [piece parity][row]
  static constexpr int kOffMl = kOffFactor + (C8 ? 2 * kRows * 4 : 0);       // [group][128] (m, l)
  static constexpr int kOffScratch = kOffMl + 2 * kTile * 8;
  static constexpr int kOffWork = kOffScratch + 32 * 8;
  static constexpr int kOffBar = kOffWork + kWorkRing * static_cast<int>(sizeof(Work));
  static constexpr int kMisc = kOffBar + 29 * 8;  // tmem, abort, wild[4], vs of the groups [2], plain[4]
  static constexpr int kPlan = kMisc + 12 * 4;
  static constexpr int kSmem = kPlan + static_cast<int>(tree_plan_bytes(kMaxSequences));
};
static_assert(Layout<true, true>::kSmem <= 227 * 1024 && Layout<true, false>::kSmem <= 227 * 1024, "shared memory");
static_assert(Layout<false, true>::kSmem <= 227 * 1024 && Layout<false, false>::kSmem <= 227 * 1024, "shared memory");

__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
  return h;
}
__device__ __forceinline__ float weight_of(float m, float top) { return m == -CUDART_INF_F ? 0.f : exp2_fast(m - top); }

// 2^e that brings `top`, a row's largest magnitude, to [2^7, 2^8) when it is divided by it; 1 for zeros, infinities
// and NaN
__device__ __forceinline__ float row_power(float top) {
  if (top == 0.f || !(top < CUDART_INF_F)) return 1.f;
  const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127 - 7;
  return __uint_as_float(static_cast<uint32_t>(127 + max(-126, min(e, 126))) << 23);
}
__device__ __forceinline__ float inverse_power(float p) {
  return __uint_as_float((254u << 23) - __float_as_uint(p));
}
__device__ __forceinline__ float top_of(uint4 x) {  // largest magnitude of 8 bf16 values
  float t = 0.f;
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) t = fmaxf(t, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
  return t;
}
__device__ __forceinline__ uint4 bf16_to_half(uint4 x, float factor) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_half2(__uint_as_float(w[i] << 16) * factor, __uint_as_float(w[i] & 0xffff0000u) * factor);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool BF>
__device__ __forceinline__ uint4 take_out_wild(uint4 x, bool& wild) {  // values that are not finite become 0
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t bad = not_finite2<BF>(w[i]);
    wild = wild || bad != 0u;
    w[i] &= ~((bad >> 15) * 0xffffu);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float row_max16(float t) {  // over the 16 lanes that share a row
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
  return t;
}

// Workspace behind the header and counters: (first slot, pieces) per (head, new token), then the slots:
// [rows][128] sums, [rows] (maximum, sum of weights)
__host__ __device__ constexpr size_t slot_floats(int rows) { return static_cast<size_t>(rows) * (kD + 2); }
__device__ __forceinline__ int2* table_of(const TreeArgs& p) {
  return reinterpret_cast<int2*>(static_cast<int*>(p.workspace) + kTreeHeader + kTreeCounters);
}
__host__ __device__ __forceinline__ size_t table_bytes(long long new_rows, int n_heads) {
  return (static_cast<size_t>(new_rows) * n_heads * sizeof(int2) + 255) / 256 * 256;
}
__device__ __forceinline__ float* slots_of(const TreeArgs& p) {
  return reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(table_of(p)) + table_bytes(p.new_rows, p.n_heads));
}

template <bool BF, bool C8, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const TreeArgs p) {
  using L = Layout<C8, WIDE>;
  constexpr bool kBf = BF && !C8;  // type of the operands
  constexpr int kSlots = L::kSlots;
  constexpr TreeShape kShape{L::kRows, kTile, 8, 64, kPartials};
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t G = static_cast<uint32_t>(p.n_heads) / static_cast<uint32_t>(p.n_kv_heads);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
  uint64_t* full = bars;          // [6] a slot's rows are there
  uint64_t* empty = bars + 6;     // [6] the MMAs that read it are done
  uint64_t* qfull = bars + 12;    // an item's queries are there
  uint64_t* qempty = bars + 13;   // the softmax warps are done with the piece and with their place
  uint64_t* sfull = bars + 14;    // [2] S of a chunk in tensor memory
  uint64_t* pfull = bars + 16;    // [2] P of a chunk over it
  uint64_t* odone = bars + 18;    // every P V of the piece done
  uint64_t* oread = bars + 19;    // its O read
  uint64_t* drain = bars + 20;    // every MMA done
  uint64_t* wfull = bars + 21;    // [4] a piece is described
  uint64_t* wempty = bars + 25;   // [4] and every role has read it
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* wild = reinterpret_cast<volatile int*>(tmem_slot + 2);  // [4]: piece ordinal + 1 with values taken out
  volatile float* group_vs = reinterpret_cast<volatile float*>(tmem_slot + 6);  // [2]
  volatile int* plain_of = reinterpret_cast<volatile int*>(tmem_slot + 8);      // [4]: no scales left in the chunk
  Work* works = reinterpret_cast<Work*>(smem + L::kOffWork);
  float* scales = reinterpret_cast<float*>(smem + L::kOffScale);
  float* row_factor = reinterpret_cast<float*>(smem + L::kOffFactor);
  float2* ml_of = reinterpret_cast<float2*>(smem + L::kOffMl);
  long long* scratch = reinterpret_cast<long long*>(smem + L::kOffScratch);
  constexpr int kScaleRing = L::kScaleRing > 0 ? L::kScaleRing : 1;
  if ((smem_addr(smem) & 1023u) != 0u) {  // the swizzled operands need a 1024-byte aligned base
    if (tid == 0) set_status(p.status, kStatusDeviceArg);
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < 6; ++i) {
      mbar_init(full + i, 128);
      mbar_init(empty + i, 1);
    }
    mbar_init(qfull, 128);
    mbar_init(qempty, 8);
    for (int i = 0; i < 2; ++i) {
      mbar_init(sfull + i, 1);
      mbar_init(pfull + i, 4);
    }
    mbar_init(odone, 1);
    mbar_init(oread, 8);
    mbar_init(drain, 1);
    for (int i = 0; i < kWorkRing; ++i) {
      mbar_init(wfull + i, 1);
      mbar_init(wempty + i, kWorkUsers);
    }
    *abort = 0;
    for (int i = 0; i < 4; ++i) wild[i] = 0;
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const TreePlan plan = tree_plan<kThreads>(p, kShape, smem + L::kPlan, scratch);
  fence_proxy_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(tmem_slot);
  // piece `ord` of the CTA: its description stays until every warp that uses it has given it back
  auto find_work = [&](int ord) {
    return wait_or_abort(wfull + ord % kWorkRing, (ord / kWorkRing) & 1, p.status, abort) && works[ord % kWorkRing].kvh >= 0;
  };
  auto give_back = [&](int ord) {
    __syncwarp();
    if (lane == 0) mbar_arrive(wempty + ord % kWorkRing);
  };
  // the c-th K or V chunk of the CTA (K0 V0 K1 ... through all its pieces) lies in slot c mod kSlots

  if (warp >= kMmaWarp && warp < kProdWarp) {
  leave_registers<56>();
  if (warp == kSchedWarp) {
    // ---------------------------------------------------------------- pieces
    int* header = static_cast<int*>(p.workspace);
    const long long total = plan.pieces[p.B];
    long long i = blockIdx.x;
#pragma unroll 1
    for (int ord = 0;; ++ord) {
      if (ord >= kWorkRing && !wait_or_abort(wempty + ord % kWorkRing, (ord / kWorkRing - 1) & 1, p.status, abort)) break;
      if (lane == 0) {
        Work w{};
        w.kvh = -1;
        if (i < total) {
          const TreePiece x = tree_piece(p, kShape, plan, i);
          w.c0 = x.r.c0;
          w.t0 = x.r.t0;
          w.len = x.r.len;
          w.n = x.r.n;
          w.kvh = x.kvh;
          w.row0 = x.row0;
          w.rows = min(L::kRows, x.r.n * static_cast<int>(G) - x.row0);
          w.from = x.from;
          w.chunks = x.to - x.from;
          w.pair = w.rows > kTile;
          w.has_new = x.to == x.n;
          w.slot = x.slot;
          w.j = x.j;
          w.of = x.of;
        }
        works[ord % kWorkRing] = w;
        mbar_arrive(wfull + ord % kWorkRing);
      }
      if (i >= total) break;
      if (lane == 0) i = gridDim.x + static_cast<long long>(atomicAdd(reinterpret_cast<unsigned*>(header), 1u));
      i = __shfl_sync(0xffffffffu, i, 0);
    }
    if (lane == 0 && atomicAdd(reinterpret_cast<unsigned*>(header) + 1, 1u) == gridDim.x - 1) {
      header[0] = 0;  // every CTA has taken its last piece
      header[1] = 0;
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs: the whole warp waits, one lane issues
    const bool leader = elect_lane();
    const uint32_t id_s = idesc_16(kBf, kTile, kTile, false), id_o = idesc_16(kBf, kTile, kD, true);
    const uint32_t slots = smem_addr(smem + L::kOffSlots);
    const uint64_t q_desc = sw128_desc(smem_addr(smem)), k_desc = sw128_desc(slots), v_desc = sw128_desc_mn(slots, 16384, 1024);
    bool ok = true;
    int c0 = 0, ord = 0;
    uint32_t p_count0 = 0, p_count1 = 0;
#pragma unroll 1
    for (; ok; ++ord) {
      if (!find_work(ord)) break;
      const Work& w = works[ord % kWorkRing];
      const int lag = w.pair ? 1 : 2;
      bool fresh = ord > 0;
#pragma unroll 1
      for (int j = 0; j < w.chunks + lag && ok; ++j) {
#pragma unroll 1
        for (int t = 0; t < 2; ++t) {
          if (!w.pair && t != (j & 1)) continue;
          const bool last_tile = !w.pair || t == 1;
          const uint32_t s_at = tmem + kColS + t * kTile, o_at = tmem + kColO + t * kTile;
          const int jp = j - lag;  // P V of chunk jp, then S of chunk j
          if (jp >= 0) {
            const int c = c0 + 2 * jp + 1;
            ok = wait_or_abort(pfull + t, (t ? p_count1 : p_count0) & 1, p.status, abort) &&
                 wait_or_abort(full + c % kSlots, (c / kSlots) & 1, p.status, abort) &&
                 (!fresh || wait_or_abort(oread, (ord - 1) & 1, p.status, abort));
            if (!ok) break;
            fresh = false;
            if (t) ++p_count1;
            else ++p_count0;
            tc_fence_after();
            const uint64_t vd = v_desc + (c % kSlots) * (kSlotBytes >> 4);
            const bool more = jp >= lag;  // not the group's first chunk
            const int steps = w.has_new && jp == w.chunks - 1 ? kMaxDrafts / 64 : kTile / 64;
            if (leader) {
#pragma unroll 1
              for (int h = 0; h < steps; ++h) {  // 64 keys
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  umma_f16_ta(o_at, s_at + h * 32 + k * 8, vd + (h * 4 + k) * 128, id_o, more || h > 0 || k > 0 ? 1u : 0u);
              }
              if (last_tile) {
                umma_commit(empty + c % kSlots);
                if (jp == w.chunks - 1) umma_commit(odone);
              }
            }
            __syncwarp();
          }
          if (j < w.chunks) {
            const int c = c0 + 2 * j;
            ok = (j > 0 || wait_or_abort(qfull, ord & 1, p.status, abort)) &&
                 wait_or_abort(full + c % kSlots, (c / kSlots) & 1, p.status, abort);
            if (!ok) break;
            tc_fence_after();
            const uint64_t qd = q_desc + (w.pair && t == 1 ? kSlotBytes >> 4 : 0), kd = k_desc + (c % kSlots) * (kSlotBytes >> 4);
            if (leader) {
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const uint32_t off = (k >> 2) * (16384 >> 4) + (k & 3) * 2;
                umma_f16(s_at, qd + off, kd + off, id_s, k > 0 ? 1u : 0u);
              }
              umma_commit(sfull + t);
              if (last_tile) umma_commit(empty + c % kSlots);
            }
            __syncwarp();
          }
        }
      }
      c0 += 2 * w.chunks;
      give_back(ord);
    }
    if (leader) umma_commit(drain);
    __syncwarp();
    mbar_wait(drain, 0, p.status);
  }
  } else if (warp >= kProdWarp) {
    // ---------------------------------------------------------------- producers
    leave_registers<88>();
    // A thread's units of a K or V chunk: 16-bit rows, unit u of rows r0, r0 + 8, ...; codes, units q and q + 4 of rows
    // r0, r0 + 32, ...: four lanes a row, so that the 8 lanes whose fp16 units are stored together have rows of both
    // parities and meet no bank twice.
    const int pt = tid - kProdWarp * 32;
    const int u = C8 ? pt & 3 : pt & 15, r0 = C8 ? pt >> 2 : pt >> 4;
    constexpr int kRowStep = C8 ? 32 : 8;
    constexpr int kAhead = C8 ? L::kRaw - 1 : kSlots - 2;  // K or V chunks copied ahead of the one that is made ready
    constexpr int kRaws = L::kRaw > 0 ? L::kRaw : 1;
    const long long row_bytes = static_cast<long long>(p.n_kv_heads) * kD * (C8 ? 1 : 2);
    const long long row_step = kRowStep * row_bytes;
    unsigned char* slots = smem + L::kOffSlots;
    unsigned char* raw = smem + L::kOffRaw;
    bool ok = true;
    // the next K or V chunk to copy: `ci` of piece `iord`, which is up to two pieces ahead of the one made ready
    int iord = 0, ci = 0, issued = 0, left = 0;  // left: rows from this thread's first row of the chunk to the end
    const unsigned char *src_k = nullptr, *src_v = nullptr;
    bool more = false;
    auto begin_copies = [&] {
      more = find_work(iord);
      if (more) {
        const Work& x = works[iord % kWorkRing];
        const int key0 = x.from * kTile + r0;
        left = x.len - key0;
        const long long at = (x.c0 + key0) * row_bytes + (x.kvh * kD * (C8 ? 1 : 2) + u * 16);
        src_k = static_cast<const unsigned char*>(p.k_cache) + at;
        src_v = static_cast<const unsigned char*>(p.v_cache) + at;
      }
    };
    begin_copies();
    // C8: this lane's scales of keys lane, lane + 32, ... of the next chunk that is made ready
    float ks_now[4], vs_now[4], ks_next[4], vs_next[4];
    auto load_scales = [&](const Work& x, int j) {
      const int first = (x.from + j) * kTile + lane;
      const long long at = x.kvh * p.cache_rows + x.c0 + first;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool there = first + 32 * e < x.len;
        ks_next[e] = there ? __ldg(p.k_scale + at + 32 * e) : 0.f;
        vs_next[e] = there ? __ldg(p.v_scale + at + 32 * e) : 0.f;
      }
    };
    auto issue = [&] {
      if (more) {
        const bool is_v = ci & 1;
        const Work& x = works[iord % kWorkRing];
        const bool is_new = x.has_new && (ci >> 1) == x.chunks - 1;
        const unsigned char* src = is_v ? src_v : src_k;
        if (!C8) {
          ok = ok && (issued < kSlots || wait_or_abort(empty + issued % kSlots, (issued / kSlots - 1) & 1, p.status, abort));
          if (ok) {
            long long step = row_step;
            int rows = left;
            if (is_new) {
              step = kRowStep * p.new_stride * 2;
              rows = x.n - r0;
              src = static_cast<const unsigned char*>(is_v ? p.v_new : p.k_new) + ((x.t0 + r0) * p.new_stride + x.kvh * kD) * 2 + u * 16;
            }
            const uint32_t dst = smem_addr(slots + (issued % kSlots) * kSlotBytes + tile_off(r0, u));  // rows 8 on lie 1024 bytes on
#pragma unroll 4
            for (int m = 0; m < 16; ++m, src += step) copy16(dst + m * 1024, src, kRowStep * m < rows);
          }
        } else if (!is_new) {
          const uint32_t dst = smem_addr(raw + (issued % kRaws) * kRawBytes + pt * 16);
#pragma unroll
          for (int m = 0; m < 4; ++m, src += row_step) {
            copy16(dst + m * 4096, src, kRowStep * m < left);
            copy16(dst + m * 4096 + 2048, src + 64, kRowStep * m < left);
          }
        }
        ++issued;
        ++ci;
        if (is_v) {
          left -= kTile;
          src_k += kTile * row_bytes;
          src_v += kTile * row_bytes;
          if (ci == 2 * x.chunks) {
            ci = 0;
            ++iord;
            begin_copies();
          }
        }
      }
      cp_async_commit();
    };
    if (C8 && more) load_scales(works[0], 0);
#pragma unroll 1
    for (int k = 0; k < kAhead; ++k) issue();
    bool plain = true;
    int c = 0, chunk_no = 0;
#pragma unroll 1
    for (int ord = 0; ok; ++ord) {
      if (!find_work(ord)) break;
      const Work& w = works[ord % kWorkRing];
      // ---- queries
      if (ord > 0) ok = wait_or_abort(qempty, (ord - 1) & 1, p.status, abort);
      if (!ok) break;
      if (C8 && ord > 0) load_scales(w, 0);
      {
        const int qu = pt & 15;
        const uint16_t* q = static_cast<const uint16_t*>(p.q) + w.t0 * p.q_stride + w.kvh * G * kD + qu * 8;
        const int to = w.pair ? 2 * kTile : kTile;
        if (!C8) {  // all on their way at once
#pragma unroll 2
          for (int r = pt >> 4; r < to; r += 8) {
            const bool there = r < w.rows;
            const uint32_t row = w.row0 + (there ? r : 0), token = row / G;
            copy16(smem_addr(smem + (r >> 7) * kSlotBytes + tile_off(r & 127, qu)), q + token * p.q_stride + (row - token * G) * kD, there);
          }
        } else {
#pragma unroll 1
          for (int r1 = pt >> 4; r1 < to; r1 += 32) {  // four rows at a time
            uint4 x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = r1 + 8 * e;
              const uint32_t row = w.row0 + r, token = row / G;
              x[e] = r < w.rows ? __ldg(reinterpret_cast<const uint4*>(q + token * p.q_stride + (row - token * G) * kD)) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = r1 + 8 * e;
              float power = 1.f;
              if (BF) {
                power = row_power(row_max16(top_of(x[e])));
                x[e] = bf16_to_half(x[e], inverse_power(power));
              }
              if (qu == 0) row_factor[(ord & 1) * L::kRows + r] = power * kScaleLog2;
              *reinterpret_cast<uint4*>(smem + (r >> 7) * kSlotBytes + tile_off(r & 127, qu)) = x[e];
            }
          }
        }
        if (C8) {
          fence_proxy_async();
          mbar_arrive(qfull);
        } else {
          // counted with the chunk copies behind them: ready when the piece's first chunk is
          cp_async_commit();
        }
      }
      // ---- chunks
#pragma unroll 1
      for (int tc = 0; tc < 2 * w.chunks && ok; ++tc, ++c) {
        const int j = tc >> 1;
        const bool is_v = tc & 1, is_new = w.has_new && j == w.chunks - 1;
        unsigned char* slot = slots + (c % kSlots) * kSlotBytes;
        if (C8) {
          issue();  // chunk c + kAhead, into the stage that chunk c - 1 was made ready from
          ok = c < kSlots || wait_or_abort(empty + c % kSlots, (c / kSlots - 1) & 1, p.status, abort);
          if (!ok) break;
          float* ks = scales + (chunk_no % kScaleRing) * 2 * kTile;
          if (!is_v) {
            // scales that leave every code exact in fp16: powers of two, 2^-15 <= s <= 2^7 (rows that are not there: 0)
            plain = true;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              ks_now[e] = ks_next[e];
              vs_now[e] = vs_next[e];
              const uint32_t x = __float_as_uint(ks_now[e]), y = __float_as_uint(vs_now[e]);
              plain = plain && ((x | y) & 0x7fffffu) == 0u && (x == 0u || x - (112u << 23) <= 22u << 23) &&
                      (y == 0u || y - (112u << 23) <= 22u << 23);
            }
            plain = __all_sync(0xffffffffu, plain);
          } else if (j + 1 < w.chunks) {
            load_scales(w, j + 1);
          }
          if (!is_new) {
            if (!is_v && pt < 32) {
              if (lane == 0) plain_of[chunk_no & 3] = plain ? 1 : 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                ks[lane + 32 * e] = plain ? 1.f : ks_now[e];
                ks[kTile + lane + 32 * e] = plain ? 1.f : vs_now[e];
              }
            }
            cp_async_wait<kAhead>();
            const unsigned char* mine = raw + (c % kRaws) * kRawBytes + pt * 16;
            unsigned char* to = slot + tile_off(r0, 2 * u);  // unit 2 u + 1 at the other place of its pair
            const int other = (r0 & 1) ? -16 : 16;
#pragma unroll
            for (int m = 0; m < 4; ++m) {  // rows r0 + 32 m lie 4096 bytes apart; the row's scale is the lane's r0 mod 32
              const float sc = __shfl_sync(0xffffffffu, is_v ? vs_now[m] : ks_now[m], r0 & 31);
              const __half2 f = __float2half2_rn(plain ? sc : 1.f);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint4 x = *reinterpret_cast<const uint4*>(mine + m * 4096 + h * 2048);
                const uint32_t y[4] = {x.x, x.y, x.z, x.w};
                uint32_t z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  const uint32_t code = e4m3x2_to_half2(y[e >> 1] >> (16 * (e & 1)));
                  const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&code), f);
                  z[e] = *reinterpret_cast<const uint32_t*>(&v);
                }
                *reinterpret_cast<uint4*>(to + m * 4096 + h * 16384) = make_uint4(z[0], z[1], z[2], z[3]);
                *reinterpret_cast<uint4*>(to + m * 4096 + h * 16384 + other) = make_uint4(z[4], z[5], z[6], z[7]);
              }
            }
          } else {
            if (!is_v && pt == 0) plain_of[chunk_no & 3] = 0;
            bool found = false;
            const int nu = pt & 15;
#pragma unroll 1
            for (int r = pt >> 4; r < kMaxDrafts; r += 8) {
              const bool there = r < w.n;
              auto row_of = [&](const void* base) {
                return there ? __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + (w.t0 + r) * p.new_stride + w.kvh * kD) + nu)
                             : make_uint4(0u, 0u, 0u, 0u);
              };
              uint4 y = row_of(p.v_new);
              bool wild_here = false;
              y = take_out_wild<BF>(y, wild_here);
              float yp = 1.f;
              if (BF) yp = row_power(row_max16(top_of(y)));
              if (!is_v) {
                uint4 x = row_of(p.k_new);
                float xp = 1.f;
                if (BF) {
                  xp = row_power(row_max16(top_of(x)));
                  x = bf16_to_half(x, inverse_power(xp));
                }
                if (nu == 0) {
                  ks[r] = xp;
                  ks[kTile + r] = there ? yp : 0.f;
                  ks[kMaxDrafts + r] = 0.f;
                  ks[kTile + kMaxDrafts + r] = 0.f;
                }
                *reinterpret_cast<uint4*>(slot + tile_off(r, nu)) = x;
              } else {
                found = found || wild_here;
                if (BF) y = bf16_to_half(y, inverse_power(yp));
                *reinterpret_cast<uint4*>(slot + tile_off(r, nu)) = y;
              }
            }
            if (found) wild[ord & 3] = ord + 1;
          }
        } else {
          // the piece's queries were committed behind the copies of the first kAhead chunks
          if (tc < kAhead) cp_async_wait<0>();
          else cp_async_wait<kAhead - 1>();
          if (is_new && is_v) {
            bool found = false;
#pragma unroll 1
            for (int r = r0; r < kMaxDrafts; r += 8) {
              uint4* at = reinterpret_cast<uint4*>(slot + tile_off(r, u));
              bool here = false;
              const uint4 y = take_out_wild<BF>(*at, here);
              if (here) *at = y;
              found = found || here;
            }
            if (found) wild[ord & 3] = ord + 1;
          }
        }
        fence_proxy_async();
        if (!C8 && tc == 0) mbar_arrive(qfull);
        mbar_arrive(full + c % kSlots);
        if (!C8) issue();
        if (is_v) ++chunk_no;
      }
      give_back(ord);
    }
    cp_async_wait<0>();
  } else {
    // ---------------------------------------------------------------- softmax of group t
    take_registers<184>();
    const int t = warp >> 2;
    const int r = tid & (kTile - 1);
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t scol = tmem + lanes + kColS + t * kTile, ocol = tmem + lanes + kColO;
    bool ok = true;
    int c0 = 0, chunk0 = 0;
    uint32_t s_count = 0;
#pragma unroll 1
    for (int ord = 0; ok; ++ord) {
      if (!find_work(ord)) break;
      const Work& w = works[ord % kWorkRing];
      const int my_row = w.pair ? t * kTile + r : r;
      const bool mine = my_row < w.rows;
      const uint32_t at = w.row0 + (mine ? my_row : 0), token = at / G;
      const int head = w.kvh * G + (at - token * G);
      float m = -CUDART_INF_F, l = 0.f, vs = C8 ? 0.f : 1.f, f = kScaleLog2;
      bool first = true;
      // O of this group times `alpha`
      auto rescale = [&](float alpha) {
#pragma unroll 1
        for (int c = 0; c < kD; c += 32) {
          uint32_t o[32];
          tmem_ld32_issue(ocol + t * kTile + c, o);
          tmem_wait_ld32(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
          tmem_st32(ocol + t * kTile + c, o);
        }
      };
#pragma unroll 1
      for (int j = w.pair ? 0 : t; j < w.chunks && ok; j += w.pair ? 1 : 2) {
        ok = wait_or_abort(sfull + t, s_count & 1, p.status, abort);
        ++s_count;
        const int cv = c0 + 2 * j + 1;
        if (C8) ok = ok && wait_or_abort(full + cv % kSlots, (cv / kSlots) & 1, p.status, abort);  // the scales, too
        if (!ok) break;
        tc_fence_after();
        const bool is_new = w.has_new && j == w.chunks - 1;
        const int left = w.len - (w.from + j) * kTile;  // cache rows of this chunk
        if (C8) f = row_factor[(ord & 1) * L::kRows + my_row];
        if (!is_new && left >= kTile && (!C8 || (plain_of[(chunk0 + j) & 3] != 0 && vs <= 1.f))) {
          // ---- a whole chunk without scales: scores in registers
          uint32_t raw[4][32];
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld32_issue(scol + 32 * i, raw[i]);
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_wait_ld32(raw[i]);
          float mx[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            mx[i] = __uint_as_float(raw[i][0]);
#pragma unroll
            for (int e = 1; e < 31; e += 2) mx[i] = max3(mx[i], __uint_as_float(raw[i][e]), __uint_as_float(raw[i][e + 1]));
            mx[i] = fmaxf(mx[i], __uint_as_float(raw[i][31]));
          }
          const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * f;
          if (__any_sync(0xffffffffu, top > m + 8.f || vs < 1.f)) {
            const float m_new = top > m + 8.f ? top : m;
            const float alpha = m_new == m ? 1.f : exp2_fast(m - m_new);
            m = m_new;
            l *= alpha;
            if (!first) rescale(alpha * vs);
            vs = 1.f;
          }
          const float nm = m == -CUDART_INF_F ? 0.f : -m;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 2; ++i) {  // 64 keys: 32 columns of P
            uint32_t pk[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              float a = __uint_as_float(raw[2 * i + (e >> 4)][2 * (e & 15)]), b = __uint_as_float(raw[2 * i + (e >> 4)][2 * (e & 15) + 1]);
              fma2(a, b, f, nm);
              a = exp2_fast(a);
              b = exp2_fast(b);
              if (e & 1) add2(sum[2], sum[3], a, b);
              else add2(sum[0], sum[1], a, b);
              pk[e] = pack16<kBf>(a, b);
            }
            tmem_st32(scol + 32 * i, pk);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        } else {
          // ---- scales, the end of the cache or the new tokens: 32 keys at a time, twice
          const float4* ks = reinterpret_cast<const float4*>(scales + ((chunk0 + j) % kScaleRing) * 2 * kTile);
          const float4* vv = ks + kTile / 4;
          const uint64_t seen = is_new && mine ? p.mask[w.t0 + token] & (w.n < 64 ? (1ull << w.n) - 1 : ~0ull) : 0ull;
          auto scores = [&](int b, float (&s)[32]) {  // times the keys' scales; -infinity where the row does not see
            uint32_t raw[32];
            tmem_ld32_issue(scol + 32 * b, raw);
            tmem_wait_ld32(raw);
            const int here = left - 32 * b;
            const uint32_t bits = is_new ? (b < 2 ? static_cast<uint32_t>(seen >> (32 * b)) : 0u)
                                         : (here >= 32 ? 0xffffffffu : here <= 0 ? 0u : (1u << here) - 1u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 k = C8 ? ks[8 * b + e] : make_float4(1.f, 1.f, 1.f, 1.f);
              s[4 * e] = (bits >> (4 * e)) & 1u ? __uint_as_float(raw[4 * e]) * k.x : -CUDART_INF_F;
              s[4 * e + 1] = (bits >> (4 * e + 1)) & 1u ? __uint_as_float(raw[4 * e + 1]) * k.y : -CUDART_INF_F;
              s[4 * e + 2] = (bits >> (4 * e + 2)) & 1u ? __uint_as_float(raw[4 * e + 2]) * k.z : -CUDART_INF_F;
              s[4 * e + 3] = (bits >> (4 * e + 3)) & 1u ? __uint_as_float(raw[4 * e + 3]) * k.w : -CUDART_INF_F;
            }
          };
          const int blocks = is_new ? 2 : 4;
          float top = -CUDART_INF_F, vtop = vs;
#pragma unroll 1
          for (int b = 0; b < blocks; ++b) {
            float s[32];
            scores(b, s);
#pragma unroll
            for (int e = 0; e < 32; e += 2) top = max3(top, s[e], s[e + 1]);
          }
          top *= f;
          if (C8) {
            const float4 x = vv[lane];  // largest value scale of the chunk, the same for every row
            vtop = fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) vtop = fmaxf(vtop, __shfl_xor_sync(0xffffffffu, vtop, o));
            vtop = fmaxf(vtop, vs);
          }
          if (__any_sync(0xffffffffu, top > m + 8.f || vtop > vs)) {
            const float m_new = top > m + 8.f ? top : m;
            float alpha = m_new == m ? 1.f : exp2_fast(m - m_new);
            m = m_new;
            l *= alpha;
            if (C8) {
              alpha *= vtop > 0.f ? vs / vtop : 1.f;
              vs = vtop;
            }
            if (!first) rescale(alpha);
          }
          const float nm = m == -CUDART_INF_F ? 0.f : -m;
          const float inv = C8 ? (vs > 0.f ? 1.f / vs : 0.f) : 1.f;
#pragma unroll 1
          for (int b = 0; b < blocks; ++b) {
            float s[32];
            scores(b, s);
            uint32_t pk[16];
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x = exp2_fast(fmaf(s[2 * e], f, nm)), y = exp2_fast(fmaf(s[2 * e + 1], f, nm));
              sum += x + y;
              if (C8) {
                const float2 v = reinterpret_cast<const float2*>(vv)[16 * b + e];
                x *= v.x * inv;
                y *= v.y * inv;
              }
              pk[e] = pack16<kBf>(x, y);
            }
            l += sum;
            // 16 columns of P over S columns 16 b .. 16 b + 15: read before by this thread's block b / 2
            asm volatile(
                "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
                    scol + 16 * b),
                "r"(pk[0]), "r"(pk[1]), "r"(pk[2]), "r"(pk[3]), "r"(pk[4]), "r"(pk[5]), "r"(pk[6]), "r"(pk[7]), "r"(pk[8]),
                "r"(pk[9]), "r"(pk[10]), "r"(pk[11]), "r"(pk[12]), "r"(pk[13]), "r"(pk[14]), "r"(pk[15])
                : "memory");
          }
        }
        first = false;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pfull + t);
      }
      // ---- the piece's result
      ok = ok && wait_or_abort(odone, ord & 1, p.status, abort);
      tc_fence_after();
      if (!w.pair) {
        ml_of[t * kTile + r] = make_float2(m, l);
        if (r == 0) group_vs[t] = vs;
      }
      // both groups, also after an abort: all leave together
      int all_ok;
      asm volatile(
          "{\n .reg .pred p, q;\n setp.ne.s32 p, %1, 0;\n barrier.red.and.pred q, 1, 256, p;\n selp.s32 %0, 1, 0, q;\n}"
          : "=r"(all_ok)
          : "r"(static_cast<int>(ok))
          : "memory");
      if (!all_ok) break;
      float w0 = 1.f, w1 = 0.f;  // of the two accumulators, for `pair` of this group's own
      if (!w.pair) {
        const float2 a = ml_of[r], b = ml_of[kTile + r];
        m = fmaxf(a.x, b.x);
        w0 = weight_of(a.x, m);
        w1 = weight_of(b.x, m);
        l = a.y * w0 + b.y * w1;
        if (C8) {
          w0 *= group_vs[0];
          w1 *= group_vs[1];
        }
      } else if (C8) {
        w0 = vs;
      }
      const bool whole = w.of == 1;
      const bool two = !w.pair && w.chunks > 1;
      const bool any_wild = w.has_new && wild[ord & 3] == ord + 1;
      const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
      w0 *= inv;
      w1 *= inv;
      // 32 columns at a time through this warp's 4 KB of the queries' place (all S are done), so that rows are
      // written in 128-byte or, as sums, 64-byte pieces by neighbouring lanes; unit u of row r lies at u ^ (r mod 8)
      float* place = reinterpret_cast<float*>(smem + warp * 4096);
      float* slot = slots_of(p) + static_cast<size_t>(w.slot + w.j) * slot_floats(L::kRows);
      uint16_t* out = static_cast<uint16_t*>(p.out);
      const int d_from = w.pair ? 0 : t * (kD / 2), d_to = w.pair ? kD : d_from + kD / 2;
      const uint32_t own = ocol + (w.pair ? t * kTile : 0);
      const int row_base = (w.pair ? t * kTile : 0) + (warp & 3) * 32;
      if (row_base < w.rows) {
#pragma unroll 1
        for (int d = d_from; d < d_to; d += 32) {
          uint32_t o[32];
          float x[32];
          tmem_ld32_issue(own + d, o);
          tmem_wait_ld32(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(o[e]) * w0;
          if (two) {
            tmem_ld32_issue(own + kTile + d, o);
            tmem_wait_ld32(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] += __uint_as_float(o[e]) * w1;
          }
          if (mine && any_wild) {
            const uint64_t seen = p.mask[w.t0 + token];
#pragma unroll 1
            for (int k = 0; k < w.n; ++k)
              if ((seen >> k) & 1u) {
                const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v_new) + (w.t0 + k) * p.new_stride + w.kvh * kD + d);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const uint32_t bad = not_finite2<BF>(v[e]);
                  const float2 y = unpack16<BF>(v[e]);
                  if (bad & 0x8000u) x[2 * e] += y.x;
                  if (bad & 0x80000000u) x[2 * e + 1] += y.y;
                }
              }
          }
          __syncwarp();  // the columns before are read
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<float4*>(place + lane * 32 + ((e ^ (lane & 7)) << 2)) = make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]);
          __syncwarp();
          const int e = lane & 7;
#pragma unroll 2
          for (int k = lane >> 3; k < 32; k += 4) {
            const int row = row_base + k;
            if (row < w.rows) {
              const float4 y = *reinterpret_cast<const float4*>(place + k * 32 + ((e ^ (k & 7)) << 2));
              if (whole) {
                const uint32_t a = w.row0 + row, to = a / G;
                *reinterpret_cast<uint2*>(out + ((w.t0 + to) * p.n_heads + w.kvh * G + (a - to * G)) * kD + d + 4 * e) =
                    make_uint2(pack16<BF>(y.x, y.y), pack16<BF>(y.z, y.w));
              } else {
                __stcg(reinterpret_cast<float4*>(slot + row * kD + d) + e, y);
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(oread);
      if (mine && (w.pair || t == 0)) {
        if (whole) {
          if (p.lse != nullptr) p.lse[head * p.new_rows + w.t0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
        } else {
          __stcg(reinterpret_cast<float2*>(slot + L::kRows * kD) + my_row, make_float2(m, l));
        }
        if (w.j == 0) table_of(p)[head * p.new_rows + w.t0 + token] = make_int2(w.slot, w.of);
      }
      c0 += 2 * w.chunks;
      chunk0 += w.chunks;
      give_back(ord);
      fence_proxy_async();  // the queries' place goes back to the tensor core
      asm volatile("bar.sync 1, 256;" ::: "memory");  // the groups' sums are read before they are written again
      if (lane == 0) mbar_arrive(qempty);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// The rows of cut items: a warp a row, 4 dims a lane, the pieces in the order of their keys. ROWS: rows of a slot.
template <bool BF, int ROWS>
__global__ void __launch_bounds__(128) tree_join_kernel(const TreeArgs p) {
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long at = static_cast<long long>(blockIdx.x) * 4 + warp;  // head * new_rows + token
  if (at >= p.new_rows * p.n_heads) return;
  const int head = static_cast<int>(at / p.new_rows);
  const long long token = at - head * p.new_rows;
  long long t0 = -1;  // first token of its request
  for (int b0 = 0; b0 < p.B && t0 < 0; b0 += 32) {
    TreeRequest r;
    const bool mine = b0 + lane < p.B && tree_request(p, b0 + lane, r) && token >= r.t0 && token < r.t0 + r.n;
    const uint32_t found = __ballot_sync(0xffffffffu, mine);
    if (found != 0u) t0 = __shfl_sync(0xffffffffu, r.t0, __ffs(found) - 1);
  }
  if (t0 < 0) return;
  const int2 entry = table_of(p)[at];
  const int of = entry.y;
  if (of <= 1 || entry.x < 0 || of > kPartials || entry.x + of > kPartials) return;
  const int G = p.n_heads / p.n_kv_heads;
  const int row = static_cast<int>((token - t0) * G + head % G) % ROWS;
  const float* first = slots_of(p) + entry.x * slot_floats(ROWS);
  const float* ml = first + ROWS * kD + 2 * row;
  float m = -CUDART_INF_F;
  for (int j = lane; j < of; j += 32) m = fmaxf(m, __ldcg(ml + j * slot_floats(ROWS)));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j0 = 0; j0 < of; j0 += 32) {
    const int count = min(32, of - j0);
    float w = 0.f;
    if (lane < count) {
      const float2 x = __ldcg(reinterpret_cast<const float2*>(ml + (j0 + lane) * slot_floats(ROWS)));
      w = weight_of(x.x, m);
      l += w * x.y;
    }
#pragma unroll 8
    for (int j = 0; j < count; ++j) {
      const float a = __shfl_sync(0xffffffffu, w, j);
      const float4 v = __ldcg(reinterpret_cast<const float4*>(first + (j0 + j) * slot_floats(ROWS) + row * kD) + lane);
      o.x += a * v.x;
      o.y += a * v.y;
      o.z += a * v.z;
      o.w += a * v.w;
    }
  }
  l = warp_sum(l);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + (token * p.n_heads + head) * kD + 4 * lane) =
      make_uint2(pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv));
  if (p.lse != nullptr && lane == 0) p.lse[at] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
}

struct Kernels {
  const void* main;
  const void* join;
  size_t smem;
};
template <bool BF, bool C8, bool WIDE>
Kernels kernels_for() {
  return {reinterpret_cast<const void*>(&tree_tc_kernel<BF, C8, WIDE>),
          reinterpret_cast<const void*>(&tree_join_kernel<BF, Layout<C8, WIDE>::kRows>), Layout<C8, WIDE>::kSmem};
}
template <bool BF>
Kernels kernels_of(bool cache8, bool wide) {
  return cache8 ? (wide ? kernels_for<BF, true, true>() : kernels_for<BF, true, false>())
                : (wide ? kernels_for<BF, false, true>() : kernels_for<BF, false, false>());
}

bool is_wide(long long new_rows, int group) { return (new_rows < kMaxDrafts ? new_rows : kMaxDrafts) * group > kTile; }

}  // namespace

size_t tree_tc_workspace_bytes(long long new_rows, int n_heads, int n_kv_heads) {
  return (kTreeHeader + kTreeCounters) * sizeof(int) + table_bytes(new_rows, n_heads) +
         kPartials * slot_floats(is_wide(new_rows, n_heads / n_kv_heads) ? 2 * kTile : kTile) * sizeof(float);
}

cudaError_t launch_tree_tc(const TreeArgs& a, int dtype, bool cache8, cudaStream_t stream) {
  const bool wide = is_wide(a.new_rows, a.n_heads / a.n_kv_heads);
  const Kernels k = dtype == FSX_BF16 ? kernels_of<true>(cache8, wide) : kernels_of<false>(cache8, wide);
  const long long join_blocks = (a.new_rows * a.n_heads + 3) / 4;
  if (join_blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  cudaError_t e = cudaFuncSetAttribute(k.main, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(k.smem));
  int dev = 0, sms = 0;
  if (e == cudaSuccess) e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<TreeArgs*>(&a)};
  e = launch_ex(k.main, dim3(static_cast<unsigned>(sms)), dim3(kThreads), k.smem, stream, false, args);
  if (e != cudaSuccess) return e;
  return launch_ex(k.join, dim3(static_cast<unsigned>(join_blocks)), dim3(128), 0, stream, true, args);
}

}  // namespace fsx
