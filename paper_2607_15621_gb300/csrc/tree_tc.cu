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
// them turns them into fp16 in the slot (exact). bf16 queries and new tokens meet an 8-bit cache as fp16 times a power
// of two per row (their 8 bits fit; components 2^-22 below the row's largest may lose their last bits); the
// new tokens' powers stand where the cache rows' scales do. Rows past the range become zeros and are never read.
// The values of new tokens are looked over on the way: a masked weight is 0, but 0 times an infinity or NaN is not,
// so these become 0 in the product and are added to the rows that see them at the end.
//
// Work is shared out as in tree_schedule.cuh (pieces in turn, not from a queue: every role finds
// its next piece by itself); cut items are put together by a second kernel, a warp a row: 256 rows
// are too many for the one CTA that comes last.
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
constexpr int kMmaWarp = 8, kProdWarp = 9;
constexpr int kThreads = 32 * 13;
constexpr uint32_t kColS = 0, kColO = 256;
constexpr int kPartials = 512;               // slots of the workspace

template <bool C8, bool WIDE>
struct Layout {
  static constexpr int kRows = WIDE ? 2 * kTile : kTile;
  static constexpr int kSlots = C8 ? (WIDE ? 3 : 4) : (WIDE ? 4 : 5);
  static constexpr int kRaw = C8 ? 3 : 0;
  static constexpr int kOffSlots = (WIDE ? 2 : 1) * kSlotBytes;
  static constexpr int kOffRaw = kOffSlots + kSlots * kSlotBytes;
  static constexpr int kOffScale = kOffRaw + kRaw * kRawBytes;  // C8: [ring][k, v][128]
  // The scales of K chunk c are copied while chunk c - 2 is made ready, so when the MMAs of chunk c - 3 - kSlots
  // are done: with 3 slots S, with 4 P V of a chunk whose weights are 4 chunks and more behind.
  static constexpr int kScaleRing = C8 ? 4 : 0;
  static constexpr int kOffFactor = kOffScale + kScaleRing * 2 * kTile * 4;  // C8: [piece parity][row]
  static constexpr int kOffMl = kOffFactor + (C8 ? 2 * kRows * 4 : 0);       // [group][128] (m, l)
  static constexpr int kOffScratch = kOffMl + 2 * kTile * 8;
  static constexpr int kOffBar = kOffScratch + 32 * 8;
  static constexpr int kMisc = kOffBar + 21 * 8;  // tmem, abort, wild[4], vs of the groups [2]
  static constexpr int kPlan = kMisc + 8 * 4;
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

// What every role derives from a piece
struct Work {
  TreePiece x;
  int rows;    // rows of the item
  bool pair;   // more than 128: a group per tile; else a group per chunk parity
  int chunks;  // of this piece
  bool has_new;
};
template <int ROWS>
__device__ __forceinline__ Work work_of(const TreeArgs& p, const TreeShape& shape, const TreePlan& plan, long long i, int G) {
  Work w;
  w.x = tree_piece(p, shape, plan, i);
  w.rows = min(ROWS, w.x.r.n * G - w.x.row0);
  w.pair = w.rows > kTile;
  w.chunks = w.x.to - w.x.from;
  w.has_new = w.x.to == w.x.n;
  return w;
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
  const int G = p.n_heads / p.n_kv_heads;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
  uint64_t* full = bars;         // [6] a slot's rows are there
  uint64_t* empty = bars + 6;    // [6] the MMAs that read it are done
  uint64_t* qfull = bars + 12;   // an item's queries are there
  uint64_t* qempty = bars + 13;  // every S of the piece is done
  uint64_t* sfull = bars + 14;   // [2] S of a chunk in tensor memory
  uint64_t* pfull = bars + 16;   // [2] P of a chunk over it
  uint64_t* odone = bars + 18;   // every P V of the piece done
  uint64_t* oread = bars + 19;   // its O read
  uint64_t* drain = bars + 20;   // every MMA done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* wild = reinterpret_cast<volatile int*>(tmem_slot + 2);  // [4]: piece ordinal + 1 with values taken out
  volatile float* group_vs = reinterpret_cast<volatile float*>(tmem_slot + 6);  // [2]
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
    mbar_init(qempty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(sfull + i, 1);
      mbar_init(pfull + i, 4);
    }
    mbar_init(odone, 1);
    mbar_init(oread, 8);
    mbar_init(drain, 1);
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
  const long long total = plan.pieces[p.B];
  const long long step = gridDim.x;
  // the c-th K or V chunk of the CTA (K0 V0 K1 ... through all its pieces) lies in slot c mod kSlots

  if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMAs: the whole warp waits, one lane issues
    const bool leader = elect_lane();
    const uint32_t id_s = idesc_16(kBf, kTile, kTile, false), id_o = idesc_16(kBf, kTile, kD, true);
    const uint32_t slots = smem_addr(smem + L::kOffSlots);
    const uint64_t q_desc = sw128_desc(smem_addr(smem)), k_desc = sw128_desc(slots), v_desc = sw128_desc_mn(slots, 16384, 1024);
    bool ok = true;
    int c0 = 0, ord = 0;
    uint32_t p_count0 = 0, p_count1 = 0;
#pragma unroll 1
    for (long long i = blockIdx.x; i < total && ok; i += step, ++ord) {
      const Work w = work_of<L::kRows>(p, kShape, plan, i, G);
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
              if (last_tile) {
                umma_commit(empty + c % kSlots);
                if (j == w.chunks - 1) umma_commit(qempty);
              }
            }
            __syncwarp();
          }
        }
      }
      c0 += 2 * w.chunks;
    }
    if (leader) umma_commit(drain);
    __syncwarp();
    mbar_wait(drain, 0, p.status);
  } else if (warp >= kProdWarp) {
    // ---------------------------------------------------------------- producers
    const int pt = tid - kProdWarp * 32;
    constexpr int kUnits = C8 ? 8 : 16;  // 16-byte units of a row
    const int u = pt % kUnits, r0 = pt / kUnits;
    constexpr int kRowStep = 128 / kUnits;
    constexpr int kAhead = C8 ? L::kRaw - 1 : kSlots - 2;  // K or V chunks copied ahead of the one that is made ready
    const long long row_bytes = static_cast<long long>(p.n_kv_heads) * kD * (C8 ? 1 : 2);
    unsigned char* slots = smem + L::kOffSlots;
    unsigned char* raw = smem + L::kOffRaw;
    bool ok = true;
    // the next K or V chunk to copy: `ci` of piece `ii`
    long long ii = blockIdx.x;
    int ci = 0, issued = 0;
    Work iw;
    if (ii < total) iw = work_of<L::kRows>(p, kShape, plan, ii, G);
    auto issue = [&] {
      if (ii < total) {
        const int j = ci >> 1, key0 = (iw.x.from + j) * kTile;
        const bool is_v = ci & 1, is_new = iw.has_new && j == iw.chunks - 1;
        if (!C8) {
          ok = ok && (issued < kSlots || wait_or_abort(empty + issued % kSlots, (issued / kSlots - 1) & 1, p.status, abort));
          if (ok) {
            unsigned char* slot = slots + (issued % kSlots) * kSlotBytes;
            const int left = is_new ? iw.x.r.n : iw.x.r.len - key0;
            const unsigned char* src;
            long long pitch;
            if (is_new) {
              src = static_cast<const unsigned char*>(is_v ? p.v_new : p.k_new) + (iw.x.r.t0 * p.new_stride + iw.x.kvh * kD) * 2;
              pitch = p.new_stride * 2;
            } else {
              src = static_cast<const unsigned char*>(is_v ? p.v_cache : p.k_cache) + (iw.x.r.c0 + key0) * row_bytes + iw.x.kvh * kD * 2;
              pitch = row_bytes;
            }
            src += r0 * pitch + u * 16;
#pragma unroll
            for (int m = 0; m < 16; ++m)
              copy16(smem_addr(slot + tile_off(r0 + 8 * m, u)), src + m * kRowStep * pitch, r0 + 8 * m < left);
          }
        } else if (!is_new) {
          const int left = iw.x.r.len - key0;
          const unsigned char* src = static_cast<const unsigned char*>(is_v ? p.v_cache : p.k_cache) +
                                     (iw.x.r.c0 + key0 + r0) * row_bytes + iw.x.kvh * kD + u * 16;
          const uint32_t dst = smem_addr(raw + (issued % (L::kRaw > 0 ? L::kRaw : 1)) * kRawBytes + pt * 16);
#pragma unroll
          for (int m = 0; m < 8; ++m) copy16(dst + m * 2048, src + m * kRowStep * row_bytes, r0 + kRowStep * m < left);
          if (!is_v) {
            float* ks = scales + (issued / 2 % kScaleRing) * 2 * kTile + pt;
            const long long at = iw.x.kvh * p.cache_rows + iw.x.r.c0 + key0 + pt;
            copy4(smem_addr(ks), p.k_scale + at, pt < left);
            copy4(smem_addr(ks + kTile), p.v_scale + at, pt < left);
          }
        }
        ++issued;
        if (++ci == 2 * iw.chunks) {
          ci = 0;
          ii += step;
          if (ii < total) iw = work_of<L::kRows>(p, kShape, plan, ii, G);
        }
      }
      cp_async_commit();
    };
    // 16-bit caches: the copies themselves wait for free slots, which free only as chunks are made ready below
#pragma unroll 1
    for (int k = 0; k < kAhead; ++k) issue();
    int c = 0, chunk_no = 0, ord = 0;
#pragma unroll 1
    for (long long i = blockIdx.x; i < total && ok; i += step, ++ord) {
      const Work w = work_of<L::kRows>(p, kShape, plan, i, G);
      // ---- queries
      if (ord > 0) ok = wait_or_abort(qempty, (ord - 1) & 1, p.status, abort);
      if (ok) {
        const uint16_t* q = static_cast<const uint16_t*>(p.q);
        const int qu = pt & 15;
#pragma unroll 1
        for (int r = pt >> 4; r < (w.pair ? 2 * kTile : kTile); r += 8) {
          const int row = w.x.row0 + r, token = row / G;
          uint4 x = make_uint4(0u, 0u, 0u, 0u);
          if (r < w.rows)
            x = __ldg(reinterpret_cast<const uint4*>(q + (w.x.r.t0 + token) * p.q_stride + (w.x.kvh * G + row - token * G) * kD) + qu);
          if (C8) {
            float power = 1.f;
            if (BF) {
              power = row_power(row_max16(top_of(x)));
              x = bf16_to_half(x, inverse_power(power));
            }
            if (qu == 0) row_factor[(ord & 1) * L::kRows + r] = power * kScaleLog2;
          }
          *reinterpret_cast<uint4*>(smem + (r >> 7) * kSlotBytes + tile_off(r & 127, qu)) = x;
        }
        fence_proxy_async();
        mbar_arrive(qfull);
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
          if (!is_new) {
            cp_async_wait<kAhead>();
            const unsigned char* mine = raw + (c % (L::kRaw > 0 ? L::kRaw : 1)) * kRawBytes + pt * 16;
#pragma unroll 4
            for (int m = 0; m < 8; ++m) {
              const uint4 x = *reinterpret_cast<const uint4*>(mine + m * 2048);
              const uint4 a = make_uint4(e4m3x2_to_half2(x.x), e4m3x2_to_half2(x.x >> 16), e4m3x2_to_half2(x.y), e4m3x2_to_half2(x.y >> 16));
              const uint4 b = make_uint4(e4m3x2_to_half2(x.z), e4m3x2_to_half2(x.z >> 16), e4m3x2_to_half2(x.w), e4m3x2_to_half2(x.w >> 16));
              const int r = r0 + kRowStep * m, hi = u >> 2;  // units 4 to 7 the other way round: no bank twice
              *reinterpret_cast<uint4*>(slot + tile_off(r, 2 * u + hi)) = hi ? b : a;
              *reinterpret_cast<uint4*>(slot + tile_off(r, 2 * u + 1 - hi)) = hi ? a : b;
            }
          } else {
            bool found = false;
            const int nu = pt & 15;
#pragma unroll 1
            for (int r = pt >> 4; r < kMaxDrafts; r += 8) {
              const bool there = r < w.x.r.n;
              auto row_of = [&](const void* base) {
                return there ? __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + (w.x.r.t0 + r) * p.new_stride + w.x.kvh * kD) + nu)
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
          cp_async_wait<kAhead - 1>();
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
        mbar_arrive(full + c % kSlots);
        if (!C8) issue();
        if (is_v) ++chunk_no;
      }
    }
    cp_async_wait<0>();
  } else {
    // ---------------------------------------------------------------- softmax of group t
    const int t = warp >> 2;
    const int r = tid & (kTile - 1);
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t scol = tmem + lanes + kColS + t * kTile, ocol = tmem + lanes + kColO;
    bool ok = true;
    int c0 = 0, chunk0 = 0, ord = 0;
    uint32_t s_count = 0;
#pragma unroll 1
    for (long long i = blockIdx.x; i < total; i += step, ++ord) {
      const Work w = work_of<L::kRows>(p, kShape, plan, i, G);
      const int my_row = w.pair ? t * kTile + r : r;
      const bool mine = my_row < w.rows;
      const int at = w.x.row0 + (mine ? my_row : 0), token = at / G, head = w.x.kvh * G + at - token * G;
      float m = -CUDART_INF_F, l = 0.f, vs = C8 ? 0.f : 1.f, f = kScaleLog2;
      bool first = true;
#pragma unroll 1
      for (int j = w.pair ? 0 : t; j < w.chunks && ok; j += w.pair ? 1 : 2) {
        ok = wait_or_abort(sfull + t, s_count & 1, p.status, abort);
        ++s_count;
        const int cv = c0 + 2 * j + 1;
        if (C8) ok = ok && wait_or_abort(full + cv % kSlots, (cv / kSlots) & 1, p.status, abort);  // the scales, too
        if (!ok) break;
        tc_fence_after();
        const bool is_new = w.has_new && j == w.chunks - 1;
        const float4* ks = reinterpret_cast<const float4*>(scales + ((chunk0 + j) % kScaleRing) * 2 * kTile);
        const float4* vv = ks + kTile / 4;
        if (C8) f = row_factor[(ord & 1) * L::kRows + my_row];
        const int left = w.x.r.len - (w.x.from + j) * kTile;  // cache rows of this chunk
        const uint64_t seen = is_new && mine ? p.mask[w.x.r.t0 + token] & (w.x.r.n < 64 ? (1ull << w.x.r.n) - 1 : ~0ull) : 0ull;
        // scores of 32 keys, times the keys' scales; -infinity where the row does not see
        auto scores = [&](int b, float (&s)[32]) {
          uint32_t raw[32];
          tmem_ld32_issue(scol + 32 * b, raw);
          tmem_wait_ld32(raw);
#pragma unroll
          for (int e = 0; e < 32; ++e) s[e] = __uint_as_float(raw[e]);
          if (C8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 k = ks[8 * b + e];
              s[4 * e] *= k.x;
              s[4 * e + 1] *= k.y;
              s[4 * e + 2] *= k.z;
              s[4 * e + 3] *= k.w;
            }
          }
          if (is_new) {
            const uint32_t bits = b < 2 ? static_cast<uint32_t>(seen >> (32 * b)) : 0u;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!((bits >> e) & 1u)) s[e] = -CUDART_INF_F;
          } else if (32 * (b + 1) > left) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (32 * b + e >= left) s[e] = -CUDART_INF_F;
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
          if (!first) {
#pragma unroll 1
            for (int c = 0; c < kD; c += 32) {
              uint32_t o[32];
              tmem_ld32_issue(ocol + t * kTile + c, o);
              tmem_wait_ld32(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
              tmem_st32(ocol + t * kTile + c, o);
            }
          }
        }
        first = false;
        const float nm = m == -CUDART_INF_F ? 0.f : -m;
        const float inv = C8 ? (vs > 0.f ? 1.f / vs : 0.f) : 1.f;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int b = 0; b < blocks; ++b) {
          float s[32];
          scores(b, s);
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x = s[2 * e], y = s[2 * e + 1];
            fma2(x, y, f, nm);
            x = exp2_fast(x);
            y = exp2_fast(y);
            if (e & 1) add2(sum[2], sum[3], x, y);
            else add2(sum[0], sum[1], x, y);
            if (C8) {
              const float2 v = reinterpret_cast<const float2*>(vv)[16 * b + e];
              x *= v.x * inv;
              y *= v.y * inv;
            }
            pk[e] = pack16<kBf>(x, y);
          }
          // 16 columns of P over S columns 16 b .. 16 b + 15: read before by this thread's block b / 2
          asm volatile(
              "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
                  scol + 16 * b),
              "r"(pk[0]), "r"(pk[1]), "r"(pk[2]), "r"(pk[3]), "r"(pk[4]), "r"(pk[5]), "r"(pk[6]), "r"(pk[7]), "r"(pk[8]),
              "r"(pk[9]), "r"(pk[10]), "r"(pk[11]), "r"(pk[12]), "r"(pk[13]), "r"(pk[14]), "r"(pk[15])
              : "memory");
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
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
      const bool whole = w.x.of == 1;
      const bool two = !w.pair && w.chunks > 1;
      const bool any_wild = w.has_new && wild[ord & 3] == ord + 1;
      const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
      float* slot = slots_of(p) + (w.x.slot + w.x.j) * slot_floats(L::kRows);
      uint16_t* out = static_cast<uint16_t*>(p.out) + ((w.x.r.t0 + token) * p.n_heads + head) * kD;
      const int d_from = w.pair ? 0 : t * (kD / 2), d_to = w.pair ? kD : d_from + kD / 2;
      const uint32_t own = ocol + (w.pair ? t * kTile : 0);
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
          const uint64_t seen = p.mask[w.x.r.t0 + token];
          for (int k = 0; k < w.x.r.n; ++k)
            if ((seen >> k) & 1u) {
              const uint32_t* v = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.v_new) + (w.x.r.t0 + k) * p.new_stride + w.x.kvh * kD + d);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const uint32_t bad = not_finite2<BF>(v[e]);
                const float2 y = unpack16<BF>(v[e]);
                if (bad & 0x8000u) x[2 * e] += y.x;
                if (bad & 0x80000000u) x[2 * e + 1] += y.y;
              }
            }
        }
        if (mine && whole) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t y[4];
#pragma unroll
            for (int h = 0; h < 4; ++h)
              y[h] = l == 0.f ? 0u : pack16<BF>(x[8 * e + 2 * h] * inv, x[8 * e + 2 * h + 1] * inv);
            *reinterpret_cast<uint4*>(out + d + 8 * e) = make_uint4(y[0], y[1], y[2], y[3]);
          }
        } else if (mine) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            __stcg(reinterpret_cast<float4*>(slot + my_row * kD + d) + e, make_float4(x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]));
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(oread);
      if (mine && (w.pair || t == 0)) {
        if (whole) {
          if (p.lse != nullptr) p.lse[head * p.new_rows + w.x.r.t0 + token] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
        } else {
          __stcg(reinterpret_cast<float2*>(slot + L::kRows * kD) + my_row, make_float2(m, l));
        }
        if (w.x.j == 0) table_of(p)[head * p.new_rows + w.x.r.t0 + token] = make_int2(w.x.slot, w.x.of);
      }
      c0 += 2 * w.chunks;
      chunk0 += w.chunks;
      asm volatile("bar.sync 1, 256;" ::: "memory");  // the groups' sums are read before they are written again
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
