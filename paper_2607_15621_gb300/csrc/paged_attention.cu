// Attention of one new token of each request over its cache in pages (fsx_paged_attention), all of them or those that a
// list picks for each kv head.
//
// The queries of a kv head's group are the rows, 8 NT of them an item, over the warps' steps of few_rows.cuh: 16 keys a step, keys
// as M of the matrix instructions. Bound by the cache's bytes. A page holds 16 rows or more, so the 16 keys of a step lie in one page and
// a warp needs one page number a step: at the start of a piece its lanes look up the pages of 32 steps at once, and a
// step's comes by a shuffle, so that no copy waits for the table.
//
// Items (request, tile of the group, kv head) are cut into pieces of at most 28 chunks of 64 keys, by the count of all chunks, and
// CTAs take pieces from one queue; the pieces of an item are joined by the CTA that ends last, in the order of the keys.
// A piece that meets a page number outside the cache marks its result, and its item writes nothing.
#include <math_constants.h>

#include "few_rows.cuh"
#include "fsx.h"
#include "kernels.h"
#include "pages.h"

namespace fsx {

namespace {

constexpr int kFew = 8, kMany = 28;  // chunks of an item that is not cut, and of a piece
constexpr int kHeader = 64;          // ints of the workspace: [0] pieces taken from the queue, [1] CTAs that are done
constexpr int kCounters = 8192;      // then one for each slot

struct Plan {
  uint32_t* pieces;  // [B + 1] pieces of the requests before
  int* slots;        // [B + 1] slots of the requests before
  int most;          // chunks of a piece
};
__host__ __device__ constexpr size_t plan_bytes(int B) { return (B + 1) * 2 * sizeof(int); }

struct Request {
  int len;    // rows
  int pages;  // that hold them
  int steps;  // of 16 keys, over all pages or the picked ones
};
// false: the length is negative or more than the table's pages hold; no steps then and no items
__device__ __forceinline__ bool request_of(const PagedArgs& p, int b, Request& r) {
  const long long len = p.pages.lengths[b];
  r.len = r.pages = r.steps = 0;
  if (len < 0 || len > static_cast<long long>(p.pages.width) << p.pages.shift || len > 0x7fffffffll - 64) return false;
  r.len = static_cast<int>(len);
  r.pages = static_cast<int>((len + (1 << p.pages.shift) - 1) >> p.pages.shift);
  r.steps = p.picked != nullptr ? min(r.pages, p.n_picked) << (p.pages.shift - 4) : (r.len + 15) >> 4;
  return true;
}
__device__ __forceinline__ int chunks_of(const Request& r) { return max(1, (r.steps + kWarps - 1) / kWarps); }
__device__ __forceinline__ int pieces_of(int n, int most) { return n <= kFew ? 1 : (n + most - 1) / most; }

// By all threads of the CTA; `scratch`: 2 values per warp. `items`: of a request that is in order.
__device__ __forceinline__ Plan make_plan(const PagedArgs& p, long long items, int slots, void* at, long long* scratch) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = p.pages.B;
  const int per = (B + kThreads - 1) / kThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
  Plan plan;
  plan.pieces = static_cast<uint32_t*>(at);
  plan.slots = reinterpret_cast<int*>(plan.pieces + B + 1);
  long long total = 0;
  for (int b = b0; b < b1; ++b) {
    Request r;
    const bool fine = request_of(p, b, r);
    if (!fine && blockIdx.x == 0) set_status(p.status, kStatusDeviceArg);
    plan.slots[b] = fine ? chunks_of(r) : 0;  // for the second look
    total += plan.slots[b];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) scratch[warp] = total;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += scratch[w];
  total *= items;
  // an even share or a part of it; cut items of n > most chunks take at most 2 n / most slots
  if (total < 0x3fffffff) {
    const uint32_t even = (static_cast<uint32_t>(total) + gridDim.x - 1) / gridDim.x, turns = (even + kMany - 1) / kMany;
    const uint32_t share = turns > 0 ? (even + turns - 1) / turns : 1;
    plan.most = static_cast<int>(max(max(share, (2 * static_cast<uint32_t>(total) + slots - 1) / slots), (kFew + 1u) / 2));
  } else {
    plan.most = static_cast<int>(min((2 * total + slots - 1) / slots, 0x7fffffffll));
  }
  long long mine = 0, mine_slots = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = plan.slots[b], of = n > 0 ? pieces_of(n, plan.most) : 0;
    plan.pieces[b] = static_cast<uint32_t>(mine);  // within this thread's requests
    plan.slots[b] = static_cast<int>(mine_slots);
    mine += items * of;
    mine_slots += of > 1 ? items * of : 0;
  }
  long long sum = mine, sum_slots = mine_slots;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long up = __shfl_up_sync(0xffffffffu, sum, o), up_slots = __shfl_up_sync(0xffffffffu, sum_slots, o);
    if (lane >= o) {
      sum += up;
      sum_slots += up_slots;
    }
  }
  __syncthreads();
  if (lane == 31) {
    scratch[warp] = sum;
    scratch[kWarps + warp] = sum_slots;
  }
  __syncthreads();
  sum -= mine;
  sum_slots -= mine_slots;
  for (int w = 0; w < warp; ++w) {
    sum += scratch[w];
    sum_slots += scratch[kWarps + w];
  }
  for (int b = b0; b < b1; ++b) {
    plan.pieces[b] += static_cast<uint32_t>(sum);
    plan.slots[b] += static_cast<int>(sum_slots);
  }
  if (tid == kThreads - 1) plan.pieces[B] = static_cast<uint32_t>(sum + mine);
  __syncthreads();
  return plan;
}

struct Piece {
  Request r;
  int b, kvh, row0;  // request, kv head, first row (head of the group) of the tile
  int from, to;      // chunks
  int slot, j, of;   // piece j of `of`; `slot` is that of piece 0
};
__device__ __forceinline__ Piece piece_at(const PagedArgs& p, const Plan& plan, int tile_rows, uint32_t i) {
  int lo = 0, hi = p.pages.B;  // pieces[lo] <= i < pieces[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (plan.pieces[mid] <= i) lo = mid;
    else hi = mid;
  }
  Piece x;
  x.b = lo;
  request_of(p, lo, x.r);
  const int n = chunks_of(x.r);
  x.of = pieces_of(n, plan.most);
  const uint32_t rel = i - plan.pieces[lo], item = rel / static_cast<uint32_t>(x.of);
  x.j = static_cast<int>(rel - item * x.of);
  x.slot = plan.slots[lo] + static_cast<int>(rel) - x.j;
  const uint32_t least = static_cast<uint32_t>(n) / static_cast<uint32_t>(x.of), more = n - least * x.of;
  x.from = static_cast<int>(x.j * least + min(static_cast<uint32_t>(x.j), more));
  x.to = static_cast<int>(x.from + least + (static_cast<uint32_t>(x.j) < more ? 1 : 0));
  const uint32_t tile = item / static_cast<uint32_t>(p.n_kv_heads);
  x.kvh = static_cast<int>(item - tile * p.n_kv_heads);
  x.row0 = static_cast<int>(tile) * tile_rows;
  return x;
}

// First cache row of step `step` and how many of its 16 rows are keys of the request. False: no page of the cache.
__device__ __forceinline__ bool look_up(const PagedArgs& p, const Piece& it, int step, int& row, int& left) {
  row = left = 0;
  if (step >= it.r.steps) return true;
  const int shift = p.pages.shift, in_page = step & ((1 << (shift - 4)) - 1);
  int page = step >> (shift - 4);
  if (p.picked != nullptr) {
    page = __ldg(p.picked + (static_cast<long long>(it.b) * p.n_kv_heads + it.kvh) * p.n_picked + page);
    if (page == -1) return true;
    if (page < 0 || page >= it.r.pages) return false;
  }
  left = min(16, it.r.len - ((page << shift) + in_page * 16));
  if (left <= 0) {
    left = 0;
    return true;
  }
  const int at = __ldg(p.pages.table + static_cast<long long>(it.b) * p.pages.width + page);
  if (at < 0 || at >= p.pages.n_pages) {
    left = 0;
    return false;
  }
  row = (at << shift) + in_page * 16;
  return true;
}

template <bool C8, int NT>
struct Shared {  // and the plan behind it
  long long scratch[2 * kWarps];
  __align__(128) unsigned char ring[kWarps][Fit<C8, NT>::kStages * Stage<C8>::kBytes];
  float m[kWarps][8 * NT], l[kWarps][8 * NT];
  float o[kWarps][Fit<C8, NT>::kPass][kD];
  int left[kWarps][4];  // keys of the ring's stages
  int bad[kWarps];
  uint32_t next;
  int last;
};

constexpr size_t slot_floats(int nt) { return static_cast<size_t>(8) * nt * (kD + 2); }
constexpr int slots_of(int nt) { return kCounters / nt; }  // 34 MB

template <int NT>
__device__ __forceinline__ float* slot_at(const PagedArgs& p, int slot) {
  return reinterpret_cast<float*>(static_cast<int*>(p.workspace) + kHeader + kCounters) +
         static_cast<size_t>(slot) * slot_floats(NT);
}

// Queries of the item's rows, as they lie
template <bool C8, int NT>
__device__ __forceinline__ void load_queries(uint32_t (&qf)[NT][8][2], const PagedArgs& p, const Piece& it, int G) {
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint16_t* q = static_cast<const uint16_t*>(p.q) + it.b * p.q_stride + static_cast<long long>(it.kvh) * G * kD;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = it.row0 + 8 * t + g;
    const bool there = row < G;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int d = C8 ? (k >> 2) * 64 + 16 * c + 4 * (k & 3) : 8 * (c + 4 * (k >> 1)) + 4 * (k & 1);
      const uint2 w = there ? __ldg(reinterpret_cast<const uint2*>(q + row * kD + d)) : make_uint2(0u, 0u);
      qf[t][k][0] = w.x;
      qf[t][k][1] = w.y;
    }
  }
}

template <bool BF, bool C8, int NT>
__global__ void __launch_bounds__(kThreads, Fit<C8, NT>::kCtas) paged_kernel(const PagedArgs p) {
  using S = Stage<C8>;
  constexpr int kStages = Fit<C8, NT>::kStages, kPass = Fit<C8, NT>::kPass;
  constexpr int kPerRow = S::kRow / 16;
  constexpr int kTile = 8 * NT;
  extern __shared__ __align__(128) unsigned char raw_smem[];
  Shared<C8, NT>& sm = *reinterpret_cast<Shared<C8, NT>*>(raw_smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const int G = p.n_heads / p.n_kv_heads;
  int* header = static_cast<int*>(p.workspace);
  const long long items = static_cast<long long>((G + kTile - 1) / kTile) * p.n_kv_heads;
  const Plan plan = make_plan(p, items, slots_of(NT), raw_smem + sizeof(sm), sm.scratch);
  const uint32_t total = plan.pieces[p.pages.B];
  const long long row_bytes = static_cast<long long>(p.n_kv_heads) * S::kRow;
  const uint32_t ring = smem_addr(sm.ring[warp]);

  // this warp's copies of a piece: chunks staged .. count - 1, of which it takes every one's `warp`-th 16 keys
  Piece it;
  const unsigned char *kc = nullptr, *vc = nullptr;
  const float* scales = nullptr;
  int staged = 0, count = 0, slot_in = 0, rows_of = 0, left_of = 0;
  bool bad = false;
  auto copy_next = [&](const Piece& x) {
    if (staged < count) {
      if ((staged & 31) == 0)  // a lane a step
        bad = !look_up(p, x, staged + lane < count ? (x.from + staged + lane) * kWarps + warp : 0x7fffffff, rows_of, left_of) || bad;
      const int row = __shfl_sync(0xffffffffu, rows_of, staged & 31), left = __shfl_sync(0xffffffffu, left_of, staged & 31);
      if (left > 0) {
        const uint32_t dst = ring + slot_in * S::kBytes;
        copy_rows<C8, false>(dst, kc + row * row_bytes, row_bytes, left);
        copy_rows<C8, true>(dst, vc + row * row_bytes, row_bytes, left);
        if (C8) copy4(dst + S::kOffScale + lane * 4, scales + row, (lane & 15) < left);
      }
      if (lane == 0) sm.left[warp][slot_in] = left;
    }
    cp_async_commit();
    ++staged;
    slot_in = slot_in + 1 == kStages ? 0 : slot_in + 1;
  };
  auto begin = [&](const Piece& x) {
    staged = 0;
    count = x.to - x.from;
    const long long at = static_cast<long long>(lane / kPerRow) * row_bytes + x.kvh * S::kRow + (lane % kPerRow) * 16;
    kc = static_cast<const unsigned char*>(p.k_cache) + at;
    vc = static_cast<const unsigned char*>(p.v_cache) + at;
    if (C8) scales = (lane < 16 ? p.k_scale : p.v_scale) + x.kvh * p.cache_rows + (lane & 15);
    slot_in = 0;
    bad = false;
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) copy_next(x);
  };

  uint32_t i = blockIdx.x;
  uint32_t qf[NT][8][2];
  if (i < total) {
    it = piece_at(p, plan, kTile, i);
    load_queries<C8, NT>(qf, p, it, G);
    begin(it);
  }
#pragma unroll 1
  while (i < total) {
    if (tid == 0) sm.next = gridDim.x + atomicAdd(reinterpret_cast<unsigned*>(header), 1u);
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
    int slot_out = 0;
    const int chunks = it.to - it.from;
#pragma unroll 1
    for (int n = 0; n < chunks; ++n) {
      cp_async_wait<kStages - 2>();
      __syncwarp();  // every lane's copies of the stage; and the stage before is read
      const int left = sm.left[warp][slot_out];
      copy_next(it);
      if (left > 0) cache_step<BF, C8, NT>(st, sm.ring[warp] + slot_out * S::kBytes, qf, f, left);
      slot_out = slot_out + 1 == kStages ? 0 : slot_out + 1;
    }
    cp_async_wait<0>();
    const bool any_bad = __any_sync(0xffffffffu, bad);
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

    const int rows = min(kTile, G - it.row0);
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
    if (lane == 0) sm.bad[warp] = any_bad;
    __syncthreads();
    // ---- the next piece's first copies go out before this one's results are put together
    const bool wrong = (sm.bad[0] | sm.bad[1] | sm.bad[2] | sm.bad[3]) != 0;
    if (wrong && tid == 0) set_status(p.status, kStatusDeviceArg);
    const uint32_t i_next = sm.next;
    Piece next = it;
    if (i_next < total) {
      next = piece_at(p, plan, kTile, i_next);
      load_queries<C8, NT>(qf, p, next, G);
      begin(next);
    }
    // ---- the four warps' results, kPass rows at a time; a thread a dim
    auto lse_at = [&](int head) -> float& { return p.lse[static_cast<long long>(head) * p.pages.B + it.b]; };
    float* slot = slot_at<NT>(p, it.slot + it.j);
#pragma unroll
    for (int base = 0; base < kTile; base += kPass) {
      if (base >= rows) break;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = 8 * t + 2 * c + r;
          if (row >= base && row < base + kPass && row < rows) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<float2*>(&sm.o[warp][row - base][out_dim<C8>(g, j, 0)]) = make_float2(st.o[j][t][r], st.o[j][t][2 + r]);
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
        const int head = it.kvh * G + it.row0 + row;
        if (it.of > 1) {
          __stcg(slot + row * kD + tid, o);
          if (tid == 0) __stcg(reinterpret_cast<float2*>(slot + kTile * kD) + row, make_float2(m, wrong ? -1.f : l));
        } else if (!wrong) {
          const float y = l == 0.f ? 0.f : o / l;
          static_cast<uint16_t*>(p.out)[(static_cast<long long>(it.b) * p.n_heads + head) * kD + tid] = static_cast<uint16_t>(pack16<BF>(y, y));
          if (p.lse != nullptr && tid == 0) lse_at(head) = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
        }
      }
      __syncthreads();
    }
    if (it.of > 1) {
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        int* counter = header + kHeader + it.slot;
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
          bool refused = false;
#pragma unroll 1
          for (int j0 = 0; j0 < it.of; j0 += kJoin) {  // in the order of the keys; the loads of kJoin pieces at once
            float2 x[kJoin];
            float4 v[kJoin];
#pragma unroll
            for (int j = 0; j < kJoin; ++j) {
              const float* other = first + min(j0 + j, it.of - 1) * slot_floats(NT);
              x[j] = __ldcg(reinterpret_cast<const float2*>(other + kTile * kD) + row);
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
              refused = refused || x[j].y < 0.f;
              if (j0 + j < it.of) {
                l += a * x[j].y;
                o.x += a * v[j].x;
                o.y += a * v[j].y;
                o.z += a * v[j].z;
                o.w += a * v[j].w;
              }
            }
          }
          if (refused) continue;
          const int head = it.kvh * G + it.row0 + row;
          const float inv = l == 0.f ? 0.f : 1.f / l;
          uint16_t* out = static_cast<uint16_t*>(p.out) + (static_cast<long long>(it.b) * p.n_heads + head) * kD + 4 * lane;
          *reinterpret_cast<uint2*>(out) = make_uint2(pack16<BF>(o.x * inv, o.y * inv), pack16<BF>(o.z * inv, o.w * inv));
          if (p.lse != nullptr && lane == 0) lse_at(head) = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
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
  return {reinterpret_cast<const void*>(&paged_kernel<BF, C8, NT>), sizeof(Shared<C8, NT>), Fit<C8, NT>::kCtas};
}
template <bool BF, bool C8>
Kernel kernel_of(int nt) {
  return nt == 1 ? kernel_for<BF, C8, 1>() : kernel_for<BF, C8, 2>();
}

int tile_count(int n_heads, int n_kv_heads) { return n_heads / n_kv_heads <= 8 ? 1 : 2; }

}  // namespace

size_t paged_attention_workspace_bytes(int B, int n_heads, int n_kv_heads) {
  const int nt = tile_count(n_heads, n_kv_heads);
  return (kHeader + kCounters) * sizeof(int) + slots_of(nt) * slot_floats(nt) * sizeof(float);
}

cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, bool cache8, cudaStream_t stream) {
  const int nt = tile_count(a.n_heads, a.n_kv_heads);
  const Kernel k = dtype == FSX_BF16 ? (cache8 ? kernel_of<true, true>(nt) : kernel_of<true, false>(nt))
                                     : (cache8 ? kernel_of<false, true>(nt) : kernel_of<false, false>(nt));
  const size_t smem = k.smem + plan_bytes(a.pages.B);
  const int sms = sm_count();
  if (sms == 0) return cudaErrorNoDevice;
  const cudaError_t e = allow_shared_memory(k.fn, smem);
  if (e != cudaSuccess) return e;
  void* args[] = {const_cast<PagedArgs*>(&a)};
  return launch_ex(k.fn, dim3(static_cast<unsigned>(sms * k.ctas)), dim3(kThreads), smem, stream, false, args);
}

}  // namespace fsx
