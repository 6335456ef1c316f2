// What the tensor-core attention kernels of prompts and drafts share: bounded waits that end together,
// operand descriptors and tensor-memory moves for 128-row tiles, and exponentials.
#pragma once

#include <cuda.h>
#include <math_constants.h>

#include "device_util.cuh"
#include "tcgen05.cuh"

namespace fsx {

// exponents are taken of log2(e) / sqrt(128) times the raw score
constexpr float kScaleLog2 = 1.4426950408889634f * 0.08838834764831845f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// (a0, a1) * (b0, b1) + (c0, c1) and (a0, a1) + (b0, b1), one instruction each
__device__ __forceinline__ void fma2(float& a0, float& a1, float b, float c) {
  asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %2};\n mov.b64 z, {%3, %3};\n"
      " fma.rn.f32x2 x, x, y, z;\n mov.b64 {%0, %1}, x;\n}"
      : "+f"(a0), "+f"(a1)
      : "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float& a0, float& a1, float b0, float b1) {
  asm("{\n .reg .b64 x, y;\n mov.b64 x, {%0, %1};\n mov.b64 y, {%2, %3};\n add.rn.f32x2 x, x, y;\n"
      " mov.b64 {%0, %1}, x;\n}"
      : "+f"(a0), "+f"(a1)
      : "f"(b0), "f"(b1));
}

template <bool BF>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {  // round to nearest even, lo in the low half
  uint32_t r;
  if (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// bits 15 / 31 where a packed 16-bit value is an infinity or a NaN
template <bool BF>
__device__ __forceinline__ uint32_t not_finite2(uint32_t v) {
  return ((v & 0x7fff7fffu) + (BF ? 0x00800080u : 0x04000400u)) & 0x80008000u;
}
template <bool BF>
__device__ __forceinline__ float2 unpack16(uint32_t v) {
  if (BF) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

// N- (or M-)contiguous operand, 128-byte swizzle: `lbo` between 64-value blocks along N, `sbo` between
// groups of 8 along K
__device__ __forceinline__ uint64_t sw128_desc_mn(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | static_cast<uint64_t>((lbo >> 4) & 0x3FFFu) << 16 |
         static_cast<uint64_t>((sbo >> 4) & 0x3FFFu) << 32 | static_cast<uint64_t>(1) << 46 |
         static_cast<uint64_t>(2) << 61;
}
// kind::f16 with fp32 sums: bf16 or fp16 operands, B K-major or N-contiguous
__host__ __device__ constexpr uint32_t idesc_16(bool bf, int m, int n, bool b_mn) {
  return (1u << 4) | (bf ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? (1u << 16) : 0u) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
// D[tmem] (+)= A[tmem] B[smem], one K = 16 step
__device__ __forceinline__ void umma_f16_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One lane of a converged warp, the same one every time. MMAs of a loop are issued under this predicate while the
// warp stays together: under `if (lane == 0)` their operands are moved to uniform registers one after another (4 MMAs
// of N = 128 in a loop: 631 cycles against 260).
__device__ __forceinline__ bool elect_lane() {
  uint32_t e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(e));
  return e != 0u;
}

// 32 columns of this thread's lane, from registers
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 16 bytes to shared memory, zeros if not `there` (then nothing is read)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

__device__ __forceinline__ uint32_t try_bar(uint32_t addr, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(addr), "r"(parity)
      : "memory");
  return done;
}
// Waits for phase `parity` of an mbarrier; false once a wait of the CTA has given up (about one second:
// the status word and `abort` are set). The timer's low word wraps after 4.3 s. A lane whose time is up leaves by the flag, which
// its whole warp reads at once: the lanes of a warp get the same answer.
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, int* status, volatile int* abort) {
  const uint32_t addr = smem_addr(bar);
  if (__builtin_expect(try_bar(addr, parity) != 0u, 1)) return true;
  uint32_t t0;
  asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t0));
#pragma unroll 1
  for (;;) {
    if (try_bar(addr, parity)) return true;
    if (*abort) return false;
    uint32_t now;
    asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(now));
    if (now - t0 > kWaitLimitNs && now - t0 < 0x80000000u) {
      set_status(status, kStatusTimeout);
      *abort = 1;
    }
  }
}

// The warpgroup's share of the block's registers from here on (a multiple of 8 per thread). The shares of
// all warpgroups together stay within what the block was launched with.
template <int N>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void leave_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// a tile of two swizzled blocks of 64 columns through a map of encode_kv_map (row, block 0, head) or encode_q_map
// (head, row, block 0)
__device__ __forceinline__ void tma_load_chunk(void* dst, const CUtensorMap* map, int y, int z, int w, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];" ::"r"(smem_addr(dst)),
      "l"(map), "r"(0), "r"(y), "r"(z), "r"(w), "r"(smem_addr(bar))
      : "memory");
}

// The other way, in the caller's bulk group
__device__ __forceinline__ void tma_store_chunk(const CUtensorMap* map, const void* src, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"(map), "r"(0),
               "r"(y), "r"(z), "r"(w), "r"(smem_addr(src))
               : "memory");
}

// Byte offset of 16-byte unit u (0..15) of row r in a [128][128] tile of 16-bit values: two swizzled
// blocks of 64 columns, 16 KB apart.
__device__ __forceinline__ uint32_t tile_off(int r, int u) {
  return static_cast<uint32_t>((u >> 3) * 16384 + (r >> 3) * 1024 + (r & 7) * 128 + (((u & 7) ^ (r & 7)) << 4));
}

}  // namespace fsx
