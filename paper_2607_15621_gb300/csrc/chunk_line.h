// Counts of the line of work of tree_tc.cu: every (request, tile of its rows, kv head) is an item of some chunks of keys.
// 1024 requests of 64 x 64 rows over one shared cache of 4 million rows and 8 kv heads are 2^32 chunks and more, so sums are
// kept in 64 bits; places on the line have 32, and a longer line is not cut. No CUDA in here: the host compiles it too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define FSX_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define FSX_HOST_DEVICE inline
#endif

namespace fsx {

constexpr uint64_t kLineEnd = 1ull << 31;  // of a line that is cut
constexpr uint32_t kLeastRange = 4;        // chunks of a range or of a piece of a cut item

FSX_HOST_DEVICE uint32_t above(uint32_t a, uint32_t b) { return (a + b - 1) / b; }

// The chunks of one lane's requests, in two parts whose sums over 32 lanes fit 32 bits: 32 requests of at most 4096 items of
// 2^24 + 1 chunks are below 2^42.
struct ChunkCount {
  static constexpr int kLow = 26;
  uint64_t n = 0;
  FSX_HOST_DEVICE void add(uint32_t items, uint32_t chunks) { n += static_cast<uint64_t>(items) * chunks; }
  FSX_HOST_DEVICE uint32_t low() const { return static_cast<uint32_t>(n) & ((1u << kLow) - 1); }
  FSX_HOST_DEVICE uint32_t high() const { return static_cast<uint32_t>(n >> kLow); }
  FSX_HOST_DEVICE static uint64_t sum(uint32_t lows, uint32_t highs) { return (static_cast<uint64_t>(highs) << kLow) + lows; }
};

// Chunks of a range, one range per CTA; 0: the line is too long to be cut
FSX_HOST_DEVICE uint32_t range_of(uint64_t total, uint32_t ctas) {
  if (total >= kLineEnd) return 0;
  const uint32_t even = above(static_cast<uint32_t>(total), ctas);
  return even > kLeastRange ? even : kLeastRange;
}

}  // namespace fsx
