// The counts of csrc/chunk_line.h against plain 128-bit sums: requests go to 32 lanes in turn, as in the kernel.
#include <cstdio>
#include <initializer_list>

#include "chunk_line.h"

namespace {

struct Shape {
  int B, tokens, group, kv_heads;
  long long rows;  // of each request's cache
  int tile;
};

int check(const Shape& s, unsigned ctas) {
  const unsigned items = fsx::above(s.tokens * s.group, s.tile) * s.kv_heads;
  const unsigned chunks = static_cast<unsigned>((s.rows + 127) / 128 + 1);
  fsx::ChunkCount lane[32];
  unsigned __int128 want = 0;
  for (int b = 0; b < s.B; ++b) {
    lane[b % 32].add(items, chunks);
    want += static_cast<unsigned __int128>(items) * chunks;
  }
  uint32_t lows = 0, highs = 0;  // sums of 32 bits, as a warp adds
  for (const fsx::ChunkCount& x : lane) lows += x.low(), highs += x.high();
  const uint64_t total = fsx::ChunkCount::sum(lows, highs);
  const uint32_t per = fsx::range_of(total, ctas);
  if (total != want) return 1;
  if (want >= (1ull << 31)) return per == 0 ? 0 : 2;
  // whole ranges end within 32 bits and hold everything
  const uint64_t end = static_cast<uint64_t>(per) * ctas;
  return per >= 4 && end >= total && (per == 4 || end - total < ctas) ? 0 : 3;
}

}  // namespace

int main() {
  const Shape shapes[] = {
      {1, 1, 17, 1, 0, 128},
      {16, 11, 4, 8, 480, 128},
      {1, 50, 4, 8, 32768, 256},
      {1024, 64, 64, 8, 1 << 20, 128},
      {1024, 64, 64, 8, 1 << 22, 128},        // 2^32 chunks and more
      {1024, 64, 64, 64, 17000000, 128},      // every HBM byte of one shared cache
      {1024, 64, 1, 4096, 2147483647, 128},   // what the entry point accepts
      {1, 64, 64, 64, 2147483647, 128},
  };
  int n = 0;
  for (const Shape& s : shapes)
    for (unsigned ctas : {1u, 148u, 152u, 256u}) {
      const int bad = check(s, ctas);
      if (bad) {
        std::printf("bad %d: shape %d, %u CTAs\n", bad, static_cast<int>(&s - shapes), ctas);
        return 1;
      }
      ++n;
    }
  std::printf("ok %d\n", n);
  return 0;
}
