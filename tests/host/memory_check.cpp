// Host-only check of the overlap test, built with AddressSanitizer and UBSan: against every byte marked one by one, over
// random buffers in one piece and of rows, apart, touching, interleaved and overlapping.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "memory.hpp"

using namespace caramel;

int main() {
  std::mt19937_64 rng(11);
  uint32_t met[2] = {0, 0}, interleaved = 0;
  for (int it = 0; it < 400000; ++it) {
    auto below = [&](uint64_t n) { return rng() % n; };
    const uint64_t es = 2 + 2 * below(2), pitch = 1 + below(9), far = 1 + below(60), count = 2 + below(3);
    Memory m;
    std::vector<int> readers(1200), writers(1200);
    bool want = false, extents = false;
    std::vector<std::vector<uint64_t>> ends;
    for (uint64_t b = 0; b < count; ++b) {
      const bool written = below(3) != 0, rows = below(4) != 0;
      const uint64_t at = below(far) * es, n = below(6), columns = rows ? 1 + below(pitch) : below(30);
      if (rows) m.add_rows(1000 + at, n, pitch, columns, es, written);
      else m.add(1000 + at, columns * es, written);
      for (uint64_t r = 0; r < (rows ? n : 1); ++r)
        for (uint64_t c = 0; c < columns * es; ++c) {
          const uint64_t byte = at + r * pitch * es + c;
          ++(written ? writers : readers)[byte];
          want = want || writers[byte] > 1 || (writers[byte] && readers[byte]);
        }
      if (rows && n) ends.push_back({at, at + ((n - 1) * pitch + columns) * es});
    }
    for (size_t i = 0; i < ends.size(); ++i)
      for (size_t j = 0; j < i; ++j) extents = extents || (ends[i][0] < ends[j][1] && ends[j][0] < ends[i][1]);
    if (m.overlap() != want) {
      std::printf("FAIL case %d: %d wanted\n", it, int(want));
      return 1;
    }
    ++met[want];
    interleaved += extents && !want;
  }
  // the most buffers that a call has, side by side in one array
  Memory m;
  for (uint64_t w = 0; w < CARAMEL_MAX_WORLD; ++w) m.add_rows(4096 + w * 12, 1000, 3 * CARAMEL_MAX_WORLD, 3, 4, true);
  for (uint64_t w = 0; w < 3 * CARAMEL_MAX_WORLD + 1; ++w) m.add(1u << 28, 64, false);
  if (m.overlap() || met[0] < 1000 || met[1] < 1000 || interleaved < 1000) return 1;
  std::printf("memory_check ok: %u apart (%u interleaved), %u overlapping\n", met[0], interleaved, met[1]);
  return 0;
}
