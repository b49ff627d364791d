// Host-only check of the overlap test where rows of different pitch meet, built with AddressSanitizer and UBSan: what it lets pass shares
// no byte, marked one by one; what it refuses shares one, or is two buffers of several rows whose stretches meet.
#include <cstdio>
#include <random>
#include <vector>

#include "memory.hpp"

using namespace caramel;

int main() {
  std::mt19937_64 rng(5);
  auto below = [&](uint64_t n) { return rng() % n; };
  uint32_t met[2] = {0, 0};
  for (int it = 0; it < 400000; ++it) {
    Memory m;
    std::vector<int> bytes(2000);
    bool shared = false;
    uint64_t lo[2], hi[2], pitch[2], rows[2];
    for (int b = 0; b < 2; ++b) {
      const uint64_t es = 2 + 2 * below(2);
      pitch[b] = (1 + below(9)) * es;
      rows[b] = below(6);
      const uint64_t at = 1000 + below(80) * 2, columns = 1 + below(pitch[b] / es);
      m.add_rows(at, rows[b], pitch[b] / es, columns, es, true);
      lo[b] = at;
      hi[b] = rows[b] ? at + (rows[b] - 1) * pitch[b] + columns * es : at;
      for (uint64_t r = 0; r < rows[b]; ++r)
        for (uint64_t c = 0; c < columns * es; ++c) shared = ++bytes[at + r * pitch[b] + c] > 1 || shared;
    }
    const bool refused = m.overlap();
    const bool unlike = pitch[0] != pitch[1] && rows[0] > 1 && rows[1] > 1 && lo[0] < hi[1] && lo[1] < hi[0];
    if (refused != (shared || unlike)) {
      std::printf("FAIL case %d: shared %d, refused %d\n", it, int(shared), int(refused));
      return 1;
    }
    ++met[refused];
  }
  if (met[0] < 1000 || met[1] < 1000) return 1;
  std::printf("pitch_check ok: %u apart, %u refused\n", met[0], met[1]);
  return 0;
}
