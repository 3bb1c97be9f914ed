// Sanitizer driver for the streaming product's loop over blocks (test infrastructure; runs on the CPU only): the runs of
// its waves and the scale byte that each place takes, by the functions that the kernel uses, for every part of a sum of up to
// some hundred blocks.  Prints "ok <places>", or names the first mistake.
#include <stdio.h>
#include <vector>

#include "fp8_tile.h"

int main() {
  long places = 0;
  for (int waves : {4, 8})
    for (int U : {2, 4})
      for (int k0 = 0; k0 < 9; ++k0)
        for (int k1 = k0 - 2; k1 < 150; ++k1) {
          std::vector<int> seen(160, 0);
          for (int wave = 0; wave < waves; ++wave) {
            const spl::Fp8Run r = spl::fp8_run(k0, k1, wave, waves);
            for (int b = r.b0; b < r.b1 && r.first < r.b1; b += U)
              for (int u = 0; u < U; ++u) {
                ++places;
                const int word = b & ~3;
                const uint32_t bytes = (uint32_t)(word & 0xff) | (uint32_t)((word + 1) & 0xff) << 8 |
                                       (uint32_t)((word + 2) & 0xff) << 16 | (uint32_t)((word + 3) & 0xff) << 24;
                const uint32_t scale = spl::fp8_scale_at(bytes, b + u) & 255u;
                if (b + u < k0 || b + u >= r.b1) continue;
                ++seen[b + u];
                if (scale != (uint32_t)((b + u) & 0xff)) return printf("scale of block %d of [%d, %d)\n", b + u, k0, k1), 1;
              }
          }
          for (int b = 0; b < 160; ++b)
            if (seen[b] != (b >= k0 && b < k1)) return printf("block %d of [%d, %d) %d times\n", b, k0, k1, seen[b]), 1;
        }
  printf("ok %ld\n", places);
  return 0;
}
