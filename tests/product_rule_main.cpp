// The rule's answers for calls on standard input, "T V H z_bytes" a line: the way that it takes and what it gives for each, the strips
// of each and whether a launch of them holds (fewer than 2^32 threads).
#include <cstdio>

#include "product_rule.h"

int main() {
  long long T;
  int V, H, z_bytes;
  while (std::scanf("%lld %d %d %d", &T, &V, &H, &z_bytes) == 4) {
    const int pitch = (H + 127) / 128 * 128;
    std::printf("%d", adwin::product_tile(T, V, pitch, z_bytes));
    for (const adwin::ProductWay& p : adwin::kProductWays) {
      const long long tiles = (T + p.tokens - 1) / p.tokens;
      const int strips = adwin::product_strips(tiles, (V + p.entries - 1) / p.entries);
      std::printf(" %.2f %d %d", adwin::product_us(p, T, V, pitch, z_bytes), strips, tiles * strips * 256 < (1ll << 32));
    }
    std::printf("\n");
  }
  return 0;
}
