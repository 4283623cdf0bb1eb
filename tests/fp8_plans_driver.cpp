// Which tiles the products in 8-bit floating point take: reads lines "tile M N k exact" and "dw rows in out 0", writes the tile, and
// of dw the tile, its splits and the blocks of 128 rows of each.
#include <cstdio>
#include <cstring>

#include "gosh_fp8.hip"

int main() {
  using namespace gosh;
  char what[8];
  long long a, b, c, exact;
  while (std::scanf("%7s %lld %lld %lld %lld", what, &a, &b, &c, &exact) == 5) {
    if (std::strcmp(what, "tile") == 0) {
      std::printf("%d\n", fp8_tile_for(a, b, ceil_div(c, kFp8Block), exact != 0));
    } else {
      const Fp8DwPlan p = plan_dw_fp8(a, static_cast<int32_t>(b), static_cast<int32_t>(c));
      std::printf("%d %d %lld\n", p.tile, p.splits, static_cast<long long>(p.blocks_per_split));
    }
  }
  return 0;
}
