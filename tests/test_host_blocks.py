"""The count of tiles under a sequence's blocks, compiled and run on the CPU."""
from tests.test_host_headers import run_cpp  # noqa: F401  (the fixture)


def test_tiles_of_blocks_one_by_one(run_cpp):  # noqa: F811
    """Every width of a block, ends at every place of a tile, up to some hundred blocks; and sizes near the largest."""
    run_cpp(r"""
#include <cstdio>
#include "xkv_blocks.h"
int main() {
  for (int w = 1; w <= 128; ++w)
    for (int b = 0; b < 400; b += (w % 7 == 0 ? 1 : 13)) {
      long long sum = 0;
      for (int n = 0; n < 700; ++n) {
        if (xkv::sum_of_tiles(n, w, b) != sum) { printf("n %d, w %d, b %d: %lld, not %lld\n", n, w, b, xkv::sum_of_tiles(n, w, b), sum); return 1; }
        sum += (b + n * w) / 128;
      }
    }
  const int ws[] = {1, 7, 8, 9, 18, 25, 64, 127, 128}, bs[] = {0, 127, 128, 4194303, 4194431};
  for (int w : ws)
    for (int b : bs) {
      const int n = 4194304 / w;
      long long sum = 0;
      for (long long v = 0; v < n; ++v) sum += (b + v * w) / 128;
      if (xkv::sum_of_tiles(n, w, b) != sum) { printf("large: w %d, b %d\n", w, b); return 1; }
    }
  return 0;
}
""")
