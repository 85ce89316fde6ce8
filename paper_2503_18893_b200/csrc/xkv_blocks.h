// How many tiles of 128 rows the blocks of a sequence go over (plain C++, also for the host).
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define XKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define XKV_HOST_DEVICE inline
#endif

namespace xkv {

// Blocks v = 0 .. n-1 end at row b + v w, in the tile (b + v w) / 128 rounded down: the sum of those numbers (1 <= w <= 128; b, n w >= 0, their sum
// below 2^31).  With g the largest power of two in w, 128 / g blocks on is w / g tiles on exactly, and the places of those blocks in their
// tiles are b mod g, and g, 2 g, ... behind it, each once: whole periods are a product, and fewer than 128 / g blocks are left to go over.
XKV_HOST_DEVICE long long sum_of_tiles(int n, int w, int b) {
  const int g = w & -w, period = 128 / g, step = w / g;
  const long long whole = n / period, place = whole * period;
  // of all blocks of the first period: their rows, less their places in their tiles
  const long long pairs = (long long)period * (period - 1) / 2;
  const long long first = (period * (long long)b + w * pairs - period * (long long)(b & (g - 1)) - g * pairs) / 128;
  long long sum = whole * first + period * step * (whole * (whole - 1) / 2);
  const int rest = n - (int)place;
  int tiles = 0;
  for (int v = 0; v < rest; ++v) tiles += ((b & 127) + v * w) >> 7;
  return sum + tiles + rest * ((b >> 7) + whole * step);
}

}  // namespace xkv
