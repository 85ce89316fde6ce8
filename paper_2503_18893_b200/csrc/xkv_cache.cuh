// Shared by the kernels over an uncompressed cache (xkv_tree.cu, xkv_weigh.cu): waits that give up, even pieces of a list.
#pragma once

#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

constexpr int kTile = 128;                     // cache rows per tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr unsigned long long kCacheWaitNs = 250000000ull;      // a wait that lasts a quarter of a second has failed

// A thread that has waited too long raises the CTA's word, which makes the others give up too, and the caller's flag.
struct Wait {
  volatile int* abort;
  unsigned int* flags;
  unsigned long long limit_ns;
};
__device__ __forceinline__ unsigned long long wait_limit(unsigned int inject) { return inject ? 2000000ull : kCacheWaitNs; }
static __device__ __forceinline__ bool wait_slow(const Wait& w, uint32_t bar, uint32_t parity) {
  unsigned long long t0, t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
  do {
    for (int i = 0; i < 64; ++i) {
      if (ptx::mbar_try_wait(bar, parity)) return true;
      if (*w.abort) return false;
    }
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  } while (t - t0 < w.limit_ns);
  *w.abort = 1;
  if (w.flags) atomicOr(w.flags, XKV_FLAG_TIMEOUT);
  return false;
}
__device__ __forceinline__ bool wait_bar(const Wait& w, uint32_t bar, uint32_t parity) {
  if (ptx::mbar_try_wait(bar, parity)) return true;
  return wait_slow(w, bar, parity);
}
// The same by a whole warp, with one answer for all its lanes.
__device__ __forceinline__ bool wait_warp(const Wait& w, uint32_t bar, uint32_t parity) {
  const bool ok = wait_bar(w, bar, parity);
  return __all_sync(0xffffffffu, ok);
}

// `total` units of work in `ctas` even pieces: where piece c begins, and the piece that holds unit u.
__device__ __forceinline__ int piece_begin(int total, int ctas, int c) { return (int)((long long)total * c / ctas); }
__device__ __forceinline__ int piece_of(int total, int ctas, int u) { return (int)(((long long)(u + 1) * ctas - 1) / total); }

}  // namespace xkv
