// Shared by the attention kernels over a paged cache of 8-bit codes (xkv_attend8.cu, xkv_attend8_wide.cu): what a call is given, the list
// of tiles, e4m3.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "xkv_blocks.h"
#include "xkv_cache.cuh"

namespace xkv {

// A weight is 2^(z - m) in 16 bits (fp16): 11 bits from 2^-14 up, steps of 2^-24 below, 2^16 at most.  The largest of a query row is put
// between 2^9 and 2^15.75: m moves when one would pass that, and then so that it becomes 2^9.  So a weight is off by 2^-11 of itself or
// 2^-34 of the largest; 2^22 rows together by 2^-12 of it.  (With the largest between 1 and 2^8, an even rest of weights 2^-24 of the
// largest beside it was off by a third, and gone from 2^-26 on.  The higher the largest is put, the more often it moves: a chunk of 512
// tokens over 12301 rows takes 221 us with 2^8, 226 with 2^9, 236 with 2^11; 16 query rows of 131072 220, 220, 228.  m moves for its own
// row's sake only: what a token attends to does not depend on the tokens beside it.)
constexpr float kTop = 15.75f, kSet = 9.0f;    // log2
// What is taken off z where the largest is m, and the largest z that it holds for; rounded so that a weight is at most 2^kTop also where
// logits are too large for fp32 to hold m - kSet.
__device__ __forceinline__ float taken_off(float m) { return __fadd_ru(m, -kSet); }
__device__ __forceinline__ float weight_bound(float off) { return __fadd_rd(off, kTop); }

// A whole warp waits (as wait_warp does), asleep for most of the time: warps that poll take their SM's issue slots from those that work.
static __device__ bool wait8_slow(const Wait& w, uint32_t bar, uint32_t parity) {
  unsigned long long t0, t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t0));
  do {
    if (ptx::mbar_try_wait_for(bar, parity, 10000u)) return true;
    if (*w.abort) return false;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  } while (t - t0 < w.limit_ns);
  *w.abort = 1;
  if (w.flags) atomicOr(w.flags, XKV_FLAG_TIMEOUT);
  return false;
}
__device__ __forceinline__ bool wait8(const Wait& w, uint32_t bar, uint32_t parity) {
  const bool ok = ptx::mbar_test(bar, parity) || wait8_slow(w, bar, parity);
  return __all_sync(0xffffffffu, ok);
}

struct Attend8Args {
  int batch, H_kv, H_q, n_rep, n_pages, max_pages, page_shift, n_tok, max_new, l0, layers;
  int block_tok;                               // tokens of a block of query rows
  uint32_t rep_inv;                            // ceil(2^16 / n_rep)
  float scale2;                                // softmax scale times log2(e)
  const __nv_bfloat16* q;
  const int32_t* first;
  const int32_t* table;
  const int32_t* length;
  const uint8_t* V8;                           // (codes that are NaN)
  const float* k_scale;
  const float* v_scale;
  int block_rows;                              // room for query rows in a piece's results
  struct Piece8* pieces;                       // [CTA]
  float* part;                                 // [CTA][2][block_rows][d_h]
  float2* part_ml;                             // [CTA][2][block_rows] (m, l)
  __nv_bfloat16* out;
  float* lse;
  unsigned int* flags;
  unsigned int inject;                         // XKV_INJECT_CACHE_* bits; 0 in normal use
};

// A sequence: its first token, how many of its tokens are looked after, its rows, and those before its first new one (below zero if
// it has more new tokens than rows).
struct Seq {
  int f0, n, base, len;
};
__device__ __forceinline__ Seq load_seq(const Attend8Args& a, int b, bool* bad) {
  const int w0 = a.first ? a.first[b] : b, w1 = a.first ? a.first[b + 1] : b + 1, wl = a.length[b];
  const int f0 = min(max(w0, 0), a.n_tok), f1 = min(max(w1, f0), a.n_tok), len = min(max(wl, 0), a.max_pages << a.page_shift);
  *bad = f0 != w0 || f1 != w1 || len != wl || f1 - f0 > a.max_new;
  return Seq{f0, min(f1 - f0, a.max_new), len - (f1 - f0), len};
}
__device__ __forceinline__ int blocks_of(const Attend8Args& a, const Seq& s) { return (s.n + a.block_tok - 1) / a.block_tok; }
// Rows that the last token of block qp sees, and the tiles that they lie in (one for tokens that see nothing: it says so).
__device__ __forceinline__ int rows_seen(const Attend8Args& a, const Seq& s, int qp) {
  return min(max(s.base + min(s.n, (qp + 1) * a.block_tok), 0), s.len);
}
__device__ __forceinline__ int tiles_of(int rows) { return max(1, (rows + kTile - 1) / kTile); }

// Tiles of one head in blocks 0 .. qp-1 of a sequence of n_qp blocks; those before the last are full: their rows grow by block_tok.
static __device__ long long tiles_before(const Attend8Args& a, const Seq& s, int qp, int n_qp) {
  if (qp == 0) return 0;
  if (qp == n_qp) return tiles_before(a, s, qp - 1, n_qp) + tiles_of(rows_seen(a, s, qp - 1));
  const int most = kTile - s.base;             // blocks that see up to one tile count one
  const int ones = most > 0 ? min(qp, most / a.block_tok) : 0;
  static_assert(kTile == 128, "tiles of sum_of_tiles");
  return ones + sum_of_tiles(qp - ones, a.block_tok, s.base + (ones + 1) * a.block_tok + kTile - 1);
}
__device__ __forceinline__ long long tiles_of_head(const Attend8Args& a, const Seq& s) {
  if (s.n <= a.block_tok) return s.n > 0 ? tiles_of(rows_seen(a, s, 0)) : 0;
  const int n_qp = blocks_of(a, s);
  return tiles_before(a, s, n_qp, n_qp);
}

// A place in the list of tiles.  Order: layer, head, sequence, block, tile.
struct Place {
  int l, g, b, qp, t, nt, n_qp;
  Seq s;
};
__device__ __forceinline__ void set_block(const Attend8Args& a, Place& p) { p.nt = tiles_of(rows_seen(a, p.s, p.qp)); }
// Moves to the next problem (there is one: the caller counts).
__device__ __forceinline__ void next_problem(const Attend8Args& a, Place& p) {
  p.t = 0;
  if (++p.qp >= p.n_qp) {
    p.qp = 0;
    do {
      if (++p.b == a.batch) {
        p.b = 0;
        if (++p.g == a.H_kv) { p.g = 0; ++p.l; }
      }
      bool bad;
      p.s = load_seq(a, p.b, &bad);
      p.n_qp = blocks_of(a, p.s);
    } while (p.n_qp == 0 && p.l < a.layers);
  }
  set_block(a, p);
}

__device__ __forceinline__ long long warp_sum(long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Lane: tiles of one head in sequence b0 + lane.
__device__ __forceinline__ long long lane_tiles(const Attend8Args& a, int b0, Seq* s, bool report) {
  const int b = b0 + (int)(threadIdx.x & 31);
  if (b >= a.batch) return 0;
  bool bad;
  *s = load_seq(a, b, &bad);
  if (bad && report && a.flags) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
  return tiles_of_head(a, *s);
}
// What a CTA has: `count` tiles from a place on.
struct Piece8 {
  Place at;
  long long count;
};

// By a whole warp: the tiles of CTA c.  They are written down for the merge, too.
__device__ __forceinline__ Place find_piece(const Attend8Args& a, int c, int grid, long long* count, bool report) {
  Seq s = {};
  const long long mine = lane_tiles(a, 0, &s, report);         // (most batches have 32 sequences at most: they are looked at once)
  long long head = mine;
  for (int b0 = 32; b0 < a.batch; b0 += 32) {
    Seq x;
    head += lane_tiles(a, b0, &x, report);
  }
  head = warp_sum(head);
  const long long total = head * a.H_kv * a.layers;
  const int ctas = (int)min((long long)grid, total);
  Place p = {};
  *count = 0;
  if (c >= ctas) {
    if ((threadIdx.x & 31) == 0) a.pieces[c] = Piece8{p, 0};
    return p;
  }
  const long long u0 = total * c / ctas;
  *count = total * (c + 1) / ctas - u0;
  const long long lg = u0 / head;
  long long rest = u0 - lg * head;
  p.l = (int)(lg / a.H_kv);
  p.g = (int)(lg - (long long)p.l * a.H_kv);
  for (int b0 = 0; b0 < a.batch; b0 += 32) {   // (u0 is in the list: the search ends inside the batch)
    const long long v = b0 == 0 ? mine : lane_tiles(a, b0, &s, false);
    long long upto = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, upto, o);
      if ((int)(threadIdx.x & 31) >= o) upto += x;
    }
    const unsigned holds = __ballot_sync(0xffffffffu, rest < upto);
    if (holds) {
      const int at = __ffs(holds) - 1;
      rest -= __shfl_sync(0xffffffffu, upto - v, at);
      p.b = b0 + at;
      p.s.f0 = __shfl_sync(0xffffffffu, s.f0, at);
      p.s.n = __shfl_sync(0xffffffffu, s.n, at);
      p.s.base = __shfl_sync(0xffffffffu, s.base, at);
      p.s.len = __shfl_sync(0xffffffffu, s.len, at);
      break;
    }
    rest -= __shfl_sync(0xffffffffu, upto, 31);
  }
  p.n_qp = blocks_of(a, p.s);
  int lo = 0, hi = p.n_qp - 1;                 // the last block that begins at or before `rest`
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tiles_before(a, p.s, mid, p.n_qp) <= rest) lo = mid; else hi = mid - 1;
  }
  p.qp = lo;
  p.t = (int)(rest - tiles_before(a, p.s, lo, p.n_qp));
  set_block(a, p);
  if ((threadIdx.x & 31) == 0) a.pieces[c] = Piece8{p, *count};
  return p;
}

// ---- 8-bit codes
// 2^(127 - e), finite for every e of 0 .. 255: rows that are left out are multiplied by it, too.
__device__ __forceinline__ float turned_over(int e) { return __int_as_float(max((254 - e) << 23, 0x400000)); }
// Does one of four codes say NaN?
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); }

// By a warp of a CTA that has given up: the results of its n tiles from place x on say so, also to a caller without a flag word.
template <int DH>
__device__ __forceinline__ void results_are_nan(const Attend8Args& a, Place x, long long n) {
  const float nan = __int_as_float(0x7fffffff);
  for (uint32_t seg = 0; n > 0; ++seg) {
    const int t1 = (int)min((long long)x.nt, x.t + n), tok0 = x.qp * a.block_tok;
    const int rows = min(a.block_tok, x.s.n - tok0) * a.n_rep;
    for (int r = threadIdx.x & 31; r < rows; r += 32) {
      if (x.t == 0 && t1 == x.nt) {
        const size_t qh = ((size_t)(a.l0 + x.l) * a.n_tok + x.s.f0 + tok0 + r / a.n_rep) * a.H_q + x.g * a.n_rep + r % a.n_rep;
        for (int c = 0; c < DH; c += 8) *reinterpret_cast<uint4*>(a.out + qh * DH + c) = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (a.lse) a.lse[qh] = nan;
      } else {                                 // (the merge makes it the whole problem's)
        a.part_ml[((size_t)blockIdx.x * 2 + (seg == 0 ? 0 : 1)) * a.block_rows + r] = make_float2(nan, nan);
      }
    }
    n -= t1 - x.t;
    if (n > 0) next_problem(a, x);
  }
}

// The copies of a CTA's tiles, by one producer's warp or one for keys and one for values: a page is one box of the copy engine; lane i has the i-th page of a tile, its
// entry of the table and its scales (asynchronous copies of four bytes, which report to a barrier of their own: a tile's scales are read
// until its values have met their weights, and its keys' slot may be filled again before).  Keys go through a ring of KS slots, values
// through one of VS behind it, scales through one of SR tiles.  Barriers: keys full, keys empty, values full, values empty,
// scales full.  Returns how many tiles were asked for.
template <int KS, int VS, int SR>
struct Ring8 {
  static constexpr int kBars = 2 * KS + 2 * VS + SR;
  uint32_t slots, bars;
  float2 (*scales)[8];                         // keys', values'
  __device__ __forceinline__ uint32_t k_full(uint32_t k) const { return bars + 8 * (k % KS); }
  __device__ __forceinline__ uint32_t k_empty(uint32_t k) const { return bars + 8 * (KS + k % KS); }
  __device__ __forceinline__ uint32_t v_full(uint32_t k) const { return bars + 8 * (2 * KS + k % VS); }
  __device__ __forceinline__ uint32_t v_empty(uint32_t k) const { return bars + 8 * (2 * KS + VS + k % VS); }
  __device__ __forceinline__ uint32_t scales_full(uint32_t k) const { return bars + 8 * (2 * KS + 2 * VS + k % SR); }
  static __device__ __forceinline__ uint32_t k_parity(uint32_t k) { return (k / KS) & 1u; }
  static __device__ __forceinline__ uint32_t v_parity(uint32_t k) { return (k / VS) & 1u; }
  static __device__ __forceinline__ uint32_t scales_parity(uint32_t k) { return (k / SR) & 1u; }
  // By one thread: how many arrivals empty a slot.
  __device__ __forceinline__ void init(int k_done, int v_done) const {
    for (int i = 0; i < KS; ++i) { ptx::mbar_init(k_full(i), 1); ptx::mbar_init(k_empty(i), k_done); }
    for (int i = 0; i < VS; ++i) { ptx::mbar_init(v_full(i), 1); ptx::mbar_init(v_empty(i), v_done); }
    for (int i = 0; i < SR; ++i) ptx::mbar_init(scales_full(i), 32);           // (every lane reports)
  }
  template <int DH, bool KEYS, bool VALUES>
  __device__ __forceinline__ uint32_t produce(const Attend8Args& a, const Wait& wt, const CUtensorMap* k_map, const CUtensorMap* v_map, Place p, long long left) const {
    const int lane = threadIdx.x & 31;
    const int ppt_shift = 7 - a.page_shift, ppt = 1 << ppt_shift, tpb = 32 >> ppt_shift;       // pages of a tile, tiles of a batch of entries
    const uint32_t page_bytes = (uint32_t)DH << a.page_shift;
    bool ok = !(a.inject & XKV_INJECT_CACHE_NO_LOAD);
    uint32_t k = 0;
    while (left > 0 && ok) {
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left);
      left -= t1 - t0;
      const int rows = rows_seen(a, p.s, p.qp), pages = min((rows + (1 << a.page_shift) - 1) >> a.page_shift, t1 << ppt_shift);
      const int32_t* entries = a.table + (size_t)p.b * a.max_pages;
      auto entry = [&](int t) {                // lane: an entry of the batch that begins with tile t
        const int i = (t << ppt_shift) + lane;
        if (i >= pages) return -1;
        const int e = entries[i];
        if (e >= 0 && e < a.n_pages) return e;
        if (KEYS && a.flags) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
        return -1;
      };
      int now = 0, next = entry(t0);
      for (int t = t0; t < t1 && ok; ++t, ++k) {
        const int in = (t - t0) & (tpb - 1);
        if (in == 0) { now = next; next = entry(t + tpb); }
        const int mine = __shfl_sync(0xffffffffu, now, ((in << ppt_shift) + lane) & 31), id = lane < ppt ? mine : -1;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, id >= 0)) * page_bytes;
        const size_t head = ((size_t)(a.l0 + p.l) * a.n_pages + (id >= 0 ? id : 0)) * a.H_kv + p.g;
        const int y = (int)(head << a.page_shift);
        if constexpr (KEYS) {
          if (!(ok = wait8(wt, k_empty(k), k_parity(k) ^ 1u))) break;
          if (lane == 0) ptx::mbar_expect_tx(k_full(k), bytes);
          __syncwarp();
          if (id >= 0) ptx::tma_load_2d(slots + (k % KS) * (kTile * DH) + lane * page_bytes, k_map, 0, y, k_full(k));
          if (lane < ppt) {
            const uint32_t at = ptx::smem_u32(&scales[k % SR][lane]), n = id >= 0 ? 4u : 0u;  // (a page that is not there gets zeros)
            ptx::cp_async4(at, a.k_scale + head, n);
            ptx::cp_async4(at + 4, a.v_scale + head, n);
          }
          ptx::cp_async_arrive_noinc(scales_full(k));
        }
        if constexpr (VALUES) {
          if (!(ok = wait8(wt, v_empty(k), v_parity(k) ^ 1u))) { k += KEYS ? 1u : 0u; break; }
          if (lane == 0) ptx::mbar_expect_tx(v_full(k), bytes);
          __syncwarp();
          if (id >= 0) ptx::tma_load_2d(slots + (KS + k % VS) * (kTile * DH) + lane * page_bytes, v_map, 0, y, v_full(k));
        }
      }
      if (left > 0) next_problem(a, p);
    }
    __syncwarp();
    return k;
  }
  // By a producer's warp of a CTA that has given up: tiles may still be on their way into its shared memory; stay (with a limit) for them.
  template <bool KEYS, bool VALUES>
  __device__ __forceinline__ void drain(uint32_t loaded) const {
    asm volatile("cp.async.wait_all;" ::: "memory");
    for (uint32_t k = loaded > KS ? loaded - KS : 0u; KEYS && k < loaded; ++k)
      for (uint32_t i = 0; i < (1u << 16); ++i) if (__all_sync(0xffffffffu, ptx::mbar_try_wait(k_full(k), k_parity(k)))) break;
    for (uint32_t k = loaded > VS ? loaded - VS : 0u; VALUES && k < loaded; ++k)
      for (uint32_t i = 0; i < (1u << 16); ++i) if (__all_sync(0xffffffffu, ptx::mbar_try_wait(v_full(k), v_parity(k)))) break;
  }
};

// Eight elements of a query row as two codes each, by a lane of the C that hold the row side by side: the row's largest element lies in
// [128, 256) times 2^ex, the first code is e4m3, and what it leaves goes to the second, as 2^5 times it in e4m3 (SCALED: columns of their
// own) or as it is in e5m2 (a product into the same columns).  A bf16 value's 8 bits are exact from 2^-14 of the largest element up
// (e5m2: 2^-13); below, off by 2^-22 of it at most (2^-21).  (Both codes in e4m3 without a factor: 2^-17, from 2^-9 down.)  A row with an element that is not finite becomes NaN.
template <int C, bool SCALED>
__device__ __forceinline__ void encode_query(const uint4& x, uint2* hi, uint2* lo, int* ex) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = __vmaxu2(top, w[e] & 0x7fff7fffu);
  top = max(top & 0xffffu, top >> 16);
#pragma unroll
  for (int o = C / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  *ex = max((int)(top >> 7) - 127 - 7, -60);                   // (with a scale's 2^-60 still a normal number)
  const float f = __int_as_float((127 - *ex) << 23);
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x0 = __uint_as_float(w[e] << 16) * f, x1 = __uint_as_float(w[e] & 0xffff0000u) * f;
    h[e] = ptx::pack_e4m3(x0, x1);
    const uint32_t back = ptx::unpack_e4m3(h[e]);
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&back));
    l[e] = SCALED ? ptx::pack_e4m3((x0 - b.x) * 32.0f, (x1 - b.y) * 32.0f) : ptx::pack_e5m2(x0 - b.x, x1 - b.y);
  }
  *hi = make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
  *lo = make_uint2(l[0] | (l[1] << 16), l[2] | (l[3] << 16));
  if (top >= 0x7f80u) *hi = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
}
// Where eight bytes of a tile with rows of DH bytes and as wide a swizzle lie.
template <int DH>
__device__ __forceinline__ uint32_t tile_place(int r, int c) {
  const int unit = DH == 128 ? (c >> 1) ^ (r & 7) : (c >> 1) ^ ((r >> 1) & 3);
  return (uint32_t)(r * DH + unit * 16 + (c & 1) * 8);
}

// xkv_attend8_wide.cu: blocks of 128 query rows
cudaError_t launch_attend8_wide(const CUtensorMap& k_map, const CUtensorMap& v_map, int d_h, const Attend8Args& a, int grid, int device,
                                cudaStream_t s);

}  // namespace xkv
