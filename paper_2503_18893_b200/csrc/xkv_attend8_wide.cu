// Attention over a paged cache of 8-bit codes for many query rows (drafted tokens, a prompt's chunk): blocks of 128 rows, the rows of Q
// being the wide side of both products.
//   S = Q8 K8^T      e4m3 as the keys lie in memory, queries as two codes (e4m3 and e5m2: encode_query): two products into the same S
//   O += P V         16 bits (fp16, which holds every code): a tile's values are converted once for all rows of the block, and weights need
//                    no splitting, so that this product takes half of what four 8-bit ones would
// Scales as there: a key's multiplies the logits, a value's exponent joins the weight's.
//
//   producer   pages by the copy engine, with their scales (Ring8)
//   scales     a warp: what 16 columns of a page need, worked out once per page
//   converters four warps: a tile of value codes becomes fp16 in one of two buffers; rows that no token of the block sees become 0, NaN is
//              taken out of rows that only some see, and listed
//   issuer     S of a tile two ahead, O += P V with P in tensor memory, where it lies over S
//   softmax    two warpgroups; a query row is a TMEM lane, which two threads share, each with half of a tile's columns.  O is rescaled only
//              when a weight would pass 2^15.75 (kTop): one vote of the two warps per tile
// Bound by the softmax: what a warp does for a row of a tile (logits from tensor memory, maximum, exponentials, weights back) is longer than
// its instructions, and two warps of an SM's quarter do not fill it; warps that poll beside them make it worse.  131072 rows of four layers of
// eight heads with four query heads: 8 tokens 327 us, 16 341, 32 368; a chunk of 512 tokens over 12301 rows of two sequences, seven query
// heads, 227 (0.63 PFLOP/s).  What did not help, with a merge that took 12 us more: one thread a row and blocks of 256 rows (steps of half a
// tile) 231 for the chunk and 412 for 32 tokens; softmax warps that poll 275 and 431; two threads a row and 256 rows 323 (registers); 256
// rows with whole tiles, S once, 251.
#include <math.h>

#include "xkv_attend8.cuh"

namespace xkv {

namespace {

constexpr int kRows8 = 128;                    // query rows of a block

template <int DH>
struct Wide8 {
  static constexpr int kSlot = kTile * DH;                     // a tile of codes
  static constexpr int kSlab = kTile * 128;                    // 128 rows x 64 values in 16 bits
  static constexpr int kValues = kSlab * (DH / 64);
  static constexpr int kKeys = DH == 64 ? 4 : 3, kCodes = kKeys;           // tiles of keys, of values
  static constexpr int kQPart = kRows8 * DH, kQBytes = 2 * kQPart;         // queries: high, low
  static constexpr int kBytes = 1024 + (kKeys + kCodes) * kSlot + 2 * kValues + kQBytes;
};
constexpr int kSoftmax8 = 8, kConvert8 = 8, kCopies8 = 12, kScales8 = 13, kIssuer8 = 14, kWide8Threads = 512;    // warps; whole warpgroups
// Registers a thread: softmax warpgroups keep their logits; the sum over four warpgroups stays that of the launch, 128 a thread.
constexpr int kSoftmaxRegs = 152, kOtherRegs = 104;

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int DH>
__global__ void __launch_bounds__(kWide8Threads, 1)
attend8_wide_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const Attend8Args a) {
  using namespace ptx;
  using L = Wide8<DH>;
  constexpr int SR = 8;
  using Ring = Ring8<L::kKeys, L::kCodes, SR>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars_s[Ring::kBars + 12 + SR];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  __shared__ Place place_s;
  __shared__ long long count_s;
  __shared__ float2 scale_s[SR][8];
  __shared__ float4 page_s[SR][8];             // of a tile's pages: keys' scale, values' exponent, its power of two turned over
  __shared__ uint32_t dead_s[SR];              // which of them hold nothing (bits 0-7), which have a scale that is not finite (8-15)
  // New rows of a block with value codes that are NaN, by segment: converters are less than eight segments ahead of the softmax.
  __shared__ uint32_t bad_s[16][4];
  // Of a query row: its factor; what the two threads that share it tell one another
  __shared__ float qs_s[kRows8], tell_s[2][kRows8];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  constexpr uint32_t kVAt = (L::kKeys + L::kCodes) * L::kSlot, kQAt = kVAt + 2 * L::kValues;
  const uint32_t bars = smem_u32(bars_s);
  const Ring ring{base, bars, scale_s};
  const uint32_t b_s = bars + 8 * Ring::kBars, b_p = b_s + 16, b_o = b_p + 16, b_vf = b_o + 16, b_ve = b_vf + 16, b_q = b_ve + 16, b_drain = b_q + 8,
                 b_pg = b_drain + 8;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    ring.init(1, 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_s + 8 * i, 1);
      mbar_init(b_p + 8 * i, 8);
      mbar_init(b_o + 8 * i, 1);
      mbar_init(b_vf + 8 * i, 4);
      mbar_init(b_ve + 8 * i, 1);
    }
    mbar_init(b_q, 8);
    mbar_init(b_drain, 1);
    for (int i = 0; i < SR; ++i) mbar_init(b_pg + 8 * i, 1);
    fence_mbar_init();
    abort_s = 0;
  }
  if (tid < 64) bad_s[tid >> 2][tid & 3] = 0u;
  if (warp == kIssuer8) {
    tmem_alloc(smem_u32(&tmem_s), 512);
    tmem_relinquish();
  }
  grid_dependency_wait();                      // everything below may come from the kernel before
  grid_dependency_launch();                    // (before this CTA is sure to hold tensor memory: the merge, which comes next, takes none)
  if (warp == kCopies8) {
    long long count;
    const Place p = find_piece(a, blockIdx.x, gridDim.x, &count, blockIdx.x == 0);
    if (lane == 0) { place_s = p; count_s = count; }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  const Wait wt{&abort_s, a.flags, wait_limit(a.inject)};
  long long left = count_s;
  Place p = place_s;
  uint32_t n_loaded = 0;                       // producer: tiles asked for

  if (left > 0 && warp < kSoftmax8) {
    regs_more<kSoftmaxRegs>();
    // Two threads share a query row (TMEM lane), each with half of a step's columns: four warps then work where one would wait.
    const int side = warp >> 2, row = tid & 127, pair = 1 + (warp & 3);        // (a barrier for each two warps)
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    uint8_t* q_gen = gen + kQAt;
    const uint32_t o_addr = tmem + lane_base + 256u;
    uint32_t k0 = 0, n_o = 0, seg = 0;         // tiles, commits on b_o and segments so far
    bool ok = true, gone = false;              // this warp's waits; the two warps have given up
    while (left > 0 && !gone) {
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left);
      left -= t1 - t0;
      const int tok0 = p.qp * a.block_tok, rows = min(a.block_tok, p.s.n - tok0) * a.n_rep;    // query rows
      const int new0 = p.s.base + tok0;        // row of the block's first token
      const size_t qh0 = ((size_t)(a.l0 + p.l) * a.n_tok + p.s.f0 + tok0) * a.H_q + (size_t)p.g * a.n_rep;
      auto token_of = [&](int m) { return (int)(((uint32_t)m * a.rep_inv) >> 16); };
      auto place_of = [&](int m) { return qh0 + (size_t)token_of(m) * a.H_q + (m - token_of(m) * a.n_rep); };
      {
        // the two warps bring their 32 rows, sixteen each; their place is theirs in the epilogue too
        constexpr int C = DH / 8, STEP = 32 / C, U = 4;        // lanes of a row; rows per round; rounds in flight
        const int c = lane % C;
#pragma unroll 1
        for (int i0 = side * 16; i0 < side * 16 + 16; i0 += U * STEP) {
          uint4 v[U];
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int m = (warp & 3) * 32 + i0 + i * STEP + lane / C;
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (m < rows) v[i] = *reinterpret_cast<const uint4*>(a.q + place_of(m) * DH + c * 8);
          }
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int r = (warp & 3) * 32 + i0 + i * STEP + lane / C;
            uint2 hi, lo;
            int ex;
            encode_query<C, false>(v[i], &hi, &lo, &ex);
            uint8_t* at = q_gen + tile_place<DH>(r, c);
            *reinterpret_cast<uint2*>(at) = hi;
            *reinterpret_cast<uint2*>(at + L::kQPart) = lo;
            if (c == 0) qs_s[r] = __int_as_float((127 + ex) << 23) * a.scale2;
          }
        }
      }
      fence_proxy_async();
      named_bar_sync(pair, 64);
      if (lane == 0) mbar_arrive(b_q);
      const float qs = qs_s[row];
      const int m = row;
      const bool live = m < rows, warp_live = (m & ~31) < rows;
      const int limit = new0 + (live ? token_of(m) : 0) + 1;   // rows of the cache that this query row sees
      float m_used = -INFINITY, l = 0.0f;      // what is taken off z, the sum of weights
      const int n = t1 - t0;
      for (int s = 0; s < n; ++s) {
        constexpr int CW = kTile / 2, NC = CW / 32, NP = CW / 16;              // columns of a thread
        const int col0 = side * CW;
        const uint32_t k = k0 + (uint32_t)s, buf = k & 1u;
        ok = ok && wait8(wt, b_pg + 8 * (k % SR), (k / SR) & 1u) && wait8(wt, b_s + 8 * buf, (k >> 1) & 1u);
        tc_fence_after();
        const uint32_t s_addr = tmem + lane_base + buf * 128u;
        const int j0 = (t0 + s) * kTile + col0;                // the cache's row of the first column
        const uint32_t dead = dead_s[k % SR];
        uint32_t z[NC][32];
        float f[NP], e[NP], e_inv[NP];         // sixteen columns lie in one page
        float top = -INFINITY;
        if (warp_live) {
#pragma unroll
          for (int i = 0; i < NC; ++i) tmem_ld32_nb(s_addr + (uint32_t)col0 + 32u * i, z[i]);
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float4 x = page_s[k % SR][(col0 + 16 * i) >> a.page_shift];
            // neither 0 nor infinite: a masked column stays minus infinity, and what is 0 has the logit 0
            f[i] = fminf(fmaxf(x.x * qs, 0x1p-126f), 0x1.fffffep127f);
            e[i] = x.y;
            e_inv[i] = x.z;
          }
#pragma unroll
          for (int i = 0; i < NC; ++i) tc_wait_ld32_nb(z[i]);
          if (j0 + CW > new0 + 1 || dead) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              const uint32_t is = dead >> ((col0 + 16 * i) >> a.page_shift), nan = is & 0x100u ? 0x7fffffffu : 0u;
              const int see = is & 1u ? 0 : limit - (j0 + 16 * i);
#pragma unroll
              for (int x = 0; x < 16; ++x) z[i / 2][16 * (i & 1) + x] = x < see ? z[i / 2][16 * (i & 1) + x] | nan : 0xff800000u;
            }
          }
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int x = 0; x < 16; x += 2)
              mx[(x >> 1) & 1] = fmaxf(fmaxf(mx[(x >> 1) & 1], __uint_as_float(z[i / 2][16 * (i & 1) + x])), __uint_as_float(z[i / 2][16 * (i & 1) + x + 1]));
            top = fmaxf(top, fmaf(fmaxf(mx[0], mx[1]), f[i], e[i]));
          }
        }
        // Both have their logits in registers now: weights may go where the other's lay.  Does a maximum move (or has a wait run out)?
        tc_fence_before();
        const bool vote = !ok || (warp_live && top > weight_bound(m_used));
        if (named_bar_any(pair, 64, vote)) {
          // O holds the tiles before this one once the last product is done, which the commit of the next S tells, or its own
          const bool next = s + 1 < n;
          if (ok && s > 0) ok = wait8(wt, next ? b_s + 8 * (buf ^ 1u) : b_o + 8 * (n_o & 1u), ((next ? k + 1 : n_o) >> 1) & 1u);
          tell_s[side][row] = top;
          if (named_bar_any(pair, 64, !ok)) { gone = true; break; }
          tc_fence_after();
          const float m = fmaxf(top, tell_s[side ^ 1][row]);
          const bool grow = m > weight_bound(m_used);
          const float g = grow ? (m_used == -INFINITY ? 0.0f : ex2_approx(m_used - taken_off(m))) : 1.0f;
          if (grow) m_used = taken_off(m);
          l *= g;
          if (s > 0 && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
            for (int c = side * (DH / 2); c < (side + 1) * (DH / 2); c += 16) {
              float o[16];
              uint32_t r[16];
              tmem_ld<16>(o_addr + (uint32_t)c, o);
              tc_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) r[x] = __float_as_uint(o[x] * g);
              tmem_st16(o_addr + (uint32_t)c, r);
            }
          }
          named_bar_sync(pair, 64);            // (what they told is read before they tell again)
        }
        tc_fence_after();
        if (warp_live) {
          const float shift = m_used == -INFINITY ? 0.0f : -m_used;
          const u64 shift2 = pack2(shift, shift);
#pragma unroll
          for (int i = 0; i < NC; ++i) {       // P, two to a column, in the upper half of S's columns
            uint32_t r[16];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = 2 * i + h;
              const u64 f2 = pack2(f[c], f[c]), e2 = pack2(e[c], e[c]);
              u64 sum = 0ull;
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                // (first what the maximum was formed of, so that no weight passes its bound, however large logits are)
                float2 w = unpack2(add2(fma2(pack2u(z[i][16 * h + 2 * x], z[i][16 * h + 2 * x + 1]), f2, e2), shift2));
                w.x = ex2_approx(w.x);
                w.y = ex2_approx(w.y);
                sum = add2(sum, pack2(w.x, w.y));
                r[8 * h + x] = pack_f16(w.x, w.y);
              }
              const float2 two = unpack2(sum);
              l = fmaf(two.x + two.y, e_inv[c], l);
            }
            tmem_st16(s_addr + 64u + (uint32_t)(col0 / 2) + 16u * i, r);
          }
          tc_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && ok && !(a.inject & XKV_INJECT_CACHE_NO_HANDOVER)) mbar_arrive(b_p + 8 * buf);
      }
      if (gone) break;
      // ---- the segment's result (the last two products commit to two barriers in turn: by now both may be done)
      n_o += (uint32_t)min(2, n);
      ok = ok && wait8(wt, b_o + 8 * ((n_o - 1u) & 1u), ((n_o - 1u) >> 1) & 1u);
      tell_s[side][row] = l;
      if (named_bar_any(pair, 64, !ok)) break;
      k0 += (uint32_t)n;
      tc_fence_after();
      l += tell_s[side ^ 1][row];
      const bool whole = t0 == 0 && t1 == p.nt;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const size_t pr = ((size_t)blockIdx.x * 2 + (seg == 0 ? 0 : 1)) * a.block_rows + m;
      const size_t qh = live ? place_of(m) : 0;
      const bool odd = t1 * kTile > new0 + 1;  // tiles of this segment held rows that not all see
      // each half of the columns; of 64 one warp has all (they go through the place of both warps' rows of Q)
      const int c_begin = DH == 128 ? side * 64 : 0, c_end = DH == 128 ? c_begin + 64 : side == 0 ? 64 : 0;
      if (warp_live) {
#pragma unroll 1
        for (int c = c_begin; c < c_end; c += 32) {
          float o[32];
          tmem_ld32(o_addr + (uint32_t)c, o);
          tc_wait_ld();
          if (odd) {
#pragma unroll 1
            for (int w = 0; w < 4; ++w) {
              uint32_t bad = bad_s[seg & 15u][w];              // (entered before the product that this result waited for)
              while (bad) {
                const int j = new0 + 32 * w + __ffs(bad) - 1;
                bad &= bad - 1u;
                if (j >= limit) continue;
                const size_t head = ((size_t)(a.l0 + p.l) * a.n_pages + a.table[(size_t)p.b * a.max_pages + (j >> a.page_shift)]) * a.H_kv + p.g;
                const uint8_t* v = a.V8 + ((head << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * DH + c;
#pragma unroll
                for (int x = 0; x < 32; ++x) o[x] = (v[x] & 0x7f) == 0x7f ? __int_as_float(0x7fffffff) : o[x];
              }
            }
          }
          if (live && whole) {
            uint4* dst = reinterpret_cast<uint4*>(a.out + qh * DH + c);
#pragma unroll
            for (int x = 0; x < 4; ++x)
              dst[x] = make_uint4(pack_bf16(o[8 * x] * inv, o[8 * x + 1] * inv), pack_bf16(o[8 * x + 2] * inv, o[8 * x + 3] * inv),
                                  pack_bf16(o[8 * x + 4] * inv, o[8 * x + 5] * inv), pack_bf16(o[8 * x + 6] * inv, o[8 * x + 7] * inv));
          } else if (!whole) {
            // through the places of these rows of Q (a part each of two of 128 columns), so that a store writes whole lines
            auto own = [&](int i) {
              constexpr int UNITS = 32 * DH / 16;              // of the rows in either part of Q
              const int part = DH == 128 ? side : i >= UNITS;
              return reinterpret_cast<float4*>(q_gen + part * L::kQPart + (warp & 3) * (32 * DH)) + (i & (UNITS - 1));
            };
            __syncwarp();
#pragma unroll
            for (int x = 0; x < 8; ++x) *own(lane * 8 + (x ^ (lane & 7))) = make_float4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
            __syncwarp();
            float* dst = a.part + (pr - row + (warp & 3) * 32) * DH + c + (lane & 7) * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = 4 * i + (lane >> 3);
              *reinterpret_cast<float4*>(dst + (size_t)r * DH) = *own(r * 8 + ((lane & 7) ^ (r & 7)));
            }
          }
        }
        if (side == 0 && live && whole && a.lse) a.lse[qh] = l == 0.0f ? -INFINITY : (m_used + log2f(l)) * 0.6931471805599453f;
        if (side == 0 && live && !whole) a.part_ml[pr] = make_float2(m_used, l);
      }
      named_bar_sync(pair, 64);                // the next problem's queries go where the other warp may still be reading
      tc_fence_before();
      ++seg;
      if (left > 0) next_problem(a, p);
    }
  } else if (left > 0 && warp < kCopies8) {
    regs_fewer<kOtherRegs>();
    constexpr int C = DH / 16, STEP = 128 / C; // 16-byte units of a row of codes; rows per round
    const int ct = tid - kConvert8 * 32, c = ct % C;
    uint32_t k = 0, seg = 0;
    bool ok = true;
    while (left > 0 && ok) {
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left);
      left -= t1 - t0;
      const int seen = rows_seen(a, p.s, p.qp), new0 = p.s.base + p.qp * a.block_tok;
      if (ct < 4) bad_s[(seg + 8) & 15u][ct] = 0u;
      for (int t = t0; t < t1; ++t, ++k) {
        if (!(ok = wait8(wt, ring.v_full(k), Ring::v_parity(k)) && wait8(wt, b_pg + 8 * (k % SR), (k / SR) & 1u) &&
                   wait8(wt, b_ve + 8 * (k & 1u), ((k >> 1) & 1u) ^ 1u))) break;
        const uint8_t* src = gen + (L::kKeys + k % L::kCodes) * L::kSlot;
        uint8_t* dst = gen + kVAt + (k & 1u) * L::kValues;
        const bool some = (t + 1) * kTile > new0 + 1;          // rows that not all tokens of the block see
        const uint32_t dead = dead_s[k % SR];
#pragma unroll 2
        for (int r0 = 0; r0 < kTile; r0 += STEP) {
          // (the upper units of a row go with the lower ones of its neighbour: then stores of eight lanes meet all banks)
          const int r = r0 + ((ct / C) ^ (c >> 2)), j = t * kTile + r;
          uint4 x = *reinterpret_cast<const uint4*>(src + tile_place<DH>(r, 2 * c));
          if (dead || some) {
            if (j >= seen || (dead >> (r >> a.page_shift) & 1u)) x = make_uint4(0u, 0u, 0u, 0u);
            if (j > new0) {
              const uint4 m = make_uint4(nan_codes(x.x), nan_codes(x.y), nan_codes(x.z), nan_codes(x.w));
              if (m.x | m.y | m.z | m.w) {
                atomicOr(&bad_s[seg & 15u][(j - new0) >> 5], 1u << ((j - new0) & 31));
                x = make_uint4(x.x & ~m.x, x.y & ~m.y, x.z & ~m.z, x.w & ~m.w);
              }
            }
          }
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[2 * e] = unpack_e4m3(w[e]);
            h[2 * e + 1] = unpack_e4m3(w[e] >> 16);
          }
          uint8_t* row = dst + (c >> 2) * L::kSlab + r * 128;  // 64 columns: four units of codes, eight of values
          const int u = 2 * (c & 3);
          *reinterpret_cast<uint4*>(row + ((u ^ (r & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(row + (((u + 1) ^ (r & 7)) << 4)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(b_vf + 8 * (k & 1u));
          mbar_arrive(ring.v_empty(k));
        }
      }
      ++seg;
      if (left > 0 && ok) next_problem(a, p);
    }
  } else if (left > 0) {
    regs_fewer<kOtherRegs>();
    if (warp == kCopies8) {
      n_loaded = ring.template produce<DH, true, true>(a, wt, &k_map, &v_map, p, left);
    } else if (warp == kScales8) {
      for (uint32_t k = 0; k < (uint32_t)count_s; ++k) {
        if (!wait8(wt, ring.scales_full(k), Ring::scales_parity(k))) break;
        const float2 sc = scale_s[k % SR][min(lane, 127 >> a.page_shift)];
        const int ke = (__float_as_int(sc.x) >> 23) & 255, ve = (__float_as_int(sc.y) >> 23) & 255;
        const uint32_t dead = __ballot_sync(0xffffffffu, ke == 0 || ve == 0) & 0xffu, odd = __ballot_sync(0xffffffffu, ke == 255 || ve == 255) & 0xffu;
        if (lane < 8) page_s[k % SR][lane] = make_float4(ke == 0 || ke == 255 ? 1.0f : __int_as_float(ke << 23), (float)(ve - 127), turned_over(ve), 0.0f);
        if (lane == 0) dead_s[k % SR] = dead | odd << 8;
        __syncwarp();
        if (lane == 0) mbar_arrive(b_pg + 8 * (k % SR));
      }
    } else if (warp == kIssuer8) {
      // ---- branches outside the issue are taken on a vote and descriptors differ by constants, so that they stay in uniform registers
      constexpr uint32_t idesc_s = idesc_e4m3_f32(128, 128), e5m2_a = 1u << 7;
      constexpr uint32_t idesc_o = (1u << 4) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((128u >> 4) << 24);   // fp16; V is read along its rows
      const uint64_t q_desc = smem_desc_rows<DH>(base + kQAt), k_desc = smem_desc_rows<DH>(base);
      const uint64_t v_desc = (smem_desc_sw128(base + kVAt, 0) & ~(0xFFFFull << 16)) | ((uint64_t)(L::kSlab >> 4) << 16);
      uint32_t k0 = 0, n_o = 0, seg = 0;       // tiles, commits on b_o and segments so far
      bool ok = true;
      auto logits = [&](uint32_t k) {
        const uint64_t kd = k_desc + (uint64_t)((k % L::kKeys) * (uint32_t)(L::kSlot >> 4));
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < DH / 32; ++i)
            tc_mma_8bit(tmem + (k & 1u) * 128u, q_desc + (uint64_t)(h * (L::kQPart >> 4) + 2 * i), kd + (uint64_t)(2 * i), h ? idesc_s | e5m2_a : idesc_s, h | i ? 1u : 0u);
        tc_commit(b_s + 8 * (k & 1u));
        tc_commit(ring.k_empty(k));
      };
      auto keys = [&](uint32_t k) { return wait8(wt, ring.k_full(k), Ring::k_parity(k)); };
      while (left > 0 && ok) {
        const int n = (int)min((long long)p.nt, p.t + left) - p.t;
        left -= n;
        ok = wait8(wt, b_q, seg & 1u);
        for (int s = 0; s < min(2, n) && ok; ++s) {            // S of two tiles ahead
          if (!(ok = keys(k0 + s))) break;
          tc_fence_after();
          if (elect_one()) logits(k0 + s);
          __syncwarp();
        }
        for (int s = 0; s < n && ok; ++s) {
          const uint32_t k = k0 + s, buf = k & 1u;
          const bool more = s + 2 < n;
          if (!(ok = wait8(wt, b_vf + 8 * buf, (k >> 1) & 1u))) break;
          if (more && !(ok = keys(k + 2))) break;
          if (!(ok = wait8(wt, b_p + 8 * buf, (k >> 1) & 1u))) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t vd = v_desc + (uint64_t)(buf * (uint32_t)(L::kValues >> 4));
#pragma unroll
            for (int i = 0; i < kTile / 16; ++i)
              tc_mma_bf16_ts(tmem + 256u, tmem + buf * 128u + 64u + (uint32_t)i * 8u, vd + (uint64_t)(i * (2048 >> 4)), idesc_o, (s | i) ? 1u : 0u);
            tc_commit(b_ve + 8 * buf);
            // S after the next follows the product that reads P, which lies where it goes; its commit tells of both
            if (more) logits(k + 2); else tc_commit(b_o + 8 * (n_o & 1u));
          }
          __syncwarp();
          n_o += more ? 0u : 1u;
        }
        k0 += n;
        ++seg;
        if (left > 0 && ok) next_problem(a, p);
      }
    }
  }

  // wind down: nothing of this CTA may still touch shared or tensor memory
  tc_fence_before();
  __syncthreads();
  if (abort_s) {                               // given up: nothing may still write tensor memory when it is freed
    if (warp == kIssuer8) {
      if (elect_one()) tc_commit(b_drain);
      for (uint32_t i = 0; i < (1u << 16); ++i) if (__all_sync(0xffffffffu, mbar_try_wait(b_drain, 0))) break;
    }
    __syncthreads();
  }
  if (warp == kIssuer8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (abort_s && warp == kCopies8) {
    ring.template drain<true, true>(n_loaded);
    results_are_nan<DH>(a, place_s, count_s);
  }
}

template <int DH>
cudaError_t launch_wide(const CUtensorMap& k_map, const CUtensorMap& v_map, const Attend8Args& a, int grid, int device, cudaStream_t s) {
  const cudaError_t e = ensure_dyn_smem<attend8_wide_kernel<DH>>(Wide8<DH>::kBytes, device);
  return e != cudaSuccess ? e : launch_pdl(attend8_wide_kernel<DH>, dim3(grid), dim3(kWide8Threads), Wide8<DH>::kBytes, s, k_map, v_map, a);
}

}  // namespace

cudaError_t launch_attend8_wide(const CUtensorMap& k_map, const CUtensorMap& v_map, int d_h, const Attend8Args& a, int grid, int device,
                                cudaStream_t s) {
  return d_h == 128 ? launch_wide<128>(k_map, v_map, a, grid, device, s) : launch_wide<64>(k_map, v_map, a, grid, device, s);
}

}  // namespace xkv
