// Attention over a paged cache of 8-bit codes for many query rows (a prompt's chunk): blocks of 128 or 256 rows, the rows of Q being the
// wide side of both products.
//   S = Q8 K8^T      e4m3 as the keys lie in memory, queries as two codes (see xkv_attend8.cu): two products into the same S
//   O += P V         16 bits (fp16, which holds every code): a tile's values are converted once for all rows of the block, and weights need
//                    no splitting, so that this product takes two thirds of what three e4m3 ones would
// Scales as there: a key's multiplies the logits, a value's exponent joins the weight's.
//
//   producer   pages by the copy engine, with their scales (Ring8)
//   converters four warps: a tile of value codes becomes fp16 in one of two buffers; rows that no token of the block sees become 0, NaN is
//              taken out of rows that only some see, and listed
//   issuers    a warp for each 128 rows of Q: S two steps ahead, O += P V with P in tensor memory, where it lies over S
//   softmax    a warpgroup for each 128 rows of Q: thread = row, so that maxima and sums need no shuffle.  O is rescaled only when a
//              maximum has grown by more than 2^8 (fp16 holds weights of 2^8, and of 2^-24).
//   scales     a warp: what 16 columns of a page need, worked out once per page
// A step is a tile of 128 rows of the cache for 128 rows of Q, and half a tile for 256 (tensor memory holds two steps of S and O).
#include <math.h>

#include "xkv_attend8.cuh"

namespace xkv {

namespace {

constexpr int kQRows8 = 128;                   // query rows per warpgroup
constexpr float kGrow8 = 8.0f;                 // log2 of the growth of a maximum that makes O be rescaled

template <int DH, int QT>
struct Wide8 {
  static constexpr int kSlot = kTile * DH;                     // a tile of codes
  static constexpr int kSlab = kTile * 128;                    // 128 rows x 64 values in 16 bits
  static constexpr int kValues = kSlab * (DH / 64);
  static constexpr int kKeys = DH == 64 ? 4 : 3, kCodes = DH == 64 ? 4 : QT == 2 ? 2 : 3;
  static constexpr int kQPart = kQRows8 * DH, kQBytes = 2 * kQPart;        // a warpgroup's queries: high, low
  static constexpr int kBytes = 1024 + (kKeys + kCodes) * kSlot + 2 * kValues + QT * kQBytes;
};
template <int QT>
constexpr int wide_threads() { return QT * 128 + 256; }      // (whole warpgroups: registers move between them)
// Registers a thread: a softmax warpgroup keeps 128 logits; the sum over warpgroups stays that of the launch (128 and 168 a thread).
template <int QT>
constexpr int kSoftmaxRegs = QT == 2 ? 168 : 232;
template <int QT>
constexpr int kOtherRegs = QT == 2 ? 88 : 128;

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int DH, int QT>
__global__ void __launch_bounds__(wide_threads<QT>(), 1)
attend8_wide_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const Attend8Args a) {
  using namespace ptx;
  using L = Wide8<DH, QT>;
  constexpr int SR = 8;
  using Ring = Ring8<L::kKeys, L::kCodes, SR>;
  constexpr int KW = QT == 2 ? 64 : 128, SPT = kTile / KW;     // rows of the cache of a step, steps of a tile
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars_s[Ring::kBars + 20 + SR];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  __shared__ Place place_s;
  __shared__ long long count_s;
  __shared__ float2 scale_s[SR][8];
  __shared__ float4 page_s[SR][8];             // of a tile's pages: keys' scale, values' exponent, its power of two turned over
  __shared__ uint32_t dead_s[SR];              // which of them hold nothing
  // New rows of a block with value codes that are NaN, by segment: converters are less than eight segments ahead of the slower warpgroup.
  __shared__ uint32_t bad_s[16][8];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  constexpr uint32_t kVAt = (L::kKeys + L::kCodes) * L::kSlot, kQAt = kVAt + 2 * L::kValues;
  const uint32_t bars = smem_u32(bars_s);
  const Ring ring{base, bars, scale_s};
  const uint32_t b_s = bars + 8 * Ring::kBars, b_p = b_s + 32, b_o = b_p + 32, b_q = b_o + 32, b_vf = b_q + 16, b_ve = b_vf + 16, b_drain = b_ve + 16, b_pg = b_drain + 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kConvert = QT * 4, kProducer = kConvert + 4, kScales = kProducer + 1, kIssuer = kScales + 1;

  if (tid == 0) {
    ring.init(QT, 4);
    for (int i = 0; i < 4; ++i) { mbar_init(b_s + 8 * i, 1); mbar_init(b_p + 8 * i, 4); mbar_init(b_o + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(b_q + 8 * i, 4); mbar_init(b_vf + 8 * i, 4); mbar_init(b_ve + 8 * i, QT); mbar_init(b_drain + 8 * i, 1); }
    for (int i = 0; i < SR; ++i) mbar_init(b_pg + 8 * i, 1);
    fence_mbar_init();
    abort_s = 0;
  }
  if (tid < 128) bad_s[tid >> 3][tid & 7] = 0u;
  if (warp == kIssuer) {
    tmem_alloc(smem_u32(&tmem_s), 512);
    tmem_relinquish();
  }
  grid_dependency_wait();                      // everything below may come from the kernel before
  grid_dependency_launch();                    // (before this CTA is sure to hold tensor memory: the merge, which comes next, takes none)
  if (warp == kProducer) {
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

  if (left > 0 && warp < kConvert) {
    regs_more<kSoftmaxRegs<QT>>();
    // A warpgroup alone polls (412 us for 32 tokens over 128k rows of four layers of eight heads, asleep 483); two sleep (a chunk of 512
    // tokens over 12k rows 231 us, polling 237).
    auto wait = [&](uint32_t bar, uint32_t parity) { return QT == 1 ? wait_warp(wt, bar, parity) : wait8(wt, bar, parity); };
    const int qt = warp >> 2, row = tid & 127;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    uint8_t* q_gen = gen + kQAt + qt * L::kQBytes;
    const uint32_t o_addr = tmem + lane_base + 256u + (uint32_t)qt * 128u;
    uint32_t k0 = 0, st = 0, n_o = 0, seg = 0; // tiles, steps, commits on b_o and segments so far
    bool ok = true;
    while (left > 0 && ok) {
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left);
      left -= t1 - t0;
      const int tok0 = p.qp * a.block_tok, rows = min(a.block_tok, p.s.n - tok0) * a.n_rep;    // query rows
      const int new0 = p.s.base + tok0;        // row of the block's first token
      const size_t qh0 = ((size_t)(a.l0 + p.l) * a.n_tok + p.s.f0 + tok0) * a.H_q + (size_t)p.g * a.n_rep;
      auto token_of = [&](int m) { return (int)(((uint32_t)m * a.rep_inv) >> 16); };
      auto place_of = [&](int m) { return qh0 + (size_t)token_of(m) * a.H_q + (m - token_of(m) * a.n_rep); };
      float qs = 0.0f;                         // factor of this thread's row
      {
        // a warp brings its own 32 rows, and their place is its own in the epilogue too
        constexpr int C = DH / 8, STEP = 32 / C, U = 4;        // lanes of a row; rows per round; rounds in flight
        const int c = lane % C;
#pragma unroll 1
        for (int i0 = 0; i0 < 32; i0 += U * STEP) {
          uint4 v[U];
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int m = qt * kQRows8 + (warp & 3) * 32 + i0 + i * STEP + lane / C;
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (m < rows) v[i] = *reinterpret_cast<const uint4*>(a.q + place_of(m) * DH + c * 8);
          }
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int r = i0 + i * STEP + lane / C;            // of the warp's
            uint2 hi, lo;
            int ex;
            encode_query<C>(v[i], &hi, &lo, &ex);
            uint8_t* at = q_gen + tile_place<DH>((warp & 3) * 32 + r, c);
            *reinterpret_cast<uint2*>(at) = hi;
            *reinterpret_cast<uint2*>(at + L::kQPart) = lo;
            const int mine = __shfl_sync(0xffffffffu, ex, (lane - (i0 + i * STEP)) * C & 31);
            if (lane >= i0 + i * STEP && lane < i0 + (i + 1) * STEP) qs = __int_as_float((127 + mine) << 23) * a.scale2;
          }
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(b_q + 8 * qt);
      const int m = qt * kQRows8 + row;
      const bool live = m < rows, warp_live = (m & ~31) < rows;
      const int limit = new0 + (live ? token_of(m) : 0) + 1;   // rows of the cache that this query row sees
      float m_used = -INFINITY, l = 0.0f;
      const int steps = (t1 - t0) * SPT;
      for (int s = 0; s < steps; ++s, ++st) {
        const int half = s % SPT;
        const uint32_t buf = st & 1u, k = k0 + (uint32_t)(s / SPT);
        if (!(ok = wait(b_pg + 8 * (k % SR), (k / SR) & 1u) && wait(b_s + 16 * qt + 8 * buf, (st >> 1) & 1u))) break;
        tc_fence_after();
        const uint32_t s_addr = tmem + lane_base + (uint32_t)qt * 128u + buf * KW;
        const int j0 = (t0 + s / SPT) * kTile + half * KW;     // first row of the step
        const uint32_t dead = dead_s[k % SR];
        if (warp_live) {
          constexpr int NC = KW / 32, NP = KW / 16;
          uint32_t z[NC][32];
#pragma unroll
          for (int i = 0; i < NC; ++i) tmem_ld32_nb(s_addr + 32u * i, z[i]);
          float f[NP], e[NP], e_inv[NP];       // sixteen columns lie in one page
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float4 x = page_s[k % SR][(half * KW + 16 * i) >> a.page_shift];
            f[i] = x.x * qs;
            e[i] = x.y;
            e_inv[i] = x.z;
          }
#pragma unroll
          for (int i = 0; i < NC; ++i) tc_wait_ld32_nb(z[i]);
          if (j0 + KW > new0 + 1 || dead) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              const int see = dead >> ((half * KW + 16 * i) >> a.page_shift) & 1u ? 0 : limit - (j0 + 16 * i);
#pragma unroll
              for (int x = 0; x < 16; ++x) z[i / 2][16 * (i & 1) + x] = x < see ? z[i / 2][16 * (i & 1) + x] : 0xff800000u;
            }
          }
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int x = 0; x < 16; x += 2)
              mx[(x >> 1) & 1] = fmaxf(fmaxf(mx[(x >> 1) & 1], __uint_as_float(z[i / 2][16 * (i & 1) + x])), __uint_as_float(z[i / 2][16 * (i & 1) + x + 1]));
            top = fmaxf(top, fmaf(fmaxf(mx[0], mx[1]), f[i], e[i]));
          }
          const float m_new = fmaxf(m_used, top);
          if (s == 0) {
            m_used = m_new;
          } else {
            const bool grow = m_new > m_used + kGrow8 || (m_used == -INFINITY && m_new > -INFINITY);
            if (__any_sync(0xffffffffu, grow)) {
              // O holds the steps before this one once the last product is done, which the next logits' commit tells, or its own
              const bool next = s + 1 < steps;
              if (!(ok = wait((next ? b_s + 8 * (buf ^ 1u) : b_o + 8 * (n_o & 1u)) + 16 * qt, ((next ? st + 1 : n_o) >> 1) & 1u))) break;
              tc_fence_after();
              const float g = grow ? (m_used == -INFINITY ? 0.0f : ex2_approx(m_used - m_new)) : 1.0f;
              if (grow) m_used = m_new;
              l *= g;
#pragma unroll 1
              for (int c = 0; c < DH; c += 16) {
                float o[16];
                uint32_t r[16];
                tmem_ld<16>(o_addr + (uint32_t)c, o);
                tc_wait_ld();
#pragma unroll
                for (int x = 0; x < 16; ++x) r[x] = __float_as_uint(o[x] * g);
                tmem_st16(o_addr + (uint32_t)c, r);
              }
            }
          }
          const float shift = m_used == -INFINITY ? 0.0f : m_used;
#pragma unroll
          for (int i = 0; i < NC; ++i) {       // P, two to a column, in the upper half of S's columns
            uint32_t r[16];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int c = 2 * i + h;
              const u64 f2 = pack2(f[c], f[c]), b2 = pack2(e[c] - shift, e[c] - shift);
              u64 sum = 0ull;
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                float2 w = unpack2(fma2(pack2u(z[i][16 * h + 2 * x], z[i][16 * h + 2 * x + 1]), f2, b2));
                w.x = ex2_approx(w.x);
                w.y = ex2_approx(w.y);
                sum = add2(sum, pack2(w.x, w.y));
                r[8 * h + x] = pack_f16(w.x, w.y);
              }
              const float2 two = unpack2(sum);
              l = fmaf(two.x + two.y, e_inv[c], l);
            }
            tmem_st16(s_addr + KW / 2 + 16u * i, r);
          }
          tc_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && !(a.inject & XKV_INJECT_CACHE_NO_HANDOVER)) mbar_arrive(b_p + 16 * qt + 8 * buf);
      }
      if (!ok) break;
      // ---- the segment's result (the last two products commit to two barriers in turn: by now both may be done)
      n_o += (uint32_t)min(2, steps);
      if (!(ok = wait(b_o + 16 * qt + 8 * ((n_o - 1u) & 1u), ((n_o - 1u) >> 1) & 1u))) break;
      k0 += (uint32_t)(t1 - t0);
      tc_fence_after();
      const bool whole = t0 == 0 && t1 == p.nt;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const size_t pr = ((size_t)blockIdx.x * 2 + (seg == 0 ? 0 : 1)) * a.block_rows + m;
      const size_t qh = live ? place_of(m) : 0;
      const bool odd = t1 * kTile > new0 + 1;  // tiles of this segment held rows that not all see
      if (warp_live) {
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          float o[32];
          tmem_ld32(o_addr + (uint32_t)c, o);
          tc_wait_ld();
          if (odd) {
#pragma unroll 1
            for (int w = 0; w < 8; ++w) {
              uint32_t bad = bad_s[seg & 15u][w];              // (entered before the product that this result waited for)
              while (bad) {
                const int j = new0 + 32 * w + __ffs(bad) - 1;
                bad &= bad - 1u;
                if (j >= limit) continue;
                const size_t head = ((size_t)(a.l0 + p.l) * a.n_pages + a.table[(size_t)p.b * a.max_pages + (j >> a.page_shift)]) * a.H_kv + p.g;
                const uint8_t* v = a.V8 + ((head << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * DH + c;
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = (v[e] & 0x7f) == 0x7f ? __int_as_float(0x7fffffff) : o[e];
              }
            }
          }
          if (live && whole) {
            uint4* dst = reinterpret_cast<uint4*>(a.out + qh * DH + c);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              dst[e] = make_uint4(pack_bf16(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                                  pack_bf16(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
          } else if (!whole) {
            // through the places of this warp's rows of Q, so that a store writes whole lines
            auto own = [&](int i) {
              constexpr int HALF = 32 * DH / 16;               // units of the warp's rows in either part of Q
              return reinterpret_cast<float4*>(q_gen + (i < HALF ? 0 : L::kQPart) + (warp & 3) * (32 * DH)) + (i < HALF ? i : i - HALF);
            };
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) *own(lane * 8 + (e ^ (lane & 7))) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
            __syncwarp();
            float* dst = a.part + (pr - row + (warp & 3) * 32) * DH + c + (lane & 7) * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = 4 * i + (lane >> 3);
              *reinterpret_cast<float4*>(dst + (size_t)r * DH) = *own(r * 8 + ((lane & 7) ^ (r & 7)));
            }
          }
        }
        __syncwarp();                          // the next problem's queries go where other lanes may still be reading
        if (live && whole && a.lse) a.lse[qh] = l == 0.0f ? -INFINITY : (m_used + log2f(l)) * 0.6931471805599453f;
        if (live && !whole) a.part_ml[pr] = make_float2(m_used, l);
      }
      tc_fence_before();
      ++seg;
      if (left > 0) next_problem(a, p);
    }
  } else if (left > 0 && warp < kProducer) {
    regs_fewer<kOtherRegs<QT>>();
    constexpr int C = DH / 16, STEP = 128 / C; // 16-byte units of a row of codes; rows per round
    const int ct = tid - kConvert * 32, c = ct % C;
    uint32_t k = 0, seg = 0;
    bool ok = true;
    while (left > 0 && ok) {
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left);
      left -= t1 - t0;
      const int seen = rows_seen(a, p.s, p.qp), new0 = p.s.base + p.qp * a.block_tok;
      if (ct < 8) bad_s[(seg + 8) & 15u][ct] = 0u;
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
            const __half2 lo = decode_f16x2(w[e]), hi = decode_f16x2(w[e] >> 16);
            h[2 * e] = *reinterpret_cast<const uint32_t*>(&lo);
            h[2 * e + 1] = *reinterpret_cast<const uint32_t*>(&hi);
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
    regs_fewer<kOtherRegs<QT>>();
    if (warp == kProducer) {
      n_loaded = ring.template produce<DH, true, true>(a, wt, &k_map, &v_map, p, left);
    } else if (warp == kScales) {
      for (uint32_t k = 0; k < (uint32_t)count_s; ++k) {
        if (!wait8(wt, ring.scales_full(k), Ring::scales_parity(k))) break;
        const float2 sc = scale_s[k % SR][min(lane, 127 >> a.page_shift)];
        const int kb = __float_as_int(sc.x) & 0x7f800000, ve = (__float_as_int(sc.y) >> 23) & 255;
        const uint32_t dead = __ballot_sync(0xffffffffu, kb == 0 || ve == 0);
        if (lane < 8) page_s[k % SR][lane] = make_float4(kb == 0 ? 1.0f : __int_as_float(kb), (float)(ve - 127), __int_as_float((254 - ve) << 23), 0.0f);
        if (lane == 0) dead_s[k % SR] = dead;
        __syncwarp();
        if (lane == 0) mbar_arrive(b_pg + 8 * (k % SR));
      }
    } else if (warp < kIssuer + QT) {
      // ---- branches outside the issue are taken on a vote and descriptors differ by constants, so that they stay in uniform registers
      const int qt = warp - kIssuer;
      constexpr uint32_t idesc_s = idesc_e4m3_f32(128, KW);
      constexpr uint32_t idesc_o = (1u << 4) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((128u >> 4) << 24);   // fp16; V is read along its rows
      const uint64_t q_desc = smem_desc_rows<DH>(base + kQAt + qt * L::kQBytes), k_desc = smem_desc_rows<DH>(base);
      const uint64_t v_desc = (smem_desc_sw128(base + kVAt, 0) & ~(0xFFFFull << 16)) | ((uint64_t)(L::kSlab >> 4) << 16);
      const uint32_t s_tmem = tmem + (uint32_t)qt * 128u, o_tmem = tmem + 256u + (uint32_t)qt * 128u;
      uint32_t k0 = 0, st = 0, n_o = 0, seg = 0;               // tiles, steps, commits on b_o and segments so far
      bool ok = true;
      auto logits = [&](uint32_t buf, uint32_t k, int half) {
        const uint64_t kd = k_desc + (uint64_t)((k % L::kKeys) * (uint32_t)(L::kSlot >> 4) + (uint32_t)half * (KW * DH >> 4));
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < DH / 32; ++i)
            tc_mma_e4m3(s_tmem + buf * KW, q_desc + (uint64_t)(h * (L::kQPart >> 4) + 2 * i), kd + (uint64_t)(2 * i), idesc_s, h | i ? 1u : 0u);
        tc_commit(b_s + 16 * qt + 8 * buf);
        if (half == SPT - 1) tc_commit(ring.k_empty(k));
      };
      auto keys = [&](uint32_t k) { return wait8(wt, ring.k_full(k), Ring::k_parity(k)); };
      while (left > 0 && ok) {
        const int n = (int)min((long long)p.nt, p.t + left) - p.t, steps = n * SPT;
        left -= n;
        ok = wait8(wt, b_q + 8 * qt, seg & 1u);
        for (int s = 0; s < min(2, steps) && ok; ++s) {        // two steps of logits ahead
          if (s % SPT == 0 && !(ok = keys(k0 + s / SPT))) break;
          tc_fence_after();
          if (elect_one()) logits((st + s) & 1u, k0 + s / SPT, s % SPT);
          __syncwarp();
        }
        for (int s = 0; s < steps && ok; ++s) {
          const uint32_t buf = (st + s) & 1u, k = k0 + s / SPT, kn = k0 + (s + 2) / SPT;
          const bool more = s + 2 < steps;
          if (s % SPT == 0 && !(ok = wait8(wt, b_vf + 8 * (k & 1u), (k >> 1) & 1u))) break;
          if (more && s % SPT == 0 && !(ok = keys(kn))) break;
          if (!(ok = wait8(wt, b_p + 16 * qt + 8 * buf, ((st + s) >> 1) & 1u))) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t vd = v_desc + (uint64_t)((k & 1u) * (uint32_t)(L::kValues >> 4) + (uint32_t)(s % SPT) * (KW * 8));
#pragma unroll
            for (int i = 0; i < KW / 16; ++i)
              tc_mma_bf16_ts(o_tmem, s_tmem + buf * KW + KW / 2 + (uint32_t)i * 8u, vd + (uint64_t)(i * (2048 >> 4)), idesc_o, (s | i) ? 1u : 0u);
            if (s % SPT == SPT - 1) tc_commit(b_ve + 8 * (k & 1u));
            // the logits after the next follow the product that reads P, which lies where they go; their commit tells of both
            if (more) logits(buf, kn, (s + 2) % SPT); else tc_commit(b_o + 16 * qt + 8 * (n_o & 1u));
          }
          __syncwarp();
          n_o += more ? 0u : 1u;
        }
        st += steps;
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
    if (warp >= kIssuer && warp < kIssuer + QT) {
      const uint32_t bar = b_drain + 8 * (warp - kIssuer);
      if (elect_one()) tc_commit(bar);
      for (uint32_t i = 0; i < (1u << 16); ++i) if (__all_sync(0xffffffffu, mbar_try_wait(bar, 0))) break;
    }
    __syncthreads();
  }
  if (warp == kIssuer) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (abort_s && warp == kProducer) {
    ring.template drain<true, true>(n_loaded);
    results_are_nan<DH>(a, place_s, count_s);
  }
}

template <int DH, int QT>
cudaError_t launch_wide(const CUtensorMap& k_map, const CUtensorMap& v_map, const Attend8Args& a, int grid, int device, cudaStream_t s) {
  const cudaError_t e = ensure_dyn_smem<attend8_wide_kernel<DH, QT>>(Wide8<DH, QT>::kBytes, device);
  return e != cudaSuccess ? e : launch_pdl(attend8_wide_kernel<DH, QT>, dim3(grid), dim3(wide_threads<QT>()), Wide8<DH, QT>::kBytes, s, k_map, v_map, a);
}

}  // namespace

cudaError_t launch_attend8_wide(const CUtensorMap& k_map, const CUtensorMap& v_map, int d_h, const Attend8Args& a, int grid, int device,
                                cudaStream_t s) {
  if (d_h == 128) return a.block_rows == 256 ? launch_wide<128, 2>(k_map, v_map, a, grid, device, s) : launch_wide<128, 1>(k_map, v_map, a, grid, device, s);
  return a.block_rows == 256 ? launch_wide<64, 2>(k_map, v_map, a, grid, device, s) : launch_wide<64, 1>(k_map, v_map, a, grid, device, s);
}

}  // namespace xkv
