// Attention over a paged cache of 8-bit codes (xkv_cache8_attend): out_i = softmax(scale q_i K^T) V over the rows of token i's sequence
// up to its own, K and V being e4m3 codes times their pages' scales, powers of two.
//
// For few query rows, 8 or 16 of a KV head (decode steps, a draft or two): the codes go from memory into the tensor core as they are, and
// the products are turned around, so that the 128 rows of a tile of the cache are the wide side and the block of query rows (tokens times
// the query heads of a KV head) the narrow one:
//   S^T = K8 Q8^T       M = 128 rows of the cache, N = 2 x query rows
//   O^T += V8^T P8^T    M = d_h, N = 4 x query rows, K = 128 rows of the cache
// Both operands of such a product have to be 8-bit codes; a query and a weight are split into several:
//   q 2^-x = q_hi + 2^-5 q_lo   (x: its row's largest element lies in [128, 256)): a bf16 value's 8 bits are two e4m3 codes (encode_query),
//                          two columns of S
//   w = w_0 + 2^-3 w_1 + 2^-6 w_2 + 2^-9 w_3   of a weight in 16 bits (fp16), exactly, in e5m2: that is an fp16 number's upper byte, so a code
//                          is cut off, not converted, and the next is that of 2^3 times what it left (3 bits of 11 each; 2^-9 times the
//                          smallest code is 2^-25).  Four groups of columns of O, joined at the end.  What 16 bits mean to a weight
//                          stands at kTop.  (Three e4m3 codes, 2^-10 of the first's steps, lost an even rest below 2^-24 of the
//                          largest weight and were off by 6 % at 2^-20.)
// A key's scale multiplies the row's logits.  A value's scale 2^e joins the exponent: w_j = 2^(z_j + e_j - m), so that codes meet weights
// that hold their scale, and m is the maximum of z_j + e_j; the denominator sums w_j 2^-e_j in fp32.
//
//   producers pages by the copy engine, with their scales (Ring8): a warp for keys, one for values (pages of 16 rows are 16 boxes a tile)
//   issuers   a warp for S, up to four tiles ahead, and one for O; the commits that free a tile's slots are what tells of S and O, too
//   softmax   two warpgroups, tile by tile in turns, each with its own maxima, sums and O; thread = row of the cache, so that a token's
//             view (rows up to its own) is a comparison of the column with one number per thread.  Maxima move only when a weight would
//             pass its bound: one vote per tile.
//   helpers   a warpgroup: queries of the next problem while this one is worked on, results of the last (S, queries and O are there twice)
// All tiles of all problems form one list that is cut into as many even pieces as there are CTAs; a piece that holds a whole problem
// writes its output, the others leave (O, m, l) for the merge.  Lengths are read on the device only.
//
// Bound by HBM.  131072 rows of four layers of eight heads, four query heads each: 168-174 us for pages of 16 to 128 rows (6.2-6.4 TB/s, 0.96
// of the copy's rate); eight sequences of up to 8191 rows 76-79; 32 of 2047 rows 102-117 (floor 84); 300 rows 10, latencies of two kernels.
// The fourth code of a weight and what keeps scales' extremes apart cost nothing where HBM bounds, 3 % at 32 sequences.  What a step
// brought (128k rows; eight sequences; pages of 16): warps that wait asleep instead of polling 187 -> 174, 99 -> 77, 105 -> 76; one
// issuing warp, two products for the two codes of a query 199, 102; the merge finding places for itself 105.
#include <cuda.h>
#include <math.h>

#include "xkv_attend8.cuh"

namespace xkv {

namespace {

constexpr int kThreads8 = 512;                 // two warpgroups of softmax, one of queries and results; two producers, two issuers
constexpr int kHelper8 = 8, kProducer8 = 12, kLogits8 = 13, kValues8 = 14, kProducerV8 = 15;
constexpr int kMergeWarps8 = 8;
constexpr int kCodes8 = 4;                     // of a weight

// N columns, and the N behind them.
template <int N>
__device__ __forceinline__ void load_columns(uint32_t addr, float (&u)[N], float (&v)[N]) {
  ptx::tmem_ld<N>(addr, u);
  ptx::tmem_ld<N>(addr + N, v);
  ptx::tc_wait_ld();
}

template <int DH, int RB>
struct Shape8 {
  static constexpr int kQ = 2 * RB;                            // columns of S: two codes of a query
  static constexpr int kP = kCodes8 * RB;                      // columns of O: the codes of a weight
  static constexpr int kSlot = kTile * DH;
  static constexpr int kSlots = DH == 64 ? 8 : 5;              // tiles of keys, and as many of values
  static constexpr int kAhead = 4;                             // tiles of S in tensor memory
  static constexpr int kQBytes = kQ * DH, kPBytes = kP * kTile;
  static constexpr int kBytes = 1024 + 2 * kSlots * kSlot + 2 * kPBytes + 2 * kQBytes;
  static constexpr int kTmem = RB == 8 ? 256 : 512;            // S of tiles ahead, O of two warpgroups for two problems; rounded up
};

// Sums of N columns over the lanes of a warp: lane i gets those of columns i, i + 32, ...
template <int N>
__device__ __forceinline__ void sum_columns(float (&v)[N], float* dst) {
  const int lane = threadIdx.x & 31;
  constexpr int W = N < 32 ? N : 32;
#pragma unroll
  for (int c0 = 0; c0 < N; c0 += W) {
    // halves change places: after each step a lane has half as many columns, summed over twice as many lanes
#pragma unroll
    for (int w = W / 2; w > 0; w >>= 1) {
      const bool up = lane & w;
#pragma unroll
      for (int i = 0; i < w; ++i) {
        const float give = up ? v[c0 + i] : v[c0 + i + w], keep = up ? v[c0 + i + w] : v[c0 + i];
        v[c0 + i] = keep + __shfl_xor_sync(0xffffffffu, give, w);
      }
    }
    float x = v[c0];
#pragma unroll
    for (int o = W; o < 32; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane < W) dst[c0 + lane] = x;
  }
}

template <int DH, int RB>
__global__ void __launch_bounds__(kThreads8, 1)
attend8_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const Attend8Args a) {
  using namespace ptx;
  using L = Shape8<DH, RB>;
  using Ring = Ring8<L::kSlots, L::kSlots, 2 * L::kSlots>;
  constexpr int NQ = L::kQ, NP = L::kP, SR = 2 * L::kSlots, NB = L::kAhead;
  static_assert(L::kSlots >= NB, "S of a tile is read before its keys' slot is multiplied again");
  static_assert(SR >= L::kSlots + NB, "and its scales before theirs is filled again");
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars_s[Ring::kBars + 12];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  __shared__ Place place_s;
  __shared__ long long count_s;
  __shared__ float2 scale_s[SR][8];            // of a tile's pages: keys', values'
  // By segment (two in turns) and warpgroup, of a column: factor of its query, bound that its z may not pass; what is taken off z (m);
  // sums of weights
  __shared__ float2 info_s[2][2][RB];
  __shared__ __align__(16) float sub_s[2][2][RB];
  __shared__ float sum_s[2][2][4][RB];
  __shared__ float fac_s[2][RB], top_s[2][4][RB];
  __shared__ uint32_t bad_s[2];                // by segment: new rows of the block's tokens with value codes that are NaN
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  constexpr uint32_t kPAt = 2 * L::kSlots * L::kSlot, kQAt = kPAt + 2 * L::kPBytes;         // ring, weights, queries
  const uint32_t bars = smem_u32(bars_s);
  // A slot is empty when its product is done, which is also what tells of S and O: k_empty of a tile "S is there", v_empty "O has it"
  const Ring ring{base, bars, scale_s};
  const uint32_t b_p = bars + 8 * Ring::kBars, b_q = b_p + 32, b_done = b_q + 16, b_free = b_done + 16, b_drain = b_free + 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    ring.init(1, 1);
    for (int i = 0; i < 4; ++i) mbar_init(b_p + 8 * i, 4);
    for (int i = 0; i < 2; ++i) { mbar_init(b_q + 8 * i, 4); mbar_init(b_done + 8 * i, 9); mbar_init(b_free + 8 * i, 4); mbar_init(b_drain + 8 * i, 1); }
    fence_mbar_init();
    abort_s = 0;
  }
  if (warp == kLogits8) {
    tmem_alloc(smem_u32(&tmem_s), L::kTmem);
    tmem_relinquish();
  }
  grid_dependency_wait();                      // everything below may come from the kernel before
  grid_dependency_launch();                    // (before this CTA is sure to hold tensor memory: the merge, which comes next, takes none)
  if (warp == kProducer8) {
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
  const uint64_t ring_desc = smem_desc_rows<DH>(base);

  if (left > 0 && warp == kProducer8) {
    n_loaded = ring.template produce<DH, true, false>(a, wt, &k_map, &v_map, p, left);
  } else if (left > 0 && warp == kProducerV8) {
    n_loaded = ring.template produce<DH, false, true>(a, wt, &k_map, &v_map, p, left);
  } else if (left > 0 && warp == kLogits8) {
    // ---- S of tile k, as soon as its keys are in and the weights of the tile that had its place are formed
    constexpr uint32_t idesc = idesc_e4m3_f32(128, NQ);
    uint32_t k = 0, seg = 0;
    bool ok = true;
    while (left > 0 && ok) {
      const int n = (int)min((long long)p.nt, p.t + left) - p.t;
      left -= n;
      ok = wait8(wt, b_q + 8 * (seg & 1u), (seg >> 1) & 1u);
      const uint64_t qd = smem_desc_rows<DH>(base + kQAt + (seg & 1u) * L::kQBytes);
      for (int s = 0; s < n && ok; ++s, ++k) {
        if (!(ok = wait8(wt, ring.k_full(k), Ring::k_parity(k)))) break;
        if (k >= NB && !(ok = wait8(wt, b_p + 8 * (k % NB), (k / NB - 1) & 1u))) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t kd = ring_desc + (uint64_t)((k % L::kSlots) * (uint32_t)(L::kSlot >> 4));
#pragma unroll
          for (int i = 0; i < DH / 32; ++i) tc_mma_8bit(tmem + (k % NB) * NQ, kd + (uint64_t)(2 * i), qd + (uint64_t)(2 * i), idesc, i ? 1u : 0u);
          tc_commit(ring.k_empty(k));
        }
        __syncwarp();
      }
      ++seg;
      if (left > 0 && ok) next_problem(a, p);
    }
  } else if (left > 0 && warp == kValues8) {
    // ---- O += weights of tile k times its values
    constexpr uint32_t idesc = idesc_e4m3_f32(DH, NP) | (1u << 10) | (1u << 15);             // P is e5m2; V is read along its rows
    const uint64_t p_desc = smem_desc_rows<128>(base + kPAt);
    uint32_t k = 0, seg = 0;
    bool ok = true;
    while (left > 0 && ok) {
      const int n = (int)min((long long)p.nt, p.t + left) - p.t;
      left -= n;
      ok = wait8(wt, b_free + 8 * (seg & 1u), ((seg >> 1) & 1u) ^ 1u);     // the results of the problem before last have been read
      const uint32_t o = tmem + NB * NQ + (seg & 1u) * (2 * NP);
      for (int s = 0; s < n && ok; ++s, ++k) {
        if (!(ok = wait8(wt, ring.v_full(k), Ring::v_parity(k)) && wait8(wt, b_p + 8 * (k % NB), (k / NB) & 1u))) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = ring_desc + (uint64_t)((L::kSlots + k % L::kSlots) * (uint32_t)(L::kSlot >> 4)), pd = p_desc + (uint64_t)((k & 1u) * (uint32_t)(L::kPBytes >> 4));
#pragma unroll
          for (int i = 0; i < kTile / 32; ++i)
            tc_mma_8bit(o + (k & 1u) * NP, vd + (uint64_t)(i * (32 * DH >> 4)), pd + (uint64_t)(2 * i), idesc, (s >= 2) | (i > 0) ? 1u : 0u);
          tc_commit(ring.v_empty(k));
          if (s + 1 == n) tc_commit(b_done + 8 * (seg & 1u));
        }
        __syncwarp();
      }
      ++seg;
      if (left > 0 && ok) next_problem(a, p);
    }
  } else if (left > 0 && warp >= kHelper8 && warp < kProducer8) {
    // ---- queries of the problem that comes next, results of the one that is done
    const int ht = tid - kHelper8 * 32;
    const uint32_t o_base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + NB * NQ;
    bool ok = true;
    auto queries = [&](const Place& x, uint32_t par) {
      const int tok0 = x.qp * a.block_tok, rows = min(a.block_tok, x.s.n - tok0) * a.n_rep;
      const size_t qh0 = ((size_t)(a.l0 + x.l) * a.n_tok + x.s.f0 + tok0) * a.H_q + (size_t)x.g * a.n_rep;
      constexpr int C = DH / 8;                // lanes of a row, eight elements each
#pragma unroll
      for (int i0 = 0; i0 < RB * C; i0 += 128) {
        const int i = i0 + ht, r = i / C, c = i % C;
        if (RB * C < 128 && i >= RB * C) break;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        const int tok = (int)(((uint32_t)r * a.rep_inv) >> 16);
        if (r < rows) v = *reinterpret_cast<const uint4*>(a.q + (qh0 + (size_t)tok * a.H_q + (r - tok * a.n_rep)) * DH + c * 8);
        uint2 hi, lo;
        int ex;
        encode_query<C, true>(v, &hi, &lo, &ex);
        uint8_t* at = gen + kQAt + par * L::kQBytes + tile_place<DH>(r, c);
        *reinterpret_cast<uint2*>(at) = hi;
        *reinterpret_cast<uint2*>(at + RB * DH) = lo;
        if (c == 0) {
          const float qs = __int_as_float((127 + ex) << 23) * a.scale2;
          info_s[par][0][r] = info_s[par][1][r] = make_float2(qs, r < rows ? -INFINITY : INFINITY);            // (nobody's column: no bound)
          sub_s[par][0][r] = sub_s[par][1][r] = 0.0f;
        }
      }
      if (ht == 0) bad_s[par] = 0u;
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(b_q + 8 * par);
    };
    queries(p, 0);
    uint32_t k0 = 0;
    for (uint32_t seg = 0; left > 0; ++seg) {
      const uint32_t par = seg & 1u;
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left), n = t1 - t0;
      left -= n;
      Place x = p;
      if (left > 0) {
        next_problem(a, p);
        queries(p, par ^ 1u);
      }
      ok = wait8(wt, b_done + 8 * par, (seg >> 1) & 1u);
      tc_fence_after();
      if (named_bar_any(3, 128, !ok)) break;
      const int tok0 = x.qp * a.block_tok, rows = min(a.block_tok, x.s.n - tok0) * a.n_rep, new0 = x.s.base + tok0;
      const size_t qh0 = ((size_t)(a.l0 + x.l) * a.n_tok + x.s.f0 + tok0) * a.H_q + (size_t)x.g * a.n_rep;
      const bool whole = t0 == 0 && t1 == x.nt;
      const bool has0 = n > (int)(k0 & 1u), has1 = n > (int)((k0 ^ 1u) & 1u);    // does a warpgroup have tiles of this segment?
      const int d = DH == 128 ? ht : (warp & 3) * 16 + lane;
      const bool owns = DH == 128 || lane < 16;
      const size_t pr = ((size_t)blockIdx.x * 2 + (seg == 0 ? 0 : 1)) * a.block_rows;
#pragma unroll 1
      for (int c0 = 0; c0 < rows; c0 += 4) {
        float o[2][kCodes8][4];
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int g = 0; g < kCodes8; ++g) tmem_ld<4>(o_base + par * (2 * NP) + (uint32_t)(w * NP + g * RB + c0), o[w][g]);
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = c0 + i;
          if (r >= rows) break;
          // a warpgroup's maxima; what it has not seen counts nothing
          const float m0 = info_s[par][0][r].y == -INFINITY ? -INFINITY : sub_s[par][0][r], m1 = info_s[par][1][r].y == -INFINITY ? -INFINITY : sub_s[par][1][r];
          const float M = fmaxf(m0, m1);
          const float f0 = m0 == M ? 1.0f : exp2f(m0 - M), f1 = m1 == M ? 1.0f : exp2f(m1 - M);
          float y = 0.0f, sum = 0.0f;
          if (has0) {
            y = f0 * (o[0][0][i] + 0x1p-3f * (o[0][1][i] + 0x1p-3f * (o[0][2][i] + 0x1p-3f * o[0][3][i])));
            sum = f0 * (sum_s[par][0][0][r] + sum_s[par][0][1][r] + sum_s[par][0][2][r] + sum_s[par][0][3][r]);
          }
          if (has1) {
            y += f1 * (o[1][0][i] + 0x1p-3f * (o[1][1][i] + 0x1p-3f * (o[1][2][i] + 0x1p-3f * o[1][3][i])));
            sum += f1 * (sum_s[par][1][0][r] + sum_s[par][1][1][r] + sum_s[par][1][2][r] + sum_s[par][1][3][r]);
          }
          uint32_t bad = bad_s[par];
          while (owns && bad) {                // rows that were taken out, given back to the columns that see them
            const int tok = __ffs(bad) - 1;
            bad &= bad - 1u;
            if (tok * a.n_rep > r) continue;
            const int jj = new0 + tok, page = a.table[(size_t)x.b * a.max_pages + (jj >> a.page_shift)];
            const size_t head = ((size_t)(a.l0 + x.l) * a.n_pages + page) * a.H_kv + x.g;
            if ((a.V8[((head << a.page_shift) + (jj & ((1 << a.page_shift) - 1))) * DH + d] & 0x7f) == 0x7f) y = __int_as_float(0x7fffffff);
          }
          if (whole) {
            const int tok = (int)(((uint32_t)r * a.rep_inv) >> 16);
            const size_t qh = qh0 + (size_t)tok * a.H_q + (r - tok * a.n_rep);
            if (owns) a.out[qh * DH + d] = __float2bfloat16_rn(sum == 0.0f ? 0.0f : y / sum);
            if (ht == 0 && a.lse) a.lse[qh] = sum == 0.0f ? -INFINITY : (M + log2f(sum)) * 0.6931471805599453f;
          } else {
            if (owns) a.part[(pr + r) * DH + d] = y;
            if (ht == 0) a.part_ml[pr + r] = make_float2(M, sum);
          }
        }
      }
      k0 += n;
      tc_fence_before();
      named_bar_sync(3, 128);                  // the columns of the problem after next go where another warp may still be reading
      if (lane == 0) mbar_arrive(b_free + 8 * par);
    }
  } else if (left > 0 && warp < kHelper8) {
    const int wg = warp >> 2, row = tid & 127;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    uint8_t* p_row = gen + kPAt + wg * L::kPBytes + (row & 15);
    uint32_t k0 = 0, seg = 0;                  // tiles and segments so far
    bool ok = true, gone = false;              // this warp's waits; the warpgroup has given up
    while (left > 0 && !gone) {
      const uint32_t par = seg & 1u;
      const int t0 = p.t, t1 = (int)min((long long)p.nt, p.t + left), n = t1 - t0;
      left -= n;
      const int tok0 = p.qp * a.block_tok, rows = min(a.block_tok, p.s.n - tok0) * a.n_rep;    // query rows
      const int seen = rows_seen(a, p.s, p.qp), new0 = p.s.base + tok0;                        // row of the block's first token
      ok = ok && wait8(wt, b_q + 8 * par, (seg >> 1) & 1u);
      const float2* info = info_s[par][wg];
      const float* sub = sub_s[par][wg];
      const uint32_t o_base = tmem + lane_base + NB * NQ + par * (2 * NP) + (uint32_t)wg * NP;
      float l[RB];
#pragma unroll
      for (int r = 0; r < RB; ++r) l[r] = 0.0f;
      bool any = false;                        // this warpgroup has tiles of the segment behind it

      for (int s = (int)((k0 ^ (uint32_t)wg) & 1u); s < n; s += 2) {
        const uint32_t k = k0 + s;
        ok = ok && wait8(wt, ring.scales_full(k), Ring::scales_parity(k));
        const float2 sc = scale_s[k % SR][row >> a.page_shift];
        const int ke = (__float_as_int(sc.x) >> 23) & 255, ve = (__float_as_int(sc.y) >> 23) & 255;
        const float ks = __int_as_float(ke << 23);
        const int j = (t0 + s) * kTile + row;
        // columns from `from` on see the row
        const bool dead = j >= seen || ke == 0 || ve == 0;
        const int from = dead ? RB : max(0, min(j - new0, 64) * a.n_rep);
        const float e = ke == 255 || ve == 255 ? __int_as_float(0x7fffffff) : (float)(ve - 127), e_inv = turned_over(ve);
        ok = ok && wait8(wt, ring.k_empty(k), Ring::k_parity(k));
        tc_fence_after();
        float z[RB];
        {
          float lo[RB];
          load_columns<RB>(tmem + lane_base + (k % NB) * NQ, z, lo);
#pragma unroll
          for (int r = 0; r < RB; ++r) z[r] = fmaf(lo[r], 0x1p-5f, z[r]);
        }
        bool grow = !ok;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          if (r % 4 == 0 && r >= rows) break;
          const float2 col = info[r];
          z[r] = fmaf(z[r] * ks, col.x, e);    // (in this order: what is 0 has the logit 0 also where the factors' product is infinite)
          z[r] = r >= from ? z[r] : -INFINITY;
          grow |= z[r] > col.y;
        }
        bool waited = false;
        if (named_bar_any(1 + wg, 128, grow)) {
          // ---- a weight would pass its bound (or a wait has run out): maxima move
          if (ok && k >= 2) ok = wait8(wt, ring.v_empty(k - 2), Ring::v_parity(k - 2));
          waited = true;
          if (named_bar_any(1 + wg, 128, !ok)) { gone = true; break; }
          tc_fence_after();
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            if (r % 4 == 0 && r >= rows) break;
            const int b = __float_as_int(fmaxf(z[r], -INFINITY));              // (NaN counts as minus infinity); as an ordered integer
            const int m = __reduce_max_sync(0xffffffffu, b ^ ((b >> 31) & 0x7fffffff));
            if (lane == 0) top_s[wg][warp & 3][r] = __int_as_float(m ^ ((m >> 31) & 0x7fffffff));
          }
          named_bar_sync(1 + wg, 128);
          if (row < RB) {
            const float m = fmaxf(fmaxf(top_s[wg][0][row], top_s[wg][1][row]), fmaxf(top_s[wg][2][row], top_s[wg][3][row]));
            float f = 1.0f;
            if (row < rows && m > info[row].y) {
              const float off = taken_off(m);
              f = info[row].y == -INFINITY ? 0.0f : exp2f(sub[row] - off);
              sub_s[par][wg][row] = off;
              info_s[par][wg][row].y = weight_bound(off);
            }
            fac_s[wg][row] = f;
          }
          named_bar_sync(1 + wg, 128);
#pragma unroll
          for (int r = 0; r < RB; ++r) {
            if (r % 4 == 0 && r >= rows) break;
            l[r] *= fac_s[wg][r];
          }
          if (any) {
#pragma unroll 1
            for (int g = 0; g < kCodes8; ++g) {
#pragma unroll 1
              for (int c = 0; c < RB; c += 8) {
                if (c >= rows) break;
                const uint32_t at = o_base + (uint32_t)(g * RB + c);
                float o[8];
                tmem_ld<8>(at, o);
                tc_wait_ld();
                uint32_t x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = __float_as_uint(o[i] * fac_s[wg][c + i]);
                tmem_st8(at, x);
              }
            }
            tc_wait_st();
          }
        }
        // ---- weights, as four codes each; the product before has to have read the last ones
        if (ok && !waited && k >= 2) ok = wait8(wt, ring.v_empty(k - 2), Ring::v_parity(k - 2));
#pragma unroll
        for (int r = 0; r < RB; r += 2) {
          if (r % 4 == 0 && r >= rows) break;
          const float w0 = ex2_approx(z[r] - sub[r]), w1 = ex2_approx(z[r + 1] - sub[r + 1]);
          l[r] = fmaf(w0, e_inv, l[r]);
          l[r + 1] = fmaf(w1, e_inv, l[r + 1]);
          const __half2 step = __float2half2_rn(8.0f);
          __half2 h = __floats2half2_rn(w0, w1);
#pragma unroll
          for (int g = 0; g < kCodes8; ++g) {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(&h) & 0xff00ff00u;
            const int n0 = g * RB + r, n1 = n0 + 1;
            p_row[n0 * 128 + (((row >> 4) ^ (n0 & 7)) << 4)] = (uint8_t)(c >> 8);
            p_row[n1 * 128 + (((row >> 4) ^ (n1 & 7)) << 4)] = (uint8_t)(c >> 24);
            if (g < kCodes8 - 1) h = __hmul2(__hsub2(h, *reinterpret_cast<const __half2*>(&c)), step);
          }
        }
        if (__any_sync(0xffffffffu, dead || from > 0)) {
          // thread = value row: what no column sees is zeroed, NaN is taken out of what only some see, and listed
          ok = ok && wait8(wt, ring.v_full(k), Ring::v_parity(k));
          if (ok && (dead || from > 0)) {
            uint4* v = reinterpret_cast<uint4*>(gen + (L::kSlots + k % L::kSlots) * L::kSlot + row * DH);      // (the order of its units does not matter)
            uint32_t hit = 0;
#pragma unroll
            for (int c = 0; c < DH / 16; ++c) {
              uint4 x = dead || from >= rows ? make_uint4(0u, 0u, 0u, 0u) : v[c];
              const uint4 m = make_uint4(nan_codes(x.x), nan_codes(x.y), nan_codes(x.z), nan_codes(x.w));
              hit |= m.x | m.y | m.z | m.w;
              v[c] = make_uint4(x.x & ~m.x, x.y & ~m.y, x.z & ~m.z, x.w & ~m.w);
            }
            if (hit) atomicOr(&bad_s[par], 1u << (j - new0));
          }
        }
        fence_proxy_async();
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && ok && !(a.inject & XKV_INJECT_CACHE_NO_HANDOVER)) mbar_arrive(b_p + 8 * (k % NB));
        any = true;
      }
      if (gone) break;
      sum_columns<RB>(l, sum_s[par][wg][warp & 3]);
      __syncwarp();
      if (lane == 0 && ok) mbar_arrive(b_done + 8 * par);
      k0 += n;
      ++seg;
      if (left > 0) next_problem(a, p);
    }
  }

  // wind down: nothing of this CTA may still touch shared or tensor memory
  tc_fence_before();
  __syncthreads();
  if (abort_s) {                               // given up: nothing may still write tensor memory when it is freed
    if (warp == kLogits8 || warp == kValues8) {
      const uint32_t bar = b_drain + 8 * (warp - kLogits8);
      if (elect_one()) tc_commit(bar);
      for (uint32_t i = 0; i < (1u << 16); ++i) if (__all_sync(0xffffffffu, mbar_try_wait(bar, 0))) break;
    }
    __syncthreads();
  }
  if (warp == kLogits8) {
    tc_fence_after();
    tmem_dealloc(tmem, L::kTmem);
  }
  if (abort_s && warp == kProducer8) {
    ring.template drain<true, false>(n_loaded);
    results_are_nan<DH>(a, place_s, count_s);
  }
  if (abort_s && warp == kProducerV8) ring.template drain<false, true>(n_loaded);
}

// Joins the pieces of a problem: O = sum_c 2^(m_c - M) O_c, l likewise.  A problem that lies in several pieces is joined where its second
// piece begins (so there are at most as many as CTAs); a warp has one of its query rows, lane = d_h / 32 columns.
// AT_ONCE pieces of a row are in flight: sixteen where there are few rows, four where there are many (four CTAs an SM instead of two).
template <int DH, int AT_ONCE>
__global__ void __launch_bounds__(kMergeWarps8 * 32) attend8_merge_kernel(const Attend8Args a) {
  constexpr int V = DH / 32;
  const int lane = threadIdx.x & 31, r = blockIdx.y * kMergeWarps8 + (threadIdx.x >> 5), c_second = blockIdx.x + 1;
  ptx::grid_dependency_wait();                 // every CTA waits, so that who waits for this kernel has waited for the one before
  ptx::grid_dependency_launch();
  const Place p = a.pieces[c_second].at;
  const long long second = a.pieces[c_second].count, first = a.pieces[c_second - 1].count;
  if (second == 0 || p.t == 0 || p.t > first) return;          // nothing; a problem's first piece; not its second
  const int tok0 = p.qp * a.block_tok;
  if (r >= min(a.block_tok, p.s.n - tok0) * a.n_rep) return;
  const int c0 = c_second - 1;
  int c1 = c_second;
  for (long long rest = p.nt - p.t - second; rest > 0; rest -= a.pieces[c1].count) ++c1;
  // a problem that begins inside a piece is that piece's last one, and in the others the first
  auto slot = [&](int c) { return ((size_t)c * 2 + (c == c0 && p.t < first ? 1 : 0)) * a.block_rows + r; };
  float M = -INFINITY, sum = 0.0f, acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.0f;
  for (int cb = c0; cb <= c1; cb += 32) {      // lane: the weight of one piece of 32
    const int n = min(32, c1 - cb + 1);
    float x[AT_ONCE][V];
    auto load = [&](int j0) {
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const float* src = a.part + slot(cb + min(j0 + j, n - 1)) * DH + lane * V;
        if constexpr (V == 4) *reinterpret_cast<float4*>(x[j]) = *reinterpret_cast<const float4*>(src);
        else *reinterpret_cast<float2*>(x[j]) = *reinterpret_cast<const float2*>(src);
      }
    };
    const float2 ml = lane < n ? a.part_ml[slot(cb + lane)] : make_float2(-INFINITY, 0.0f);
    load(0);                                   // (asked for before the weights are known)
    float top = ml.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float M_new = fmaxf(M, top), old = M == -INFINITY ? 1.0f : exp2f(M - M_new);
    const float f = ml.x == -INFINITY ? (ml.y == 0.0f ? 0.0f : 1.0f) : exp2f(ml.x - M_new);    // (a piece of NaNs stays one)
    M = M_new;
    float part = f * ml.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    sum = fmaf(sum, old, part);
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] *= old;
    for (int j0 = 0; j0 < n; j0 += AT_ONCE) {
      if (j0 > 0) load(j0);
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const float w = __shfl_sync(0xffffffffu, f, (j0 + j) & 31);
        if (j0 + j < n && w != 0.0f) {
#pragma unroll
          for (int i = 0; i < V; ++i) acc[i] = fmaf(w, x[j][i], acc[i]);
        }
      }
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const size_t qh = ((size_t)(a.l0 + p.l) * a.n_tok + p.s.f0 + tok0 + r / a.n_rep) * a.H_q + p.g * a.n_rep + r % a.n_rep;
  uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + qh * DH + lane * V);
#pragma unroll
  for (int i = 0; i < V; i += 2) dst[i / 2] = ptx::pack_bf16(acc[i] * inv, acc[i + 1] * inv);
  if (a.lse && lane == 0) a.lse[qh] = sum == 0.0f ? -INFINITY : (M + log2f(sum)) * 0.6931471805599453f;
}

template <int DH, int RB>
cudaError_t launch_as(const CUtensorMap& k_map, const CUtensorMap& v_map, const Attend8Args& a, int grid, int device, cudaStream_t s) {
  const cudaError_t e = ensure_dyn_smem<attend8_kernel<DH, RB>>(Shape8<DH, RB>::kBytes, device);
  return e != cudaSuccess ? e : launch_pdl(attend8_kernel<DH, RB>, dim3(grid), dim3(kThreads8), Shape8<DH, RB>::kBytes, s, k_map, v_map, a);
}

template <int DH>
cudaError_t launch_width(const CUtensorMap& k_map, const CUtensorMap& v_map, const Attend8Args& a, int grid, int device, cudaStream_t s) {
  cudaError_t e = a.block_rows == 8 ? launch_as<DH, 8>(k_map, v_map, a, grid, device, s) : a.block_rows == 16 ? launch_as<DH, 16>(k_map, v_map, a, grid, device, s)
                : launch_attend8_wide(k_map, v_map, DH, a, grid, device, s);
  if (e != cudaSuccess) return e;
  if (grid > 1) {
    const dim3 ctas(grid - 1, a.block_rows / kMergeWarps8), threads(kMergeWarps8 * 32);
    e = a.block_rows <= 16 ? launch_pdl(attend8_merge_kernel<DH, 16>, ctas, threads, 0, s, a) : launch_pdl(attend8_merge_kernel<DH, 4>, ctas, threads, 0, s, a);
  }
  count_launch(kFamAttend8, 2);
  return e;
}

// Query rows of a block: as few as hold the tokens of the longest sequence.  From 17 on they are the wide side of the products (32 rows a
// head over 131072 rows of four layers of eight heads: 321 us, as the narrow side, with three codes of a weight, 357; over 8191 rows of one
// layer 29 and 38; 21 rows over 3000 of three sequences 32.5 and 34.5).  One choice for all sequences of a call: beside a chunk's tokens a
// single one takes a block of 128 rows, too.
int block_rows(int max_new, int n_rep) {
  const long long rows = (long long)max_new * n_rep;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : 128;
}

}  // namespace

// A piece leaves at most two results: its first and its last problem.
size_t cache8_workspace_bytes(const xkv_cache8_config* c, int max_new) {
  return (size_t)kPlanSms * (2 * block_rows(max_new, c->H_q / c->H_kv) * (c->d_h + 2) * sizeof(float) + sizeof(Piece8));
}

cudaError_t launch_cache8_attend(const xkv_cache8_config* c, int l0, int l1, const __nv_bfloat16* q, const int32_t* first, int n_tok,
                                 int max_new, const int32_t* table, const int32_t* length, const void* K8, const void* V8,
                                 const float* k_scale, const float* v_scale, void* workspace, __nv_bfloat16* out, float* lse,
                                 unsigned int* flags, int device, cudaStream_t s) {
  CUtensorMap k_map, v_map;
  const uint64_t rows = (uint64_t)c->G * c->n_pages * c->H_kv * c->page;
  if (!encode_byte_map(&k_map, K8, rows, c->d_h, c->page) || !encode_byte_map(&v_map, V8, rows, c->d_h, c->page)) return cudaErrorInvalidValue;
  int sms = 0;
  const cudaError_t e = device_sms(device, &sms);
  if (e != cudaSuccess) return e;
  Attend8Args a;
  a.batch = c->batch; a.H_kv = c->H_kv; a.H_q = c->H_q; a.n_rep = c->H_q / c->H_kv; a.n_pages = c->n_pages; a.max_pages = c->max_pages;
  a.page_shift = __builtin_ctz((unsigned)c->page);
  a.n_tok = n_tok; a.max_new = max_new; a.l0 = l0; a.layers = l1 - l0;
  a.block_rows = block_rows(max_new, a.n_rep);
  a.block_tok = a.block_rows / a.n_rep;
  a.rep_inv = (65536u + a.n_rep - 1u) / a.n_rep;
  a.scale2 = (c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / sqrtf((float)c->d_h)) * kLog2e;
  a.q = q; a.first = first; a.table = table; a.length = length; a.V8 = (const uint8_t*)V8;
  a.k_scale = k_scale; a.v_scale = v_scale; a.out = out; a.lse = lse; a.flags = flags;
  a.inject = cache_fault_injection();
  const int grid = sms < kPlanSms ? sms : kPlanSms;
  a.part = (float*)workspace;
  a.part_ml = reinterpret_cast<float2*>(a.part + (size_t)kPlanSms * 2 * a.block_rows * c->d_h);
  a.pieces = reinterpret_cast<Piece8*>(a.part_ml + (size_t)kPlanSms * 2 * a.block_rows);
  return c->d_h == 128 ? launch_width<128>(k_map, v_map, a, grid, device, s) : launch_width<64>(k_map, v_map, a, grid, device, s);
}

}  // namespace xkv
