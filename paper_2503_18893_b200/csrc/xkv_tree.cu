// Attention of drafted tokens over an uncompressed cache (xkv_tree_attend).
//
// A sequence has `len` committed rows, which every drafted token attends to, and behind them its drafts' own rows, which
// token i attends to where bit j of its mask is set.  For one (layer, sequence, KV head) the queries of all tokens and of the
// head's n_rep query heads are the rows of one matrix Q, row token * n_rep + head, and
//   S = scale Q K^T,   p = exp2(S log2(e) - m),   O += p V,   l += sum p
// runs over 128-row tiles of the cache with a running maximum m.  The cache is read once for up to 256 rows of Q: with 256
// an element of two bytes meets 256 multiply-adds, 256 flops a byte, where B200's tensor cores (1651 TFLOP/s) and its HBM (6548 GB/s,
// 252 flops a byte) take about as long.
//
//   producer  TMA: K and V tiles through one ring of shared-memory slots, across the borders of problems
//   issuer    tcgen05.mma, a warp for each 128 rows of Q: S (both operands in shared memory) two steps ahead, and O += P V with
//             P in tensor memory, where it lies over S
//   softmax   a warpgroup for each 128 rows of Q: thread = row = TMEM lane, so a row's maximum and sum need no shuffle.
//             O stays in tensor memory; it is rescaled only when a row's maximum has grown by more than 2^8 (a weight is then
//             at most 2^8, which fp32 sums and bf16's relative precision do not notice; a published technique for such kernels).
// Weights are rounded to bf16 for the tensor core (by half a step, relative 2^-8 at most, as the output is); the denominator
// sums them unrounded in fp32.
//
// Up to 128 query rows a step is a tile of 128 cache rows; a CTA with 256 has the tensor memory for two steps of 64.  Measured on
// B200s, the first 50 ms of calls (in brackets: after a second of them, at the power limit): 131072 rows, 64 query rows a head, four
// layers of eight heads 320-344 us (375-410), 6.2-6.7 TB/s: HBM.  Eight sequences of up to 16411 rows, 231 query rows a head 227-234
// (268-275), 3.7 TB/s and 0.69 PFLOP/s of products (tensor cores 46 % busy, special-function units 37 %: bound by the hand-overs between
// the two, see the steps that did not help: one step of 128 rows 245, exponentials in turns 256, two warpgroups per 128 rows in turns
// 256, the next step's logits loaded part by part 240).  One layer of 8192 rows, 256 query rows a head 33.5, by time stamps of a CTA:
// start and place 2.2, queries 3.3, first logits 0.8, four tiles 9.7 (14 in the slowest CTA), last product and partial result 2.8, a
// second problem in four CTAs 2-5, to the merge 1.4, merge 5.2.  300 rows, one small window 10-10.6: place 1.0, queries 1.6, logits 0.6,
// weights 1.9, product 0.5, result 0.8, to the merge 1.1, merge 2.5: latencies of two kernels.
//
// The tiles of all problems form one list that is cut into as many even pieces as there are CTAs, whatever the lengths of the
// sequences: a CTA that holds a whole problem writes its output, the others leave (O, m, l) for tree_merge_kernel.  Lengths are
// read on the device only, so a captured call serves sequences as they grow.
//
// Rows that a token does not attend to have no influence on it whatever they hold: logits are selected, not added to, and a
// weight of zero meets only finite values, since value rows behind the last draft are zeroed in shared memory and elements of
// the drafts' value rows that are not finite are taken out there and given to the rows that do attend to them at the end.
#include <cuda.h>
#include <math.h>

#include "xkv_cache.cuh"

namespace xkv {

namespace {

constexpr int kQRows = 128;                    // query rows per warpgroup
constexpr float kGrow = 8.0f;                  // log2 of the growth of a maximum that makes O be rescaled
constexpr int kMergeWarps = 8;

struct TreeArgs {
  int batch, H_kv, H_q, n_rep, cap, n_draft, words, l0, layers;
  uint32_t rep_inv;                            // ceil(2^16 / n_rep)
  float scale2;                                // softmax scale times log2(e)
  const __nv_bfloat16* q;
  const uint32_t* mask;                        // nullptr: token i attends to drafts 0 .. i
  const int32_t* draft_len;
  const __nv_bfloat16* V;                      // (the rows of drafts that are not finite)
  const int32_t* len;
  float* part;                                 // [CTA][2][rows of a CTA][d_h]
  float2* part_ml;                             // [CTA][2][rows of a CTA] (m, l)
  __nv_bfloat16* out;
  float* lse;
  unsigned int* flags;
  unsigned int inject;                         // XKV_INJECT_CACHE_* bits; 0 in normal use
};

// m / n_rep for rows of Q: m < 4096, n_rep <= 16 and rep_inv = ceil(2^16 / n_rep), so the product's excess stays below one.
__device__ __forceinline__ int token_of(const TreeArgs& a, int m) { return (int)(((uint32_t)m * a.rep_inv) >> 16); }

// Rows and drafts of a sequence, brought into range; *bad reports what was not.
__device__ __forceinline__ void tree_lengths(const TreeArgs& a, int b, int* len, int* drafts, bool* bad) {
  const int want_dl = a.draft_len ? __ldcg(a.draft_len + b) : a.n_draft, dl = min(max(want_dl, 0), a.n_draft);
  const int want_ln = a.len ? __ldcg(a.len + b) : a.cap - a.n_draft, ln = min(max(want_ln, 0), a.cap - dl);
  *len = ln;
  *drafts = dl;
  *bad = want_dl != dl || want_ln != ln;
}

// A place in the list of tiles: problem (l, b, g, block of query rows), tile t of nt.  Order: layer, sequence, head, block, tile.
struct Place {
  int l, b, g, qp, t, nt, n_qp, len, drafts;
};

template <int QT>
__device__ __forceinline__ void load_sequence(const TreeArgs& a, Place& p) {
  bool bad;
  tree_lengths(a, p.b, &p.len, &p.drafts, &bad);
  p.nt = p.drafts > 0 ? (p.len + p.drafts + kTile - 1) / kTile : 0;
  p.n_qp = (p.drafts * a.n_rep + QT * kQRows - 1) / (QT * kQRows);
}

// Moves to the next problem that has tiles (there is one: the caller counts).
template <int QT>
__device__ __forceinline__ void next_problem(const TreeArgs& a, Place& p) {
  p.t = 0;
  if (++p.qp < p.n_qp) return;
  p.qp = 0;
  if (++p.g < a.H_kv) return;
  p.g = 0;
  do {
    if (++p.b == a.batch) { p.b = 0; ++p.l; }
    load_sequence<QT>(a, p);
  } while (p.nt == 0 && p.l < a.layers);
}

// Inclusive prefix sum over a warp.
__device__ __forceinline__ int warp_prefix(int v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v, o);
    if ((int)(threadIdx.x & 31) >= o) v += x;
  }
  return v;
}

// Lane: tiles of one head, all blocks of query rows, in sequence b0 + lane.
template <int QT>
__device__ __forceinline__ int lane_tiles(const TreeArgs& a, int b0, Place& s, bool report) {
  s.b = b0 + (int)(threadIdx.x & 31);
  if (s.b >= a.batch) return 0;
  load_sequence<QT>(a, s);
  if (report && a.flags) {
    int x, y;
    bool bad;
    tree_lengths(a, s.b, &x, &y, &bad);
    if (bad) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
  }
  return s.nt * s.n_qp;
}

// By a whole warp: tiles of one head over the batch, and over the sequences before b.
template <int QT>
__device__ __forceinline__ int head_tiles(const TreeArgs& a, int b, int* before) {
  int all = 0;
  *before = 0;
#pragma unroll 4
  for (int b0 = 0; b0 < a.batch; b0 += 32) {
    Place s;
    const int v = lane_tiles<QT>(a, b0, s, false);
    all += __reduce_add_sync(0xffffffffu, v);
    *before += __reduce_add_sync(0xffffffffu, s.b < b ? v : 0);
  }
  return all;
}

// By a whole warp: the tiles [range[0], range[1]) of CTA c, and the place of the first.
template <int QT>
__device__ __forceinline__ Place find_piece(const TreeArgs& a, int c, int grid, int* range, bool report) {
  const int lane = threadIdx.x & 31;
  Place s;                                     // of this lane's sequence
  const int mine = lane_tiles<QT>(a, 0, s, report);
  int upto = warp_prefix(mine), head = __shfl_sync(0xffffffffu, upto, 31);
#pragma unroll 4
  for (int b0 = 32; b0 < a.batch; b0 += 32) {
    Place x;
    head += __reduce_add_sync(0xffffffffu, lane_tiles<QT>(a, b0, x, report));
  }
  const int per_layer = head * a.H_kv, total = per_layer * a.layers, ctas = min(grid, total);
  int u0 = 0, u1 = 0;
  if (c < ctas) { u0 = piece_begin(total, ctas, c); u1 = piece_begin(total, ctas, c + 1); }
  if (lane == 0) { range[0] = u0; range[1] = u1; }
  Place p = s;
  if (u1 == u0) return p;
  p.l = u0 / per_layer;
  int rest = u0 - p.l * per_layer, own = mine;
  for (int b0 = 0;; ) {                        // (u0 is in the list: the search ends inside the batch)
    const unsigned holds = __ballot_sync(0xffffffffu, rest < upto * a.H_kv);
    if (holds || b0 + 32 >= a.batch) {
      const int at = holds ? __ffs(holds) - 1 : 0;
      rest -= __shfl_sync(0xffffffffu, upto - own, at) * a.H_kv;
      p.b = b0 + at;
      p.len = __shfl_sync(0xffffffffu, s.len, at);
      p.drafts = __shfl_sync(0xffffffffu, s.drafts, at);
      p.nt = __shfl_sync(0xffffffffu, s.nt, at);
      p.n_qp = __shfl_sync(0xffffffffu, s.n_qp, at);
      break;
    }
    rest -= __shfl_sync(0xffffffffu, upto, 31) * a.H_kv;
    b0 += 32;
    own = lane_tiles<QT>(a, b0, s, false);
    upto = warp_prefix(own);
  }
  const int per_head = p.nt * p.n_qp;
  p.g = rest / per_head;
  rest -= p.g * per_head;
  p.qp = rest / p.nt;
  p.t = rest - p.qp * p.nt;
  return p;
}

// What rows base .. base + 31 of the cache are to a token: bit = it attends to the row.
__device__ __forceinline__ uint32_t row_bits(const TreeArgs& a, const uint32_t* mask_row, int token, int base, int len, int drafts) {
  const int d0 = base - len;                   // draft index of bit 0
  if (d0 >= drafts) return 0u;
  if (d0 <= -32) return 0xffffffffu;
  uint32_t w;
  if (!mask_row) {                             // a chain: drafts up to the token itself
    const int n = token + 1 - d0;              // bits from 0 that are set
    w = n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
  } else if (d0 < 0) {
    w = (mask_row[0] << -d0) | ((1u << -d0) - 1u);
  } else {
    const int i = d0 >> 5, s = d0 & 31;
    w = mask_row[i] >> s;
    if (s && i + 1 < a.words) w |= mask_row[i + 1] << (32 - s);
  }
  const int n = drafts - d0;                   // bits behind the last draft are nobody's
  return n >= 32 ? w : w & ((1u << n) - 1u);
}

template <int DH, int QT>
struct TreeSmem {
  static constexpr int kSlab = kTile * 128;                    // 128 rows x 64 columns, 128-byte swizzle
  static constexpr int kSlot = kSlab * (DH / 64);
  static constexpr int kSlots = DH == 128 ? (QT == 2 ? 5 : 6) : 8;
  static constexpr int kBytes = 1024 + QT * kSlot + kSlots * kSlot;
};

// Warpgroups of query rows, the producer, an issuer for each warpgroup.
template <int QT>
constexpr int tree_threads() { return QT * 128 + 32 + QT * 32; }

// By a warp of a CTA that has given up: the results of its n tiles from place x on say so, also to a caller without a flag word.
template <int DH, int QT>
__device__ __forceinline__ void results_are_nan(const TreeArgs& a, Place x, int n) {
  const float nan = __int_as_float(0x7fffffff);
  for (uint32_t seg = 0; n > 0; ++seg) {
    const int t1 = min(x.nt, x.t + n);
    for (int row = threadIdx.x & 31; row < QT * kQRows; row += 32) {
      const int m = x.qp * (QT * kQRows) + row, token = token_of(a, m);
      if (m >= x.drafts * a.n_rep) break;
      if (x.t == 0 && t1 == x.nt) {
        const size_t qh = (((size_t)(a.l0 + x.l) * a.batch + x.b) * a.n_draft + token) * a.H_q + (size_t)x.g * a.n_rep + (m - token * a.n_rep);
        for (int c = 0; c < DH; c += 8) *reinterpret_cast<uint4*>(a.out + qh * DH + c) = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (a.lse) a.lse[qh] = nan;
      } else {                                 // (the merge makes it the whole problem's)
        a.part_ml[((size_t)blockIdx.x * 2 + (seg == 0 ? 0 : 1)) * (QT * kQRows) + row] = make_float2(nan, nan);
      }
    }
    n -= t1 - x.t;
    if (n > 0) next_problem<QT>(a, x);
  }
}

template <int DH, int QT>
__global__ void __launch_bounds__(tree_threads<QT>(), 1)
tree_attend_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const TreeArgs a) {
  using namespace ptx;
  using L = TreeSmem<DH, QT>;
  // A step is KW rows of a tile, and S has room for two steps (512 columns of tensor memory: S and O of QT * 128 rows).
  constexpr int KW = QT == 2 ? 64 : 128, SPT = kTile / KW;
  constexpr int NS = L::kSlots;
  constexpr uint32_t kSlab16 = L::kSlab >> 4;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars_s[2 * NS + 17];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  __shared__ Place place_s;
  __shared__ int range_s[2];
  // Drafts with elements that are not finite, by segment: a warpgroup is ahead of the other by a ring of tiles at most, so by
  // less than eight segments.
  __shared__ uint32_t bad_s[16][8];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t ring = base + QT * L::kSlot;
  const uint32_t bars = smem_u32(bars_s);
  const uint32_t b_full = bars, b_empty = bars + 8 * NS, b_s = bars + 16 * NS, b_p = b_s + 32, b_o = b_p + 32, b_q = b_o + 32,
                 b_drain = b_q + 16, b_first = b_drain + 16;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kProducer = QT * 4, kIssuer = QT * 4 + 1;

  if (tid == 0) {
    for (int i = 0; i < NS; ++i) { mbar_init(b_full + 8 * i, 1); mbar_init(b_empty + 8 * i, QT); }
    for (int i = 0; i < 4; ++i) { mbar_init(b_s + 8 * i, 1); mbar_init(b_p + 8 * i, 4); mbar_init(b_o + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) mbar_init(b_q + 8 * i, 4);      // (a warp arrives once: 128 arrivals take their time)
    mbar_init(b_first, QT * 4);
    mbar_init(b_drain, 1);
    mbar_init(b_drain + 8, 1);
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
    const Place p = find_piece<QT>(a, blockIdx.x, gridDim.x, range_s, blockIdx.x == 0);
    if (lane == 0) place_s = p;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  const Wait wt{&abort_s, a.flags, wait_limit(a.inject)};
  int left = range_s[1] - range_s[0];
  Place p = place_s;
  uint32_t n_loaded = 0;                       // producer: tiles (K and V each) asked for

  if (left > 0 && warp == kProducer) {
    if (lane == 0 && !(a.inject & XKV_INJECT_CACHE_NO_LOAD)) { // (the others of the warp wait at its end)
      bool ok = true;
      while (left > 0 && ok) {
        const int t1 = min(p.nt, p.t + left);
        const int row0 = (((a.l0 + p.l) * a.batch + p.b) * a.H_kv + p.g) * a.cap;
        left -= t1 - p.t;
        for (int t = p.t; t < t1 && ok; ++t) {
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            const uint32_t slot = n_loaded % NS;
            // the first queries come before the rest of the ring, which takes the memory a while
            if (n_loaded == 2 && !wait_bar(wt, b_first, 0u)) { ok = false; break; }
            if (!wait_bar(wt, b_empty + 8 * slot, ((n_loaded / NS) & 1u) ^ 1u)) { ok = false; break; }
            mbar_expect_tx(b_full + 8 * slot, L::kSlot);
#pragma unroll
            for (int x = 0; x < DH / 64; ++x)
              tma_load_2d(ring + slot * L::kSlot + x * L::kSlab, kv ? &v_map : &k_map, x * 64, row0 + t * kTile, b_full + 8 * slot);
            ++n_loaded;
          }
        }
        if (left > 0) next_problem<QT>(a, p);
      }
    }
    __syncwarp();
  } else if (left > 0 && warp >= kIssuer) {
    // ---- an issuing warp for each 128 rows of Q (a thread spends 70 to 130 cycles on an MMA and 235 on a commit).  Branches
    // outside the issue are taken on a vote and descriptors differ by constants, so that they stay in uniform registers.
    const int qt = warp - kIssuer;
    constexpr uint32_t idesc_s = idesc_bf16_f32(128, KW);
    constexpr uint32_t idesc_o = idesc_bf16_f32(128, DH) | (1u << 16);         // V is read along its rows (MN-major)
    const uint64_t q_desc = smem_desc_sw128(base + qt * L::kSlot, 0), k_desc = smem_desc_sw128(ring, 0);
    const uint64_t v_desc = (k_desc & ~(0xFFFFull << 16)) | ((uint64_t)kSlab16 << 16);
    const uint32_t s_tmem = tmem + (uint32_t)qt * 128u, o_tmem = tmem + 256u + (uint32_t)qt * 128u;
    uint32_t n = 0, st = 0, n_o = 0, seg = 0;  // ring position of the segment's first K tile; steps, commits on b_o, segments so far
    bool ok = true;
    auto logits = [&](uint32_t buf, uint32_t n_of, int half) {
      const uint64_t kd = k_desc + (uint64_t)((n_of % NS) * (uint32_t)(L::kSlot >> 4) + (uint32_t)half * (KW * 8));
#pragma unroll
      for (int k = 0; k < DH / 16; ++k) {
        const uint64_t off = (uint64_t)((k >> 2) * (int)kSlab16 + (k & 3) * 2);
        tc_mma_bf16(s_tmem + buf * KW, q_desc + off, kd + off, idesc_s, k ? 1u : 0u);
      }
      tc_commit(b_s + 16 * qt + 8 * buf);
      if (half == SPT - 1) tc_commit(b_empty + 8 * (n_of % NS));
    };
    auto wait_slot = [&](uint32_t n_of) { return wait_warp(wt, b_full + 8 * (n_of % NS), (n_of / NS) & 1u); };
    while (left > 0 && ok) {
      const int t1 = min(p.nt, p.t + left), steps = (t1 - p.t) * SPT;
      left -= t1 - p.t;
      ok = wait_warp(wt, b_q + 8 * qt, seg & 1u);
      for (int s = 0; s < min(2, steps) && ok; ++s) {          // two steps of logits ahead
        if (s % SPT == 0 && !(ok = wait_slot(n + 2 * (s / SPT)))) break;
        tc_fence_after();
        if (elect_one()) logits((st + s) & 1u, n + 2 * (s / SPT), s % SPT);
        __syncwarp();
      }
      for (int s = 0; s < steps && ok; ++s) {
        const uint32_t buf = (st + s) & 1u, nv = n + 2 * (s / SPT) + 1, nk = n + 2 * ((s + 2) / SPT);
        const bool more = s + 2 < steps;
        if (s % SPT == 0 && !(ok = wait_slot(nv))) break;
        if (more && s % SPT == 0 && !(ok = wait_slot(nk))) break;
        if (!(ok = wait_warp(wt, b_p + 16 * qt + 8 * buf, ((st + s) >> 1) & 1u))) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = v_desc + (uint64_t)((nv % NS) * (uint32_t)(L::kSlot >> 4) + (uint32_t)(s % SPT) * (KW * 8));
#pragma unroll
          for (int k = 0; k < KW / 16; ++k)
            tc_mma_bf16_ts(o_tmem, s_tmem + buf * KW + KW / 2 + (uint32_t)k * 8u, vd + (uint64_t)(k * (2048 >> 4)), idesc_o, (s | k) ? 1u : 0u);
          if (s % SPT == SPT - 1) tc_commit(b_empty + 8 * (nv % NS));
          // the logits after the next follow the product that reads P, which lies where they go; their commit tells of both
          if (more) logits(buf, nk, (s + 2) % SPT); else tc_commit(b_o + 16 * qt + 8 * (n_o & 1u));
        }
        __syncwarp();
        n_o += more ? 0u : 1u;
      }
      st += steps;
      n += 2 * (t1 - p.t);
      ++seg;
      if (left > 0 && ok) next_problem<QT>(a, p);
    }
  } else if (left > 0) {
    const int qt = warp >> 2, row = tid & 127;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    uint8_t* q_gen = gen + qt * L::kSlot;
    const uint32_t o_addr = tmem + lane_base + 256u + (uint32_t)qt * 128u;
    uint32_t it = 0, st = 0, n_o = 0, seg = 0; // tiles, steps, commits on b_o and segments so far
    bool ok = true;
    while (left > 0 && ok) {
      const int t0 = p.t, t1 = min(p.nt, p.t + left);
      left -= t1 - t0;
      const int rows_q = p.drafts * a.n_rep;                   // rows of Q of this sequence
      const int m0 = (p.qp * QT + qt) * kQRows;                // this warpgroup's first
      // ---- Q as the A operand: 64-column slabs, 128-byte rows, 16-byte units swizzled by the row; rows behind the last are 0
      // (a warp brings its own 32 rows, and their place is its own in the epilogue too)
      {
        constexpr int C = DH / 8, STEP = 32 / C, U = 8;        // 16-byte units of a row; rows per round; rounds in flight
        const int c = lane % C, r0 = (warp & 3) * 32 + lane / C;
        const __nv_bfloat16* q0 = a.q + (((size_t)(a.l0 + p.l) * a.batch + p.b) * a.n_draft * a.H_q + (size_t)p.g * a.n_rep) * DH + c * 8;
#pragma unroll
        for (int i0 = 0; i0 < C; i0 += U) {
          uint4 v[U];
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int mm = m0 + r0 + (i0 + i) * STEP, token = token_of(a, mm);
            v[i] = make_uint4(0u, 0u, 0u, 0u);
            if (mm < rows_q) v[i] = *reinterpret_cast<const uint4*>(q0 + ((size_t)token * a.H_q + (mm - token * a.n_rep)) * DH);
          }
#pragma unroll
          for (int i = 0; i < U; ++i) {
            const int r = r0 + (i0 + i) * STEP;
            *reinterpret_cast<uint4*>(q_gen + (c >> 3) * L::kSlab + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[i];
          }
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(b_q + 8 * qt);
        if (seg == 0) mbar_arrive(b_first);
      }
      const int m = m0 + row;
      const bool live = m < rows_q;
      const bool warp_live = m0 + (row & ~31) < rows_q;
      const int token = live ? token_of(a, m) : 0;
      const uint32_t* mask_row = a.mask ? a.mask + ((size_t)p.b * a.n_draft + token) * a.words : nullptr;
      float m_used = -INFINITY;
      u64 l2[2] = {0ull, 0ull};                // four partial sums of the weights
      bool odd = false;                        // tiles of this segment held drafts
      const int steps = (t1 - t0) * SPT;
      for (int s = 0; s < steps; ++s, ++st) {
        const int t = t0 + s / SPT, half = s % SPT;
        const uint32_t buf = st & 1u, nk = 2u * (it + (uint32_t)(s / SPT));    // ring position of the tile's keys
        if (!(ok = wait_warp(wt, b_s + 16 * qt + 8 * buf, (st >> 1) & 1u))) break;
        tc_fence_after();
        if (qt == 0 && s == 0 && row < 8) bad_s[(seg + 8) & 15u][row] = 0u;
        const uint32_t s_addr = tmem + lane_base + (uint32_t)qt * 128u + buf * KW;
        const int j0 = t * kTile + half * KW;  // first row of the step
        if (warp_live) {
          constexpr int NC = KW / 32;
          const bool masked = j0 + KW > p.len;
          uint32_t z[NC][32];
#pragma unroll
          for (int i = 0; i < NC; ++i) tmem_ld32_nb(s_addr + 32u * i, z[i]);
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < NC; ++i) {
            tc_wait_ld32_nb(z[i]);
            if (masked) {
              const uint32_t w = row_bits(a, mask_row, token, j0 + 32 * i, p.len, p.drafts);
#pragma unroll
              for (int e = 0; e < 32; ++e) z[i][e] = (w >> e) & 1u ? z[i][e] : 0xff800000u;
            }
#pragma unroll
            for (int e = 0; e < 32; e += 2)
              mx[(e >> 1) & 3] = fmaxf(fmaxf(mx[(e >> 1) & 3], __uint_as_float(z[i][e])), __uint_as_float(z[i][e + 1]));
          }
          const float m_new = fmaxf(m_used, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale2);
          if (s == 0) {
            m_used = m_new;
          } else {
            const bool grow = m_new > m_used + kGrow || (m_used == -INFINITY && m_new > -INFINITY);
            if (__any_sync(0xffffffffu, grow)) {
              // O holds the steps before this one once the last product is done, which the next logits' commit tells, or its own
              const bool next = s + 1 < steps;
              if (!(ok = wait_warp(wt, (next ? b_s + 8 * (buf ^ 1u) : b_o + 8 * (n_o & 1u)) + 16 * qt, ((next ? st + 1 : n_o) >> 1) & 1u))) break;
              tc_fence_after();
              const float f = grow ? (m_used == -INFINITY ? 0.0f : ex2_approx(m_used - m_new)) : 1.0f;
              if (grow) m_used = m_new;
              const u64 f2 = pack2(f, f);
              l2[0] = mul2(l2[0], f2);
              l2[1] = mul2(l2[1], f2);
#pragma unroll 1
              for (int c = 0; c < DH; c += 16) {
                float o[16];
                uint32_t r[16];
                tmem_ld<16>(o_addr + (uint32_t)c, o);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(o[e] * f);
                tmem_st16(o_addr + (uint32_t)c, r);
              }
            }
          }
          const float shift = m_used == -INFINITY ? 0.0f : m_used;
          const u64 scale_2 = pack2(a.scale2, a.scale2), shift_2 = pack2(-shift, -shift);
#pragma unroll
          for (int i = 0; i < NC; ++i) {       // P, two to a column, in the upper half of S's columns
            uint32_t r[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float2 w = unpack2(fma2(pack2u(z[i][2 * e], z[i][2 * e + 1]), scale_2, shift_2));
              w.x = ex2_approx(w.x);
              w.y = ex2_approx(w.y);
              l2[e & 1] = add2(l2[e & 1], pack2(w.x, w.y));
              r[e] = pack_bf16(w.x, w.y);
            }
            tmem_st16(s_addr + KW / 2 + 16u * i, r);
          }
          tc_wait_st();
        }
        if (half == 0 && (t + 1) * kTile > p.len) {
          odd = true;
          // thread = value row: what no token holds is zeroed, what is not finite in a draft's row is taken out.  Both warpgroups do
          // it, to the same effect; one that finds a row cleared finds it listed, too.
          const uint32_t nv = nk + 1u, slot = nv % NS;
          if (!(ok = wait_warp(wt, b_full + 8 * slot, (nv / NS) & 1u))) break;
          const int draft = t * kTile + row - p.len;
          if (draft >= 0) {
            uint8_t* v = gen + QT * L::kSlot + slot * L::kSlot + row * 128;
#pragma unroll 1
            for (int c = 0; c < DH / 8; ++c) {
              uint4* at = reinterpret_cast<uint4*>(v + (c >> 3) * L::kSlab + (((c & 7) ^ (row & 7)) << 4));
              uint4 x = draft < p.drafts ? *at : make_uint4(0u, 0u, 0u, 0u);
              uint32_t* w = reinterpret_cast<uint32_t*>(&x);
              bool hit = draft >= p.drafts;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; hit = true; }
                if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; hit = true; }
              }
              if (hit) {
                if (draft < p.drafts) {
                  atomicOr(&bad_s[seg & 15u][draft >> 5], 1u << (draft & 31));
                  __threadfence_block();
                }
                *at = x;
              }
            }
          }
          fence_proxy_async();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && !(a.inject & XKV_INJECT_CACHE_NO_HANDOVER)) mbar_arrive(b_p + 16 * qt + 8 * buf);
      }
      if (!ok) break;
      // ---- the segment's result
      // (the last two products commit to two barriers in turn: by now both may be done)
      n_o += (uint32_t)min(2, steps);
      if (!(ok = wait_warp(wt, b_o + 16 * qt + 8 * ((n_o - 1u) & 1u), ((n_o - 1u) >> 1) & 1u))) break;
      it += (uint32_t)(t1 - t0);
      tc_fence_after();
      const bool whole = t0 == 0 && t1 == p.nt;
      const float2 la = unpack2(add2(l2[0], l2[1]));
      const float l = la.x + la.y;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const size_t qh = (((size_t)(a.l0 + p.l) * a.batch + p.b) * a.n_draft + token) * a.H_q + (size_t)p.g * a.n_rep + (m - token * a.n_rep);
      const size_t pr = ((size_t)blockIdx.x * 2 + (seg == 0 ? 0 : 1)) * (QT * kQRows) + qt * kQRows + row;
      if (warp_live) {
#pragma unroll 1
        for (int c = 0; c < DH; c += 32) {
          float o[32];
          tmem_ld32(o_addr + (uint32_t)c, o);
          tc_wait_ld();
          if (odd) {
#pragma unroll 1
            for (int w = 0; w < a.words; ++w) {
              uint32_t bad = bad_s[seg & 15u][w];              // (entered before the product that this result waited for)
              while (bad) {
                const int j = 32 * w + __ffs(bad) - 1;
                bad &= bad - 1u;
                if (!(row_bits(a, mask_row, token, p.len + 32 * w, p.len, p.drafts) >> (j & 31) & 1u)) continue;
                const __nv_bfloat16* v = a.V + ((((size_t)(a.l0 + p.l) * a.batch + p.b) * a.H_kv + p.g) * (size_t)a.cap + p.len + j) * DH + c;
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  const float x = __bfloat162float(v[e]);
                  if (!isfinite(x)) o[e] += x;
                }
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
            // through the place of this warp's rows of Q, so that a store writes whole lines
            float4* own = reinterpret_cast<float4*>(q_gen + (warp & 3) * 4096);
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) own[lane * 8 + (e ^ (lane & 7))] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
            __syncwarp();
            float* dst = a.part + (pr - row + (warp & 3) * 32) * DH + c + (lane & 7) * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int r = 4 * i + (lane >> 3);
              *reinterpret_cast<float4*>(dst + (size_t)r * DH) = own[r * 8 + ((lane & 7) ^ (r & 7))];
            }
          }
        }
        __syncwarp();                          // the next problem's queries go where other lanes may still be reading
        if (live && whole && a.lse) a.lse[qh] = l == 0.0f ? -INFINITY : (m_used + log2f(l)) * 0.6931471805599453f;
        if (live && !whole) a.part_ml[pr] = make_float2(m_used, l);
      }
      tc_fence_before();
      ++seg;
      if (left > 0) next_problem<QT>(a, p);
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
    // given up: tiles may still be on their way into this CTA's shared memory; stay (with a limit) for them
    if (lane == 0) {
      for (uint32_t n = n_loaded > NS ? n_loaded - NS : 0u; n < n_loaded; ++n)
        for (uint32_t i = 0; i < (1u << 16); ++i) if (mbar_try_wait(b_full + 8 * (n % NS), (n / NS) & 1u)) break;
    }
    results_are_nan<DH, QT>(a, place_s, range_s[1] - range_s[0]);
  }
}

// Joins the pieces of a problem: O = sum_c 2^(m_c - M) O_c, l likewise.  A warp has ROWS query rows, lane = d_h / 32 columns.
// Sixteen pieces of one row, or two of four, are in flight (twenty of one: 1 us less for 18 pieces, 0.5 more for three).
template <int DH, int QT, int ROWS>
__global__ void __launch_bounds__(kMergeWarps * 32)
tree_merge_kernel(const TreeArgs a, int attend_grid) {
  constexpr int V = DH / 32, AT_ONCE = ROWS == 1 ? 16 : 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int py = blockIdx.x, l = py / (a.batch * a.H_kv), b = (py / a.H_kv) % a.batch, g = py % a.H_kv;
  // The lengths come from before the kernel that this one waits for, which had waited for them before it let this one start: they
  // are read (past L1) while that kernel runs.
  const int m0 = (blockIdx.y * kMergeWarps + warp) * ROWS;     // first row of Q (32 rows of a CTA lie in one block of rows)
  Place p;
  p.b = b;
  load_sequence<QT>(a, p);
  int before;
  const int head = head_tiles<QT>(a, b, &before);
  const int total = head * a.H_kv * a.layers, ctas = min(attend_grid, total);
  const int qp = m0 / (QT * kQRows), live = p.drafts * a.n_rep - m0;
  const int u0 = (l * head + before) * a.H_kv + (g * p.n_qp + qp) * p.nt, u1 = u0 + p.nt;
  const int c0 = live > 0 ? piece_of(total, ctas, u0) : 0, c1 = live > 0 ? piece_of(total, ctas, u1 - 1) : 0;  // (else there may be no tiles)
  ptx::grid_dependency_wait();                 // the pieces come from the kernel before; every CTA waits, so that who waits for this
  ptx::grid_dependency_launch();               // kernel has waited for that one
  if (c0 == c1) return;                        // one piece: written where it was computed
  // a problem that begins inside a piece is that piece's last one, and in the others the first
  const size_t r0 = (size_t)(m0 - qp * QT * kQRows), first = (size_t)c0 * 2 + (piece_begin(total, ctas, c0) == u0 ? 0 : 1);
  auto slot = [&](int c) { return (c == c0 ? first : (size_t)c * 2) * (QT * kQRows) + r0; };
  float M[ROWS], sum[ROWS], acc[ROWS][V];
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    M[k] = -INFINITY;
    sum[k] = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[k][i] = 0.0f;
  }
  for (int cb = c0; cb <= c1; cb += 32) {      // lane: the weight of one piece of 32, for every row
    const int n = min(32, c1 - cb + 1);
    float2 ml[ROWS];
    float f[ROWS], x[AT_ONCE][ROWS][V];
    auto load = [&](int j0) {
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
          const float* src = a.part + (slot(cb + min(j0 + j, n - 1)) + min(k, live - 1)) * DH + lane * V;
          if constexpr (V == 4) *reinterpret_cast<float4*>(x[j][k]) = *reinterpret_cast<const float4*>(src);
          else *reinterpret_cast<float2*>(x[j][k]) = *reinterpret_cast<const float2*>(src);
        }
      }
    };
#pragma unroll
    for (int k = 0; k < ROWS; ++k) ml[k] = lane < n && k < live ? a.part_ml[slot(cb + lane) + k] : make_float2(-INFINITY, 0.0f);
    load(0);                                   // (asked for before the weights are known)
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      float top = ml[k].x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float M_new = fmaxf(M[k], top), old = M[k] == -INFINITY ? 1.0f : exp2f(M[k] - M_new);
      f[k] = ml[k].x == -INFINITY ? (ml[k].y == 0.0f ? 0.0f : 1.0f) : exp2f(ml[k].x - M_new);         // (a piece of NaNs stays one)
      M[k] = M_new;
      float part = f[k] * ml[k].y;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
      sum[k] = fmaf(sum[k], old, part);
#pragma unroll
      for (int i = 0; i < V; ++i) acc[k][i] *= old;
    }
    for (int j0 = 0; j0 < n; j0 += AT_ONCE) {
      if (j0 > 0) load(j0);
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
          const float w = __shfl_sync(0xffffffffu, f[k], (j0 + j) & 31);
          if (j0 + j < n) {
#pragma unroll
            for (int i = 0; i < V; ++i) acc[k][i] = fmaf(w, x[j][k][i], acc[k][i]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    if (k >= live) break;
    const float inv = sum[k] == 0.0f ? 0.0f : 1.0f / sum[k];
    const int m = m0 + k, token = token_of(a, m);
    const size_t qh = (((size_t)(a.l0 + l) * a.batch + b) * a.n_draft + token) * a.H_q + (size_t)g * a.n_rep + (m - token * a.n_rep);
    uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + qh * DH + lane * V);
#pragma unroll
    for (int i = 0; i < V; i += 2) dst[i / 2] = ptx::pack_bf16(acc[k][i] * inv, acc[k][i + 1] * inv);
    if (a.lse && lane == 0) a.lse[qh] = sum[k] == 0.0f ? -INFINITY : (M[k] + log2f(sum[k])) * 0.6931471805599453f;
  }
}

template <int DH, int QT>
cudaError_t launch_tree_as(const CUtensorMap& k_map, const CUtensorMap& v_map, const TreeArgs& a, int grid, int device, cudaStream_t s) {
  cudaError_t e = ensure_dyn_smem<tree_attend_kernel<DH, QT>>(TreeSmem<DH, QT>::kBytes, device);
  if (e == cudaSuccess) e = launch_pdl(tree_attend_kernel<DH, QT>, dim3(grid), dim3(tree_threads<QT>()), TreeSmem<DH, QT>::kBytes, s, k_map, v_map, a);
  if (e != cudaSuccess) return e;
  // Few rows are a matter of latency: a warp each.  Many are one of the CTAs that they take: four a warp.  Whole calls, one and four rows
  // a warp: 2048 rows 33.3 and 38.3 us (64 drafts over one layer of 8192), 18.3 and 19.6; 2560 36.6 and 37.8, 25.7 and 25.6; 3584 42.5
  // and 42.3, 29.0 and 27.5; 4096 46.4 and 45.9; 8192 69.7 and 62.2, 44.3 and 37.1; 24576 113 and 88.6.
  const int rows = a.n_draft * a.n_rep, problems = a.layers * a.batch * a.H_kv;
  auto merge = [&](auto kernel, int per_warp) {
    const int per_cta = kMergeWarps * per_warp;
    return launch_pdl(kernel, dim3(problems, (rows + per_cta - 1) / per_cta), dim3(kMergeWarps * 32), 0, s, a, grid);
  };
  e = (long long)rows * problems <= 3500 ? merge(tree_merge_kernel<DH, QT, 1>, 1) : merge(tree_merge_kernel<DH, QT, 4>, 4);
  count_launch(kFamTree, 2);
  return e;
}

}  // namespace

// Floats of workspace: a piece leaves at most two results (its first and its last problem) of a CTA's query rows.
size_t tree_part_floats(const xkv_cache_config* c, int n_draft) {
  const int rows = n_draft * (c->H_q / c->H_kv) > kQRows ? 2 * kQRows : kQRows;
  return (size_t)kPlanSms * 2 * rows * (c->d_h + 2);
}

cudaError_t launch_tree_attend(const xkv_cache_config* c, int l0, int l1, const __nv_bfloat16* q, int n_draft, const uint32_t* mask,
                               const int32_t* draft_len, const __nv_bfloat16* K, const __nv_bfloat16* V, const int32_t* len,
                               float* workspace, __nv_bfloat16* out, float* lse, unsigned int* flags, int device, cudaStream_t s) {
  CUtensorMap k_map, v_map;
  const uint64_t rows = (uint64_t)c->G * c->batch * c->H_kv * c->cap;
  if (!encode_bf16_map(&k_map, K, rows, c->d_h, c->d_h, kTile) || !encode_bf16_map(&v_map, V, rows, c->d_h, c->d_h, kTile))
    return cudaErrorInvalidValue;
  int sms = 0;
  const cudaError_t e = device_sms(device, &sms);
  if (e != cudaSuccess) return e;
  TreeArgs a;
  a.batch = c->batch; a.H_kv = c->H_kv; a.H_q = c->H_q; a.n_rep = c->H_q / c->H_kv; a.cap = c->cap; a.n_draft = n_draft;
  a.words = (n_draft + 31) / 32; a.l0 = l0; a.layers = l1 - l0;
  a.rep_inv = (65536u + a.n_rep - 1u) / a.n_rep;
  a.scale2 = (c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / sqrtf((float)c->d_h)) * kLog2e;
  a.q = q; a.mask = mask; a.draft_len = draft_len; a.V = V; a.len = len; a.out = out; a.lse = lse; a.flags = flags;
  a.inject = cache_fault_injection();
  const int rows_q = n_draft * a.n_rep, qt = rows_q > kQRows ? 2 : 1;
  const int grid = sms < kPlanSms ? sms : kPlanSms;
  a.part = workspace;
  a.part_ml = reinterpret_cast<float2*>(workspace + (size_t)kPlanSms * 2 * qt * kQRows * c->d_h);
  if (c->d_h == 128) return qt == 2 ? launch_tree_as<128, 2>(k_map, v_map, a, grid, device, s) : launch_tree_as<128, 1>(k_map, v_map, a, grid, device, s);
  return qt == 2 ? launch_tree_as<64, 2>(k_map, v_map, a, grid, device, s) : launch_tree_as<64, 1>(k_map, v_map, a, grid, device, s);
}

}  // namespace xkv
