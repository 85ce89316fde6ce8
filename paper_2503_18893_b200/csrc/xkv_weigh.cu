// Accumulated attention weights of the rows of an uncompressed cache (xkv_cache_weigh):
//   w[j] = (j < seen ? decay w[j] : 0) + sum over queries c that saw row j of exp2(scale log2(e) k_j . q_c - lse_c log2(e)).
// The log-sum-exp is known, so a weight needs no maximum: the cache's keys are read once for up to 128 queries of a KV head.
//
// Rows of the cache are the rows of the tensor core's product and queries its columns, S[row][query] = K Q^T (tcgen05.mma,
// M = 128 rows, N up to 128 queries of one KV head, in tensor memory): a thread then owns a row, adds up its columns in
// registers and writes one weight, without a shuffle and in the same order in every call.  Only queries of tokens that saw a
// row at all become columns.  More than 128 are taken 128 at a time, each with another pass over the keys of a CTA's tiles, which
// comes from HBM again where those of all CTAs do not fit L2: 131072 rows, four layers of eight heads, 128 queries 198 us, 132 337
// (two reads of the keys are 330), 192 354, 256 390, 260 526.
//
//   producer  TMA: K tiles through a ring of shared-memory slots
//   issuer    tcgen05.mma into four accumulators in turn
//   4 warpgroups, one for each accumulator: the exponentials and their sums.  The special-function unit takes 8 cycles for a
//             warp's exponentials, one warp alone spends 10 and as long again on its loads and waits: four to a scheduler
//             keep it fed (two, with accumulators of 256 columns: 224 us at 131072 rows, 32 tokens, four layers of eight heads).
// As in the attention of drafted tokens, the tiles of all problems are one list in even pieces, one per CTA.  Exponentials are the
// hardware's (relative error 2^-22): a weight is off by 0.3e-7 to 6e-7 of itself against 64 bits, with exp() by 0.2e-7 to 2.3e-7.
//
// Measured on a B200, four layers of eight heads, the first 50 ms of calls: 131072 rows, one token 170 us, 16 tokens 174 (6.5 and
// 6.4 TB/s: HBM), 32 tokens 198-204 (5.5 TB/s; 537 M exponentials a call, for which the special-function units need 120 at the clock
// that the call runs at; 227-239 after a second of such calls, at the power limit); one layer of 8192 rows, one token 7.8 us, of
// which 3 are its bytes.
#include <cuda.h>
#include <math.h>

#include "xkv_cache.cuh"

namespace xkv {

namespace {

constexpr int kCols = 128;                     // queries per pass over the keys, columns of an accumulator
constexpr int kGroups = 4;                     // accumulators, and warpgroups that sum them up
constexpr int kMaxTokens = XKV_TREE_MAX_DRAFT;

struct WeighArgs {
  int batch, H_kv, H_q, n_rep, cap, n_tok, l0, layers;
  float scale2, decay;
  const __nv_bfloat16* q;
  const float* lse;
  const int32_t* len;
  const int32_t* visible;
  const int32_t* seen;
  float* weights;
  unsigned int* flags;
  unsigned int inject;                         // XKV_INJECT_CACHE_* bits; 0 in normal use
};

__device__ __forceinline__ int clamp_to(int v, int most, bool* bad) {
  const int x = min(max(v, 0), most);
  *bad |= x != v;
  return x;
}
__device__ __forceinline__ int weigh_length(const WeighArgs& a, int b, bool* bad) {
  return a.len ? clamp_to(a.len[b], a.cap, bad) : a.cap;
}

// A problem (layer l, sequence b, head g) and a tile of it.  Order: layer, sequence, head, tile.
struct Spot {
  int l, b, g, t, nt, len;
};
__device__ __forceinline__ void load_rows(const WeighArgs& a, Spot& p) {
  bool bad = false;
  p.len = weigh_length(a, p.b, &bad);
  p.nt = (p.len + kTile - 1) / kTile;
}
__device__ __forceinline__ void next_spot(const WeighArgs& a, Spot& p) {
  p.t = 0;
  if (++p.g < a.H_kv) return;
  p.g = 0;
  do {
    if (++p.b == a.batch) { p.b = 0; ++p.l; }
    load_rows(a, p);
  } while (p.nt == 0 && p.l < a.layers);
}

// Tokens of sequence b that saw a row, by a whole warp: their number, their list (may be nullptr).
__device__ __forceinline__ int seen_tokens(const WeighArgs& a, int b, int len, uint8_t* list) {
  const int lane = threadIdx.x & 31;
  int n = 0;
  for (int i0 = 0; i0 < a.n_tok; i0 += 32) {
    const int i = i0 + lane;
    bool bad = false;
    const int v = i < a.n_tok ? (a.visible ? clamp_to(a.visible[(size_t)b * a.n_tok + i], len, &bad) : len) : 0;
    const unsigned on = __ballot_sync(0xffffffffu, v > 0);
    if (v > 0 && list) list[n + __popc(on & ((1u << lane) - 1u))] = (uint8_t)i;
    n += __popc(on);
  }
  return n;
}

template <int DH>
struct WeighSmem {
  static constexpr int kSlab = kTile * 128;                    // 128 rows x 64 columns, 128-byte swizzle
  static constexpr int kSlot = kSlab * (DH / 64);
  static constexpr int kSlots = DH == 128 ? 5 : 8;
  static constexpr int kQ = kCols * DH * 2;
  static constexpr int kBytes = 1024 + kQ + kSlots * kSlot;
};
constexpr int kWeighThreads = kGroups * 128 + 64;

template <int DH>
__global__ void __launch_bounds__(kWeighThreads, 1)
cache_weigh_kernel(const __grid_constant__ CUtensorMap k_map, const WeighArgs a) {
  using namespace ptx;
  using L = WeighSmem<DH>;
  constexpr int NS = L::kSlots;
  constexpr uint32_t kSlab16 = L::kSlab >> 4;
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars_s[2 * NS + 2 * kGroups + 3];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s, range_s[2];
  __shared__ Spot spot_s;
  __shared__ __align__(16) float bias_s[kCols];               // -lse log2(e) of a column
  __shared__ int vis_s[kCols];                 // rows that a column's token saw; none where its log-sum-exp is -inf
  __shared__ uint8_t list_s[4 * kGroups][kMaxTokens];    // every warp's own copy of the tokens that saw a row
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* q_gen = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t ring = base + L::kQ;
  const uint32_t bars = smem_u32(bars_s);
  const uint32_t b_full = bars, b_empty = bars + 8 * NS, b_s = bars + 16 * NS, b_free = b_s + 8 * kGroups, b_done = b_free + 8 * kGroups, b_q = b_done + 8,
                 b_drain = b_q + 8;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kProducer = 4 * kGroups, kIssuer = kProducer + 1;

  if (tid == 0) {
    for (int i = 0; i < NS; ++i) { mbar_init(b_full + 8 * i, 1); mbar_init(b_empty + 8 * i, 1); }
    for (int i = 0; i < kGroups; ++i) { mbar_init(b_s + 8 * i, 1); mbar_init(b_free + 8 * i, 4); }     // (a warp arrives once)
    mbar_init(b_done, 4 * kGroups);
    mbar_init(b_q, 4 * kGroups);
    mbar_init(b_drain, 1);
    fence_mbar_init();
    abort_s = 0;
  }
  if (warp == kIssuer) {
    tmem_alloc(smem_u32(&tmem_s), 512);
    tmem_relinquish();
  }
  grid_dependency_wait();                      // everything below may come from the kernel before
  if (warp == kProducer) {
    // the list: tiles of a head over the batch, and the place of this CTA's first
    int head = 0;
    for (int b = lane; b < a.batch; b += 32) {
      Spot p;
      p.b = b;
      load_rows(a, p);
      head += p.nt;
    }
    head = __reduce_add_sync(0xffffffffu, head);
    const int per_layer = head * a.H_kv, total = per_layer * a.layers;
    int u0 = 0, u1 = 0;
    const int ctas = min((int)gridDim.x, total), c = blockIdx.x;
    if (c < ctas) { u0 = piece_begin(total, ctas, c); u1 = piece_begin(total, ctas, c + 1); }
    if (u1 > u0) {
      Spot p;
      p.l = u0 / per_layer;
      int rest = u0 - p.l * per_layer;
      for (int b0 = 0;; b0 += 32) {
        Spot s;
        s.b = min(b0 + lane, a.batch - 1);
        load_rows(a, s);
        const int mine = b0 + lane < a.batch ? s.nt * a.H_kv : 0;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        const unsigned holds = __ballot_sync(0xffffffffu, rest < upto);
        if (holds || b0 + 32 >= a.batch) {
          const int at = holds ? __ffs(holds) - 1 : 0;
          rest -= __shfl_sync(0xffffffffu, upto - mine, at);
          p.b = b0 + at;
          break;
        }
        rest -= __shfl_sync(0xffffffffu, upto, 31);
      }
      load_rows(a, p);
      p.g = rest / p.nt;
      p.t = rest - p.g * p.nt;
      if (lane == 0) spot_s = p;
    }
    if (lane == 0) { range_s[0] = u0; range_s[1] = u1; }
  } else if (warp == 0 && a.flags) {           // (every CTA looks at its share)
    bool bad = false;
    for (int i = blockIdx.x * 32 + lane; i < a.batch * a.n_tok; i += gridDim.x * 32) {
      const int b = i / a.n_tok, ln = weigh_length(a, b, &bad);
      if (a.visible) clamp_to(a.visible[i], ln, &bad);
      if (a.seen) clamp_to(a.seen[b], ln, &bad);
    }
    if (bad) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Only now that this CTA holds its tensor memory: a kernel started earlier could take some on this SM while the allocation above
  // still waits for another stream's, and then wait for this kernel, which waits for it.
  grid_dependency_launch();
  const uint32_t tmem = tmem_s;
  const Wait wt{&abort_s, a.flags, wait_limit(a.inject)};
  int left = range_s[1] - range_s[0];
  Spot p = spot_s;
  uint32_t n_loaded = 0;                       // producer: tiles asked for

  if (left > 0 && warp == kProducer) {
    bool ok = true;
    while (left > 0 && ok) {
      const int t1 = min(p.nt, p.t + left);
      const int row0 = (((a.l0 + p.l) * a.batch + p.b) * a.H_kv + p.g) * a.cap;
      const int cols = seen_tokens(a, p.b, p.len, nullptr) * a.n_rep;
      left -= t1 - p.t;
      if (lane == 0 && !(a.inject & XKV_INJECT_CACHE_NO_LOAD)) {
        for (int c0 = 0; c0 < max(cols, 1) && ok; c0 += kCols) {
          for (int t = p.t; t < t1; ++t) {
            const uint32_t slot = n_loaded % NS;
            if (!wait_bar(wt, b_empty + 8 * slot, ((n_loaded / NS) & 1u) ^ 1u)) { ok = false; break; }
            mbar_expect_tx(b_full + 8 * slot, L::kSlot);
#pragma unroll
            for (int x = 0; x < DH / 64; ++x)
              tma_load_2d(ring + slot * L::kSlot + x * L::kSlab, &k_map, x * 64, row0 + t * kTile, b_full + 8 * slot);
            ++n_loaded;
          }
        }
      }
      __syncwarp();
      ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
      if (left > 0) next_spot(a, p);
    }
  } else if (left > 0 && warp == kIssuer) {
    const uint64_t hi = smem_desc_sw128(0, 0) & 0xFFFFFFFF00000000ull;
    const uint32_t k_lo = (uint32_t)smem_desc_sw128(ring, 0), q_lo = (uint32_t)smem_desc_sw128(base, 0);
    uint32_t it = 0, chunk = 0;
    bool ok = true;
    while (left > 0 && ok) {
      const int t1 = min(p.nt, p.t + left), cnt = t1 - p.t;
      left -= cnt;
      const int cols = seen_tokens(a, p.b, p.len, nullptr) * a.n_rep;
      for (int c0 = 0; c0 < max(cols, 1) && ok; c0 += kCols, ++chunk) {
        const int n16 = max(16, (min(cols - c0, kCols) + 15) & ~15);
        const uint32_t idesc = idesc_bf16_f32(128, 0) | ((uint32_t)(n16 >> 3) << 17);
        if (!(ok = wait_warp(wt, b_q, chunk & 1u))) break;
        tc_fence_after();
        for (int t = 0; t < cnt; ++t, ++it) {
          const uint32_t slot = it % NS, buf = it % kGroups;
          if (!(ok = wait_warp(wt, b_full + 8 * slot, (it / NS) & 1u))) break;
          if (!(ok = wait_warp(wt, b_free + 8 * buf, ((it / kGroups) & 1u) ^ 1u))) break;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t ka = k_lo + slot * (uint32_t)(L::kSlot >> 4);
#pragma unroll
            for (int k = 0; k < DH / 16; ++k)
              tc_mma_bf16(tmem + buf * kCols, hi | (ka + (uint32_t)(k >> 2) * kSlab16 + (uint32_t)(k & 3) * 2u),
                          hi | (q_lo + (uint32_t)(k >> 2) * (uint32_t)(kCols * 128 >> 4) + (uint32_t)(k & 3) * 2u), idesc, k ? 1u : 0u);
            tc_commit(b_s + 8 * buf);
            tc_commit(b_empty + 8 * slot);
          }
        }
      }
      if (left > 0 && ok) next_spot(a, p);
    }
  } else if (left > 0) {
    const int wg = warp >> 2, row = tid & 127;
    const uint32_t acc = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)wg * kCols;
    uint8_t* list = list_s[warp];
    uint32_t it = 0, chunk = 0;
    bool ok = true;
    while (left > 0 && ok) {
      const int t0 = p.t, t1 = min(p.nt, p.t + left);
      left -= t1 - t0;
      __syncwarp();
      const int tokens = seen_tokens(a, p.b, p.len, list), cols = tokens * a.n_rep;
      __syncwarp();
      bool bad = false;
      const int old_rows = a.decay == 0.0f ? 0 : a.seen ? clamp_to(a.seen[p.b], p.len, &bad) : p.len;
      const size_t tok0 = ((size_t)(a.l0 + p.l) * a.batch + p.b) * a.n_tok;
      float* w_head = a.weights + (((size_t)(a.l0 + p.l) * a.batch + p.b) * a.H_kv + p.g) * (size_t)a.cap;
      for (int c0 = 0; c0 < max(cols, 1) && ok; c0 += kCols, ++chunk) {
        const int nc = min(cols - c0, kCols), n16 = max(16, (nc + 15) & ~15);
        // all warpgroups are done with the columns before (and with them the tensor core is with their queries)
        __syncwarp();
        if (lane == 0) mbar_arrive(b_done);
        if (!(ok = wait_warp(wt, b_done, chunk & 1u))) break;
        for (int i = tid; i < n16 * (DH / 8); i += kGroups * 128) {
          const int r = i / (DH / 8), c = i % (DH / 8);
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (r < nc) {
            const int at = (c0 + r) / a.n_rep, h = c0 + r - at * a.n_rep;
            v = *reinterpret_cast<const uint4*>(a.q + ((tok0 + list[at]) * a.H_q + (size_t)p.g * a.n_rep + h) * DH + c * 8);
          }
          *reinterpret_cast<uint4*>(q_gen + (c >> 3) * (kCols * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
        }
        if (tid < n16) {
          float bias = -INFINITY;
          int vis = 0;
          if (tid < nc) {
            const int at = (c0 + tid) / a.n_rep, h = c0 + tid - at * a.n_rep, tok = list[at];
            const float l = a.lse[(tok0 + tok) * a.H_q + (size_t)p.g * a.n_rep + h];
            // (a bias of -inf alone would not do: it makes a NaN of a logit that is not finite)
            if (l != -INFINITY) {
              bias = -l * kLog2e;
              vis = a.visible ? clamp_to(a.visible[(size_t)p.b * a.n_tok + tok], p.len, &bad) : p.len;
            }
          }
          bias_s[tid] = bias;
          vis_s[tid] = vis;
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_q);
        if (!(ok = wait_warp(wt, b_q, chunk & 1u))) break;
        int least = INT32_MAX;                                 // rows that every column saw
        for (int i = lane; i < nc; i += 32) least = min(least, vis_s[i]);
        least = __reduce_min_sync(0xffffffffu, least);
        for (int t = t0; t < t1; ++t, ++it) {
          if ((int)(it % kGroups) != wg) continue;
          const int j = t * kTile + row;
          float sum = 0.0f;
          const bool has_old = j < (c0 ? p.len : old_rows);
          const float old = has_old ? w_head[j] : 0.0f;        // (asked for before the wait)
          if (!(ok = wait_warp(wt, b_s + 8 * wg, (it / kGroups) & 1u))) break;
          tc_fence_after();
          const bool all_see = (t + 1) * kTile <= least;       // every column saw every row of the tile
          // 32 columns at a time
          const int full = all_see ? nc >> 5 : 0;
          if (full > 0) {
            const u64 scale_2 = pack2(a.scale2, a.scale2);
            u64 acc2[2] = {0ull, 0ull};
#pragma unroll 1
            for (int g = 0; g < full; ++g) {
              uint32_t z[32];
              tmem_ld32_nb(acc + 32u * g, z);
              tc_wait_ld32_nb(z);
              const ulonglong2* bias = reinterpret_cast<const ulonglong2*>(bias_s + 32 * g);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const ulonglong2 bb = bias[e];
                const float2 x = unpack2(fma2(pack2u(z[4 * e], z[4 * e + 1]), scale_2, bb.x));
                const float2 y = unpack2(fma2(pack2u(z[4 * e + 2], z[4 * e + 3]), scale_2, bb.y));
                acc2[0] = add2(acc2[0], pack2(ex2_approx(x.x), ex2_approx(x.y)));
                acc2[1] = add2(acc2[1], pack2(ex2_approx(y.x), ex2_approx(y.y)));
              }
            }
            const float2 s2 = unpack2(add2(acc2[0], acc2[1]));
            sum = s2.x + s2.y;
          }
          for (int g = 32 * full; g < nc; g += 8) {            // (columns behind the last have seen nothing)
            float z[8];
            tmem_ld<8>(acc + (uint32_t)g, z);
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x = ex2_approx(fmaf(z[e], a.scale2, bias_s[g + e]));
              sum += j < vis_s[g + e] ? x : 0.0f;
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0 && !(a.inject & XKV_INJECT_CACHE_NO_HANDOVER)) mbar_arrive(b_free + 8 * wg);
          if (j < p.len) w_head[j] = has_old ? fmaf(old, c0 ? 1.0f : a.decay, sum) : sum;
        }
      }
      if (left > 0 && ok) next_spot(a, p);
    }
  }

  // wind down: nothing of this CTA may still touch shared or tensor memory
  tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) {
    tc_fence_after();
    if (abort_s) {                             // given up: nothing may still write tensor memory when it is freed
      if (elect_one()) tc_commit(b_drain);
      for (uint32_t i = 0; i < (1u << 16); ++i) if (__all_sync(0xffffffffu, mbar_try_wait(b_drain, 0))) break;
    }
    tmem_dealloc(tmem, 512);
  }
  if (abort_s) {                               // given up: this CTA's rows say so, also to a caller without a flag word
    Spot x = spot_s;
    for (int n = range_s[1] - range_s[0]; n > 0; ) {
      const int t1 = min(x.nt, x.t + n);
      float* w = a.weights + (((size_t)(a.l0 + x.l) * a.batch + x.b) * a.H_kv + x.g) * (size_t)a.cap;
      for (int j = x.t * kTile + tid; j < min(t1 * kTile, x.len); j += kWeighThreads) w[j] = __int_as_float(0x7fffffff);
      n -= t1 - x.t;
      if (n > 0) next_spot(a, x);
    }
  }
  if (abort_s && warp == kProducer && lane == 0) {
    // given up: tiles may still be on their way into this CTA's shared memory; stay (with a limit) for them
    for (uint32_t n = n_loaded > NS ? n_loaded - NS : 0u; n < n_loaded; ++n)
      for (uint32_t i = 0; i < (1u << 16); ++i) if (mbar_try_wait(b_full + 8 * (n % NS), (n / NS) & 1u)) break;
  }
}

}  // namespace

cudaError_t launch_cache_weigh(const xkv_cache_config* c, int l0, int l1, const __nv_bfloat16* q, int n_tok, const float* lse,
                               const __nv_bfloat16* K, const int32_t* len, const int32_t* visible, const int32_t* seen, float decay,
                               float* weights, unsigned int* flags, int device, cudaStream_t s) {
  CUtensorMap k_map;
  if (!encode_bf16_map(&k_map, K, (uint64_t)c->G * c->batch * c->H_kv * c->cap, c->d_h, c->d_h, kTile)) return cudaErrorInvalidValue;
  int sms = 0;
  cudaError_t e = device_sms(device, &sms);
  if (e != cudaSuccess) return e;
  WeighArgs a;
  a.batch = c->batch; a.H_kv = c->H_kv; a.H_q = c->H_q; a.n_rep = c->H_q / c->H_kv; a.cap = c->cap; a.n_tok = n_tok;
  a.l0 = l0; a.layers = l1 - l0;
  a.scale2 = (c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / sqrtf((float)c->d_h)) * kLog2e;
  a.decay = decay; a.q = q; a.lse = lse; a.len = len; a.visible = visible; a.seen = seen; a.weights = weights; a.flags = flags;
  a.inject = cache_fault_injection();
  if (c->d_h == 128) {
    e = ensure_dyn_smem<cache_weigh_kernel<128>>(WeighSmem<128>::kBytes, device);
    if (e == cudaSuccess) e = launch_pdl(cache_weigh_kernel<128>, dim3(sms), dim3(kWeighThreads), WeighSmem<128>::kBytes, s, k_map, a);
  } else {
    e = ensure_dyn_smem<cache_weigh_kernel<64>>(WeighSmem<64>::kBytes, device);
    if (e == cudaSuccess) e = launch_pdl(cache_weigh_kernel<64>, dim3(sms), dim3(kWeighThreads), WeighSmem<64>::kBytes, s, k_map, a);
  }
  count_launch(kFamWeigh);
  return e;
}

}  // namespace xkv
