// Moves and choices over an uncompressed cache: the commit of an accepted path (xkv_tree_commit), which rows stay
// (xkv_evict_select) and the move that closes the holes (xkv_evict_compact).
#include <cooperative_groups.h>
#include <math.h>

#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace cg = cooperative_groups;

namespace {

// Every array may come from the kernel before, which may still be writing it while these kernels start (they wait for it, but the
// read-only path is for memory that does not change while a kernel lives): no input is loaded as read-only, nor named as unaliased.
__device__ __forceinline__ void raise(unsigned int* flags, unsigned int bit) {
  if (flags) atomicOr(flags, bit);
}

// ---------------------------------------------------------------------------------------------
// Commit.  A path may read a row that it also writes, so every row is in registers before the first store: a CTA takes 64
// bytes of every row of one head's K or V, four lanes to a row.  Bound by latency: four sequences, up to 8 of 64 drafts, four layers of
// eight heads 2.9 us; eight sequences, up to 200 of 256 drafts (20.6 MB) 5.1 us.
constexpr int kCommitThreads = 256;
constexpr int kCommitRows = XKV_TREE_MAX_DRAFT / (kCommitThreads / 4);         // rows per thread

template <int DH>
__global__ void __launch_bounds__(kCommitThreads)
tree_commit_kernel(int batch, int H_kv, int cap, int l0, __nv_bfloat16* K, __nv_bfloat16* V, const int32_t* len,
                   const int32_t* path, const int32_t* path_len, int n_path, int32_t* pos,
                   const int32_t* first_pos, unsigned int* flags) {
  const int py = blockIdx.x, b = (py / H_kv) % batch;
  const size_t head = ((size_t)l0 * batch * H_kv + py) * (size_t)cap;
  const int tid = threadIdx.x;
  constexpr int SLICES = DH / 32;
  const int slice = blockIdx.y % SLICES;
  uint4* base = reinterpret_cast<uint4*>((blockIdx.y < SLICES ? K : V) + head * DH + slice * 32);
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int ln = len[b], want = path_len ? path_len[b] : n_path;
  const int n = min(max(want, 0), n_path);
  bool bad = n != want || ln < 0;
  uint4 x[kCommitRows];
  bool has[kCommitRows];
#pragma unroll
  for (int i = 0; i < kCommitRows; ++i) {
    const int j = i * (kCommitThreads / 4) + tid / 4;
    has[i] = false;
    if (j < n && ln >= 0) {
      const int p = path[(size_t)b * n_path + j];
      // (64 bits: an entry near 2^31 must not wrap)
      has[i] = p >= 0 && (long long)ln + p < cap && (long long)ln + j < cap;
      bad |= !has[i];
      if (has[i]) x[i] = base[(size_t)(ln + p) * (DH / 8) + (tid & 3)];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kCommitRows; ++i) {
    const int j = i * (kCommitThreads / 4) + tid / 4;
    if (has[i]) {
      base[(size_t)(ln + j) * (DH / 8) + (tid & 3)] = x[i];
      if (pos && blockIdx.y == 0 && (tid & 3) == 0) pos[head + ln + j] = first_pos[b] + j;
    }
  }
  if (bad && blockIdx.y == 0 && py % H_kv == 0) raise(flags, XKV_FLAG_INDEX_RANGE);
}

// ---------------------------------------------------------------------------------------------
// Compaction.  Sources are at or behind `keep`, destinations before it, so rows move independently.  A CTA looks at 256
// entries of a head's map, lists those that move, and copies their rows in 16-byte pieces, several in flight per thread.  Bound by
// HBM where many rows move: 65531 rows to 16384, four layers of eight heads (411 MB) 70 us, 5.9 TB/s; 4224 to 4096 2.4 us in a graph of such calls, 3.3 to 3.6 called one by one.
constexpr int kCompactThreads = 256;

template <int DH>
__global__ void __launch_bounds__(kCompactThreads)
evict_compact_kernel(int cap, size_t head0, __nv_bfloat16* K, __nv_bfloat16* V, const int32_t* src, int keep,
                     float* weights, int32_t* pos, unsigned int* flags) {
  __shared__ int to_s[kCompactThreads], from_s[kCompactThreads], count_s;
  const int tid = threadIdx.x;
  const size_t head = head0 + blockIdx.y, rows0 = head * (size_t)cap;
  if (tid == 0) count_s = 0;
  __syncthreads();
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int j = blockIdx.x * kCompactThreads + tid;
  if (j < keep) {
    const int s = src[head * (size_t)keep + j];
    if (s >= 0 && s != j) {
      if (s >= keep && s < cap) {
        const int at = atomicAdd(&count_s, 1);           // (the order of the list does not matter: rows are independent)
        to_s[at] = j;
        from_s[at] = s;
        if (weights) weights[rows0 + j] = weights[rows0 + s];
        if (pos) pos[rows0 + j] = pos[rows0 + s];
      } else {
        raise(flags, XKV_FLAG_INDEX_RANGE);
      }
    }
  }
  __syncthreads();
  constexpr int PPR = DH / 8, U = 4;                     // 16-byte pieces of a row; rounds in flight
  const int pieces = count_s * PPR;
  uint4* k = reinterpret_cast<uint4*>(K + rows0 * DH);
  uint4* v = reinterpret_cast<uint4*>(V + rows0 * DH);
  for (int i0 = tid; i0 < pieces; i0 += U * kCompactThreads) {
    uint4 a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kCompactThreads;
      if (i < pieces) {
        const size_t at = (size_t)from_s[i / PPR] * PPR + i % PPR;
        a[u] = k[at];
        b[u] = v[at];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kCompactThreads;
      if (i < pieces) {
        const size_t at = (size_t)to_s[i / PPR] * PPR + i % PPR;
        k[at] = a[u];
        v[at] = b[u];
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Selection.  A cluster of CTAs per head; every thread holds the weights of ITEMS rows, 1024 apart, in registers as 32-bit keys
// that order like the weights.  The recent rows are counted with the first digit: either they fill `keep` and are the only
// candidates, or they all stay and the others compete for the rest.  The key of the last row that stays is found digit by
// digit (11, 11, 10 bits) from histograms in shared memory, which a warp of every CTA adds up over the cluster: first 64 sums
// of 32 bins, then the bins of one of them, so that little crosses between SMs.  Rows with that very key stay in row order as
// far as there is room.  Ranks in row order -- of ties, of holes, of the rows that fill them -- are ballots and a prefix sum
// over (round, warp), so the map does not depend on timing.
// Bound by latency (11 barriers of the CTA or the cluster) and, where heads take several waves of CTAs, by instructions, about 130 a
// row and lane: 32 heads of 4224 rows 9.8 us, 128 heads of 32768 to 65536 rows 85 us (9.6 for their bytes).  With keys in shared
// memory, all 2048 bins read from every CTA and a thread's rows side by side it took 16.7 and 304.  (Not all keys stay in registers
// through the first digit's loads: 32 rounds spill 132 bytes a thread, 16 rounds 8.)
constexpr int kSelThreads = 1024;
constexpr int kSelBins = 2048;
constexpr int kSelMaxCluster = 8;
constexpr uint32_t kOut = 0u, kStays = 0xffffffffu;      // no weight maps to these (they would be NaNs)

__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(fmaxf(w + 0.0f, -INFINITY));              // -0 becomes 0, NaN the lowest weight
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

struct SelShared {
  uint32_t hist[4][kSelBins];                            // first digit of other rows, of recent rows; second; third
  uint32_t coarse[4][64];                                // sums of 32 bins
  uint32_t table[kSelThreads];                           // per (round, warp): counts, then their exclusive prefix
  uint32_t warp[32];
  uint32_t count;                                        // holes | movers << 16 of this CTA
  uint32_t digit, need, recent_only, ties_before, all_ties, holes_before, movers_upto[kSelMaxCluster];
};

// table[] becomes its exclusive prefix; returns the sum.
__device__ __forceinline__ uint32_t scan_table(SelShared& s) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __syncthreads();
  const uint32_t v = s.table[tid];
  uint32_t upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) s.warp[warp] = upto;
  __syncthreads();
  const uint32_t w = s.warp[lane];
  s.table[tid] = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u) + upto - v;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, w);
}

// By a whole warp: the bin from the top of histogram h, summed over the cluster, that holds the need-th entry (from 1), what is
// needed inside it, and its entries.
__device__ __forceinline__ void find_bin(cg::cluster_group& cl, SelShared& s, int h, int n_cta, uint32_t need, uint32_t* bin, uint32_t* rest,
                                         uint32_t* entries) {
  const int lane = threadIdx.x & 31;
  auto locate = [&](uint32_t v, uint32_t* before) {      // lane whose running sum reaches `need`
    uint32_t upto = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    const unsigned holds = __ballot_sync(0xffffffffu, upto >= need);
    const int at = holds ? __ffs(holds) - 1 : 31;
    *before = __shfl_sync(0xffffffffu, upto - v, at);
    return at;
  };
  uint32_t hi = 0, lo = 0, before;
#pragma unroll
  for (int c = 0; c < kSelMaxCluster; ++c) {             // (unrolled: the reads of other SMs' memory are all in flight at once)
    if (c < n_cta) {
      const uint2 v = *reinterpret_cast<const uint2*>(&cl.map_shared_rank(&s, c)->coarse[h][62 - 2 * lane]);
      hi += v.y;
      lo += v.x;
    }
  }
  const int at = locate(hi + lo, &before);
  need -= before;
  const uint32_t top = __shfl_sync(0xffffffffu, hi, at);
  int group = 63 - 2 * at;
  if (need > top) { need -= top; --group; }
  uint32_t v = 0;
#pragma unroll
  for (int c = 0; c < kSelMaxCluster; ++c)
    if (c < n_cta) v += cl.map_shared_rank(&s, c)->hist[h][group * 32 + 31 - lane];
  const int b = locate(v, &before);
  *bin = (uint32_t)(group * 32 + 31 - b);
  *rest = need - before;
  *entries = __shfl_sync(0xffffffffu, v, b);
}

template <int ITEMS>
__global__ void __launch_bounds__(kSelThreads, 1)
evict_select_kernel(int batch, int H_kv, int cap, int l0, const float* weights, const int32_t* pos,
                    const int32_t* since, const int32_t* len, int keep, int32_t* src,
                    unsigned int* flags) {
  extern __shared__ int list_s[];                        // rows at or behind `keep` that stay, ascending
  __shared__ __align__(16) SelShared s;
  cg::cluster_group cl = cg::this_cluster();
  const int n_cta = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int py = blockIdx.x / n_cta, b = (py / H_kv) % batch;
  const size_t head = (size_t)l0 * batch * H_kv + py, rows0 = head * (size_t)cap;
  auto cluster_sync = [&] {
    if (n_cta > 1) cl.sync(); else __syncthreads();
  };
  for (int i = tid; i < 4 * kSelBins; i += kSelThreads) s.hist[0][i] = 0u;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int want = len ? len[b] : cap, ln = min(max(want, 0), cap);
  if (want != ln && blockIdx.x % (n_cta * H_kv) == 0 && tid == 0) raise(flags, XKV_FLAG_INDEX_RANGE);
  int32_t* dst = src + head * (size_t)keep;
  if (ln <= keep) {
    for (int j = rank * kSelThreads + tid; j < keep; j += n_cta * kSelThreads) dst[j] = j < ln ? j : -1;
    return;                                              // (the whole cluster does: ln and keep are the same for all)
  }
  // rounds that this length needs (the head's rows are spread evenly over the cluster); this thread's rows: r0 + 1024 k, of
  // which the first `held` exist, and the first `front` are before `keep`
  const int items = (ln + n_cta * kSelThreads - 1) / (n_cta * kSelThreads);
  const int r0 = rank * (kSelThreads * items) + tid;
  auto rounds_below = [&](int end) { return min(max((end - r0 + kSelThreads - 1) / kSelThreads, 0), items); };
  const int held = r0 < ln ? rounds_below(ln) : 0, front = r0 < keep ? rounds_below(keep) : 0;
  // ---- keys, the recent rows, the first digit of both kinds
  uint32_t key[ITEMS], recent = 0;
  {
    const float* wp = weights + rows0 + r0;
    constexpr int U = ITEMS < 16 ? ITEMS : 16;           // rounds whose loads are in flight at once
#pragma unroll
    for (int k0 = 0; k0 < ITEMS; k0 += U) {
      float w[U];
#pragma unroll
      for (int k = 0; k < U; ++k) w[k] = k0 + k < held ? __ldcg(wp + (k0 + k) * kSelThreads) : 0.0f;
#pragma unroll
      for (int k = 0; k < U; ++k) key[k0 + k] = k0 + k < held ? weight_key(w[k]) : kOut;
    }
    if (since) {
      const int since_b = since[b];
      const int32_t* pp = pos ? pos + rows0 + r0 : nullptr;
#pragma unroll
      for (int k0 = 0; k0 < ITEMS; k0 += U) {
        int at[U];
#pragma unroll
        for (int k = 0; k < U; ++k) at[k] = pp && k0 + k < held ? __ldcg(pp + (k0 + k) * kSelThreads) : r0 + (k0 + k) * kSelThreads;
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (k0 + k < held && at[k] >= since_b) recent |= 1u << (k0 + k);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    if (k >= items) break;
    if (k < held) atomicAdd(&s.hist[0][((recent >> k) & 1u) * kSelBins + (key[k] >> 21)], 1u);
  }
  auto sum_bins = [&](int h) {                           // a warp sums two groups of 32 bins
    const uint32_t x = __reduce_add_sync(0xffffffffu, s.hist[h][warp * 64 + lane]);
    const uint32_t y = __reduce_add_sync(0xffffffffu, s.hist[h][warp * 64 + 32 + lane]);
    if (lane == 0) { s.coarse[h][2 * warp] = x; s.coarse[h][2 * warp + 1] = y; }
  };
  __syncthreads();
  sum_bins(0);
  sum_bins(1);
  cluster_sync();
  if (warp == 0) {
    uint32_t n = 0;
#pragma unroll
    for (int c = 0; c < kSelMaxCluster; ++c) {
      if (c < n_cta) {
        const uint32_t* g = cl.map_shared_rank(&s, c)->coarse[1];
        n += g[lane] + g[lane + 32];
      }
    }
    n = __reduce_add_sync(0xffffffffu, n);
    const bool only = n >= (uint32_t)keep;
    uint32_t bin, rest, entries;
    find_bin(cl, s, only ? 1 : 0, n_cta, only ? (uint32_t)keep : (uint32_t)keep - n, &bin, &rest, &entries);   // (at least one is needed)
    if (lane == 0) { s.digit = bin; s.need = rest; s.recent_only = only; }
  }
  __syncthreads();
  uint32_t prefix = s.digit << 21;
  if (since) {
    const bool only = s.recent_only != 0;
    const uint32_t set = only ? ~recent : recent, to = only ? kOut : kStays;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
      if ((set >> k) & 1u && k < held) key[k] = to;
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    if (k >= items) break;
    if (key[k] - prefix < 1u << 21) atomicAdd(&s.hist[2][(key[k] >> 10) & 2047u], 1u);         // (kOut and kStays have other digits)
  }
  __syncthreads();
  sum_bins(2);
  cluster_sync();
  if (warp == 0) {
    uint32_t bin, rest, entries;
    find_bin(cl, s, 2, n_cta, s.need, &bin, &rest, &entries);
    if (lane == 0) { s.digit = bin; s.need = rest; }
  }
  __syncthreads();
  prefix |= s.digit << 10;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    if (k >= items) break;
    if (key[k] - prefix < 1u << 10) atomicAdd(&s.hist[3][key[k] & 1023u], 1u);
  }
  __syncthreads();
  sum_bins(3);
  cluster_sync();
  if (warp == 0) {
    uint32_t bin, rest, entries;
    find_bin(cl, s, 3, n_cta, s.need, &bin, &rest, &entries);
    const uint32_t t = __reduce_add_sync(0xffffffffu, lane < rank ? cl.map_shared_rank(&s, lane)->hist[3][bin] : 0u);
    if (lane == 0) { s.digit = bin; s.need = rest; s.ties_before = t; s.all_ties = entries == rest; }
  }
  s.table[tid] = 0u;
  __syncthreads();
  prefix |= s.digit;
  // ---- who stays: all keys above the last one's, and its ties, in row order if there is not room for all of them
  const uint32_t below = (1u << lane) - 1u;
  uint32_t stays = 0;
  if (s.all_ties) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
      if (key[k] >= prefix) stays |= 1u << k;            // (kStays is above every key, kOut below)
  } else {
    const uint32_t need = s.need, ties_before = s.ties_before;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      if (k >= items) break;
      const unsigned t = __ballot_sync(0xffffffffu, key[k] == prefix);
      if (lane == 0) s.table[k * 32 + warp] = __popc(t);
    }
    scan_table(s);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      if (k >= items) break;
      const bool tie = key[k] == prefix;
      const unsigned t = __ballot_sync(0xffffffffu, tie);
      const uint32_t nth = ties_before + s.table[k * 32 + warp] + __popc(t & below);
      if (key[k] > prefix || (tie && nth < need)) stays |= 1u << k;
    }
    __syncthreads();
    if (tid >= items * 32) s.table[tid] = 0u;            // (the scan left its sum there)
  }
  // ---- holes and movers in row order: a row before `keep` that does not stay, a row behind that does.  (From here on bits of
  // rounds, not keys: the loops need not be unrolled.)
  const uint32_t fronts = front == 32 ? 0xffffffffu : (1u << front) - 1u;
  const uint32_t hole = fronts & ~stays, mover = stays & ~fronts;
#pragma unroll 4
  for (int k = 0; k < items; ++k) {
    const unsigned ho = __ballot_sync(0xffffffffu, (hole >> k) & 1u), mo = __ballot_sync(0xffffffffu, (mover >> k) & 1u);
    if (lane == 0) s.table[k * 32 + warp] = __popc(ho) | __popc(mo) << 16;     // (at most 32768 of each in a CTA)
  }
  const uint32_t sums = scan_table(s);
  if (tid == 0) s.count = sums;
  const int k_back = __reduce_min_sync(0xffffffffu, front), k_front = __reduce_max_sync(0xffffffffu, front);
#pragma unroll 4
  for (int k = k_back; k < items; ++k) {
    const bool mv = (mover >> k) & 1u;
    const unsigned mo = __ballot_sync(0xffffffffu, mv);
    if (mv) list_s[(s.table[k * 32 + warp] >> 16) + __popc(mo & below)] = r0 + k * kSelThreads;
  }
  cluster_sync();
  if (warp == 0) {
    const uint32_t c = lane < n_cta ? cl.map_shared_rank(&s, lane)->count : 0u;
    const uint32_t holes = __reduce_add_sync(0xffffffffu, lane < rank ? c & 0xffffu : 0u);
    uint32_t upto = c >> 16;
#pragma unroll
    for (int o = 1; o < kSelMaxCluster; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane < kSelMaxCluster) s.movers_upto[lane] = upto;
    if (lane == 0) s.holes_before = holes;
  }
  __syncthreads();
  const uint32_t holes_before = s.holes_before;
#pragma unroll 4
  for (int k = 0; k < k_front; ++k) {
    const int row = r0 + k * kSelThreads;
    const bool ho = (hole >> k) & 1u;
    const unsigned hs = __ballot_sync(0xffffffffu, ho);
    int from = row;
    if (ho) {                                            // the i-th hole takes the i-th mover, which some CTA has listed
      const uint32_t i = holes_before + (s.table[k * 32 + warp] & 0xffffu) + __popc(hs & below);
      uint32_t of = 0;
      int c = 0;
      for (int d = 0; d < n_cta - 1; ++d)
        if (i >= s.movers_upto[d]) { c = d + 1; of = s.movers_upto[d]; }
      from = cl.map_shared_rank(list_s, c)[i - of];
    }
    if (k < front) dst[row] = from;
  }
  cluster_sync();                                        // no CTA's lists go before they have been read
}

}  // namespace

cudaError_t launch_tree_commit(const xkv_cache_config* c, int l0, int l1, __nv_bfloat16* K, __nv_bfloat16* V, const int32_t* len,
                               const int32_t* path, const int32_t* path_len, int n_path, int32_t* pos, const int32_t* first_pos,
                               unsigned int* flags, cudaStream_t s) {
  const dim3 grid((l1 - l0) * c->batch * c->H_kv, 2 * c->d_h / 32), block(kCommitThreads);
  const cudaError_t e = c->d_h == 128
      ? launch_pdl(tree_commit_kernel<128>, grid, block, 0, s, c->batch, c->H_kv, c->cap, l0, K, V, len, path, path_len, n_path, pos, first_pos, flags)
      : launch_pdl(tree_commit_kernel<64>, grid, block, 0, s, c->batch, c->H_kv, c->cap, l0, K, V, len, path, path_len, n_path, pos, first_pos, flags);
  count_launch(kFamTree);
  return e;
}

cudaError_t launch_evict_compact(const xkv_cache_config* c, int l0, int l1, __nv_bfloat16* K, __nv_bfloat16* V, const int32_t* src,
                                 int keep, float* weights, int32_t* pos, unsigned int* flags, cudaStream_t s) {
  const dim3 grid((keep + kCompactThreads - 1) / kCompactThreads, (l1 - l0) * c->batch * c->H_kv), block(kCompactThreads);
  const size_t head0 = (size_t)l0 * c->batch * c->H_kv;
  const cudaError_t e = c->d_h == 128
      ? launch_pdl(evict_compact_kernel<128>, grid, block, 0, s, c->cap, head0, K, V, src, keep, weights, pos, flags)
      : launch_pdl(evict_compact_kernel<64>, grid, block, 0, s, c->cap, head0, K, V, src, keep, weights, pos, flags);
  count_launch(kFamEvict);
  return e;
}

template <int ITEMS>
static cudaError_t launch_select_as(const xkv_cache_config* c, int l0, int l1, int n_cta, size_t smem, const float* weights, const int32_t* pos,
                                    const int32_t* since, const int32_t* len, int keep, int32_t* src, unsigned int* flags, int device,
                                    cudaStream_t s) {
  cudaError_t e = ensure_dyn_smem<evict_select_kernel<ITEMS>>(smem, device);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((l1 - l0) * c->batch * c->H_kv * n_cta);
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = n_cta;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, evict_select_kernel<ITEMS>, (int)c->batch, (int)c->H_kv, (int)c->cap, l0, weights, pos, since, len, keep, src, flags);
  count_launch(kFamEvict);
  return e;
}

cudaError_t launch_evict_select(const xkv_cache_config* c, int l0, int l1, const float* weights, const int32_t* pos,
                                const int32_t* since, const int32_t* len, int keep, int32_t* src, unsigned int* flags, int device,
                                cudaStream_t s) {
  // CTAs per head.  A CTA holds 1024 rows a round in its registers, up to 32 rounds, and is alone on its SM.  Measured: 7 us and
  // 0.55 us a round for one CTA; 9.3 us and 0.8 us a round in a cluster, whose barriers cross SMs; and so many clusters of n at
  // once.  32 heads of 65500 rows: 35 us in pairs, 23 in fours, 48 in eights; 128 of them: 77, 96, 152; 128 of up to 65539 rows, which
  // two CTAs do not hold: 85 in threes, 104 in fours; 32 of 4200 rows: 9.0 us alone, 10.6 in pairs.  The rule goes by the cache's room,
  // since lengths are on the device: 128 heads half to quite full take 63 with room for 65536 rows each and 85 with room for 65537.
  constexpr int kAtOnce[kSelMaxCluster] = {148, 74, 43, 32, 26, 21, 14, 14};
  const int heads = (l1 - l0) * c->batch * c->H_kv;
  int n_cta = 0, rounds = 0;
  float least = 0.0f;
  for (int n = 1; n <= kSelMaxCluster; ++n) {
    const int r = (c->cap + n * kSelThreads - 1) / (n * kSelThreads), waves = (heads + kAtOnce[n - 1] - 1) / kAtOnce[n - 1];
    const float cost = (float)waves * (n == 1 ? 7.0f + 0.55f * (float)r : 9.3f + 0.8f * (float)r);
    if (r <= 32 && (n_cta == 0 || cost < least)) { n_cta = n; rounds = r; least = cost; }
  }
  const size_t smem = (size_t)rounds * kSelThreads * sizeof(int);
  if (rounds <= 8) return launch_select_as<8>(c, l0, l1, n_cta, smem, weights, pos, since, len, keep, src, flags, device, s);
  if (rounds <= 16) return launch_select_as<16>(c, l0, l1, n_cta, smem, weights, pos, since, len, keep, src, flags, device, s);
  return launch_select_as<32>(c, l0, l1, n_cta, smem, weights, pos, since, len, keep, src, flags, device, s);
}

}  // namespace xkv
