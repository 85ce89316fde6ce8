// Moves and choices over an uncompressed cache: the commit of an accepted path (xkv_tree_commit), which rows stay
// (xkv_evict_select) and the move that closes the holes (xkv_evict_compact).
#include <cooperative_groups.h>
#include <math.h>

#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace cg = cooperative_groups;

namespace {

__device__ __forceinline__ void raise(unsigned int* flags, unsigned int bit) {
  if (flags) atomicOr(flags, bit);
}

// ---------------------------------------------------------------------------------------------
// Commit.  A path may read a row that it also writes, so every row is in registers before the first store: a CTA takes 64
// bytes of every row of one head's K or V, four lanes to a row.
constexpr int kCommitThreads = 256;
constexpr int kCommitRows = XKV_TREE_MAX_DRAFT / (kCommitThreads / 4);         // rows per thread

template <int DH>
__global__ void __launch_bounds__(kCommitThreads)
tree_commit_kernel(int batch, int H_kv, int cap, int l0, __nv_bfloat16* K, __nv_bfloat16* V, const int32_t* __restrict__ len,
                   const int32_t* __restrict__ path, const int32_t* __restrict__ path_len, int n_path, int32_t* pos,
                   const int32_t* __restrict__ first_pos, unsigned int* flags) {
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
// entries of a head's map, lists those that move, and copies their rows in 16-byte pieces, several in flight per thread.
constexpr int kCompactThreads = 256;

template <int DH>
__global__ void __launch_bounds__(kCompactThreads)
evict_compact_kernel(int cap, size_t head0, __nv_bfloat16* K, __nv_bfloat16* V, const int32_t* __restrict__ src, int keep,
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
// Selection.  A cluster of CTAs per head, each with an even slice of the rows in shared memory as 32-bit keys that order
// like the weights.  The recent rows are counted first: either they fill `keep` and are the only candidates, or they all stay
// and the others compete for the rest.  The key of the last row that stays is found digit by digit (11, 11, 10 bits) from
// histograms summed over the cluster; rows with that very key stay in row order as far as there is room.  Ranks of holes and of
// the rows that fill them are prefix sums in row order, so the map does not depend on timing.
constexpr int kSelThreads = 1024;
constexpr int kSelBins = 2048;
constexpr int kSelMaxCluster = 8;
constexpr uint32_t kOut = 0u, kStays = 0xffffffffu;      // no weight maps to these (they would be NaNs)

__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) w = -INFINITY;
  if (w == 0.0f) w = 0.0f;                               // -0 orders like 0
  const uint32_t u = __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct SelShared {
  uint32_t hist[kSelBins];
  uint32_t warp[32];
  uint32_t count[4];                                     // what the cluster adds up: recent rows, ties, holes, movers
  uint32_t pick[2];                                      // digit, what is still needed inside it
};

// Sum over the CTA, for every thread.
__device__ __forceinline__ uint32_t block_sum(SelShared& s, uint32_t v) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if (lane == 0) s.warp[warp] = v;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, s.warp[lane]);
}
// Exclusive prefix over the CTA's threads; *all: the sum.
__device__ __forceinline__ uint32_t block_prefix(SelShared& s, uint32_t v, uint32_t* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  __syncthreads();
  if (lane == 31) s.warp[warp] = upto;
  __syncthreads();
  const uint32_t w = s.warp[lane];
  const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u);
  *all = __reduce_add_sync(0xffffffffu, w);
  return before + upto - v;
}

__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(int batch, int H_kv, int cap, int per_cta, int l0, const float* __restrict__ weights,
                    const int32_t* __restrict__ pos, const int32_t* __restrict__ since, const int32_t* __restrict__ len, int keep,
                    int32_t* src, unsigned int* flags) {
  extern __shared__ uint32_t key_s[];                    // [per_cta] keys, then one bit per row: recent
  __shared__ SelShared s;
  cg::cluster_group cl = cg::this_cluster();
  const int n_cta = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int tid = threadIdx.x, lane = tid & 31;
  const int py = blockIdx.x / n_cta, b = (py / H_kv) % batch;
  const size_t head = (size_t)l0 * batch * H_kv + py, rows0 = head * (size_t)cap;
  uint32_t* bit_s = key_s + per_cta;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int want = len ? len[b] : cap, ln = min(max(want, 0), cap);
  if (want != ln && blockIdx.x % (n_cta * H_kv) == 0 && tid == 0) raise(flags, XKV_FLAG_INDEX_RANGE);
  int32_t* dst = src + head * (size_t)keep;
  const int r0 = rank * per_cta;                         // this CTA's rows: r0 .. r0 + n - 1
  const int n = max(0, min(ln - r0, per_cta)), n_up = (n + kSelThreads - 1) / kSelThreads * kSelThreads;
  if (ln <= keep) {
    for (int j = rank * kSelThreads + tid; j < keep; j += n_cta * kSelThreads) dst[j] = j < ln ? j : -1;
    return;                                              // (the whole cluster does: ln and keep are the same for all)
  }

  // ---- keys and recent rows
  const int since_b = since ? since[b] : INT32_MAX;
  uint32_t recent = 0;
  for (int i = tid; i < n_up; i += kSelThreads) {
    bool rec = false;
    if (i < n) {
      const int row = r0 + i;
      key_s[i] = weight_key(weights[rows0 + row]);
      if (since) rec = (pos ? pos[rows0 + row] : row) >= since_b;
    }
    const uint32_t bits = __ballot_sync(0xffffffffu, rec);
    if (lane == 0) bit_s[i >> 5] = bits;
    recent += rec ? 1u : 0u;
  }
  recent = block_sum(s, recent);
  if (tid == 0) s.count[0] = recent;
  cl.sync();
  uint32_t all_recent = 0;
  for (int c = 0; c < n_cta; ++c) all_recent += cl.map_shared_rank(&s, c)->count[0];
  const bool only_recent = all_recent >= (uint32_t)keep;
  uint32_t need = only_recent ? (uint32_t)keep : (uint32_t)keep - all_recent;  // at least one, at most the candidates
  for (int i = tid; i < n; i += kSelThreads) {
    const bool rec = (bit_s[i >> 5] >> (i & 31)) & 1u;
    if (only_recent && !rec) key_s[i] = kOut;
    if (!only_recent && rec) key_s[i] = kStays;
  }
  // ---- the key of the last row that stays
  uint32_t prefix = 0, known = 0;                        // digits found, as bits and as a mask
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t digits = pass == 2 ? 1023u : 2047u;
    for (int i = tid; i < kSelBins; i += kSelThreads) s.hist[i] = 0u;
    __syncthreads();
    for (int i = tid; i < n; i += kSelThreads) {
      const uint32_t k = key_s[i];
      if (k != kOut && k != kStays && (k & known) == prefix) atomicAdd(&s.hist[(k >> shift) & digits], 1u);
    }
    cl.sync();
    // thread t: bins 2t and 2t + 1 of the cluster, from the top
    const int hi = kSelBins - 1 - 2 * tid;
    uint32_t a0 = 0, a1 = 0;
    for (int c = 0; c < n_cta; ++c) {
      const uint32_t* h = cl.map_shared_rank(&s, c)->hist;
      a0 += h[hi];
      a1 += h[hi - 1];
    }
    uint32_t all;
    const uint32_t before = block_prefix(s, a0 + a1, &all);
    if (before < need && need <= before + a0) { s.pick[0] = (uint32_t)hi; s.pick[1] = need - before; }
    else if (before + a0 < need && need <= before + a0 + a1) { s.pick[0] = (uint32_t)hi - 1u; s.pick[1] = need - before - a0; }
    cl.sync();                                           // everyone has read the histograms
    prefix |= s.pick[0] << shift;
    known |= digits << shift;
    need = s.pick[1];
  }
  // ---- ties in row order: a thread's rows are consecutive
  const int each = (n + kSelThreads - 1) / kSelThreads, i0 = min(n, tid * each), i1 = min(n, i0 + each);
  uint32_t ties = 0;
  for (int i = i0; i < i1; ++i) ties += key_s[i] == prefix ? 1u : 0u;
  uint32_t all_ties;
  uint32_t tie = block_prefix(s, ties, &all_ties);
  if (tid == 0) s.count[1] = all_ties;
  cl.sync();
  for (int c = 0; c < rank; ++c) tie += cl.map_shared_rank(&s, c)->count[1];
  uint32_t holes = 0, movers = 0;
  for (int i = i0; i < i1; ++i) {
    const uint32_t k = key_s[i];
    const bool stays = k > prefix || (k == prefix && tie++ < need);            // (kStays is above every key, kOut below)
    key_s[i] = stays ? kStays : kOut;
    if (r0 + i < keep) holes += stays ? 0u : 1u;
    else movers += stays ? 1u : 0u;
  }
  uint32_t all_holes, all_movers;
  uint32_t hole = block_prefix(s, holes, &all_holes), mover = block_prefix(s, movers, &all_movers);
  if (tid == 0) { s.count[2] = all_holes; s.count[3] = all_movers; }
  cl.sync();
  for (int c = 0; c < rank; ++c) {
    hole += cl.map_shared_rank(&s, c)->count[2];
    mover += cl.map_shared_rank(&s, c)->count[3];
  }
  // ---- the i-th mover goes through entry i of the map to the i-th hole (which is at or behind entry i)
  for (int i = i0; i < i1; ++i)
    if (r0 + i >= keep && key_s[i] == kStays) dst[mover++] = r0 + i;
  __threadfence();
  cl.sync();
  for (int i = i0; i < i1; ++i)
    if (r0 + i < keep && key_s[i] == kOut) key_s[i] = (uint32_t)__ldcg(dst + hole++);
  cl.sync();
  for (int i = tid; i < n && r0 + i < keep; i += kSelThreads) dst[r0 + i] = key_s[i] == kStays ? r0 + i : (int32_t)key_s[i];
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

cudaError_t launch_evict_select(const xkv_cache_config* c, int l0, int l1, const float* weights, const int32_t* pos,
                                const int32_t* since, const int32_t* len, int keep, int32_t* src, unsigned int* flags, int device,
                                cudaStream_t s) {
  int n_cta = 1;
  while (n_cta < kSelMaxCluster && c->cap > 4 * kSelThreads * n_cta) n_cta *= 2;
  const int per_cta = ((c->cap + n_cta - 1) / n_cta + kSelThreads - 1) / kSelThreads * kSelThreads;
  const size_t smem = (size_t)per_cta * 4 + (size_t)per_cta / 8;
  cudaError_t e = ensure_dyn_smem<evict_select_kernel>(smem, device);
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
  e = cudaLaunchKernelEx(&cfg, evict_select_kernel, (int)c->batch, (int)c->H_kv, (int)c->cap, per_cta, l0, weights, pos, since, len, keep, src, flags);
  count_launch(kFamEvict);
  return e;
}

}  // namespace xkv
