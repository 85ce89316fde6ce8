// Pages of a paged cache from lengths (xkv_page_assign): who takes which free pages, who gives pages back, where new tokens go.
//
// Sequences that lack pages take them from the ring in their order, so a sequence's share is a prefix sum of what those before it want;
// what shrinking sequences give back is another, and the places of new tokens a third.  One CTA goes over the sequences in blocks of
// its threads, carrying the three sums; within a block, pages and tokens are then dealt out by whole warps and by binary search.
// Pages given back go to places of the ring that held no free page before the call, so nothing that is read is written.
// Bound by latency: 48 sequences with eight drafts each 4.3 us a call, 300 with up to 128 new tokens and back 5.8 (a cluster of eight from
// 2048 tokens on).  Dealt out sequence after sequence by whole warps they took 18 and 26: a page's way is a load and a store that waits for it.
#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kSeqs = 1024;                    // threads, and sequences of a block
constexpr int kRanks = 8;                      // CTAs of a cluster, where there are many tokens

struct PageArgs {
  int batch, page_shift, n_pages, max_pages, n_tok;
  const int32_t* held;
  const int32_t* want;
  int32_t* table;
  int32_t* ring;
  int32_t* state;
  int32_t* first;
  int32_t* length;
  int32_t* pos;
  int32_t* slot;
  unsigned int* flags;
};

// Inclusive prefix sums of three numbers over the CTA's threads, and their totals.
struct Sums {
  int take, give;
  long long fresh;
};
__device__ __forceinline__ Sums prefix(Sums v, Sums* warps_s, Sums* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, v.take, o), g = __shfl_up_sync(0xffffffffu, v.give, o);
    const long long f = __shfl_up_sync(0xffffffffu, v.fresh, o);
    if (lane >= o) { v.take += t; v.give += g; v.fresh += f; }
  }
  if (lane == 31) warps_s[warp] = v;
  __syncthreads();
  if (warp == 0) {
    Sums w = warps_s[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, w.take, o), g = __shfl_up_sync(0xffffffffu, w.give, o);
      const long long f = __shfl_up_sync(0xffffffffu, w.fresh, o);
      if (lane >= o) { w.take += t; w.give += g; w.fresh += f; }
    }
    warps_s[lane] = w;
  }
  __syncthreads();
  if (warp > 0) {
    const Sums w = warps_s[warp - 1];
    v.take += w.take; v.give += w.give; v.fresh += w.fresh;
  }
  *total = warps_s[31];
  return v;
}

// The last of 1024 sequences that begins at or before i: upto_s[x] <= i < upto_s[x + 1].
__device__ __forceinline__ int sequence_of(const int* upto_s, int i) {
  int lo = 0, hi = kSeqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (upto_s[mid + 1] > i) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// A cluster: every CTA forms the sums of a block for itself, then they deal out its pages and tokens among them.
__global__ void __launch_bounds__(kSeqs) page_assign_kernel(const PageArgs a) {
  __shared__ Sums warps_s[32];
  // of the block's sequences: rows before the call (-1 - rows: it got no pages); pages taken, given back, and new tokens of those before
  __shared__ int held_s[kSeqs], want_s[kSeqs], take_s[kSeqs + 1], give_s[kSeqs + 1], fresh_s[kSeqs + 1];
  __shared__ int taken_s, bad_s;
  const int tid = threadIdx.x, rank = blockIdx.x, ranks = gridDim.x;
  const int page = 1 << a.page_shift, most = a.max_pages << a.page_shift;
  if (tid == 0) { taken_s = 0; bad_s = 0; take_s[0] = give_s[0] = fresh_s[0] = 0; }
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  int head = a.state[0], count = a.state[1];
  bool bad = false;
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) {
    head = count = 0;
    bad = true;
  }
  const int room = a.n_pages - count;          // places of the ring that hold no free page
  auto place = [&](long long i) { return (int)((head + i) % a.n_pages); };
  long long take0 = 0, give0 = 0, fresh0 = 0;  // of the blocks before
  for (int b0 = 0; b0 < a.batch; b0 += kSeqs) {
    const int b = b0 + tid;
    int held = 0, want = 0;
    if (b < a.batch) {
      const int h = a.held[b], w = a.want[b];
      held = min(max(h, 0), most);
      want = min(max(w, 0), most);
      bad |= h != held || w != want;
    }
    const int have = (held + page - 1) >> a.page_shift, need = (want + page - 1) >> a.page_shift;
    const Sums mine = {max(need - have, 0), max(have - need, 0), (long long)max(want - held, 0)};
    Sums all;
    const Sums upto = prefix(mine, warps_s, &all);
    const bool ok = mine.take == 0 || take0 + upto.take <= count;
    if (mine.take > 0 && ok) atomicMax(&taken_s, (int)(take0 + upto.take));
    held_s[tid] = ok ? held : -1 - held;
    want_s[tid] = want;
    take_s[tid + 1] = upto.take;
    give_s[tid + 1] = upto.give;
    fresh_s[tid + 1] = (int)min(upto.fresh, 0x7fffffffll);
    // every CTA has read what is overwritten now (`length` may be `held` or `want`)
    ptx::cluster_sync();
    if (rank == 0 && b < a.batch) {
      const long long f = fresh0 + upto.fresh - mine.fresh, e = fresh0 + upto.fresh;
      if (a.first) {
        a.first[b] = (int)min(f, 0x7fffffffll);
        if (b == a.batch - 1) a.first[a.batch] = (int)min(e, 0x7fffffffll);
        bad |= e > 0x7fffffffll;
      }
      a.length[b] = ok ? want : held;
    }
    for (int i = rank * kSeqs + tid; i < all.take; i += ranks * kSeqs) {       // pages taken
      const int x = sequence_of(take_s, i), h = held_s[x];
      if (h >= 0) {
        const int p = a.ring[place(take0 + i)];
        a.table[(size_t)(b0 + x) * a.max_pages + ((h + page - 1) >> a.page_shift) + i - take_s[x]] = p;
        bad |= p < 0 || p >= a.n_pages;
      }
    }
    for (int i = rank * kSeqs + tid; i < all.give; i += ranks * kSeqs) {       // pages given back
      const int x = sequence_of(give_s, i);
      int32_t* entry = a.table + (size_t)(b0 + x) * a.max_pages + ((want_s[x] + page - 1) >> a.page_shift) + i - give_s[x];
      const int p = *entry;
      if (give0 + i < room) a.ring[place(count + give0 + i)] = p;
      bad |= give0 + i >= room || p < 0 || p >= a.n_pages;
      *entry = -1;
    }
    if (a.slot) {
      const int n = (int)max(0ll, min(all.fresh, (long long)a.n_tok - fresh0));
      for (uint32_t t = rank * kSeqs + tid; t < (uint32_t)n; t += ranks * kSeqs) {
        const int x = sequence_of(fresh_s, (int)t), h = held_s[x], held_x = h >= 0 ? h : -1 - h, pos = held_x + (int)t - fresh_s[x];
        int slot = -1;
        if (h >= 0) {
          // a page that was taken just now is still in the ring, in whatever order the table is written
          const int i = pos >> a.page_shift, fresh = i - ((held_x + page - 1) >> a.page_shift);
          const int p = fresh >= 0 ? a.ring[place(take0 + take_s[x] + fresh)] : a.table[(size_t)(b0 + x) * a.max_pages + i];
          if (p >= 0 && p < a.n_pages) slot = (p << a.page_shift) + (pos & (page - 1));
          else bad = true;
        }
        a.pos[fresh0 + t] = pos;
        a.slot[fresh0 + t] = slot;
      }
    }
    take0 += all.take;
    give0 += all.give;
    fresh0 += all.fresh;
    __syncthreads();
  }
  if (a.slot) {
    for (long long t = fresh0 + rank * kSeqs + tid; t < a.n_tok; t += ranks * kSeqs) { a.pos[t] = 0; a.slot[t] = -1; }
    bad |= fresh0 > a.n_tok;
  }
  if (bad) bad_s = 1;
  __syncthreads();
  if (tid == 0) {
    if (rank == 0) {
      a.state[0] = place(taken_s);
      a.state[1] = count - taken_s + (int)min(give0, (long long)room);
    }
    if (bad_s && a.flags) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
  }
}

}  // namespace

cudaError_t launch_page_assign(const xkv_cache8_config* c, const int32_t* held, const int32_t* want, int32_t* table, int32_t* ring,
                               int32_t* state, int32_t* first, int32_t* length, int32_t* pos, int32_t* slot, int32_t n_tok,
                               unsigned int* flags, cudaStream_t s) {
  PageArgs a;
  a.batch = c->batch; a.n_pages = c->n_pages; a.max_pages = c->max_pages; a.n_tok = n_tok;
  a.page_shift = __builtin_ctz((unsigned)c->page);
  a.held = held; a.want = want; a.table = table; a.ring = ring; a.state = state; a.first = first; a.length = length;
  a.pos = pos; a.slot = slot; a.flags = flags;
  const int ranks = n_tok > 2 * kSeqs ? kRanks : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks);
  cfg.blockDim = dim3(kSeqs);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ranks;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, page_assign_kernel, a);
  count_launch(kFamPages);
  return e;
}

}  // namespace xkv
