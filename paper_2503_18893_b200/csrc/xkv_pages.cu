// Pages of a paged cache from lengths (xkv_page_assign): who takes which free pages, who gives pages back, where new tokens go.
//
// Sequences that lack pages take them from the ring in their order, so a sequence's share is a prefix sum of what those before it want;
// what shrinking sequences give back is another, and the places of new tokens a third.  One CTA goes over the sequences in blocks of
// its threads, carrying the three sums; within a block, pages and tokens are then dealt out by whole warps and by binary search.
// Pages given back go to places of the ring that held no free page before the call, so nothing that is read is written.
#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kSeqs = 1024;                    // threads, and sequences of a block

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

__global__ void __launch_bounds__(kSeqs) page_assign_kernel(const PageArgs a) {
  __shared__ Sums warps_s[32];
  __shared__ int held_s[kSeqs], fresh_s[kSeqs + 1];            // rows before the call; new tokens of the sequences before, in the block
  __shared__ uint8_t ok_s[kSeqs];
  __shared__ int taken_s, bad_s;
  const int tid = threadIdx.x, lane = tid & 31;
  const int page = 1 << a.page_shift, most = a.max_pages << a.page_shift;
  if (tid == 0) { taken_s = 0; bad_s = 0; }
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  int head = a.state[0], count = a.state[1];
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) {
    head = count = 0;
    if (tid == 0) bad_s = 1;
  }
  const int room = a.n_pages - count;          // places of the ring that hold no free page
  long long take0 = 0, give0 = 0, fresh0 = 0;  // of the blocks before
  __syncthreads();
  for (int b0 = 0; b0 < a.batch; b0 += kSeqs) {
    const int b = b0 + tid;
    int held = 0, want = 0;
    bool bad = false;
    if (b < a.batch) {
      const int h = a.held[b], w = a.want[b];
      held = min(max(h, 0), most);
      want = min(max(w, 0), most);
      bad = h != held || w != want;
    }
    const int have = (held + page - 1) >> a.page_shift, need = (want + page - 1) >> a.page_shift;
    const Sums mine = {max(need - have, 0), max(have - need, 0), (long long)max(want - held, 0)};
    Sums all;
    const Sums upto = prefix(mine, warps_s, &all);
    const bool ok = mine.take == 0 || take0 + upto.take <= count;
    if (b < a.batch) {
      if (a.first) {
        const long long f = fresh0 + upto.fresh - mine.fresh, e = fresh0 + upto.fresh;
        a.first[b] = (int)min(f, 0x7fffffffll);
        if (b == a.batch - 1) a.first[a.batch] = (int)min(e, 0x7fffffffll);
        if (e > 0x7fffffffll) bad = true;
      }
      a.length[b] = ok ? want : held;
    }
    // pages, by whole warps: a sequence after the other
    const int took = ok ? mine.take : 0;
    const int from = (int)((head + take0 + upto.take - mine.take) % a.n_pages);
    const long long back = give0 + upto.give - mine.give;      // of those before this sequence
    const int to = (int)((head + count + back) % a.n_pages);
    const long long left = room - back;
    if (mine.take > 0 && ok) atomicMax(&taken_s, (int)(take0 + upto.take));
    if (mine.give > 0 && left < mine.give) bad = true;
    for (unsigned todo = __ballot_sync(0xffffffffu, took > 0 || mine.give > 0); todo; todo &= todo - 1u) {
      const int src = __ffs(todo) - 1;
      const int n_take = __shfl_sync(0xffffffffu, took, src), n_give = __shfl_sync(0xffffffffu, mine.give, src);
      const int at = __shfl_sync(0xffffffffu, n_take > 0 ? from : to, src);
      const int row = __shfl_sync(0xffffffffu, n_take > 0 ? have : need, src);
      const long long free_places = __shfl_sync(0xffffffffu, left, src);
      int32_t* entry = a.table + (size_t)(b - lane + src) * a.max_pages + row;
      for (int i = lane; i < n_take + n_give; i += 32) {
        const int p = (int)(((long long)at + i) % a.n_pages);
        if (n_take > 0) {
          entry[i] = a.ring[p];
        } else {
          if (i < free_places) a.ring[p] = entry[i];
          entry[i] = -1;
        }
      }
    }
    held_s[tid] = held;
    fresh_s[tid + 1] = (int)min(upto.fresh, 0x7fffffffll);
    if (tid == 0) fresh_s[0] = 0;
    ok_s[tid] = ok;
    __syncthreads();                           // (taken pages are in the table for the whole CTA, too)
    if (a.slot) {
      const int n = (int)max(0ll, min(all.fresh, (long long)a.n_tok - fresh0));
      for (int t = tid; t < n; t += kSeqs) {
        int lo = 0, hi = kSeqs - 1;            // the last sequence that begins at or before t: fresh_s[lo] <= t < fresh_s[lo + 1]
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (fresh_s[mid + 1] > t) hi = mid; else lo = mid + 1;
        }
        const int pos = held_s[lo] + t - fresh_s[lo];
        int slot = -1;
        if (ok_s[lo]) {
          const int p = a.table[(size_t)(b0 + lo) * a.max_pages + (pos >> a.page_shift)];
          if (p >= 0 && p < a.n_pages) slot = (p << a.page_shift) + (pos & (page - 1));
          else bad = true;
        }
        a.pos[fresh0 + t] = pos;
        a.slot[fresh0 + t] = slot;
      }
    }
    if (bad) bad_s = 1;
    take0 += all.take;
    give0 += all.give;
    fresh0 += all.fresh;
    __syncthreads();
  }
  if (a.slot) {
    for (long long t = fresh0 + tid; t < a.n_tok; t += kSeqs) { a.pos[t] = 0; a.slot[t] = -1; }
    if (tid == 0 && fresh0 > a.n_tok) bad_s = 1;
  }
  __syncthreads();
  if (tid == 0) {
    const long long joined = min(give0, (long long)room);
    a.state[0] = (int)(((long long)head + taken_s) % a.n_pages);
    a.state[1] = count - taken_s + (int)joined;
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
  const cudaError_t e = launch_pdl(page_assign_kernel, dim3(1), dim3(kSeqs), 0, s, a);
  count_launch(kFamPages);
  return e;
}

}  // namespace xkv
