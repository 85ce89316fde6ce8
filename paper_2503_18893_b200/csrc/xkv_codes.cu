// Rows of a paged cache into 8-bit codes and back (xkv_cache8_append, xkv_cache8_read).
//
// A page and head share a scale 2^e.  Multiplying by a power of two is exact, so a code is the value's own rounding to e4m3 and depends
// on nothing but the value and e: e comes from integer comparisons on the largest magnitude's bits, and no division takes place.
// When a louder row joins a page its scale grows, and the codes that are there move down by the steps it has grown: exact but where
// they leave e4m3's normal range.
//
// Append: the rows that a call brings to a page are one run of tokens.  For every run, head and tensor (keys, values) page / 16 warps
// keep 16 rows each in registers: one read of the new rows, the maximum over the warps, one write of codes.  Read: 16 codes a thread.
// Both are meant to be bound by memory.  4099 tokens of four heads in four layers: append 15.5 us (3.2 TB/s; instructions: 65 % of issue slots
// busy), their read back 10.4; 32768 rows of eight heads in four layers read back in 131-138 us (5.8-6.1 TB/s); 32 sequences' tokens 4.5.
#include <cuda_fp16.h>

#include "xkv_internal.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kLowest = -60, kHighest = 120;   // exponents of scales of rows (bf16's largest value is below 448 * 2^120)
constexpr int kAppendThreads = 256, kRunRows = 16;             // rows that a warp keeps

struct CodesArgs {
  int batch, H_kv, n_pages, max_pages, page_shift, l0, layers;
  int n_tok, per_group;                        // append: tokens of the call, and those whose runs a group of warps looks after
  int cap;                                     // read
  const __nv_bfloat16* x[2];                   // append: keys, values
  __nv_bfloat16* y[2];                         // read
  uint8_t* codes[2];
  float* scale[2];
  const int32_t* slot;
  const int32_t* table;
  const int32_t* length;
  unsigned int* flags;
};

// 2^e for -127 <= e <= 127.
__device__ __forceinline__ float two_to(int e) { return e == -127 ? 0x1p-127f : __int_as_float((127 + e) << 23); }
// The exponent of a scale; kNothing: it is 0 (or no normal number), kNotFinite: infinite or NaN.
constexpr int kNothing = -127, kNotFinite = 128;
__device__ __forceinline__ int exponent_of(float scale) { return ((__float_as_int(scale) >> 23) & 255) - 127; }
// The smallest e with top <= 448 * 2^e = 1.75 * 2^(e + 8), for the bits of a bf16 magnitude.
__device__ __forceinline__ int exponent_for(uint32_t top) {
  return min(max((int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), kLowest), kHighest);
}
__device__ __forceinline__ float2 decode2(uint32_t codes) {    // the two codes of the low half
  const uint32_t h = ptx::unpack_e4m3(codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
// Magnitudes of two bf16 values; 0 for those that are not finite.
__device__ __forceinline__ uint32_t magnitudes(uint32_t x) {
  x &= 0x7fff7fffu;
  return x & ~__vcmpgeu2(x, 0x7f807f80u);
}

// W: 32-bit words of a row that a lane holds (two values each): 2 for d_h = 128, 1 for 64.
template <int W>
__global__ void __launch_bounds__(kAppendThreads, 4) append_kernel(const CodesArgs a) {
  constexpr int DH = W * 64;
  __shared__ uint32_t top_s[kAppendThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int page = 1 << a.page_shift, warps = page / kRunRows, groups = kAppendThreads / 32 / warps;
  const int group = warp / warps, part = warp - group * warps;
  const int t0 = (int)min(((long long)blockIdx.x * groups + group) * a.per_group, (long long)a.n_tok);
  const int h = blockIdx.y, l = a.l0 + (int)(blockIdx.z >> 1), kv = blockIdx.z & 1;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  if (t0 >= a.n_tok) return;                   // (a whole group)
  const int limit = a.n_pages << a.page_shift, n = min(a.per_group, a.n_tok - t0);
  // which of the group's tokens begin a run: not the row behind the token before's, or a page's first
  unsigned begin[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = 32 * i + lane;
    bool begins = false;
    if (x < n) {
      const int s = a.slot[t0 + x], before = t0 + x > 0 ? a.slot[t0 + x - 1] : -1;
      const bool in = s >= 0 && s < limit;
      if (!in && s != -1 && a.flags && h == 0 && blockIdx.z == 0) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
      begins = in && ((s & (page - 1)) == 0 || before != s - 1);
    }
    begin[i] = __ballot_sync(0xffffffffu, begins);
  }
  for (int at = 0;; ++at) {                    // (a group has few runs: one or two of a prompt's, or one token's)
    int first = -1;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      const unsigned rest = at < 32 * i ? begin[i] : at >= 32 * i + 32 ? 0u : begin[i] & (0xffffffffu << (at - 32 * i));
      if (rest) first = 32 * i + __ffs(rest) - 1;
    }
    if (first < 0) break;
    at = first;
    const int t = t0 + first, s = a.slot[t];
    const int off = s & (page - 1), most = min(page - off, a.n_tok - t);
    int rows = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = 32 * i + lane;
      const unsigned same = __ballot_sync(0xffffffffu, x < most && a.slot[t + min(x, most - 1)] == s + x);
      if (rows == 32 * i) rows += same == 0xffffffffu ? 32 : __ffs(~same) - 1;
    }
    const size_t head = ((size_t)l * a.n_pages + (s >> a.page_shift)) * a.H_kv + h;
    uint8_t* codes = a.codes[kv] + (head << a.page_shift) * DH;
    float* scale = a.scale[kv] + head;
    const int old = off > 0 ? exponent_of(*scale) : kNothing;
    const __nv_bfloat16* x = a.x[kv] + (((size_t)l * a.n_tok + t) * a.H_kv + h) * DH + lane * (2 * W);
    uint32_t v[kRunRows][W], top = 0;
#pragma unroll
    for (int i = 0; i < kRunRows; ++i) {
      const int r = part * kRunRows + i;
#pragma unroll
      for (int w = 0; w < W; ++w) v[i][w] = 0;
      if (r < rows) {
        const __nv_bfloat16* src = x + (size_t)r * a.H_kv * DH;
        if constexpr (W == 2) *reinterpret_cast<uint2*>(v[i]) = *reinterpret_cast<const uint2*>(src);
        else v[i][0] = *reinterpret_cast<const uint32_t*>(src);
      }
    }
#pragma unroll
    for (int i = 0; i < kRunRows; ++i) {
#pragma unroll
      for (int w = 0; w < W; ++w) top = __vmaxu2(top, v[i][w] & 0x7fff7fffu);
    }
    if (__any_sync(0xffffffffu, (top & 0xffffu) >= 0x7f80u || top >= 0x7f800000u)) {           // something is not finite: without it
      top = 0;
#pragma unroll
      for (int i = 0; i < kRunRows; ++i) {
#pragma unroll
        for (int w = 0; w < W; ++w) top = __vmaxu2(top, magnitudes(v[i][w]));
      }
    }
    top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
    if (warps > 1) {                           // (every warp of the group has read the old scale by then)
      if (lane == 0) top_s[warp] = top;
      ptx::named_bar_sync(1 + group, warps * 32);
      for (int i = 0; i < warps; ++i) top = max(top, top_s[group * warps + i]);
      ptx::named_bar_sync(1 + group, warps * 32);
    }
    const int e = max(exponent_for(top), old == kNotFinite ? kLowest : old);
    if (e != old && off > 0) {
      const float f = old == kNotFinite ? __int_as_float(0x7fffffff) : two_to(max(old - e, -126));
      for (int i = part * 32 + lane; i < off * (DH / 4); i += warps * 32) {
        uint32_t* at = reinterpret_cast<uint32_t*>(codes) + i;
        const uint32_t c = old == kNothing ? 0u : *at;
        const float2 lo = decode2(c), hi = decode2(c >> 16);
        *at = ptx::pack_e4m3(lo.x * f, lo.y * f) | (ptx::pack_e4m3(hi.x * f, hi.y * f) << 16);
      }
    }
    const float f = two_to(-e);
#pragma unroll
    for (int i = 0; i < kRunRows; ++i) {
      const int r = part * kRunRows + i;
      if (r < rows) {
        uint8_t* dst = codes + (size_t)(off + r) * DH + lane * (2 * W);
        const uint32_t c = ptx::pack_e4m3(bf16_lo(v[i][0]) * f, bf16_hi(v[i][0]) * f);
        if constexpr (W == 2) *reinterpret_cast<uint32_t*>(dst) = c | (ptx::pack_e4m3(bf16_lo(v[i][1]) * f, bf16_hi(v[i][1]) * f) << 16);
        else *reinterpret_cast<uint16_t*>(dst) = (uint16_t)c;
      }
    }
    if (part == 0 && lane == 0) *scale = two_to(e);
  }
}

constexpr int kReadThreads = 256;

// CTA: rows of one (layer, sequence, head, tensor); a thread has 16 codes.
template <int DH>
__global__ void __launch_bounds__(kReadThreads) read_kernel(const CodesArgs a) {
  constexpr int C = DH / 16, ROWS = kReadThreads / C;
  const int c = threadIdx.x % C;
  const int h = blockIdx.y % a.H_kv, b = blockIdx.y / a.H_kv, l = a.l0 + (int)(blockIdx.z >> 1), kv = blockIdx.z & 1;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  if (!a.y[kv]) return;
  const int want = a.length[b], len = min(max(want, 0), min(a.cap, a.max_pages << a.page_shift));
  if (len != want && a.flags && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
  const int j = (int)blockIdx.x * ROWS + threadIdx.x / C;
  if (j >= len) return;
  const int p = a.table[(size_t)b * a.max_pages + (j >> a.page_shift)];
  if (p < 0 || p >= a.n_pages) {
    if (a.flags) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
    return;
  }
  const size_t head = ((size_t)l * a.n_pages + p) * a.H_kv + h;
  const uint4 x = *reinterpret_cast<const uint4*>(a.codes[kv] + ((head << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * DH + c * 16);
  const float f = __int_as_float(__float_as_int(a.scale[kv][head]) & 0x7f800000);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t r[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 lo = decode2(w[i]), hi = decode2(w[i] >> 16);
    r[2 * i] = ptx::pack_bf16(lo.x * f, lo.y * f);
    r[2 * i + 1] = ptx::pack_bf16(hi.x * f, hi.y * f);
  }
  uint4* dst = reinterpret_cast<uint4*>(a.y[kv] + ((((size_t)l * a.batch + b) * a.H_kv + h) * a.cap + j) * DH + c * 16);
  dst[0] = make_uint4(r[0], r[1], r[2], r[3]);
  dst[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

CodesArgs codes_args(const xkv_cache8_config* c, int l0, int l1, void* K8, void* V8, float* k_scale, float* v_scale, unsigned int* flags) {
  CodesArgs a = {};
  a.batch = c->batch; a.H_kv = c->H_kv; a.n_pages = c->n_pages; a.max_pages = c->max_pages;
  a.page_shift = __builtin_ctz((unsigned)c->page);
  a.l0 = l0; a.layers = l1 - l0;
  a.codes[0] = (uint8_t*)K8; a.codes[1] = (uint8_t*)V8;
  a.scale[0] = k_scale; a.scale[1] = v_scale;
  a.flags = flags;
  return a;
}

// Keys and values of at most as many layers at a time as a grid's third dimension has room for.
template <typename F>
cudaError_t launch_layers(CodesArgs a, F launch) {
  constexpr int kMost = 65535 / 2;
  for (int l0 = a.l0, left = a.layers; left > 0; l0 += kMost, left -= kMost) {
    a.l0 = l0;
    a.layers = left < kMost ? left : kMost;
    const cudaError_t e = launch(a, 2 * a.layers);
    count_launch(kFamCodes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_cache8_append(const xkv_cache8_config* c, int l0, int l1, const __nv_bfloat16* k, const __nv_bfloat16* v,
                                 const int32_t* slot, int n_tok, void* K8, void* V8, float* k_scale, float* v_scale, unsigned int* flags,
                                 cudaStream_t s) {
  CodesArgs a = codes_args(c, l0, l1, K8, V8, k_scale, v_scale, flags);
  a.x[0] = k; a.x[1] = v; a.slot = slot; a.n_tok = n_tok;
  // A group looks after one token as long as that gives two waves of CTAs at most (decode: every token is a run of its own, and runs
  // of a group come one after the other), then after as many as a page has rows, 32 at least: most of a prompt's tokens begin no run.
  // (4099 tokens of four heads in four layers, pages of 128: 25 us with 32 tokens a group, 22 with 128, 18 with four CTAs an SM besides, 15.5 when it
  // looks for what is not finite only where there is something.)
  const int groups = kAppendThreads / 32 / (c->page / kRunRows);
  const long long per_token = (long long)c->H_kv * 2 * a.layers;
  auto ctas = [&](int per_group) { return (int)(((long long)n_tok + groups * per_group - 1) / (groups * per_group)); };
  a.per_group = 1;
  while (a.per_group < (c->page > 32 ? c->page : 32) && ctas(a.per_group) * per_token > kPlanSms * 16) a.per_group *= 2;
  return launch_layers(a, [&](const CodesArgs& part, int z) {
    const dim3 grid(ctas(part.per_group), c->H_kv, z), threads(kAppendThreads);
    return c->d_h == 128 ? launch_pdl(append_kernel<2>, grid, threads, 0, s, part) : launch_pdl(append_kernel<1>, grid, threads, 0, s, part);
  });
}

cudaError_t launch_cache8_read(const xkv_cache8_config* c, int l0, int l1, const int32_t* table, const int32_t* length, const void* K8,
                               const void* V8, const float* k_scale, const float* v_scale, int cap, __nv_bfloat16* K, __nv_bfloat16* V,
                               unsigned int* flags, cudaStream_t s) {
  CodesArgs a = codes_args(c, l0, l1, const_cast<void*>(K8), const_cast<void*>(V8), const_cast<float*>(k_scale), const_cast<float*>(v_scale), flags);
  a.table = table; a.length = length; a.cap = cap; a.y[0] = K; a.y[1] = V;
  const int rows = kReadThreads / (c->d_h / 16), most = cap < c->max_pages * c->page ? cap : c->max_pages * c->page;
  return launch_layers(a, [&](const CodesArgs& part, int z) {
    const dim3 grid((most + rows - 1) / rows, c->batch * c->H_kv, z), threads(kReadThreads);
    return c->d_h == 128 ? launch_pdl(read_kernel<128>, grid, threads, 0, s, part) : launch_pdl(read_kernel<64>, grid, threads, 0, s, part);
  });
}

}  // namespace xkv
