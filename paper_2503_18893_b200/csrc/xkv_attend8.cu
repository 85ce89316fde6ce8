// Attention over a paged cache of 8-bit codes (xkv_cache8_attend): out_i = softmax(scale q_i K^T) V over the rows of token i's sequence
// up to its own, K and V being codes times their pages' scales.
//
// One CTA per token, query head and layer; thread = row of a 128-row tile for the logits, thread = column for the weighted sum.
#include <math.h>

#include <cuda_fp16.h>

#include "xkv_cache.cuh"

namespace xkv {

namespace {

constexpr int kThreads8 = 128;

struct Attend8Args {
  int batch, H_kv, H_q, n_rep, n_pages, max_pages, page_shift, n_tok, max_new, l0;
  float scale2;                                // softmax scale times log2(e)
  const __nv_bfloat16* q;
  const int32_t* first;
  const int32_t* table;
  const int32_t* length;
  const uint8_t* K8;
  const uint8_t* V8;
  const float* k_scale;
  const float* v_scale;
  __nv_bfloat16* out;
  float* lse;
  unsigned int* flags;
};

__device__ __forceinline__ float code_value(uint8_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)c));
  return __half2float(__ushort_as_half((unsigned short)h));
}
__device__ __forceinline__ float power_of_two(float scale) { return __int_as_float(__float_as_int(scale) & 0x7f800000); }

template <int DH>
__global__ void __launch_bounds__(kThreads8) attend8_plain_kernel(const Attend8Args a) {
  __shared__ float q_s[DH], p_s[kThreads8], red_s[2][4];
  const int t = blockIdx.x, hq = blockIdx.y, l = a.l0 + (int)blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  bool bad = false;
  auto first_of = [&](int b) {
    const int f = a.first ? a.first[b] : b, c = min(max(f, 0), a.n_tok);
    bad |= f != c;
    return c;
  };
  int lo = 0, hi = a.batch - 1;                // the sequence of token t
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (first_of(mid + 1) > t) hi = mid; else lo = mid + 1;
  }
  const int f0 = first_of(lo), f1 = first_of(lo + 1), n = f1 - f0;
  if (t < f0 || t >= f1 || t - f0 >= a.max_new) return;
  const int want = a.length[lo], len = min(max(want, 0), a.max_pages << a.page_shift);
  bad |= want != len || n > a.max_new;
  const int rows = max(0, min(len, len - n + (t - f0) + 1));
  const int g = hq / a.n_rep;
  const size_t qh = ((size_t)l * a.n_tok + t) * a.H_q + hq;
  if (tid < DH) q_s[tid] = __bfloat162float(a.q[qh * DH + tid]);
  __syncthreads();
  float m = -INFINITY, sum = 0.0f, acc = 0.0f;
  for (int j0 = 0; j0 < rows; j0 += kThreads8) {
    const int j = j0 + tid;
    float z = -INFINITY, vs = 0.0f;
    size_t row = 0;
    if (j < rows) {
      const int p = a.table[(size_t)lo * a.max_pages + (j >> a.page_shift)];
      if (p >= 0 && p < a.n_pages) {
        const size_t head = ((size_t)l * a.n_pages + p) * a.H_kv + g;
        row = (head << a.page_shift) + (j & ((1 << a.page_shift) - 1));
        const float ks = power_of_two(a.k_scale[head]);
        vs = power_of_two(a.v_scale[head]);
        if (ks > 0.0f && vs > 0.0f) {
          z = 0.0f;
          for (int d = 0; d < DH; ++d) z = fmaf(q_s[d], code_value(a.K8[row * DH + d]), z);
          z *= ks * a.scale2;
        } else {
          vs = 0.0f;
        }
      } else {
        bad = true;
      }
    }
    float top = z;
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) red_s[0][warp] = top;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(red_s[0][0], red_s[0][1]), fmaxf(red_s[0][2], red_s[0][3])));
    const float shift = m_new == -INFINITY ? 0.0f : m_new;
    const float p = vs > 0.0f ? exp2f(z - shift) : 0.0f;
    p_s[tid] = p;
    float part = p;
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
    if (lane == 0) red_s[1][warp] = part;
    __syncthreads();
    const float f = m == -INFINITY ? 0.0f : exp2f(m - shift);
    sum = sum * f + (red_s[1][0] + red_s[1][1] + red_s[1][2] + red_s[1][3]);
    acc *= f;
    m = m_new;
    if (tid < DH) {
      for (int i = 0; i < min(kThreads8, rows - j0); ++i) {
        const int p2 = a.table[(size_t)lo * a.max_pages + ((j0 + i) >> a.page_shift)];
        if (p2 < 0 || p2 >= a.n_pages) continue;
        const size_t head = ((size_t)l * a.n_pages + p2) * a.H_kv + g;
        const float v2 = power_of_two(a.v_scale[head]);
        if (!(v2 > 0.0f) || !(power_of_two(a.k_scale[head]) > 0.0f)) continue;
        acc = fmaf(p_s[i], code_value(a.V8[((head << a.page_shift) + ((j0 + i) & ((1 << a.page_shift) - 1))) * DH + tid]) * v2, acc);
      }
    }
    __syncthreads();
  }
  if (tid < DH) a.out[qh * DH + tid] = __float2bfloat16_rn(sum == 0.0f ? 0.0f : acc / sum);
  if (tid == 0 && a.lse) a.lse[qh] = sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
  if (bad && a.flags) atomicOr(a.flags, XKV_FLAG_INDEX_RANGE);
}

}  // namespace

size_t cache8_workspace_bytes(const xkv_cache8_config* c, int max_new) { return 16; }

cudaError_t launch_cache8_attend(const xkv_cache8_config* c, int l0, int l1, const __nv_bfloat16* q, const int32_t* first, int n_tok,
                                 int max_new, const int32_t* table, const int32_t* length, const void* K8, const void* V8,
                                 const float* k_scale, const float* v_scale, void* workspace, __nv_bfloat16* out, float* lse,
                                 unsigned int* flags, int device, cudaStream_t s) {
  Attend8Args a;
  a.batch = c->batch; a.H_kv = c->H_kv; a.H_q = c->H_q; a.n_rep = c->H_q / c->H_kv; a.n_pages = c->n_pages; a.max_pages = c->max_pages;
  a.page_shift = __builtin_ctz((unsigned)c->page);
  a.n_tok = n_tok; a.max_new = max_new; a.l0 = l0;
  a.scale2 = (c->softmax_scale > 0.0f ? c->softmax_scale : 1.0f / sqrtf((float)c->d_h)) * kLog2e;
  a.q = q; a.first = first; a.table = table; a.length = length; a.K8 = (const uint8_t*)K8; a.V8 = (const uint8_t*)V8;
  a.k_scale = k_scale; a.v_scale = v_scale; a.out = out; a.lse = lse; a.flags = flags;
  const dim3 grid(n_tok, c->H_q, l1 - l0);
  const cudaError_t e = c->d_h == 128 ? launch_pdl(attend8_plain_kernel<128>, grid, dim3(kThreads8), 0, s, a)
                                      : launch_pdl(attend8_plain_kernel<64>, grid, dim3(kThreads8), 0, s, a);
  count_launch(kFamAttend8);
  return e;
}

}  // namespace xkv
