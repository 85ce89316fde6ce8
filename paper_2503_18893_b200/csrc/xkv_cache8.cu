// C entry points of rotary positions and of the paged cache of 8-bit codes: argument checking and dispatch.
#include <math.h>

#include <initializer_list>

#include "xkv_internal.cuh"

namespace xkv {

namespace {

int check_cache8(const xkv_cache8_config* c) {
  if (!c || c->struct_size != sizeof(xkv_cache8_config)) return XKV_ERR_INVALID_ARG;
  if (c->G < 1 || c->batch < 1 || c->H_kv < 1 || c->H_q < 1 || c->H_q % c->H_kv != 0 || c->H_q / c->H_kv > kMaxRep) return XKV_ERR_INVALID_ARG;
  if (c->d_h != 64 && c->d_h != 128) return XKV_ERR_INVALID_ARG;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return XKV_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->max_pages < 1 || (int64_t)c->max_pages * c->page > XKV_CACHE_MAX_ROWS) return XKV_ERR_INVALID_ARG;
  if (!(c->softmax_scale >= 0.0f) || isinf(c->softmax_scale)) return XKV_ERR_INVALID_ARG;
  // heads are a grid dimension, rows of all pages a 32-bit coordinate of the copy engine
  if ((double)c->G * c->batch * c->H_kv > 65535.0 || (double)c->G * c->n_pages * c->H_kv * c->page >= 2147483648.0) return XKV_ERR_UNSUPPORTED;
  return XKV_OK;
}

int check_layers8(const xkv_cache8_config* c, int l0, int l1) {
  const int st = check_cache8(c);
  if (st != XKV_OK) return st;
  return l0 < 0 || l1 > c->G || l0 >= l1 ? XKV_ERR_INVALID_ARG : XKV_OK;
}

bool aligned_to(unsigned to, std::initializer_list<const void*> ps) {
  uintptr_t all = 0;
  for (const void* p : ps) all |= (uintptr_t)p;
  return (all & (to - 1u)) == 0;
}

int finish8(cudaError_t e) {
  if (e == cudaSuccess) return XKV_OK;
  set_cuda_error(e);
  (void)cudaGetLastError();
  return XKV_ERR_CUDA;
}

}  // namespace

}  // namespace xkv

using namespace xkv;

extern "C" {

int xkv_rope_plan_init(const xkv_rope_config* cfg, xkv_rope_plan* plan) { return rope_plan_init(cfg, plan); }

int xkv_rope(const xkv_rope_plan* plan, int direction, int type, const xkv_rope_tensor* tensors, int n_tensors, int64_t rows,
             const int32_t* pos, int64_t n_pos, void* stream) {
  if (!plan || plan->struct_size != sizeof(xkv_rope_plan) || !tensors || n_tensors < 1 || n_tensors > 2) return XKV_ERR_INVALID_ARG;
  if (plan->d_h < 2 || plan->d_h > 1024 || plan->d_h % 2 || plan->rot < 2 || plan->rot % 2 || plan->rot > plan->d_h ||
      plan->rot > XKV_ROPE_MAX_ROT || (plan->layout != XKV_ROPE_HALF && plan->layout != XKV_ROPE_INTERLEAVED) || !(plan->gain > 0.0f) || isinf(plan->gain) ||
      isinf(1.0f / plan->gain))
    return XKV_ERR_INVALID_ARG;
  if (direction < XKV_ROPE_FORWARD || direction > XKV_ROPE_INVERSE || type < XKV_BF16 || type > XKV_FP32) return XKV_ERR_INVALID_ARG;
  if (rows < 0 || n_pos < 0 || !aligned_to(4, {pos})) return XKV_ERR_INVALID_ARG;
  if (rows > 0 && (n_pos == 0 || rows % n_pos != 0 || !pos)) return XKV_ERR_INVALID_ARG;
  int64_t heads = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const xkv_rope_tensor& t = tensors[i];
    if (t.heads < 0) return XKV_ERR_INVALID_ARG;
    if (t.heads == 0 || rows == 0) continue;
    if (!t.x || !t.y || !aligned_to(type == XKV_FP32 ? 4 : 2, {t.x, t.y})) return XKV_ERR_INVALID_ARG;
    if (t.x == t.y && (t.x_row != t.y_row || t.x_head != t.y_head)) return XKV_ERR_INVALID_ARG;
    if ((double)rows * t.heads >= 2147483648.0) return XKV_ERR_UNSUPPORTED;
    heads += t.heads;
  }
  if (heads >= 2147483648LL - 1024) return XKV_ERR_UNSUPPORTED;               // (a thread steps past the last by its CTA's threads)
  int device = 0;
  const int st = current_sm100_device(&device);
  if (st != XKV_OK) return st;
  return finish8(launch_rope(plan, direction, type, tensors, n_tensors, rows, pos, n_pos, (cudaStream_t)stream));
}

int xkv_page_assign(const xkv_cache8_config* cfg, const int32_t* held, const int32_t* want, int32_t* table, int32_t* ring, int32_t* state,
                    int32_t* first, int32_t* length, int32_t* pos, int32_t* slot, int32_t n_tok, uint32_t* flags, void* stream) {
  int st = check_cache8(cfg);
  if (st != XKV_OK) return st;
  if (!held || !want || !table || !ring || !state || !length || n_tok < 0) return XKV_ERR_INVALID_ARG;
  if (!pos != !slot || (pos && !first) || (!pos && n_tok > 0)) return XKV_ERR_INVALID_ARG;
  if (!aligned_to(4, {held, want, table, ring, state, first, length, pos, slot, flags})) return XKV_ERR_INVALID_ARG;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish8(launch_page_assign(cfg, held, want, table, ring, state, first, length, pos, slot, n_tok, flags, (cudaStream_t)stream));
}

int xkv_cache8_append(const xkv_cache8_config* cfg, int layer_begin, int layer_end, const void* k, const void* v, const int32_t* slot,
                      int32_t n_tok, void* K8, void* V8, float* k_scale, float* v_scale, uint32_t* flags, void* stream) {
  int st = check_layers8(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!k || !v || !slot || !K8 || !V8 || !k_scale || !v_scale || n_tok < 0) return XKV_ERR_INVALID_ARG;
  if (!aligned_to(16, {k, v, K8, V8}) || !aligned_to(4, {slot, k_scale, v_scale, flags})) return XKV_ERR_INVALID_ARG;
  if ((double)n_tok * cfg->H_q * cfg->G >= 2147483648.0) return XKV_ERR_UNSUPPORTED;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  if (n_tok == 0) return XKV_OK;
  return finish8(launch_cache8_append(cfg, layer_begin, layer_end, (const __nv_bfloat16*)k, (const __nv_bfloat16*)v, slot, n_tok, K8, V8,
                                      k_scale, v_scale, flags, (cudaStream_t)stream));
}

int xkv_cache8_read(const xkv_cache8_config* cfg, int layer_begin, int layer_end, const int32_t* table, const int32_t* length, const void* K8,
                    const void* V8, const float* k_scale, const float* v_scale, int32_t cap, void* K, void* V, uint32_t* flags, void* stream) {
  int st = check_layers8(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!table || !length || !K8 || !V8 || !k_scale || !v_scale || (!K && !V) || cap < 1 || cap > XKV_CACHE_MAX_ROWS) return XKV_ERR_INVALID_ARG;
  if (!aligned_to(16, {K8, V8, K, V}) || !aligned_to(4, {table, length, k_scale, v_scale, flags})) return XKV_ERR_INVALID_ARG;
  if ((double)cfg->G * cfg->batch * cfg->H_kv * cap >= 2147483648.0) return XKV_ERR_UNSUPPORTED;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish8(launch_cache8_read(cfg, layer_begin, layer_end, table, length, K8, V8, k_scale, v_scale, cap, (__nv_bfloat16*)K,
                                    (__nv_bfloat16*)V, flags, (cudaStream_t)stream));
}

int xkv_cache8_workspace_bytes(const xkv_cache8_config* cfg, int32_t max_new, uint64_t* bytes) {
  const int st = check_cache8(cfg);
  if (st != XKV_OK) return st;
  if (!bytes || max_new < 1) return XKV_ERR_INVALID_ARG;
  *bytes = cache8_workspace_bytes(cfg, max_new);
  return XKV_OK;
}

int xkv_cache8_attend(const xkv_cache8_config* cfg, int layer_begin, int layer_end, const void* q, const int32_t* first, int32_t n_tok,
                      int32_t max_new, const int32_t* table, const int32_t* length, const void* K8, const void* V8, const float* k_scale,
                      const float* v_scale, void* workspace, uint64_t workspace_bytes, void* out, float* lse, uint32_t* flags, void* stream) {
  int st = check_layers8(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!q || !table || !length || !K8 || !V8 || !k_scale || !v_scale || !workspace || !out) return XKV_ERR_INVALID_ARG;
  if (n_tok < 1 || max_new < 1 || max_new > n_tok || (!first && n_tok != cfg->batch)) return XKV_ERR_INVALID_ARG;
  if (!aligned_to(16, {q, K8, V8, workspace, out}) || !aligned_to(4, {first, table, length, k_scale, v_scale, lse, flags})) return XKV_ERR_INVALID_ARG;
  if (workspace_bytes < cache8_workspace_bytes(cfg, max_new)) return XKV_ERR_INVALID_ARG;
  if ((double)n_tok * cfg->H_q * cfg->G >= 2147483648.0) return XKV_ERR_UNSUPPORTED;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish8(launch_cache8_attend(cfg, layer_begin, layer_end, (const __nv_bfloat16*)q, first, n_tok, max_new, table, length, K8, V8,
                                      k_scale, v_scale, workspace, (__nv_bfloat16*)out, lse, flags, device, (cudaStream_t)stream));
}

}  // extern "C"
