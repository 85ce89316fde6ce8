// C entry points of the operators over an uncompressed cache: argument checking and dispatch.
#include <math.h>

#include <atomic>

#include "xkv_internal.cuh"

namespace xkv {

static std::atomic<unsigned int> g_inject{0};
unsigned int cache_fault_injection() { return g_inject.load(std::memory_order_relaxed); }

namespace {

int check_cache(const xkv_cache_config* c) {
  if (!c || c->struct_size != sizeof(xkv_cache_config)) return XKV_ERR_INVALID_ARG;
  if (c->G < 1 || c->batch < 1 || c->H_kv < 1 || c->H_q < 1 || c->H_q % c->H_kv != 0 || c->H_q / c->H_kv > kMaxRep) return XKV_ERR_INVALID_ARG;
  if (c->d_h != 64 && c->d_h != 128) return XKV_ERR_INVALID_ARG;
  if (c->cap < 1 || c->cap > XKV_CACHE_MAX_ROWS) return XKV_ERR_INVALID_ARG;
  if (!(c->softmax_scale >= 0.0f) || isinf(c->softmax_scale)) return XKV_ERR_INVALID_ARG;
  // problems are a grid dimension, rows a 32-bit coordinate of the copy engine (and with at most 32 blocks of query rows for each of a
  // head's tiles, lists of tiles are below 2^31 then, too)
  const double heads = (double)c->G * c->batch * c->H_kv;
  if (heads > 65535.0 || heads * c->cap >= 2147483648.0) return XKV_ERR_UNSUPPORTED;
  return XKV_OK;
}

int check_layers(const xkv_cache_config* c, int l0, int l1) {
  const int st = check_cache(c);
  if (st != XKV_OK) return st;
  return l0 < 0 || l1 > c->G || l0 >= l1 ? XKV_ERR_INVALID_ARG : XKV_OK;
}

template <typename... P>
bool aligned(unsigned to, const P*... p) {
  return ((... | (uintptr_t)p) & (to - 1u)) == 0;
}

int finish(cudaError_t e) {
  if (e == cudaSuccess) return XKV_OK;
  set_cuda_error(e);
  (void)cudaGetLastError();
  return XKV_ERR_CUDA;
}

}  // namespace

}  // namespace xkv

using namespace xkv;

extern "C" {

int xkv_tree_workspace_bytes(const xkv_cache_config* cfg, int32_t n_draft, uint64_t* bytes) {
  const int st = check_cache(cfg);
  if (st != XKV_OK) return st;
  if (!bytes || n_draft < 1 || n_draft > XKV_TREE_MAX_DRAFT) return XKV_ERR_INVALID_ARG;
  *bytes = (uint64_t)tree_part_floats(cfg, n_draft) * sizeof(float);
  return XKV_OK;
}

int xkv_tree_attend(const xkv_cache_config* cfg, int layer_begin, int layer_end, const void* q, int32_t n_draft, const uint32_t* mask,
                    const int32_t* draft_len, const void* K, const void* V, const int32_t* len, void* workspace,
                    uint64_t workspace_bytes, void* out, float* lse, uint32_t* flags, void* stream) {
  int st = check_layers(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!q || !K || !V || !workspace || !out || n_draft < 1 || n_draft > XKV_TREE_MAX_DRAFT || n_draft > cfg->cap) return XKV_ERR_INVALID_ARG;
  if (!aligned(16, (const char*)q, (const char*)K, (const char*)V, (const char*)workspace, (const char*)out) ||
      !aligned(4, mask, draft_len, len, lse, flags))
    return XKV_ERR_INVALID_ARG;
  if (workspace_bytes < (uint64_t)tree_part_floats(cfg, n_draft) * sizeof(float)) return XKV_ERR_INVALID_ARG;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish(launch_tree_attend(cfg, layer_begin, layer_end, (const __nv_bfloat16*)q, n_draft, mask, draft_len, (const __nv_bfloat16*)K,
                                   (const __nv_bfloat16*)V, len, (float*)workspace, (__nv_bfloat16*)out, lse, flags, device, (cudaStream_t)stream));
}

int xkv_tree_commit(const xkv_cache_config* cfg, int layer_begin, int layer_end, void* K, void* V, const int32_t* len, const int32_t* path,
                    const int32_t* path_len, int32_t n_path, int32_t* pos, const int32_t* first_pos, uint32_t* flags, void* stream) {
  int st = check_layers(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!K || !V || !len || !path || n_path < 1 || n_path > XKV_TREE_MAX_DRAFT || (pos && !first_pos)) return XKV_ERR_INVALID_ARG;
  if (!aligned(16, (const char*)K, (const char*)V) || !aligned(4, len, path, path_len, pos, first_pos, flags)) return XKV_ERR_INVALID_ARG;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish(launch_tree_commit(cfg, layer_begin, layer_end, (__nv_bfloat16*)K, (__nv_bfloat16*)V, len, path, path_len, n_path, pos,
                                   first_pos, flags, (cudaStream_t)stream));
}

int xkv_cache_weigh(const xkv_cache_config* cfg, int layer_begin, int layer_end, const void* q, int32_t n_tok, const float* lse, const void* K,
                    const int32_t* len, const int32_t* visible, const int32_t* seen, float decay, float* weights, uint32_t* flags, void* stream) {
  int st = check_layers(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!q || !lse || !K || !weights || n_tok < 1 || n_tok > XKV_TREE_MAX_DRAFT || !(decay >= 0.0f && decay <= 1.0f)) return XKV_ERR_INVALID_ARG;
  if (!aligned(16, (const char*)q, (const char*)K) || !aligned(4, lse, len, visible, seen, weights, flags)) return XKV_ERR_INVALID_ARG;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish(launch_cache_weigh(cfg, layer_begin, layer_end, (const __nv_bfloat16*)q, n_tok, lse, (const __nv_bfloat16*)K, len, visible,
                                   seen, decay, weights, flags, device, (cudaStream_t)stream));
}

int xkv_evict_select(const xkv_cache_config* cfg, int layer_begin, int layer_end, const float* weights, const int32_t* pos,
                     const int32_t* since, const int32_t* len, int32_t keep, int32_t* src, uint32_t* flags, void* stream) {
  int st = check_layers(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!weights || !src || keep < 1 || keep > cfg->cap) return XKV_ERR_INVALID_ARG;
  if (!aligned(4, weights, pos, since, len, src, flags)) return XKV_ERR_INVALID_ARG;
  if (cfg->cap > XKV_EVICT_MAX_ROWS) return XKV_ERR_UNSUPPORTED;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish(launch_evict_select(cfg, layer_begin, layer_end, weights, pos, since, len, keep, src, flags, device, (cudaStream_t)stream));
}

int xkv_evict_compact(const xkv_cache_config* cfg, int layer_begin, int layer_end, void* K, void* V, const int32_t* src, int32_t keep,
                      float* weights, int32_t* pos, uint32_t* flags, void* stream) {
  int st = check_layers(cfg, layer_begin, layer_end);
  if (st != XKV_OK) return st;
  if (!K || !V || !src || keep < 1 || keep > cfg->cap) return XKV_ERR_INVALID_ARG;
  if (!aligned(16, (const char*)K, (const char*)V) || !aligned(4, src, weights, pos, flags)) return XKV_ERR_INVALID_ARG;
  int device = 0;
  if ((st = current_sm100_device(&device)) != XKV_OK) return st;
  return finish(launch_evict_compact(cfg, layer_begin, layer_end, (__nv_bfloat16*)K, (__nv_bfloat16*)V, src, keep, weights, pos, flags,
                                     (cudaStream_t)stream));
}

int xkv_debug_set_cache_fault_injection(uint32_t mask) {
  if (mask & ~(XKV_INJECT_CACHE_NO_LOAD | XKV_INJECT_CACHE_NO_HANDOVER)) return XKV_ERR_INVALID_ARG;
  g_inject.store(mask, std::memory_order_relaxed);
  return XKV_OK;
}

}  // extern "C"
