// C ABI of the 8-bit cache: host-side validation and workspace layout of epicache_kv8_append, epicache_kv8_attention and
// epicache_kv8_evict.  No kernel lives here.
#include <math.h>
#include <string.h>

#include "kv8.h"

namespace epicache {
namespace {

bool misaligned(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15) != 0; }

// What all three calls check.  with_arrays: the cache's arrays have to be there.
int make_kv8_plan(const epicache_params* prm, const epicache_kv8* cache, bool with_arrays, Kv8Plan* out) {
  if (!prm || !cache) return EPICACHE_ERR_INVALID_ARG;
  if (prm->struct_size != sizeof(epicache_params) || cache->struct_size != sizeof(epicache_kv8)) return EPICACHE_ERR_INVALID_ARG;
  if (prm->reserved != 0 || cache->reserved != 0) return EPICACHE_ERR_INVALID_ARG;
  if (prm->n_batch < 1 || prm->n_q_heads < 1 || prm->n_kv_heads < 1 || prm->head_dim < 1 || prm->n_cached < 0 ||
      prm->n_block < 0 || cache->capacity < 1)
    return EPICACHE_ERR_INVALID_ARG;
  if (prm->n_q_heads % prm->n_kv_heads != 0) return EPICACHE_ERR_INVALID_ARG;
  if (prm->dtype != EPICACHE_DTYPE_F32 && prm->dtype != EPICACHE_DTYPE_BF16) return EPICACHE_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)prm->n_cached + prm->n_block;
  if (rows < 1 || rows > cache->capacity) return EPICACHE_ERR_INVALID_ARG;
  int shift = 4;
  while (shift < 7 && cache->block_tokens != 1 << shift) shift++;
  if (cache->block_tokens != 1 << shift) return EPICACHE_ERR_INVALID_ARG;

  const int64_t nb = prm->n_batch, Hkv = prm->n_kv_heads, d = prm->head_dim, capacity = cache->capacity;
  const int64_t strides[7] = {cache->stride_b, cache->stride_h, cache->stride_t, cache->scale_stride_b, cache->scale_stride_h,
                              cache->row_stride_b, cache->row_stride_h};
  for (int i = 0; i < 7; i++)
    if (strides[i] < 0) return EPICACHE_ERR_INVALID_ARG;
  if (cache->stride_b % 16 != 0 || cache->stride_h % 16 != 0 || cache->stride_t % 16 != 0) return EPICACHE_ERR_INVALID_ARG;
  // rows of one array must not overlap; a stride of an axis of one is not looked at
  auto holds = [&](int64_t sb, int64_t sh, int64_t span) {
    if (Hkv > 1 && sh < span) return false;
    return nb == 1 || sb >= sh * (Hkv - 1) + span;
  };
  if (capacity > 1 && cache->stride_t < d) return EPICACHE_ERR_INVALID_ARG;
  if (cache->stride_t > (1 << 20)) return EPICACHE_ERR_UNSUPPORTED;
  if (!holds(cache->stride_b, cache->stride_h, cache->stride_t * (capacity - 1) + d)) return EPICACHE_ERR_INVALID_ARG;
  if (!holds(cache->scale_stride_b, cache->scale_stride_h, (capacity + cache->block_tokens - 1) / cache->block_tokens))
    return EPICACHE_ERR_INVALID_ARG;
  if ((cache->weight || cache->position) && !holds(cache->row_stride_b, cache->row_stride_h, capacity))
    return EPICACHE_ERR_INVALID_ARG;
  if (d % 16 != 0 || d > 256) return EPICACHE_ERR_UNSUPPORTED;
  if (capacity > (1 << 24)) return EPICACHE_ERR_UNSUPPORTED;
  if (nb * Hkv > 65535) return EPICACHE_ERR_UNSUPPORTED;
  if (with_arrays) {
    if (!cache->k || !cache->v || cache->k == cache->v || !cache->k_scale || !cache->v_scale || cache->k_scale == cache->v_scale)
      return EPICACHE_ERR_INVALID_ARG;
    const void* arrays[6] = {cache->k, cache->v, cache->k_scale, cache->v_scale, cache->weight, cache->position};
    for (int i = 0; i < 6; i++)
      if (misaligned(arrays[i])) return EPICACHE_ERR_INVALID_ARG;
  }

  Kv8Plan pl;
  memset(&pl, 0, sizeof(pl));
  pl.k = static_cast<uint8_t*>(cache->k), pl.v = static_cast<uint8_t*>(cache->v);
  pl.k_scale = cache->k_scale, pl.v_scale = cache->v_scale;
  pl.weight = cache->weight, pl.position = cache->position;
  pl.sb = cache->stride_b, pl.sh = cache->stride_h, pl.st = cache->stride_t;
  pl.ssb = cache->scale_stride_b, pl.ssh = cache->scale_stride_h;
  pl.rsb = cache->row_stride_b, pl.rsh = cache->row_stride_h;
  pl.nb = prm->n_batch, pl.Hq = prm->n_q_heads, pl.Hkv = prm->n_kv_heads, pl.G = pl.Hq / pl.Hkv;
  pl.d = prm->head_dim;
  pl.block_shift = shift;
  pl.n_cached = prm->n_cached, pl.n_block = prm->n_block;
  pl.dtype = prm->dtype;
  pl.p = 1, pl.R = pl.G, pl.inv_p = 1.f;
  pl.heads_magic = (uint32_t)(((uint64_t(1) << 32) + pl.Hkv - 1) / pl.Hkv);
  *out = pl;
  return EPICACHE_OK;
}

// The query side of epicache_kv8_attention.
int add_queries(const epicache_params* prm, Kv8Plan* pl) {
  if (prm->patch_len < 1) return EPICACHE_ERR_INVALID_ARG;
  if (!(prm->softmax_scale >= 0.0f) || isinf(prm->softmax_scale)) return EPICACHE_ERR_INVALID_ARG;
  if (prm->causal_patch != 0 && prm->causal_patch != 1) return EPICACHE_ERR_INVALID_ARG;
  if (prm->causal_patch && prm->patch_len != prm->n_block) return EPICACHE_ERR_INVALID_ARG;
  const int64_t p = prm->patch_len, d = prm->head_dim, Hq = prm->n_q_heads;
  const int64_t strides[3] = {prm->q_stride_b, prm->q_stride_h, prm->q_stride_t};
  for (int i = 0; i < 3; i++)
    if (strides[i] < 0 || strides[i] % 8 != 0) return EPICACHE_ERR_INVALID_ARG;
  if (p > 1 && prm->q_stride_t < d) return EPICACHE_ERR_INVALID_ARG;
  const int64_t span = prm->q_stride_t * (p - 1) + d;
  if (Hq > 1 && prm->q_stride_h < span) return EPICACHE_ERR_INVALID_ARG;
  if (prm->n_batch > 1 && prm->q_stride_b < prm->q_stride_h * (Hq - 1) + span) return EPICACHE_ERR_INVALID_ARG;
  if (prm->softmax_scale > 1.0e6f) return EPICACHE_ERR_UNSUPPORTED;
  if (prm->q_stride_t > (1 << 20)) return EPICACHE_ERR_UNSUPPORTED;
  if (p * pl->G > (1 << 20)) return EPICACHE_ERR_UNSUPPORTED;                    // rows of a KV head, exact in a float
  if (p * Hq * prm->n_batch > INT32_MAX) return EPICACHE_ERR_UNSUPPORTED;        // rows of all heads
  pl->p = prm->patch_len, pl->R = pl->G * pl->p;
  pl->inv_p = 1.0f / (float)pl->p;
  pl->causal = prm->causal_patch;
  pl->qsb = prm->q_stride_b, pl->qsh = prm->q_stride_h, pl->qst = prm->q_stride_t;
  const float scale = prm->softmax_scale > 0.0f ? prm->softmax_scale : 1.0f / sqrtf((float)pl->d);
  pl->c2 = scale * 1.44269504088896340736f;
  return EPICACHE_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? EPICACHE_OK : EPICACHE_ERR_DEVICE; }

}  // namespace
}  // namespace epicache

using namespace epicache;

extern "C" {

int epicache_kv8_workspace_size(const epicache_params* prm, const epicache_kv8* cache, size_t* bytes_out) {
  Kv8Plan pl;
  int st = make_kv8_plan(prm, cache, false, &pl);
  if (st != EPICACHE_OK) return st;
  if (!bytes_out) return EPICACHE_ERR_INVALID_ARG;
  st = add_queries(prm, &pl);
  if (st != EPICACHE_OK) return st;
  if (prm->budget < 1) return EPICACHE_ERR_INVALID_ARG;
  pl.budget = prm->budget;
  pl.accumulate = 1;
  const size_t attention = kv8_attention_workspace(pl), evict = kv8_evict_workspace(pl);
  *bytes_out = attention > evict ? attention : evict;
  return EPICACHE_OK;
}

int epicache_kv8_append(const epicache_params* prm, const epicache_kv8* cache, const void* k_new, const void* v_new,
                        const int32_t* n_ctx_opt, const int32_t* first_position_opt, void* hip_stream) {
  Kv8Plan pl;
  int st = make_kv8_plan(prm, cache, true, &pl);
  if (st != EPICACHE_OK) return st;
  const int64_t strides[3] = {prm->kv_stride_b, prm->kv_stride_h, prm->kv_stride_t};
  for (int i = 0; i < 3; i++)
    if (strides[i] < 0 || strides[i] % 8 != 0) return EPICACHE_ERR_INVALID_ARG;  // rows may be read more than once
  if (pl.n_block == 0) return EPICACHE_OK;
  if (!k_new || !v_new || misaligned(k_new) || misaligned(v_new) || misaligned(n_ctx_opt) || misaligned(first_position_opt))
    return EPICACHE_ERR_INVALID_ARG;
  pl.nsb = prm->kv_stride_b, pl.nsh = prm->kv_stride_h, pl.nst = prm->kv_stride_t;
  pl.n_ctx = n_ctx_opt;
  return status_of(launch_kv8_append(pl, k_new, v_new, first_position_opt, (hipStream_t)hip_stream));
}

int epicache_kv8_attention(const epicache_params* prm, const epicache_kv8* cache, const void* q, const int32_t* n_ctx_opt,
                           int32_t accumulate, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  Kv8Plan pl;
  int st = make_kv8_plan(prm, cache, true, &pl);
  if (st == EPICACHE_OK) st = add_queries(prm, &pl);
  if (st != EPICACHE_OK) return st;
  if ((accumulate != 0 && accumulate != 1) || (accumulate && !cache->weight)) return EPICACHE_ERR_INVALID_ARG;
  if (!q || !out || !lse_out || misaligned(q) || misaligned(out) || misaligned(lse_out) || misaligned(n_ctx_opt) ||
      misaligned(workspace))
    return EPICACHE_ERR_INVALID_ARG;
  pl.n_ctx = n_ctx_opt;
  pl.accumulate = accumulate;
  const size_t need = kv8_attention_workspace(pl);
  if (need > 0 && !workspace) return EPICACHE_ERR_INVALID_ARG;
  if (workspace_bytes < need) return EPICACHE_ERR_WORKSPACE_TOO_SMALL;
  return status_of(launch_kv8_attention(pl, q, out, lse_out, workspace, (hipStream_t)hip_stream));
}

int epicache_kv8_evict(const epicache_params* prm, const epicache_kv8* cache, int32_t n_recent, const int32_t* n_ctx_opt,
                       const int32_t* budgets_opt, int32_t* n_kept, int32_t* row_from_opt, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  Kv8Plan pl;
  const int st = make_kv8_plan(prm, cache, true, &pl);
  if (st != EPICACHE_OK) return st;
  if (prm->budget < 1 || n_recent < 0 || n_recent > prm->budget || !cache->weight) return EPICACHE_ERR_INVALID_ARG;
  if (!n_kept || !workspace || misaligned(n_kept) || misaligned(workspace) || misaligned(n_ctx_opt) ||
      misaligned(budgets_opt) || misaligned(row_from_opt))
    return EPICACHE_ERR_INVALID_ARG;
  pl.n_ctx = n_ctx_opt;
  pl.budget = prm->budget;
  pl.n_recent = n_recent;
  if (workspace_bytes < kv8_evict_workspace(pl)) return EPICACHE_ERR_WORKSPACE_TOO_SMALL;
  return status_of(launch_kv8_evict(pl, budgets_opt, n_kept, row_from_opt, workspace, (hipStream_t)hip_stream));
}

}  // extern "C"
