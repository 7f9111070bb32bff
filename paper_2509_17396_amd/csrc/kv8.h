// The 8-bit cache (include/epicache.h, epicache_kv8): what its launchers take, and the e4m3 codes and scales on the device.
#pragma once

#include "epicache_internal.h"

namespace epicache {

struct Kv8Plan {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  float* weight;      // null: none
  int32_t* position;  // null: none
  int64_t sb, sh, st;      // codes, bytes
  int64_t ssb, ssh;        // scales
  int64_t rsb, rsh;        // weight, position
  int64_t qsb, qsh, qst;   // queries, elements
  int64_t nsb, nsh, nst;   // new rows, elements
  const int32_t* n_ctx;    // null: n_cached everywhere
  int nb, Hq, Hkv, G, d, p;
  int R;                   // query rows of a KV head: G * p
  int block_shift;         // block_tokens = 1 << block_shift
  int n_cached, n_block, budget, n_recent;
  int dtype, causal, accumulate;
  uint32_t heads_magic;    // as Plan's
  float inv_p;
  float c2;                // softmax scale * log2(e)
};

__device__ __forceinline__ int kv8_batch_of(const Kv8Plan& pl, int bh) {
  return pl.Hkv == 1 ? bh : (int)__umulhi((uint32_t)bh, pl.heads_magic);
}
__device__ __forceinline__ int kv8_old_rows(const Kv8Plan& pl, int bh) {
  if (!pl.n_ctx) return pl.n_cached;
  const int n = pl.n_ctx[bh];
  return n < 0 ? 0 : n > pl.n_cached ? pl.n_cached : n;
}

// Largest number of rows that evict leaves a head.
inline int kv8_most_kept(const Kv8Plan& pl) {
  const int rows = pl.n_cached + pl.n_block;
  return pl.budget < rows ? pl.budget : rows;
}

hipError_t launch_kv8_append(const Kv8Plan& pl, const void* k_new, const void* v_new, const int32_t* first_position,
                             hipStream_t stream);
size_t kv8_attention_workspace(const Kv8Plan& pl);
hipError_t launch_kv8_attention(const Kv8Plan& pl, const void* q, void* out, float* lse, void* workspace, hipStream_t stream);
size_t kv8_evict_workspace(const Kv8Plan& pl);
hipError_t launch_kv8_evict(const Kv8Plan& pl, const int32_t* budgets, int32_t* n_kept, int32_t* row_from, void* workspace,
                            hipStream_t stream);

// ---- codes and scales

typedef __attribute__((ext_vector_type(2))) float kv8_f32x2;

constexpr uint32_t kNanCode = 0x7f;

// The smallest power of two, at least 2^-126, by which `amax` (finite) becomes at most 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float((uint32_t)(max(e, -126) + 127) << 23);
}

__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Four codes of values of at most 448 in magnitude; not finite: the NaN code.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  u = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true);
  if (!(is_finite(a) && is_finite(b) && is_finite(c) && is_finite(d))) {
    const float x[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (!is_finite(x[i])) u = (u & ~(0xff << 8 * i)) | (int)(kNanCode << 8 * i);
  }
  return (uint32_t)u;
}

__device__ __forceinline__ void decode4(uint32_t u, float* x) {
  const kv8_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
  x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
}

}  // namespace epicache
