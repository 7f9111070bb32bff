// Attention over the 8-bit cache (epicache_kv8_attention).
#include <hip/hip_bf16.h>

#include "kv8.h"
#include "select_util.h"

namespace epicache {
namespace {

__device__ __forceinline__ float to_float(__hip_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ void put(__hip_bfloat16& to, float x) { to = __float2bfloat16(x); }
__device__ __forceinline__ void put(float& to, float x) { to = x; }

__device__ __forceinline__ float block_reduce(float x, bool is_max, float* lds) {
  for (int s = 32; s >= 1; s >>= 1) {
    const float y = __shfl_xor(x, s);
    x = is_max ? fmaxf(x, y) : x + y;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return is_max ? fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3])) : (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// One workgroup per query: 256 keys at a time, a key per thread for the logits, a column per thread for the output.
template <typename T>
__global__ __launch_bounds__(256) void kv8_attention_rows(Kv8Plan pl, const T* __restrict__ q, T* __restrict__ out,
                                                          float* __restrict__ lse, float2* __restrict__ stats) {
  __shared__ float qs[256], w[256], red[4];
  const int tid = threadIdx.x;
  const size_t orow = blockIdx.x;
  const int t = (int)(orow % pl.p), hq = (int)(orow / pl.p % pl.Hq), b = (int)(orow / pl.p / pl.Hq), h = hq / pl.G;
  const int bh = b * pl.Hkv + h;
  const int old = kv8_old_rows(pl, bh), n = pl.causal ? old + t + 1 : old + pl.n_block;
  const uint8_t* k = pl.k + b * pl.sb + h * pl.sh;
  const uint8_t* v = pl.v + b * pl.sb + h * pl.sh;
  const float* ks = pl.k_scale + b * pl.ssb + h * pl.ssh;
  const float* vs = pl.v_scale + b * pl.ssb + h * pl.ssh;
  if (tid < pl.d) qs[tid] = to_float(q[b * pl.qsb + hq * pl.qsh + t * pl.qst + tid]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc = 0.f;
  for (int k0 = 0; k0 < n; k0 += 256) {
    const int i = k0 + tid;
    float z = -INFINITY;
    if (i < n) {
      float dot = 0.f;
      for (int c = 0; c < pl.d; c += 4) {
        float x[4];
        decode4(*reinterpret_cast<const uint32_t*>(k + (int64_t)i * pl.st + c), x);
        for (int j = 0; j < 4; j++) dot = fmaf(qs[c + j], x[j], dot);
      }
      z = dot * ks[i >> pl.block_shift] * pl.c2;
    }
    const float mn = fmaxf(m, block_reduce(z, true, red));
    const float e = z == -INFINITY ? 0.f : exp2f(z - mn), corr = m == mn ? 1.f : exp2f(m - mn);
    l = l * corr + block_reduce(e, false, red);
    acc *= corr;
    m = mn;
    w[tid] = e;
    __syncthreads();
    if (tid < pl.d)
      for (int j = 0; j < min(256, n - k0); j++) {
        float x[4];
        decode4(v[(int64_t)(k0 + j) * pl.st + tid], x);
        acc = fmaf(w[j] * vs[(k0 + j) >> pl.block_shift], x[0], acc);
      }
    __syncthreads();
  }
  const bool any = l > 0.f || l != l;
  if (tid < pl.d) put(out[orow * pl.d + tid], any ? acc / l : 0.f);
  if (tid == 0) {
    lse[orow] = any ? (m + log2f(l)) * 0.69314718055994530942f : -INFINITY;
    if (stats) stats[orow] = make_float2(m, any ? 1.f / l : 0.f);
  }
}

// weight += the softmax weights, a key per thread, the queries of its head one after the other.
template <typename T>
__global__ __launch_bounds__(256) void kv8_accumulate_keys(Kv8Plan pl, const T* __restrict__ q, const float2* __restrict__ stats) {
  const int bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int old = kv8_old_rows(pl, bh), n = old + pl.n_block, i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const uint8_t* k = pl.k + b * pl.sb + h * pl.sh + (int64_t)i * pl.st;
  const float scale = pl.k_scale[b * pl.ssb + h * pl.ssh + (i >> pl.block_shift)];
  float sum = 0.f;
  for (int r = 0; r < pl.R; r++) {
    const int g = r / pl.p, t = r - g * pl.p;
    if (pl.causal && i > old + t) continue;
    const T* row = q + b * pl.qsb + (h * pl.G + g) * pl.qsh + t * pl.qst;
    float dot = 0.f;
    for (int c = 0; c < pl.d; c += 4) {
      float x[4];
      decode4(*reinterpret_cast<const uint32_t*>(k + c), x);
      for (int j = 0; j < 4; j++) dot = fmaf(to_float(row[c + j]), x[j], dot);
    }
    const float2 s = stats[((size_t)b * pl.Hq + h * pl.G + g) * pl.p + t];
    if (s.y != 0.f) sum += exp2f(dot * scale * pl.c2 - s.x) * s.y;
  }
  pl.weight[b * pl.rsb + h * pl.rsh + i] += sum;
}

template <typename T>
hipError_t launch(const Kv8Plan& pl, const void* q, void* out, float* lse, float2* stats, hipStream_t stream) {
  hipLaunchKernelGGL(kv8_attention_rows<T>, dim3((unsigned)((size_t)pl.nb * pl.Hq * pl.p)), dim3(256), 0, stream, pl,
                     static_cast<const T*>(q), static_cast<T*>(out), lse, stats);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !pl.accumulate) return e;
  hipLaunchKernelGGL(kv8_accumulate_keys<T>, dim3((pl.n_cached + pl.n_block + 255) / 256, pl.nb * pl.Hkv), dim3(256), 0, stream,
                     pl, static_cast<const T*>(q), stats);
  return hipGetLastError();
}

}  // namespace

size_t kv8_attention_workspace(const Kv8Plan& pl) { return pl.accumulate ? (size_t)pl.nb * pl.Hq * pl.p * sizeof(float2) : 0; }

hipError_t launch_kv8_attention(const Kv8Plan& pl, const void* q, void* out, float* lse, void* workspace, hipStream_t stream) {
  float2* stats = pl.accumulate ? static_cast<float2*>(workspace) : nullptr;
  return pl.dtype == EPICACHE_DTYPE_BF16 ? launch<__hip_bfloat16>(pl, q, out, lse, stats, stream)
                                         : launch<float>(pl, q, out, lse, stats, stream);
}

}  // namespace epicache
