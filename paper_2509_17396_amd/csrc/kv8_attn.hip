// Attention over the 8-bit cache (epicache_kv8_attention).
#include <hip/hip_bf16.h>

#include <algorithm>
#include <type_traits>

#include "kv8.h"
#include "mfma_tiles.h"

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

// ---- Few query rows per KV head (decoding): every wave streams its own keys through registers.

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kTokenRows = 32;  // of a KV head, at most
// Two tiles of rows beside a step's keys fit the registers where head_dim is at most 128.
bool few_rows(const Kv8Plan& pl) { return pl.R <= (pl.d <= 128 ? kTokenRows : 16); }
constexpr int kMostSplits = 64;
constexpr int kTokenWaves = 4, kTokenKeys = 32;  // waves of a workgroup; keys of a wave's step
constexpr float kLazyBits = 8.f;
constexpr float kNoKey = -1.0e30f;  // the reference of a row that has seen no key

// Room in the workspace.  splits workgroups share the keys of a head.
struct TokenRoom {
  int splits, logit_pitch;
  float2* stats;   // [heads][splits][R]: reference and sum
  float* records;  // [heads][splits][R][d], where there are several splits: outputs before the division
  float* logits;   // [heads][R][logit_pitch], where weights are accumulated: in base 2
};

// Two fp32 values as bf16 parts whose sum they are, to 8 bits per part: truncated, then what is left.
template <int PARTS>
__device__ __forceinline__ void cut_pair(uint32_t (&p)[PARTS], float a, float b) {
#pragma unroll
  for (int i = 0; i < PARTS; i++) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    p[i] = __builtin_amdgcn_perm(ub, ua, 0x07060302);  // the upper halves, b's above a's
    a -= __uint_as_float(ua & 0xffff0000u), b -= __uint_as_float(ub & 0xffff0000u);
  }
}

// e4m3 codes 2 i, 2 i + 1 of a dword as bf16, which holds them exactly.
template <int HIGH>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t u) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HIGH != 0));
}
__device__ __forceinline__ bf16x8 codes_to_frag(uint32_t lo, uint32_t hi) {
  const u32x4 u = {codes_to_bf16<0>(lo), codes_to_bf16<1>(lo), codes_to_bf16<0>(hi), codes_to_bf16<1>(hi)};
  return __builtin_bit_cast(bf16x8, u);
}
__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The query row of a lane as operand parts: 16-value chunks g, g + 4, .. of the row, two steps of 8 values each; zeros behind d.
template <int NCH>
__device__ __forceinline__ void load_query(bf16x8 (&f)[1][2 * NCH], const __hip_bfloat16* row, int g, int d, bool ok) {
#pragma unroll
  for (int c = 0; c < NCH; c++) {
    const int at = (4 * c + g) * 16;
    uint4 u[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (ok && at < d) u[0] = reinterpret_cast<const uint4*>(row + at)[0], u[1] = reinterpret_cast<const uint4*>(row + at)[1];
    f[0][2 * c] = __builtin_bit_cast(bf16x8, u[0]), f[0][2 * c + 1] = __builtin_bit_cast(bf16x8, u[1]);
  }
}
template <int NCH>
__device__ __forceinline__ void load_query(bf16x8 (&f)[3][2 * NCH], const float* row, int g, int d, bool ok) {
#pragma unroll
  for (int c = 0; c < NCH; c++)
#pragma unroll
    for (int s = 0; s < 2; s++) {
      const int at = (4 * c + g) * 16 + 8 * s;
      float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (ok && at < d) {
        const float4 a = reinterpret_cast<const float4*>(row + at)[0], b = reinterpret_cast<const float4*>(row + at)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
      }
      u32x4 u[3];
#pragma unroll
      for (int j = 0; j < 4; j++) {
        uint32_t p[3];
        cut_pair<3>(p, x[2 * j], x[2 * j + 1]);
        // nothing is left of an infinity or a NaN, and a NaN stays one
#pragma unroll
        for (int e = 0; e < 2; e++) {
          const float y = x[2 * j + e];
          if (is_finite(y)) continue;
          const uint32_t top = (y != y ? 0x7fc0u : __float_as_uint(y) >> 16) << 16 * e, keep = e ? 0xffffu : 0xffff0000u;
          p[0] = (p[0] & keep) | top, p[1] &= keep, p[2] &= keep;
        }
#pragma unroll
        for (int i = 0; i < 3; i++) u[i][j] = p[i];
      }
#pragma unroll
      for (int i = 0; i < 3; i++) f[i][2 * c + s] = __builtin_bit_cast(bf16x8, u[i]);
    }
}

__device__ __forceinline__ void store4(__hip_bfloat16* to, const float (&x)[4]) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  uint2 u;
  u.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2));
  u.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2], x[3]}), bf16x2));
  *reinterpret_cast<uint2*>(to) = u;
}
__device__ __forceinline__ void store4(float* to, const float (&x)[4]) { *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]); }

// What a step of 32 keys reads.  K: lane (m, g) has chunks g, g + 4, .. of keys m and 16 + m.  V: of the keys 4 g + i and 16 + 4 g + i
// that the lane will hold weights of, the dwords at its columns.
template <int NCH>
struct Step {
  uint4 k[2][NCH];
  uint32_t v[8][NCH];
  float ks[2], vs[2];
};

// NaN codes of V in a step that some rows see and others do not: the rows that see one get a NaN in its column, and the code is
// taken out, since a weight of 0 times it would make one of the others' columns too.  Whether a row sees one is a product of
// zeros and ones.
template <int NCH, int NR>
__device__ __forceinline__ void not_numbers(Step<NCH>& s, f32x4 (&acc)[NR][4 * NCH], int key0, int g, const int (&last)[NR]) {
  auto nan_bytes = [](uint32_t u) { return ((u & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };  // 0x80 where the byte is 0x7f or 0xff
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 8; i++)
#pragma unroll
    for (int c = 0; c < NCH; c++) any |= nan_bytes(s.v[i][c]);
  if (!__any(any != 0)) return;
  bf16x8 sees[NR];
#pragma unroll
  for (int r = 0; r < NR; r++) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int key = key0 + (i >> 1) * 16 + 4 * g + 2 * (i & 1);
      u[i] = (key <= last[r] ? 0x3f80u : 0u) | (key + 1 <= last[r] ? 0x3f800000u : 0u);
    }
    sees[r] = __builtin_bit_cast(bf16x8, u);
  }
#pragma unroll
  for (int c = 0; c < NCH; c++) {
    uint32_t is[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
      is[i] = nan_bytes(s.v[i][c]);
      s.v[i][c] &= ~(is[i] | (is[i] - (is[i] >> 7)));  // 0x80 makes 0xff
    }
#pragma unroll
    for (int j = 0; j < 4; j++) {
      u32x4 u;
#pragma unroll
      for (int i = 0; i < 4; i++)
        u[i] = ((is[2 * i] >> (8 * j + 7)) & 1 ? 0x3f80u : 0u) | ((is[2 * i + 1] >> (8 * j + 7)) & 1 ? 0x3f800000u : 0u);
#pragma unroll
      for (int r = 0; r < NR; r++) {
        const f32x4 seen = mfma16(__builtin_bit_cast(bf16x8, u), sees[r], f32x4{0, 0, 0, 0});
#pragma unroll
        for (int i = 0; i < 4; i++) acc[r][4 * c + j][i] += seen[i] > 0.f ? NAN : 0.f;
      }
    }
  }
}

// EXACT: d = 64 NCH; a lane's columns of V are then 4 NCH neighbouring ones, else 4 of every 64.
// Waves per SIMD that the registers are cut for.
constexpr int token_occupancy(size_t elem, int chunks) { return chunks <= 2 ? (elem == 4 ? 2 : 3) : elem == 4 && chunks > 3 ? 1 : 2; }

template <typename T, int NCH, bool EXACT, int NR>
__global__ __launch_bounds__(kTokenWaves * 64, token_occupancy(sizeof(T), NCH * NR)) void kv8_attention_tokens(Kv8Plan pl, const T* __restrict__ q, T* __restrict__ out,
                                                                        float* __restrict__ lse, TokenRoom room) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : 2;
  constexpr int NT = 4 * NCH;  // 16-column tiles of the output
  __shared__ float merged_acc[kTokenWaves / 2][NT * 4][64];
  __shared__ float2 merged_ml[kTokenWaves][16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m16 = lane & 15, g = lane >> 4;
  const int bh = blockIdx.y, split = blockIdx.x, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int old = kv8_old_rows(pl, bh), n = old + pl.n_block;
  const int all_see = pl.causal ? old + 1 : n;  // keys that every row sees (all, of a decoding step)
  const int tiles = (n + kTokenKeys - 1) / kTokenKeys;
  const int per_split = (tiles + room.splits - 1) / room.splits;
  const int end = min(tiles, (split + 1) * per_split);

  const uint8_t* kbase = pl.k + b * pl.sb + h * pl.sh;
  const uint8_t* vbase = pl.v + b * pl.sb + h * pl.sh;
  const float* ks = pl.k_scale + b * pl.ssb + h * pl.ssh;
  const float* vs = pl.v_scale + b * pl.ssb + h * pl.ssh;
  const uint32_t pitch = (uint32_t)pl.st;
  const int last_chunk = (pl.d >> 4) - 1;
  auto chunk_of = [&](int c) { return EXACT ? 4 * c + g : min(4 * c + g, last_chunk); };
  auto column_of = [&](int c) { return EXACT ? 4 * NCH * m16 + 4 * c : min(64 * c + 4 * m16, pl.d - 4); };

  int last[NR];
  int64_t orow[NR];
  bool ok[NR];
  bf16x8 qf[NR][QP][2 * NCH];
#pragma unroll
  for (int r = 0; r < NR; r++) {
    const int row = r * 16 + m16;
    ok[r] = row < pl.R;
    int gr, t;
    head_and_token(pl.p, pl.inv_p, min(row, pl.R - 1), gr, t);
    last[r] = pl.causal ? old + t : n - 1;
    orow[r] = ((int64_t)b * pl.Hq + h * pl.G + gr) * pl.p + t;
    load_query<NCH>(qf[r], q + b * pl.qsb + (int64_t)(h * pl.G + gr) * pl.qsh + (int64_t)t * pl.qst, g, pl.d, ok[r]);
  }

  f32x4 acc[NR][NT];
  float m[NR], l[NR];
#pragma unroll
  for (int r = 0; r < NR; r++) {
    m[r] = kNoKey, l[r] = 0.f;
#pragma unroll
    for (int j = 0; j < NT; j++) acc[r][j] = f32x4{0, 0, 0, 0};
  }

  auto load = [&](Step<NCH>& s, int tile) {
    const int key0 = tile * kTokenKeys;
#pragma unroll
    for (int a = 0; a < 2; a++) {
      const int block = min(key0 + 16 * a, n - 1) >> pl.block_shift;
      s.ks[a] = ks[block], s.vs[a] = vs[block];
    }
    if (key0 + kTokenKeys <= n) {
      const uint8_t* kt = kbase + (int64_t)key0 * pitch;
      const uint8_t* vt = vbase + (int64_t)key0 * pitch;
#pragma unroll
      for (int a = 0; a < 2; a++)
#pragma unroll
        for (int c = 0; c < NCH; c++)
          s.k[a][c] = *reinterpret_cast<const uint4*>(kt + (16 * a + m16) * pitch + chunk_of(c) * 16);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const uint8_t* row = vt + ((i >> 2) * 16 + 4 * g + (i & 3)) * pitch;
#pragma unroll
        for (int c = 0; c < NCH; c++) s.v[i][c] = *reinterpret_cast<const uint32_t*>(row + column_of(c));
      }
    } else {  // rows behind the last one: K of the last one again, V 0
#pragma unroll
      for (int a = 0; a < 2; a++)
#pragma unroll
        for (int c = 0; c < NCH; c++)
          s.k[a][c] = *reinterpret_cast<const uint4*>(kbase + (int64_t)min(key0 + 16 * a + m16, n - 1) * pitch + chunk_of(c) * 16);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const int key = key0 + (i >> 2) * 16 + 4 * g + (i & 3);
        const uint8_t* row = vbase + (int64_t)min(key, n - 1) * pitch;
#pragma unroll
        for (int c = 0; c < NCH; c++) {
          const uint32_t u = *reinterpret_cast<const uint32_t*>(row + column_of(c));
          s.v[i][c] = key < n ? u : 0u;
        }
      }
    }
  };

  auto work = [&](Step<NCH>& s, int tile) {
    const int key0 = tile * kTokenKeys;
    const bool masked = key0 + kTokenKeys > all_see;
    // logits, in base 2: lane (query m16, g) has the keys 16 a + 4 g + i
    float x[NR][8];
#pragma unroll
    for (int a = 0; a < 2; a++) {
      f32x4 z[NR];
#pragma unroll
      for (int r = 0; r < NR; r++) z[r] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < NCH; c++) {
        const bf16x8 k0 = codes_to_frag(s.k[a][c].x, s.k[a][c].y), k1 = codes_to_frag(s.k[a][c].z, s.k[a][c].w);
#pragma unroll
        for (int r = 0; r < NR; r++)
#pragma unroll
          for (int part = QP - 1; part >= 0; part--) {
            z[r] = mfma16(k0, qf[r][part][2 * c], z[r]);
            z[r] = mfma16(k1, qf[r][part][2 * c + 1], z[r]);
          }
      }
      const float by = pl.c2 * s.ks[a];
#pragma unroll
      for (int r = 0; r < NR; r++)
#pragma unroll
        for (int i = 0; i < 4; i++) x[r][4 * a + i] = z[r][i] * by;
    }
    if (masked) {
#pragma unroll
      for (int r = 0; r < NR; r++)
#pragma unroll
        for (int i = 0; i < 8; i++)
          if (key0 + (i >> 2) * 16 + 4 * g + (i & 3) > last[r]) x[r][i] = -INFINITY;
    }
    if (room.logits) {
#pragma unroll
      for (int r = 0; r < NR; r++)
        if (ok[r]) {
          float* to = room.logits + ((size_t)bh * pl.R + r * 16 + m16) * room.logit_pitch + key0 + 4 * g;
#pragma unroll
          for (int a = 0; a < 2; a++)
            *reinterpret_cast<float4*>(to + 16 * a) = make_float4(x[r][4 * a], x[r][4 * a + 1], x[r][4 * a + 2], x[r][4 * a + 3]);
        }
    }
    uint32_t pf[NR][PP][4];
#pragma unroll
    for (int r = 0; r < NR; r++) {
      const float top = fmaxf(fmaxf(fmaxf(x[r][0], x[r][1]), fmaxf(x[r][2], x[r][3])),
                              fmaxf(fmaxf(x[r][4], x[r][5]), fmaxf(x[r][6], x[r][7])));
      // The reference follows the maximum lazily: fp32 sums and weights keep their relative precision up to 2^kLazyBits.
      if (__any(top > m[r] + kLazyBits)) {
        float mn = fmaxf(m[r], top);
        mn = fmaxf(mn, __shfl_xor(mn, 16));
        mn = fmaxf(mn, __shfl_xor(mn, 32));
        const float corr = ex2(m[r] - mn);
        l[r] *= corr;
#pragma unroll
        for (int j = 0; j < NT; j++) acc[r][j] *= corr;
        m[r] = mn;
      }
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; i++) e[i] = ex2(x[r][i] - m[r]);
      l[r] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
      for (int i = 0; i < 4; i++) {
        uint32_t p[PP];
        cut_pair<PP>(p, e[2 * i] * s.vs[i >> 1], e[2 * i + 1] * s.vs[i >> 1]);
#pragma unroll
        for (int part = 0; part < PP; part++) pf[r][part][i] = p[part];
      }
    }
    if (masked && pl.causal && pl.p > 1) not_numbers<NCH, NR>(s, acc, key0, g, last);
    // out^T += V^T P^T.  Bytes of one column in four keys: two byte permutations make pairs of keys of two columns each.
#pragma unroll
    for (int c = 0; c < NCH; c++)
#pragma unroll
      for (int half = 0; half < 2; half++) {
        const uint32_t sel = half ? 0x07030602u : 0x05010400u;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = __builtin_amdgcn_perm(s.v[2 * i + 1][c], s.v[2 * i][c], sel);
#pragma unroll
        for (int j = 0; j < 2; j++) {
          const u32x4 u = j == 0 ? u32x4{codes_to_bf16<0>(w[0]), codes_to_bf16<0>(w[1]), codes_to_bf16<0>(w[2]), codes_to_bf16<0>(w[3])}
                                 : u32x4{codes_to_bf16<1>(w[0]), codes_to_bf16<1>(w[1]), codes_to_bf16<1>(w[2]), codes_to_bf16<1>(w[3])};
          const bf16x8 vf = __builtin_bit_cast(bf16x8, u);
#pragma unroll
          for (int r = 0; r < NR; r++)
#pragma unroll
            for (int part = PP - 1; part >= 0; part--) {
              const u32x4 pw = {pf[r][part][0], pf[r][part][1], pf[r][part][2], pf[r][part][3]};
              acc[r][4 * c + 2 * half + j] = mfma16(vf, __builtin_bit_cast(bf16x8, pw), acc[r][4 * c + 2 * half + j]);
            }
        }
      }
  };

  {
    Step<NCH> now, next;
    int tile = split * per_split + wave;
    if (tile < end) load(now, tile);
    for (; tile < end; tile += kTokenWaves) {
      if (tile + kTokenWaves < end) load(next, tile + kTokenWaves);
      work(now, tile);
      now = next;
    }
  }

  // the waves' parts together: lanes of a row first, then the waves
#pragma unroll
  for (int r = 0; r < NR; r++) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    __syncthreads();
    if (lane < 16) merged_ml[wave][lane] = make_float2(m[r], l[r]);
    __syncthreads();
    float mn = kNoKey, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kTokenWaves; w++) mn = fmaxf(mn, merged_ml[w][m16].x);
#pragma unroll
    for (int w = 0; w < kTokenWaves; w++) sum += merged_ml[w][m16].y * ex2(merged_ml[w][m16].x - mn);
    const float corr = ex2(m[r] - mn);
#pragma unroll
    for (int j = 0; j < NT; j++) acc[r][j] *= corr;
    for (int half = kTokenWaves / 2; half >= 1; half >>= 1) {
      if (half < kTokenWaves / 2) __syncthreads();
      if (wave >= half && wave < 2 * half)
#pragma unroll
        for (int j = 0; j < NT; j++)
#pragma unroll
          for (int i = 0; i < 4; i++) merged_acc[wave - half][4 * j + i][lane] = acc[r][j][i];
      __syncthreads();
      if (wave < half)
#pragma unroll
        for (int j = 0; j < NT; j++)
#pragma unroll
          for (int i = 0; i < 4; i++) acc[r][j][i] += merged_acc[wave][4 * j + i][lane];
    }
    if (wave == 0 && ok[r]) {
      const int row = r * 16 + m16;
      const bool whole = room.splits == 1, any = sum > 0.f || sum != sum;
      const float inv = !whole ? 1.f : any ? 1.f / sum : 0.f;
      const size_t record = ((size_t)bh * room.splits + split) * pl.R + row;
      if (g == 0) {
        if (whole) lse[orow[r]] = any ? (mn + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
        if (room.stats) room.stats[record] = make_float2(mn, sum);
      }
#pragma unroll
      for (int c = 0; c < NCH; c++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int column = EXACT ? 4 * NCH * (4 * g + i) + 4 * c : 64 * c + 4 * (4 * g + i);
          if (!EXACT && column >= pl.d) continue;
          float y[4];
#pragma unroll
          for (int j = 0; j < 4; j++) y[j] = any || !whole ? acc[r][4 * c + j][i] * inv : 0.f;
          if (whole) store4(out + orow[r] * pl.d + column, y);
          else store4(room.records + record * pl.d + column, y);
        }
    }
  }
}

// What the splits left, put together: the outputs (blockIdx.x = 0, where there are several splits) and the rows' weights, 1024 keys
// to a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void kv8_join_tokens(Kv8Plan pl, T* __restrict__ out, float* __restrict__ lse, TokenRoom room,
                                                       int out_blocks) {
  __shared__ float2 row_ml[kTokenRows];  // reference and 1 / sum
  const int tid = threadIdx.x, bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int n = kv8_old_rows(pl, bh) + pl.n_block;
  const bool is_out = (int)blockIdx.x < out_blocks;
  const int key = ((int)blockIdx.x - out_blocks) * 1024 + tid * 4;
  if (!is_out && key - tid * 4 >= n) return;
  {  // eight lanes to a row
    const int row = tid >> 3;
    float mn = kNoKey, sum = 0.f;
    if (row < pl.R) {
      const float2* s = room.stats + (size_t)bh * room.splits * pl.R + row;
      for (int i = tid & 7; i < room.splits; i += 8) mn = fmaxf(mn, s[(size_t)i * pl.R].x);
#pragma unroll
      for (int x = 1; x < 8; x <<= 1) mn = fmaxf(mn, __shfl_xor(mn, x));
      for (int i = tid & 7; i < room.splits; i += 8) sum += s[(size_t)i * pl.R].y * ex2(s[(size_t)i * pl.R].x - mn);
#pragma unroll
      for (int x = 1; x < 8; x <<= 1) sum += __shfl_xor(sum, x);
      const bool any = sum > 0.f || sum != sum;
      if ((tid & 7) == 0) {
        row_ml[row] = make_float2(mn, any ? 1.f / sum : 0.f);
        if (is_out && blockIdx.x == 0) {
          int gr, t;
          head_and_token(pl.p, pl.inv_p, row, gr, t);
          lse[((size_t)b * pl.Hq + h * pl.G + gr) * pl.p + t] = any ? (mn + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
        }
      }
    }
  }
  __syncthreads();
  if (is_out) {
    const int per_row = pl.d >> 2;
    for (int at = blockIdx.x * 256 + tid; at < pl.R * per_row; at += out_blocks * 256) {
      const int row = at / per_row, column = (at - row * per_row) * 4;
      const float2 ml = row_ml[row];
      float y[4] = {0, 0, 0, 0};
      if (ml.y != 0.f) {
        for (int s = 0; s < room.splits; s++) {
          const size_t record = ((size_t)bh * room.splits + s) * pl.R + row;
          const float w = ex2(room.stats[record].x - ml.x) * ml.y;
          const float4 a = *reinterpret_cast<const float4*>(room.records + record * pl.d + column);
          y[0] += w * a.x, y[1] += w * a.y, y[2] += w * a.z, y[3] += w * a.w;
        }
      }
      int gr, t;
      head_and_token(pl.p, pl.inv_p, row, gr, t);
      store4(out + (((size_t)b * pl.Hq + h * pl.G + gr) * pl.p + t) * pl.d + column, y);
    }
    return;
  }
  if (key >= n) return;
  float w[4] = {0, 0, 0, 0};
  for (int row = 0; row < pl.R; row++) {
    const float4 x = *reinterpret_cast<const float4*>(room.logits + ((size_t)bh * pl.R + row) * room.logit_pitch + key);
    const float2 ml = row_ml[row];
    if (ml.y == 0.f) continue;
    w[0] += ex2(x.x - ml.x) * ml.y, w[1] += ex2(x.y - ml.x) * ml.y, w[2] += ex2(x.z - ml.x) * ml.y, w[3] += ex2(x.w - ml.x) * ml.y;
  }
  float* to = pl.weight + b * pl.rsb + h * pl.rsh + key;
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (key + i < n) to[i] += w[i];
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Room of the kernel for few rows; null workspace: only its size, in *bytes.
TokenRoom token_room(const Kv8Plan& pl, void* workspace, size_t* bytes) {
  const int64_t heads = (int64_t)pl.nb * pl.Hkv;
  const int tiles = (pl.n_cached + pl.n_block + kTokenKeys - 1) / kTokenKeys;
  // four workgroups for every CU, each with two steps a wave at least
  int64_t splits = (4 * kComputeUnits + heads - 1) / heads;
  splits = std::max<int64_t>(1, std::min<int64_t>({splits, tiles / (2 * kTokenWaves), kMostSplits}));
  TokenRoom room = {(int)splits, tiles * kTokenKeys, nullptr, nullptr, nullptr};
  char* ws = static_cast<char*>(workspace);
  size_t at = 0;
  auto take = [&](size_t n) {
    char* p = ws ? ws + at : nullptr;
    at += align256(n);
    return reinterpret_cast<float*>(p);
  };
  if (splits > 1 || pl.accumulate) room.stats = reinterpret_cast<float2*>(take((size_t)heads * splits * pl.R * sizeof(float2)));
  if (splits > 1) room.records = take((size_t)heads * splits * pl.R * pl.d * sizeof(float));
  if (pl.accumulate) room.logits = take((size_t)heads * pl.R * room.logit_pitch * sizeof(float));
  *bytes = at;
  return room;
}

template <typename T>
hipError_t launch_tokens(const Kv8Plan& pl, const T* q, T* out, float* lse, void* workspace, hipStream_t stream) {
  size_t bytes;
  const TokenRoom room = token_room(pl, workspace, &bytes);
  const int heads = pl.nb * pl.Hkv;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(room.splits, heads), dim3(kTokenWaves * 64), 0, stream, pl, q, out, lse, room);
  };
  auto rows = [&](auto nch, auto exact) {
    constexpr int NCH = decltype(nch)::value;
    constexpr bool EXACT = decltype(exact)::value;
    if constexpr (NCH <= 2)
      if (pl.R > 16) return go(kv8_attention_tokens<T, NCH, EXACT, 2>);
    go(kv8_attention_tokens<T, NCH, EXACT, 1>);
  };
  auto chunks = [&](auto nch) {
    if (pl.d == 64 * decltype(nch)::value) rows(nch, std::true_type{});
    else rows(nch, std::false_type{});
  };
  if (pl.d <= 64) chunks(std::integral_constant<int, 1>{});
  else if (pl.d <= 128) chunks(std::integral_constant<int, 2>{});
  else if (pl.d <= 192) chunks(std::integral_constant<int, 3>{});
  else chunks(std::integral_constant<int, 4>{});
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int out_blocks = room.splits > 1 ? 1 : 0;
  const int key_blocks = pl.accumulate ? (pl.n_cached + pl.n_block + 1023) / 1024 : 0;
  if (out_blocks + key_blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(kv8_join_tokens<T>, dim3(out_blocks + key_blocks, heads), dim3(256), 0, stream, pl, out, lse, room, out_blocks);
  return hipGetLastError();
}

}  // namespace

size_t kv8_attention_workspace(const Kv8Plan& pl) {
  if (few_rows(pl)) {
    size_t bytes;
    token_room(pl, nullptr, &bytes);
    return bytes;
  }
  return pl.accumulate ? (size_t)pl.nb * pl.Hq * pl.p * sizeof(float2) : 0;
}

hipError_t launch_kv8_attention(const Kv8Plan& pl, const void* q, void* out, float* lse, void* workspace, hipStream_t stream) {
  if (few_rows(pl)) {
    if (pl.dtype == EPICACHE_DTYPE_BF16)
      return launch_tokens(pl, static_cast<const __hip_bfloat16*>(q), static_cast<__hip_bfloat16*>(out), lse, workspace, stream);
    return launch_tokens(pl, static_cast<const float*>(q), static_cast<float*>(out), lse, workspace, stream);
  }
  float2* stats = pl.accumulate ? static_cast<float2*>(workspace) : nullptr;
  return pl.dtype == EPICACHE_DTYPE_BF16 ? launch<__hip_bfloat16>(pl, q, out, lse, stats, stream)
                                         : launch<float>(pl, q, out, lse, stats, stream);
}

}  // namespace epicache
