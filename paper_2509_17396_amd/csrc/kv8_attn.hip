// Attention over the 8-bit cache (epicache_kv8_attention): O_t = sum_i softmax_i(scale q_t . k_i) v_i and the log of the sum, k_i and v_i
// being e4m3 codes times their block's scale; with `accumulate` the softmax weights that a key receives are added to its own.
//
// An e4m3 code is a bf16 value exactly, so all products run on the bf16 matrix cores on decoded codes; scales are multiplied with the
// logits and the weights in fp32 (or, powers of two, folded into the decoded value, which stays exact).  fp32 queries and weights are cut
// into bf16 parts whose sum they are: three for fp32 outputs, two for the weights of few rows, one (rounded to bf16, 2^-8 of a weight, as
// the output itself is) for the weights of many bf16 rows, where a second part would cost half as many products again.
// The softmax is taken in one pass with a running reference and sum per row, in fp32 and base 2.
//
// Few rows per KV head (a decoding step: up to 32, 16 for head_dim above 128) are bound by the codes' way from memory: kv8_attention_tokens,
// 16 x 8 heads of 24576 rows 128 us, 6.3 TB/s.  Many rows are bound by the products and the softmax between them: kv8_attention_block, 2 x 32
// heads of 2048 rows over 6144 keys 405 us, 850 TFLOP/s.
#include <hip/hip_bf16.h>

#include <algorithm>
#include <type_traits>

#include "kv8.h"
#include "mfma_tiles.h"

namespace epicache {
namespace {

// ---- Few query rows per KV head (decoding): every wave streams its own keys through registers.
//
// Steps of 32 keys go from memory to the matrix cores without LDS.  S^T = K Q^T with 16x16x32 products: a lane holds one query and the keys
// 4 g + i and 16 + 4 g + i of the step, which is how O^T += V^T P^T wants its weights.  V^T wants 8 keys of one column in a lane, so a
// lane fetches its columns of those 8 rows and pairs the bytes of neighbouring keys with permutations, two bytes to an instruction.
// The order of the contraction over head_dim is free, so a lane's 16-byte chunks of K need no shuffling either.
// What it took: rows' tiles handled apart from the last ones and two steps in flight without spills 221 -> 147 us (16 x 8 heads of 24576
// rows), codes read past the caches 139 -> 128 us.  The workgroups of a head each leave their reference, sum and output, and where
// weights are accumulated the logits (a few bytes per key and query beside 256 of codes); kv8_join_tokens puts them together.

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

// Eight fp32 values as three operand parts; not ok: zeros.
__device__ __forceinline__ void cut_row8(bf16x8 (&f)[3], const float* row, bool ok) {
  float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (ok) {
    const float4 a = reinterpret_cast<const float4*>(row)[0], b = reinterpret_cast<const float4*>(row)[1];
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
  for (int i = 0; i < 3; i++) f[i] = __builtin_bit_cast(bf16x8, u[i]);
}

// e4m3 codes 2 i, 2 i + 1 of a dword as bf16, which holds them exactly.
// `scale`: a power of two to be multiplied with.
template <int HIGH>
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t u, float scale = 1.f) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, scale, HIGH != 0));
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
      bf16x8 parts[3];
      cut_row8(parts, row + at, ok && at < d);
#pragma unroll
      for (int i = 0; i < 3; i++) f[i][2 * c + s] = parts[i];
    }
}

__device__ __forceinline__ void store4(__hip_bfloat16* to, const float (&x)[4]) {
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

// 0x80 where a byte is the NaN code, 0x7f or 0xff.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t u) { return ((u & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// NaN codes of V in a step that some rows see and others do not: the rows that see one get a NaN in its column, and the code is
// taken out, since a weight of 0 times it would make one of the others' columns too.  Whether a row sees one is a product of
// zeros and ones.
template <int NCH, int NR>
__device__ __forceinline__ void not_numbers(Step<NCH>& s, f32x4 (&acc)[NR][4 * NCH], int key0, int g, const int (&last)[NR]) {
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

// Waves per SIMD that the registers are cut for: as many as leave the hot loop without spills.
constexpr int token_occupancy(size_t elem, int chunks) { return chunks <= 1 ? 3 : chunks <= (elem == 4 ? 2 : 3) ? 2 : 1; }

// EXACT: d = 64 NCH; a lane's columns of V are then 4 NCH neighbouring ones, else 4 of every 64.  A wave has 16 NR rows.
template <typename T, int NCH, bool EXACT, int NR>
__global__ __launch_bounds__(kTokenWaves * 64, token_occupancy(sizeof(T), NCH * NR)) void kv8_attention_tokens(
    Kv8Plan pl, const T* __restrict__ q, T* __restrict__ out, float* __restrict__ lse, TokenRoom room) {
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

  // INSIDE: all keys of the tile are there, and seen by every row
  auto load = [&](auto inside, Step<NCH>& s, int tile) {
    constexpr bool INSIDE = decltype(inside)::value;
    const int key0 = tile * kTokenKeys;
#pragma unroll
    for (int a = 0; a < 2; a++) {
      const int block = (INSIDE ? key0 + 16 * a : min(key0 + 16 * a, n - 1)) >> pl.block_shift;
      s.ks[a] = ks[block], s.vs[a] = vs[block];
    }
    if constexpr (INSIDE) {
      const uint8_t* kt = kbase + (int64_t)key0 * pitch;
      const uint8_t* vt = vbase + (int64_t)key0 * pitch;
#pragma unroll
      for (int a = 0; a < 2; a++)
#pragma unroll
        for (int c = 0; c < NCH; c++)
          s.k[a][c] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kt + (16 * a + m16) * pitch + chunk_of(c) * 16)));
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const uint8_t* row = vt + ((i >> 2) * 16 + 4 * g + (i & 3)) * pitch;
        if constexpr (EXACT && NCH != 3) {
          typedef __attribute__((ext_vector_type(NCH))) uint32_t columns;
          const columns u = __builtin_nontemporal_load(reinterpret_cast<const columns*>(row + column_of(0)));
#pragma unroll
          for (int c = 0; c < NCH; c++) s.v[i][c] = u[c];
        } else {
#pragma unroll
          for (int c = 0; c < NCH; c++) s.v[i][c] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(row + column_of(c)));
        }
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

  auto work = [&](auto inside, Step<NCH>& s, int tile) {
    constexpr bool INSIDE = decltype(inside)::value;
    const int key0 = tile * kTokenKeys;
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
    if constexpr (!INSIDE) {
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
    if constexpr (!INSIDE)
      if (pl.causal && pl.p > 1) not_numbers<NCH, NR>(s, acc, key0, g, last);
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
    // two steps' rows on their way: one is asked for as soon as its registers are free
    Step<NCH> one, two;
    const std::true_type in;
    const std::false_type any;
    const int inside_end = min(end, all_see / kTokenKeys);
    int tile = split * per_split + wave;
    if (tile < inside_end) load(in, one, tile);
    if (tile + kTokenWaves < inside_end) load(in, two, tile + kTokenWaves);
    for (; tile < inside_end; tile += 2 * kTokenWaves) {
      work(in, one, tile);
      if (tile + 2 * kTokenWaves < inside_end) load(in, one, tile + 2 * kTokenWaves);
      if (tile + kTokenWaves >= inside_end) {
        tile += kTokenWaves;
        break;
      }
      work(in, two, tile + kTokenWaves);
      if (tile + 3 * kTokenWaves < inside_end) load(in, two, tile + 3 * kTokenWaves);
    }
    for (; tile < end; tile += kTokenWaves) {  // the last ones
      load(any, one, tile);
      work(any, one, tile);
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
  // the first rows' logits are on their way while the sums are put together
  constexpr int kEarly = 4;
  const float* logits = room.logits + (size_t)bh * pl.R * room.logit_pitch + key;
  float4 early[kEarly];
  if (!is_out && key < n) {
#pragma unroll
    for (int i = 0; i < kEarly; i++)
      if (i < pl.R) early[i] = *reinterpret_cast<const float4*>(logits + (size_t)i * room.logit_pitch);
  }
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
  auto add = [&](const float4& x, int row) {
    const float2 ml = row_ml[row];
    if (ml.y == 0.f) return;
    w[0] += ex2(x.x - ml.x) * ml.y, w[1] += ex2(x.y - ml.x) * ml.y, w[2] += ex2(x.z - ml.x) * ml.y, w[3] += ex2(x.w - ml.x) * ml.y;
  };
#pragma unroll
  for (int i = 0; i < kEarly; i++)
    if (i < pl.R) add(early[i], i);
  for (int row = kEarly; row < pl.R; row++) add(*reinterpret_cast<const float4*>(logits + (size_t)row * room.logit_pitch), row);
  float* to = pl.weight + b * pl.rsb + h * pl.rsh + key;
#pragma unroll
  for (int i = 0; i < 4; i++)
    if (key + i < n) to[i] += w[i];
}

// ---- Many query rows per KV head (patches, prefilled blocks): tiles of keys through LDS, shared by the waves of a workgroup.
//
// A wave owns 32 query rows.  Tiles of 64 rows of K and V come from memory as codes, one tile ahead, are decoded to bf16 (exactly,
// with their scale where it is a power of two) by whoever fetched them, once per workgroup, and lie in LDS double buffered.  Per 32 keys: S^T = K Q^T, an online softmax, O^T += V^T P^T.

struct BlockRoom {
  int splits, split_tiles;  // workgroups that share the keys of a row, and the tiles of each
  float2* rows;             // [heads][R]: reference and 1 / sum, where weights are accumulated
  float2* stats;            // [heads][splits][R], where there are several: reference and sum
  float* records;           // [heads][splits][R][d]: outputs before the division
  int row_splits, pitch;    // workgroups that share the rows of a key, where weights are accumulated
  float* sums;              // [heads][row_splits][pitch], where there are several: what each has of a key's weight
};

constexpr int kBlockKeys = 64;

// Waves of a workgroup.  The fewer rows, the more of them only help with the tiles.  Eight share one tile where it has a chunk for each
// of their threads (head_dim above 64).
int block_waves(const Kv8Plan& pl) { return pl.R > 128 && pl.d > 64 && pl.d <= 128 && pl.dtype == EPICACHE_DTYPE_BF16 ? 8 : 4; }

__device__ __forceinline__ bool folds(float scale) {  // into the exponent of a decoded value
  const uint32_t u = __float_as_uint(scale);
  return (u & 0x7fffffu) == 0 && u != 0;
}

// Rows in LDS are padded, not swizzled, so that every operand is at one lane address plus an immediate: by 16 bytes where a
// fragment's 16 lanes read 16 rows, by 32 where the transposing load's read 32 bytes of 4 rows.  Both without bank conflicts.
template <int HD>
constexpr int row_pitch() { return HD * 2 + 16; }
template <int HD>
constexpr int value_pitch() { return HD * 2 + 32; }

// Operand fragments of 32 rows; `lane_base`: row l % 32, byte 16 (l / 32).
template <int HD, int KS>
__device__ __forceinline__ void read_rows(bf16x8 (&f)[KS], const unsigned char* lane_base, int sub) {
#pragma unroll
  for (int j = 0; j < KS; j++) f[j] = as_frag(*reinterpret_cast<const uint4*>(lane_base + sub * 32 * row_pitch<HD>() + j * 32));
}
// A operand of O^T += V^T P^T as read_vt_frag has it; `lane_base`: see value_base.
__device__ __forceinline__ int value_base(int pitch, int lane) {
  const int s = lane & 15, gh = (lane >> 4) & 1, hi = lane >> 5;
  return (4 * hi + (s >> 2)) * pitch + gh * 32 + (s & 3) * 8;
}
template <int HD>
__device__ __forceinline__ bf16x8 read_values(const unsigned char* lane_base, int half, int step, int block) {
  s16x4 part[2];
#pragma unroll
  for (int g = 0; g < 2; g++) {
    const unsigned char* p = lane_base + (32 * half + 16 * step + 8 * g) * value_pitch<HD>() + block * 64;
    part[g] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)LDS_PTR(p));
  }
  typedef __attribute__((ext_vector_type(8))) short s16x8;
  const s16x8 both = {part[0][0], part[0][1], part[0][2], part[0][3], part[1][0], part[1][1], part[1][2], part[1][3]};
  return __builtin_bit_cast(bf16x8, both);
}
// Bytes of the two buffers of K and V tiles.
template <int HD>
constexpr int block_tiles_bytes() { return 2 * kBlockKeys * (row_pitch<HD>() + value_pitch<HD>()); }

// Thread's share of a tile on its way to LDS: 16-code chunks tid, tid + NT, .. of the tile's rows, K and V.
template <int HD, int NT>
struct TileCodes {
  static constexpr int kPer = kBlockKeys * (HD / 16) / NT;
  static_assert(kPer >= 1, "every thread has a chunk");
  uint4 k[kPer], v[kPer];
  float ks[kPer], vs[kPer];  // of the 16 keys that a wave's chunks lie in: wave-uniform
};

// Waves per SIMD that the registers are cut for.
constexpr int block_occupancy(size_t elem, int hd) { return elem == 2 && hd <= 128 ? 2 : 1; }

__device__ __forceinline__ uint4 codes_to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  return make_uint4(codes_to_bf16<0>(lo, scale), codes_to_bf16<1>(lo, scale), codes_to_bf16<0>(hi, scale), codes_to_bf16<1>(hi, scale));
}

// The 8 values of chunks hi, 2 + hi, .. of a row as operand parts; zeros behind d.
template <int KS>
__device__ __forceinline__ void load_rows(bf16x8 (&f)[1][KS], const __hip_bfloat16* row, int hi, int d) {
  load_row_frags<KS>(f[0], reinterpret_cast<const bf16_t*>(row), hi, d);
}
template <int KS>
__device__ __forceinline__ void load_rows(bf16x8 (&f)[3][KS], const float* row, int hi, int d) {
#pragma unroll
  for (int j = 0; j < KS; j++) {
    bf16x8 parts[3];
    const int at = (2 * j + hi) * 8;
    cut_row8(parts, row + at, at < d);
#pragma unroll
    for (int i = 0; i < 3; i++) f[i][j] = parts[i];
  }
}

// Rows from .. to - 1 of a head: how many keys each of them sees at least, and how many at most.
__device__ __forceinline__ void rows_see(const Kv8Plan& pl, int old, int n, int from, int to, int& least, int& most) {
  least = most = n;
  if (!pl.causal) return;
  int ga, ta, gb, tb;
  head_and_token(pl.p, pl.inv_p, min(from, pl.R - 1), ga, ta);
  head_and_token(pl.p, pl.inv_p, min(to, pl.R) - 1, gb, tb);
  least = old + 1 + (ga == gb ? ta : 0), most = old + 1 + (ga == gb ? tb : pl.p - 1);
}

// HD: row layout in LDS; KS 16-element steps of Q K^T, DB 32-column blocks of the output.
template <typename T, int HD, int KS, int DB, int NW>
__global__ __launch_bounds__(NW * 64, block_occupancy(sizeof(T), HD)) void kv8_attention_block(
    Kv8Plan pl, const T* __restrict__ q, T* __restrict__ out, float* __restrict__ lse, BlockRoom room) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int PARTS = F32 ? 3 : 1, NT = NW * 64;
  constexpr int kKTile = kBlockKeys * row_pitch<HD>(), kVTile = kBlockKeys * value_pitch<HD>();
  using Codes = TileCodes<HD, NT>;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];  // K, K, V, V, then
  unsigned char* const more = smem + block_tiles_bytes<HD>();
  float(*rest)[2][4] = reinterpret_cast<float(*)[2][4]>(more);  // [buffer][K, V][16 keys]: what scales have not been folded
  int* unfolded = reinterpret_cast<int*>(more + 64);            // [buffer]: the last tile there with such a scale
  int* nan_seen = reinterpret_cast<int*>(more + 72);            // NaN codes have been taken out of a V that not all rows see
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  // XCD-aware ids: the row blocks of one head and split read the same keys and land on one XCD; the last rows, which see most, first
  const int n_rb = gridDim.x >> 3, rb = n_rb - 1 - (blockIdx.x >> 3);
  const int unit = blockIdx.y * 8 + (blockIdx.x & 7);
  if (unit >= pl.nb * pl.Hkv * room.splits) return;
  const int bh = unit / room.splits, split = unit - bh * room.splits;
  const int b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int old = kv8_old_rows(pl, bh), n = old + pl.n_block;

  const int first_row = rb * 32 * NW, row0 = first_row + wave * 32, r = row0 + l32;
  const bool active = row0 < pl.R;
  int g_row, t_row;
  head_and_token(pl.p, pl.inv_p, min(r, pl.R - 1), g_row, t_row);
  const int last_key = pl.causal ? old + t_row : n - 1;
  bf16x8 qf[PARTS][KS];
  load_rows<KS>(qf, q + b * pl.qsb + (int64_t)(h * pl.G + g_row) * pl.qsh + (int64_t)t_row * pl.qst, hi, pl.d);
  int all_see, any_sees, wave_all, wave_any;
  rows_see(pl, old, n, first_row, first_row + 32 * NW, all_see, any_sees);
  rows_see(pl, old, n, row0, row0 + 32, wave_all, wave_any);
  const int tiles = (any_sees + kBlockKeys - 1) / kBlockKeys;
  const int first_tile = split * room.split_tiles, end_tile = room.splits == 1 ? tiles : min(tiles, first_tile + room.split_tiles);

  const uint8_t* kbase = pl.k + b * pl.sb + h * pl.sh;
  const uint8_t* vbase = pl.v + b * pl.sb + h * pl.sh;
  const float* ks = pl.k_scale + b * pl.ssb + h * pl.ssh;
  const float* vs = pl.v_scale + b * pl.ssb + h * pl.ssh;
  const uint32_t pitch = (uint32_t)pl.st;

  // a row of the tile has HD / 16 chunks, of which the first d / 16 are there
  const int my_row = tid / (HD / 16), my_chunk = tid % (HD / 16);
  constexpr int kRowsApart = NT / (HD / 16);  // from a thread's chunk to its next
  const bool in_row = my_chunk * 16 < pl.d;
  const uint32_t my_column = in_row ? my_chunk * 16 : 0;
  auto fetch = [&](Codes& c, int t) {
    const int key0 = t * kBlockKeys, there = n - key0;
    const uint8_t* kt = kbase + (int64_t)key0 * pitch;
    const uint8_t* vt = vbase + (int64_t)key0 * pitch;
#pragma unroll
    for (int i = 0; i < Codes::kPer; i++) {
      const int row = my_row + i * kRowsApart;
      const int block = min(key0 + (__builtin_amdgcn_readfirstlane(row) & ~15), n - 1) >> pl.block_shift;
      c.ks[i] = ks[block], c.vs[i] = vs[block];
      const uint32_t at = __umul24(min(row, there - 1), pitch) + my_column;
      c.k[i] = *reinterpret_cast<const uint4*>(kt + at);
      c.v[i] = *reinterpret_cast<const uint4*>(vt + at);
    }
  };
  // Before a tile's codes are decoded: what is not to be in them, and what the decoded values will not have in them.
  auto check = [&](Codes& c, auto buf_c, int t) {
    constexpr int buf = decltype(buf_c)::value;
    const bool partly = (t + 1) * kBlockKeys > all_see;  // a weight of 0 times a NaN code would be a NaN in rows that do not see it
#pragma unroll
    for (int i = 0; i < Codes::kPer; i++) {
      const int row = my_row + i * kRowsApart;
      if (my_chunk == 0 && (row & 15) == 0) {
        const bool kf = folds(c.ks[i]), vf = folds(c.vs[i]);
        rest[buf][0][row >> 4] = kf ? 1.f : c.ks[i];
        rest[buf][1][row >> 4] = vf ? 1.f : c.vs[i];
        if (!kf || !vf) unfolded[buf] = t;
      }
      if (pl.d != HD && !in_row) c.k[i] = c.v[i] = make_uint4(0, 0, 0, 0);
      if (partly) {
        uint32_t* u = reinterpret_cast<uint32_t*>(&c.v[i]);
        bool nan = false;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          if (t * kBlockKeys + row >= n) u[j] = 0;
          const uint32_t is = nan_bytes(u[j]);
          nan = nan || is != 0;
          u[j] &= ~(is | (is - (is >> 7)));
        }
        if (nan) *nan_seen = 1;
      }
    }
  };
  unsigned char* const my_k = smem + my_row * row_pitch<HD>() + my_chunk * 32;
  unsigned char* const my_v = smem + 2 * kKTile + my_row * value_pitch<HD>() + my_chunk * 32;
  auto place = [&](const Codes& c, auto buf_c) {
    constexpr int buf = decltype(buf_c)::value;
#pragma unroll
    for (int i = 0; i < Codes::kPer; i++) {
      const float kfold = folds(c.ks[i]) ? c.ks[i] : 1.f, vfold = folds(c.vs[i]) ? c.vs[i] : 1.f;
      uint4* kt = reinterpret_cast<uint4*>(my_k + buf * kKTile + i * kRowsApart * row_pitch<HD>());
      uint4* vt = reinterpret_cast<uint4*>(my_v + buf * kVTile + i * kRowsApart * value_pitch<HD>());
      kt[0] = codes_to_bf16x8(c.k[i].x, c.k[i].y, kfold), kt[1] = codes_to_bf16x8(c.k[i].z, c.k[i].w, kfold);
      vt[0] = codes_to_bf16x8(c.v[i].x, c.v[i].y, vfold), vt[1] = codes_to_bf16x8(c.v[i].z, c.v[i].w, vfold);
    }
  };
  const unsigned char* const k_lane = smem + l32 * row_pitch<HD>() + hi * 16;
  const unsigned char* const v_lane = smem + 2 * kKTile + value_base(value_pitch<HD>(), lane);

  f32x16 o[DB];
#pragma unroll
  for (int j = 0; j < DB; j++) o[j] = f32x16{0};
  float m = kNoKey, l = 0.f;  // reference in base 2, this lane's sum

  // BUF is a compile-time constant (the loop below is unrolled by two), so that LDS addresses are loop-invariant lane offsets plus
  // immediates.
  // Between the products of the first half the next tile's codes, which are there by now, go to LDS, and those behind them are asked
  // for: 80 of 424 us went into that where it stood in front of the tile (2 x 32 heads x 2048 rows over 6144 keys).
  auto work = [&](auto buf_c, auto next_c, Codes& c, int t) {
    constexpr int buf = decltype(buf_c)::value;
    const unsigned char* ktile = k_lane + buf * kKTile;
    const unsigned char* vtile = v_lane + buf * kVTile;
    const bool masked = (t + 1) * kBlockKeys > wave_all, folded = __builtin_amdgcn_readfirstlane(unfolded[buf]) != t;
    bf16x8 kf[KS];
    read_rows<HD, KS>(kf, ktile, 0);
#pragma unroll
    for (int half = 0; half < 2; half++) {
      const int key0 = t * kBlockKeys + 32 * half;
      f32x16 z = f32x16{0};
      __builtin_amdgcn_s_setprio(1);  // of the two waves of a SIMD the one with products goes first: 424 -> 410 us
#pragma unroll
      for (int part = PARTS - 1; part >= 0; part--)
#pragma unroll
        for (int j = 0; j < KS; j++) mfma_step(z, kf[j], qf[part][j]);
      if (half == 0) read_rows<HD, KS>(kf, ktile, 1);  // what the arithmetic below can hide
      bf16x8 vf[DB][2];
#pragma unroll
      for (int j = 0; j < DB; j++)
#pragma unroll
        for (int st = 0; st < 2; st++) vf[j][st] = read_values<HD>(vtile, half, st, j);
      if (half == 0) place(c, next_c);
      if (masked || !folded) {
#pragma unroll
        for (int i = 0; i < 16; i++) {
          if (!folded) z[i] *= rest[buf][0][2 * half + (i >> 3)];
          if (key0 + (i >> 2) * 8 + hi * 4 + (i & 3) > last_key) z[i] = -INFINITY;
        }
      }
      __builtin_amdgcn_s_setprio(0);
      const float a0 = max3(z[0], z[1], z[2]), a1 = max3(z[3], z[4], z[5]), a2 = max3(z[6], z[7], z[8]);
      const float a3 = max3(z[9], z[10], z[11]), a4 = max3(z[12], z[13], z[14]);
      const float top = max_across_halves(max3(max3(a0, a1, a2), max3(a3, a4, z[15]), -INFINITY)) * pl.c2;
      // the reference follows the maximum lazily, as in the kernel for few rows
      if (__any(top > m + kLazyBits)) {
        const float mn = fmaxf(m, top), corr = ex2(m - mn);
        l *= corr;
#pragma unroll
        for (int j = 0; j < DB; j++)
#pragma unroll
          for (int i = 0; i < 16; i++) o[j][i] *= corr;
        m = mn;
      }
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; i++) e[i] = ex2(fmaf(z[i], pl.c2, -m));
      l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])) +
           (((e[8] + e[9]) + (e[10] + e[11])) + ((e[12] + e[13]) + (e[14] + e[15])));
      if (!folded) {
#pragma unroll
        for (int i = 0; i < 16; i++) e[i] *= rest[buf][1][2 * half + (i >> 3)];
      }
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int st = 0; st < 2; st++) {
        bf16x8 pf[PARTS];
        weight_frags<PARTS>(pf, e + 8 * st);
#pragma unroll
        for (int part = PARTS - 1; part >= 0; part--)
#pragma unroll
          for (int j = 0; j < DB; j++) o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j][st], pf[part], o[j], 0, 0, 0);
      }
      if (half == 0) fetch(c, min(t + 2, end_tile - 1));
    }
  };

  {
    Codes c;
    if (tid == 0) *nan_seen = 0, unfolded[0] = unfolded[1] = -1;
    __syncthreads();
    constexpr std::integral_constant<int, 0> even;
    constexpr std::integral_constant<int, 1> odd;
    if (first_tile < end_tile) {
      fetch(c, first_tile);
      check(c, even, first_tile);
      place(c, even);
      fetch(c, min(first_tile + 1, end_tile - 1));
    }
    __syncthreads();
    auto step = [&](auto now, auto next, int t) {
      if (t + 1 < end_tile) check(c, next, t + 1);
      if (active && t * kBlockKeys < wave_any) {
        work(now, next, c, t);
      } else {
        place(c, next);  // the last tile once more where there is no next one: nobody reads it
        fetch(c, min(t + 2, end_tile - 1));
      }
      __syncthreads();
    };
    for (int t = first_tile; t < end_tile; t += 2) {
      step(even, odd, t);
      if (t + 1 < end_tile) step(odd, even, t + 1);
    }
  }

  if (!active) return;
  const bool whole = room.splits == 1, nan = __any(*nan_seen != 0);
  const float sum = l + __shfl_xor(l, 32);
  if (r >= pl.R) return;
  const bool any = sum > 0.f || sum != sum;
  const float inv = any ? 1.f / sum : 0.f;
  const size_t orow = ((size_t)b * pl.Hq + h * pl.G + g_row) * pl.p + t_row;
  const size_t record = (size_t)unit * pl.R + r;
  if (hi == 0) {
    if (whole) lse[orow] = any ? (m + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
    if (whole && room.rows) room.rows[(size_t)bh * pl.R + r] = make_float2(m, inv);
    if (!whole) room.stats[record] = make_float2(m, sum);
  }
#pragma unroll
  for (int j = 0; j < DB; j++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int column = 32 * j + 8 * i + 4 * hi;
      if (column >= pl.d) continue;
      float y[4];
#pragma unroll
      for (int c = 0; c < 4; c++) y[c] = !whole ? o[j][4 * i + c] : any ? o[j][4 * i + c] * inv : 0.f;
      if (nan) {  // look for them again, among the keys that this row sees
        const int from = max(first_tile, all_see / kBlockKeys) * kBlockKeys, to = min(end_tile * kBlockKeys, last_key + 1);
        for (int key = from; key < to; key++) {
          const uint32_t is = nan_bytes(*reinterpret_cast<const uint32_t*>(vbase + (int64_t)key * pitch + column));
#pragma unroll
          for (int c = 0; c < 4; c++) y[c] = (is >> (8 * c + 7)) & 1 ? NAN : y[c];
        }
      }
      if (whole) store4(out + orow * pl.d + column, y);
      else store4(room.records + record * pl.d + column, y);
    }
}

// What the splits of the rows left, put together: 4 columns to a thread, d / 4 threads to a row.
template <typename T>
__global__ __launch_bounds__(256) void kv8_join_rows(Kv8Plan pl, T* __restrict__ out, float* __restrict__ lse, BlockRoom room) {
  const int per_row = pl.d >> 2;
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  const size_t row_of_all = at / per_row;
  if (row_of_all >= (size_t)pl.nb * pl.Hkv * pl.R) return;
  const int column = (int)(at - row_of_all * per_row) * 4, bh = (int)(row_of_all / pl.R), r = (int)(row_of_all - (size_t)bh * pl.R);
  const float2* s = room.stats + (size_t)bh * room.splits * pl.R + r;
  float m = kNoKey, sum = 0.f;
  for (int i = 0; i < room.splits; i++) m = fmaxf(m, s[(size_t)i * pl.R].x);
  float y[4] = {0, 0, 0, 0};
  for (int i = 0; i < room.splits; i++) {
    const float2 ml = s[(size_t)i * pl.R];
    const float w = ex2(ml.x - m);
    sum += ml.y * w;
    const float4 a = *reinterpret_cast<const float4*>(room.records + (((size_t)bh * room.splits + i) * pl.R + r) * pl.d + column);
    y[0] += w * a.x, y[1] += w * a.y, y[2] += w * a.z, y[3] += w * a.w;
  }
  const bool any = sum > 0.f || sum != sum;
  const float inv = any ? 1.f / sum : 0.f;
#pragma unroll
  for (int i = 0; i < 4; i++) y[i] = any ? y[i] * inv : 0.f;
  const int b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  int g, t;
  head_and_token(pl.p, pl.inv_p, r, g, t);
  const size_t orow = ((size_t)b * pl.Hq + h * pl.G + g) * pl.p + t;
  store4(out + orow * pl.d + column, y);
  if (column == 0) {
    lse[orow] = any ? (m + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
    if (room.rows) room.rows[(size_t)bh * pl.R + r] = make_float2(m, inv);
  }
}

constexpr int accumulate_rows(bool f32) { return f32 ? 32 : 64; }  // query rows of a tile

// weight += the softmax weights of many rows: the product with K once more, now with the keys in registers and the query rows
// through LDS, so that every key's sum has one owner and one order.  A wave has 32 NK keys, a lane one column of each 32 and half
// of its rows: a key's scale and its sum are the lane's own, what belongs to a row comes from LDS.
template <typename T, int HD, int KS, int NK, int NW>
__global__ __launch_bounds__(NW * 64, block_occupancy(sizeof(T), HD)) void kv8_accumulate_block(Kv8Plan pl, const T* __restrict__ q, BlockRoom room) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int PARTS = F32 ? 3 : 1, NT = NW * 64, QT = accumulate_rows(F32);
  constexpr int kPart = QT * row_pitch<HD>(), kTile = PARTS * kPart, kChunks = HD / 8;
  constexpr int kPer = QT * kChunks / NT;  // 8-value chunks of a tile per thread
  static_assert(kPer >= 1, "every thread has a chunk");
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  float(*info)[3][QT] = reinterpret_cast<float(*)[3][QT]>(smem + 2 * kTile);  // [buffer]: reference, 1 / sum, last key
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int old = kv8_old_rows(pl, bh), n = old + pl.n_block;
  const int first_key = blockIdx.x * (32 * NK * NW), key0 = first_key + wave * 32 * NK;
  if (first_key >= n) return;
  const uint8_t* kbase = pl.k + b * pl.sb + h * pl.sh;
  const float* ks = pl.k_scale + b * pl.ssb + h * pl.ssh;

  bf16x8 kf[NK][KS];
  float by[NK], acc[NK];  // logits of codes in base 2
#pragma unroll
  for (int x = 0; x < NK; x++) {
    const int key = min(key0 + 32 * x + l32, n - 1);
    by[x] = pl.c2 * ks[key >> pl.block_shift];
    acc[x] = 0.f;
    const uint8_t* row = kbase + (int64_t)key * pl.st;
#pragma unroll
    for (int j = 0; j < KS; j += 2) {  // chunks of 16 codes in the place of two of 8: in which order they are multiplied is free
      const int at = j * 16 + hi * 16;
      uint4 u = make_uint4(0, 0, 0, 0);
      if (at < pl.d) u = *reinterpret_cast<const uint4*>(row + at);
      kf[x][j] = codes_to_frag(u.x, u.y), kf[x][j + 1] = codes_to_frag(u.z, u.w);
    }
  }

  struct Share {
    float v[kPer][F32 ? 8 : 4];
    float2 ml;
    int last;
  };
  auto fetch = [&](Share& c, int tile) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int at = tid + i * NT, r = tile * QT + at / kChunks, column = at % kChunks * 8;
      int g, t;
      head_and_token(pl.p, pl.inv_p, min(r, pl.R - 1), g, t);
      const T* from = q + b * pl.qsb + (int64_t)(h * pl.G + g) * pl.qsh + (int64_t)t * pl.qst + column;
      float4 a = make_float4(0, 0, 0, 0), z = a;
      if (column < pl.d && r < pl.R) {  // no row: zeros, not what the last one holds, which may be NaN
        a = reinterpret_cast<const float4*>(from)[0];
        if (F32) z = reinterpret_cast<const float4*>(from)[1];
      }
      c.v[i][0] = a.x, c.v[i][1] = a.y, c.v[i][2] = a.z, c.v[i][3] = a.w;
      if constexpr (F32) c.v[i][4] = z.x, c.v[i][5] = z.y, c.v[i][6] = z.z, c.v[i][7] = z.w;
    }
    if (tid < QT) {
      const int r = tile * QT + tid;
      c.ml = make_float2(0.f, 0.f);
      int g = 0, t = 0;
      if (r < pl.R) {
        c.ml = room.rows[(size_t)bh * pl.R + r];
        head_and_token(pl.p, pl.inv_p, r, g, t);
      }
      if (c.ml.y == 0.f) c.ml.x = INFINITY;  // a row without weights: exponentials of -inf, whatever its logits
      c.last = pl.causal ? old + t : n - 1;
    }
  };
  auto place = [&](Share& c, int buf) {
    unsigned char* tile = smem + buf * kTile;
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int at = tid + i * NT, r = at / kChunks, chunk = at % kChunks;
      uint4* to = reinterpret_cast<uint4*>(tile + r * row_pitch<HD>() + chunk * 16);
      if constexpr (F32) {
        bf16x8 parts[3];
        cut_row8(parts, c.v[i], true);
#pragma unroll
        for (int p = 0; p < 3; p++) *(to + p * (kPart / 16)) = __builtin_bit_cast(uint4, parts[p]);
      } else {
        *to = make_uint4(__float_as_uint(c.v[i][0]), __float_as_uint(c.v[i][1]), __float_as_uint(c.v[i][2]), __float_as_uint(c.v[i][3]));
      }
    }
    if (tid < QT) info[buf][0][tid] = c.ml.x, info[buf][1][tid] = c.ml.y, info[buf][2][tid] = __int_as_float(c.last);
  };

  const int all_tiles = (pl.R + QT - 1) / QT, per_split = (all_tiles + room.row_splits - 1) / room.row_splits;
  const int first_tile = blockIdx.z * per_split, tiles = min(all_tiles, first_tile + per_split);
  Share c;
  fetch(c, first_tile);
  place(c, 0);
  if (first_tile + 1 < tiles) fetch(c, first_tile + 1);
  __syncthreads();
  for (int t = first_tile; t < tiles; t++) {
    const int buf = (t - first_tile) & 1;
    if (t + 1 < tiles) {
      place(c, buf ^ 1);
      if (t + 2 < tiles) fetch(c, t + 2);
    }
#pragma unroll 1
    for (int half = 0; half < QT / 32; half++) {
      int least, most;
      const int row0 = t * QT + 32 * half;
      rows_see(pl, old, n, row0, row0 + 32, least, most);
      if (row0 >= pl.R || key0 >= most) continue;
      bf16x8 qf[PARTS][KS];
#pragma unroll
      for (int p = 0; p < PARTS; p++) {
        const unsigned char* row = smem + buf * kTile + p * kPart + (32 * half + l32) * row_pitch<HD>() + hi * 32;
#pragma unroll
        for (int j = 0; j < KS; j++) qf[p][j] = as_frag(*reinterpret_cast<const uint4*>(row + (j >> 1) * 64 + (j & 1) * 16));
      }
      float m[16], inv[16];  // of the lane's rows 8 (i / 4) + 4 hi + i % 4
#pragma unroll
      for (int i = 0; i < 4; i++) {
        *reinterpret_cast<float4*>(m + 4 * i) = *reinterpret_cast<const float4*>(&info[buf][0][32 * half + 8 * i + 4 * hi]);
        *reinterpret_cast<float4*>(inv + 4 * i) = *reinterpret_cast<const float4*>(&info[buf][1][32 * half + 8 * i + 4 * hi]);
      }
#pragma unroll
      for (int x = 0; x < NK; x++) {
        f32x16 z = f32x16{0};
#pragma unroll
        for (int p = PARTS - 1; p >= 0; p--)
#pragma unroll
          for (int j = 0; j < KS; j++) mfma_step(z, qf[p][j], kf[x][j]);
        float sum[4] = {0, 0, 0, 0};
        if (key0 + 32 * x + 32 > least) {
          const int key = key0 + 32 * x + l32;
#pragma unroll
          for (int i = 0; i < 16; i++) {
            const int last = __float_as_int(info[buf][2][32 * half + 8 * (i >> 2) + 4 * hi + (i & 3)]);
            sum[i & 3] += key <= last ? ex2(fmaf(z[i], by[x], -m[i])) * inv[i] : 0.f;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; i++) sum[i & 3] = fmaf(ex2(fmaf(z[i], by[x], -m[i])), inv[i], sum[i & 3]);
        }
        acc[x] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
    }
    __syncthreads();
  }
  float* weight = pl.weight + b * pl.rsb + h * pl.rsh;
#pragma unroll
  for (int x = 0; x < NK; x++) {
    const float sum = acc[x] + __shfl_xor(acc[x], 32);
    const int key = key0 + 32 * x + l32;
    if (hi != 0 || key >= n) continue;
    if (room.row_splits == 1) weight[key] += sum;
    else room.sums[((size_t)bh * room.row_splits + blockIdx.z) * room.pitch + key] = sum;
  }
}

// weight += the row splits' sums, in their order.
__global__ __launch_bounds__(256) void kv8_add_sums(Kv8Plan pl, BlockRoom room) {
  const int bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv, key = blockIdx.x * 256 + threadIdx.x;
  if (key >= kv8_old_rows(pl, bh) + pl.n_block) return;
  float sum = 0.f;
  for (int i = 0; i < room.row_splits; i++) sum += room.sums[((size_t)bh * room.row_splits + i) * room.pitch + key];
  pl.weight[b * pl.rsb + h * pl.rsh + key] += sum;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Room of the kernel for few rows; null workspace: only its size, in *bytes.
TokenRoom token_room(const Kv8Plan& pl, void* workspace, size_t* bytes) {
  const int64_t heads = (int64_t)pl.nb * pl.Hkv;
  const int tiles = (pl.n_cached + pl.n_block + kTokenKeys - 1) / kTokenKeys;
  // A round of resident workgroups, each with two steps a wave at least (32 heads of 2049 keys: one step 16.0 us, two 13.7, four 14.9); two rounds where the steps are many, so that the last workgroups
  // to end are shorter (64 x 4 heads of 8193 keys: one 156 us, two 150; 96 heads of up to 2501 keys: one 18.3, more 23.2).
  const int64_t slots = kComputeUnits * token_occupancy(pl.dtype == EPICACHE_DTYPE_F32 ? 4 : 2, (pl.d + 63) / 64 * ((pl.R + 15) / 16));
  int64_t splits = slots / heads;
  if (splits > 0 && tiles / splits >= 16 * kTokenWaves) splits *= 2;
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

BlockRoom block_room(const Kv8Plan& pl, void* workspace, size_t* bytes) {
  const int64_t heads = (int64_t)pl.nb * pl.Hkv;
  const int nw = block_waves(pl), n_rb = (pl.R + 32 * nw - 1) / (32 * nw);
  const int tiles = (pl.n_cached + pl.n_block + kBlockKeys - 1) / kBlockKeys;
  const int64_t slots = kComputeUnits * 4 * block_occupancy(pl.dtype == EPICACHE_DTYPE_F32 ? 4 : 2, pl.d <= 128 ? 128 : 256) / nw;
  int64_t splits = slots / (heads * n_rb);  // a round of workgroups, each with four tiles at least
  splits = std::max<int64_t>(1, std::min<int64_t>({splits, tiles / 4, kMostSplits}));
  const int split_tiles = (tiles + (int)splits - 1) / (int)splits;
  splits = (tiles + split_tiles - 1) / split_tiles;
  BlockRoom room = {(int)splits, split_tiles, nullptr, nullptr, nullptr, 1, (tiles * kBlockKeys + 127) / 128 * 128, nullptr};
  char* ws = static_cast<char*>(workspace);
  size_t at = 0;
  auto take = [&](size_t n) {
    char* p = ws ? ws + at : nullptr;
    at += align256(n);
    return reinterpret_cast<float*>(p);
  };
  if (pl.accumulate) room.rows = reinterpret_cast<float2*>(take((size_t)heads * pl.R * sizeof(float2)));
  if (splits > 1) {
    room.stats = reinterpret_cast<float2*>(take((size_t)heads * splits * pl.R * sizeof(float2)));
    room.records = take((size_t)heads * splits * pl.R * pl.d * sizeof(float));
  }
  if (pl.accumulate) {
    // Few heads and keys and many rows: the rows are shared too, two tiles of them at least to a workgroup (24 heads of 1368 rows over some
    // 1400 keys: 132 us with one workgroup to 128 keys).
    const bool f32 = pl.dtype == EPICACHE_DTYPE_F32;
    const int row_tiles = (pl.R + accumulate_rows(f32) - 1) / accumulate_rows(f32);
    const int64_t workgroups = heads * (room.pitch / 128), resident = kComputeUnits * block_occupancy(f32 ? 4 : 2, pl.d <= 128 ? 128 : 256);
    const int wanted = (int)std::max<int64_t>(1, std::min<int64_t>(resident / workgroups, row_tiles / 2));
    const int per_split = (row_tiles + wanted - 1) / wanted;
    room.row_splits = (row_tiles + per_split - 1) / per_split;
    if (room.row_splits > 1) room.sums = take((size_t)heads * room.row_splits * room.pitch * sizeof(float));
  }
  *bytes = at;
  return room;
}

template <typename K, typename... A>
hipError_t launch_with_lds(K kernel, dim3 grid, int threads, size_t lds, hipStream_t stream, A... args) {
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, stream, args...);
  return hipGetLastError();
}

template <typename T, int HD, int KS, int DB, int NW>
hipError_t launch_block(const Kv8Plan& pl, const T* q, T* out, float* lse, void* workspace, hipStream_t stream) {
  size_t bytes;
  const BlockRoom room = block_room(pl, workspace, &bytes);
  const int heads = pl.nb * pl.Hkv, n_rb = (pl.R + 32 * NW - 1) / (32 * NW);
  hipError_t e = launch_with_lds(kv8_attention_block<T, HD, KS, DB, NW>, dim3(8 * n_rb, (heads * room.splits + 7) / 8), NW * 64,
                                 block_tiles_bytes<HD>() + 128, stream, pl, q, out, lse, room);
  if (e != hipSuccess) return e;
  if (room.splits > 1) {
    const size_t threads = (size_t)heads * pl.R * (pl.d / 4);
    hipLaunchKernelGGL(kv8_join_rows<T>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, pl, out, lse, room);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!pl.accumulate) return hipSuccess;
  // 32-key tiles of a wave: rounds of workgroups, each as long as its tiles and some one more for getting going (32 heads of 512 rows
  // over 8320 keys: one tile 66.8 us, two, with a third round for the last few workgroups, 74.0, three 66.2)
  constexpr int PARTS = sizeof(T) == 4 ? 3 : 1, QT = accumulate_rows(sizeof(T) == 4);
  constexpr size_t lds = 2 * PARTS * QT * row_pitch<HD>() + 2 * 3 * QT * sizeof(float);
  auto accumulate = [&](auto nk) {
    constexpr int NK = decltype(nk)::value, kKeys = 32 * NK * 4;
    return launch_with_lds(kv8_accumulate_block<T, HD, KS, NK, 4>, dim3((pl.n_cached + pl.n_block + kKeys - 1) / kKeys, heads, room.row_splits),
                           256, lds, stream, pl, q, room);
  };
  if (room.row_splits > 1) {
    e = accumulate(std::integral_constant<int, 1>{});
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kv8_add_sums, dim3((pl.n_cached + pl.n_block + 255) / 256, heads), dim3(256), 0, stream, pl, room);
    return hipGetLastError();
  }
  auto cost = [&](int nk) {
    const int64_t workgroups = (int64_t)heads * ((pl.n_cached + pl.n_block + 128 * nk - 1) / (128 * nk));
    const int64_t slots = kComputeUnits * block_occupancy(sizeof(T), HD);
    return (workgroups + slots - 1) / slots * (nk + 1);
  };
  if constexpr (HD < 256) {
    if constexpr (sizeof(T) == 2)
      if (cost(3) <= cost(2) && cost(3) <= cost(1)) return accumulate(std::integral_constant<int, 3>{});
    if (cost(2) <= cost(1)) return accumulate(std::integral_constant<int, 2>{});
  }
  return accumulate(std::integral_constant<int, 1>{});
}

template <typename T>
hipError_t launch_blocks(const Kv8Plan& pl, const T* q, T* out, float* lse, void* workspace, hipStream_t stream) {
  auto waves = [&](auto hd, auto ks, auto db) {
    constexpr int HD = decltype(hd)::value, KS = decltype(ks)::value, DB = decltype(db)::value;
    if constexpr (sizeof(T) == 2 && HD == 128)
      if (block_waves(pl) == 8) return launch_block<T, HD, KS, DB, 8>(pl, q, out, lse, workspace, stream);
    return launch_block<T, HD, KS, DB, 4>(pl, q, out, lse, workspace, stream);
  };
  using std::integral_constant;
  if (pl.d <= 64) return waves(integral_constant<int, 64>{}, integral_constant<int, 4>{}, integral_constant<int, 2>{});
  if (pl.d <= 96) return waves(integral_constant<int, 128>{}, integral_constant<int, 6>{}, integral_constant<int, 3>{});
  if (pl.d <= 128) return waves(integral_constant<int, 128>{}, integral_constant<int, 8>{}, integral_constant<int, 4>{});
  if (pl.d <= 192) return waves(integral_constant<int, 256>{}, integral_constant<int, 12>{}, integral_constant<int, 6>{});
  return waves(integral_constant<int, 256>{}, integral_constant<int, 16>{}, integral_constant<int, 8>{});
}

}  // namespace

size_t kv8_attention_workspace(const Kv8Plan& pl) {
  size_t bytes;
  if (few_rows(pl)) token_room(pl, nullptr, &bytes);
  else block_room(pl, nullptr, &bytes);
  return bytes;
}

hipError_t launch_kv8_attention(const Kv8Plan& pl, const void* q, void* out, float* lse, void* workspace, hipStream_t stream) {
  auto typed = [&](auto* rows, auto* to) {
    return few_rows(pl) ? launch_tokens(pl, rows, to, lse, workspace, stream) : launch_blocks(pl, rows, to, lse, workspace, stream);
  };
  if (pl.dtype == EPICACHE_DTYPE_BF16) return typed(static_cast<const __hip_bfloat16*>(q), static_cast<__hip_bfloat16*>(out));
  return typed(static_cast<const float*>(q), static_cast<float*>(out));
}

}  // namespace epicache
