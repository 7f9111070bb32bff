// Rows into the 8-bit cache (epicache_kv8_append) and its eviction by accumulated attention weight (epicache_kv8_evict).
//
// Both write rows into blocks that share a scale, with one rule: the scale of a block is the smallest power of two that
// brings its new values to at most 448, and at least what it was while older rows stay in it (those are rounded again where it
// has grown).  A workgroup owns a block of K or of V, so the scale has one writer: it reads the new rows into registers, takes the
// largest magnitude, and writes codes.  One pass over the data.
#include <hip/hip_bf16.h>

#include <algorithm>

#include "kv8.h"
#include "select_util.h"

namespace epicache {
namespace {

// Sixteen values of an incoming row.
__device__ __forceinline__ void load16(const __hip_bfloat16* from, float (&x)[16]) {
  const uint4 a = reinterpret_cast<const uint4*>(from)[0], b = reinterpret_cast<const uint4*>(from)[1];
  const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; i++) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
}
__device__ __forceinline__ void load16(const float* from, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float4 a = reinterpret_cast<const float4*>(from)[i];
    x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = a.z, x[4 * i + 3] = a.w;
  }
}
__device__ __forceinline__ void decode16(uint4 u, float (&x)[16], float scale) {
  decode4(u.x, x), decode4(u.y, x + 4), decode4(u.z, x + 8), decode4(u.w, x + 12);
#pragma unroll
  for (int i = 0; i < 16; i++) x[i] *= scale;
}
// The codes of x / scale; a power of two is divided by exactly with a product.
__device__ __forceinline__ uint4 encode16(float (&x)[16], float scale) {
  if ((__float_as_uint(scale) & 0x7fffffu) == 0) {
    const float by = 1.f / scale;
#pragma unroll
    for (int i = 0; i < 16; i++) x[i] *= by;
  } else {
#pragma unroll
    for (int i = 0; i < 16; i++) x[i] /= scale;
  }
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; i++) u[i] = encode4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ float finite_amax(const float (&x)[16]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; i++) m = fmaxf(m, is_finite(x[i]) ? fabsf(x[i]) : 0.f);
  return m;
}

// Rows into one block of codes, by NW waves, NC chunks of 16 values per thread.  codes: the block's first row; `scale`:
// its scale, `was` what it was.  kind(r): what becomes of row r of the block, kComes (fetch(r, column, x) has its values), kStays or
// kNone.
enum Kind { kNone, kStays, kComes };

template <int NW, int NC, typename KindOf, typename Fetch>
__device__ __forceinline__ void put_rows(uint8_t* codes, int64_t pitch, float* scale, float was, bool any_stays, int rows,
                                         int d, KindOf kind, Fetch fetch) {
  __shared__ float wave_amax[NW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per_row = d >> 4;
  const float inv = 1.f / (float)per_row;
  float x[NC][16];
  int row[NC], what[NC];
  float amax = 0.f;
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int chunk = tid + c * NW * 64;
    row[c] = (int)(((float)chunk + 0.5f) * inv);  // chunk / per_row: chunk < 2048, per_row <= 16
    what[c] = row[c] < rows ? kind(row[c]) : kNone;
    if (what[c] == kComes) {
      fetch(row[c], (chunk - row[c] * per_row) * 16, x[c]);
      amax = fmaxf(amax, finite_amax(x[c]));
    }
  }
  auto higher = [](uint32_t a, uint32_t b) { return a > b ? a : b; };  // magnitudes order as their bits
  amax = __uint_as_float(wave_reduce(__float_as_uint(amax), higher));
  if (NW > 1) {
    if (lane == 0) wave_amax[wave] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; w++) amax = fmaxf(amax, wave_amax[w]);
  }
  float now = scale_for(amax);
  if (any_stays) now = fmaxf(now, was);
  const bool grown = any_stays && now > was;
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int column = (tid + c * NW * 64 - row[c] * per_row) * 16;
    uint4* at = reinterpret_cast<uint4*>(codes + row[c] * pitch + column);
    if (what[c] == kComes) {
      *at = encode16(x[c], now);
    } else if (what[c] == kStays && grown) {
      decode16(*at, x[c], was);
      *at = encode16(x[c], now);
    }
  }
  if (tid == 0) *scale = now;
}

// Grid: blocks that a head's new rows may touch, heads, K and V.
template <typename T, int NW, int NC>
__global__ __launch_bounds__(NW * 64) void kv8_append(Kv8Plan pl, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                      const int32_t* __restrict__ first_position) {
  const int bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int old = kv8_old_rows(pl, bh), end = old + pl.n_block;
  const int block = (old >> pl.block_shift) + blockIdx.x, rows = 1 << pl.block_shift, first = block << pl.block_shift;
  if (first >= end) return;
  const bool is_v = blockIdx.z != 0;
  const T* from = (is_v ? v_new : k_new) + b * pl.nsb + h * pl.nsh;
  uint8_t* codes = (is_v ? pl.v : pl.k) + b * pl.sb + h * pl.sh + (int64_t)first * pl.st;
  float* scale = (is_v ? pl.v_scale : pl.k_scale) + b * pl.ssb + h * pl.ssh + block;
  const bool stays = first < old;
  if (!is_v) {
    for (int r = first + threadIdx.x; r < first + rows; r += NW * 64)
      if (r >= old && r < end) {
        const int64_t at = b * pl.rsb + h * pl.rsh + r;
        if (pl.weight) pl.weight[at] = 0.f;
        if (pl.position) pl.position[at] = first_position ? first_position[b] + (r - old) : r;
      }
  }
  put_rows<NW, NC>(
      codes, pl.st, scale, stays ? *scale : 0.f, stays, rows, pl.d,
      [&](int r) { return first + r < old ? kStays : first + r < end ? kComes : kNone; },
      [&](int r, int column, float(&x)[16]) { load16(from + (int64_t)(first + r - old) * pl.nst + column, x); });
}

// The order of eviction: the latest rows, then by weight.  Never 0 for a row.
__device__ __forceinline__ uint32_t evict_key(float weight, int position, int latest, int n_recent) {
  if ((int64_t)position > (int64_t)latest - n_recent) return 0xffffffffu;
  return max(min(order_key(weight), 0xff800001u), 1u);
}

// Which rows stay, and which row takes the place of one that goes.  One workgroup per head; the keys are made again in every sweep.
// Leaves row_from, n_kept, the moved rows' weight and position, and the scales of the block that K cuts (blocks below it
// take rows of it, and it takes rows itself).
__global__ __launch_bounds__(1024) void kv8_choose(Kv8Plan pl, const int32_t* __restrict__ budgets, int32_t* n_kept,
                                                   int32_t* row_from, int pitch, int32_t* sources, float2* cut_scales) {
  __shared__ uint32_t hist_rep[256 * kHistCopies];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t wave_a[16], wave_b[16];
  __shared__ int wave_latest[16];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int bh = blockIdx.x, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int n = kv8_old_rows(pl, bh) + pl.n_block;
  int M = pl.budget;
  if (budgets) M = max(0, min(M, budgets[b]));
  const int K = min(M, n);
  float* weight = pl.weight + b * pl.rsb + h * pl.rsh;
  int32_t* position = pl.position ? pl.position + b * pl.rsb + h * pl.rsh : nullptr;
  int32_t* out = row_from + (size_t)bh * pitch;
  int32_t* src = sources + (size_t)bh * pitch;
  if (tid == 0) {
    const int64_t cut = b * pl.ssb + h * pl.ssh + (K >> pl.block_shift);
    cut_scales[bh] = K < n ? make_float2(pl.k_scale[cut], pl.v_scale[cut]) : make_float2(0.f, 0.f);
  }
  if (K == n || K == 0) {  // all stay, or none
    for (int i = tid; i < pitch; i += 1024) out[i] = i < K ? i : -1;
    if (tid == 0) n_kept[bh] = K;
    return;
  }
  int latest = INT32_MIN;
  for (int i = tid; i < n; i += 1024) latest = max(latest, position ? position[i] : i);
  latest = (int)(wave_reduce((uint32_t)latest ^ 0x80000000u, [](uint32_t x, uint32_t y) { return x > y ? x : y; }) ^ 0x80000000u);
  if (lane == 0) wave_latest[wave] = latest;
  for (int i = tid; i < 256 * kHistCopies; i += 1024) hist_rep[i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; w++) latest = max(latest, wave_latest[w]);

  const int groups = (n + 1023) / 1024;  // 64-wide groups per wave
  const int base = wave * groups * 64 + lane;
  auto key_at = [&](int i) -> uint32_t { return i < n ? evict_key(weight[i], position ? position[i] : i, latest, pl.n_recent) : 0u; };

  uint32_t prefix = 0, mask = 0, kth = (uint32_t)K;
#pragma unroll 1
  for (int pass = 0; pass < 4; pass++) {
    const int shift = 24 - 8 * pass;
    for (int j = 0; j < groups; j++) {
      const uint32_t key = key_at(base + j * 64);
      if (key != 0 && (key & mask) == prefix) hist_count(hist_rep, (key >> shift) & 255u, lane);
    }
    __syncthreads();
    hist_fold(hist_rep, hist, tid);
    __syncthreads();
    uint32_t bin, above;
    locate_digit(hist, kth, lane, bin, above);
    prefix |= bin << shift;
    mask |= 255u << shift;
    kth -= above;
  }
  const uint32_t thr = prefix, need_eq = kth;

  // ties before this wave
  uint32_t ceq = 0;
  for (int j = 0; j < groups; j++) ceq += __popcll(__ballot(key_at(base + j * 64) == thr));
  if (lane == 0) wave_a[wave] = ceq;
  __syncthreads();
  uint32_t eq_first = 0;
  for (int w = 0; w < wave; w++) eq_first += wave_a[w];
  auto each = [&](auto f) {
    uint32_t eq = eq_first;
    for (int j = 0; j < groups; j++) {
      const int i = base + j * 64;
      const uint32_t key = key_at(i);
      const uint64_t beq = __ballot(key == thr);
      f(i, key > thr || (key == thr && eq + lanes_below(beq) < need_eq));
      eq += __popcll(beq);
    }
  };
  __syncthreads();  // wave_a has been read
  uint32_t holes = 0, from = 0;
  each([&](int i, bool kept) {
    holes += __popcll(__ballot(i < K && !kept));
    from += __popcll(__ballot(i >= K && kept));
  });
  if (lane == 0) wave_a[wave] = holes, wave_b[wave] = from;
  __syncthreads();
  holes = 0, from = 0;
  for (int w = 0; w < wave; w++) holes += wave_a[w], from += wave_b[w];
  each([&](int i, bool kept) {
    const uint64_t m = __ballot(i >= K && kept);
    if (i >= K && kept) src[from + lanes_below(m)] = i;
    from += __popcll(m);
  });
  __threadfence_block();
  __syncthreads();
  // weight and position below K change only in the places that are looked at no more
  each([&](int i, bool kept) {
    const bool hole = i < K && !kept;
    const uint64_t m = __ballot(hole);
    if (i < K) out[i] = hole ? src[holes + lanes_below(m)] : i;
    holes += __popcll(m);
  });
  __threadfence_block();
  __syncthreads();
  for (int i = tid; i < pitch; i += 1024) {
    if (i >= K) {
      out[i] = -1;
      continue;
    }
    const int f = out[i];
    if (f == i) continue;
    weight[i] = weight[f];
    if (position) position[i] = position[f];
  }
  if (tid == 0) n_kept[bh] = K;
}

// Grid: blocks of the kept rows, heads, K and V.
template <int NW, int NC>
__global__ __launch_bounds__(NW * 64) void kv8_move(Kv8Plan pl, const int32_t* __restrict__ n_kept,
                                                    const int32_t* __restrict__ row_from, int pitch,
                                                    const float2* __restrict__ cut_scales) {
  const int bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int K = n_kept[bh], block = blockIdx.x, rows = 1 << pl.block_shift, first = block << pl.block_shift;
  const int32_t* from = row_from + (size_t)bh * pitch + first;
  const int here = min(rows, K - first);  // kept rows of this block
  bool comes = false, stays = false;
  for (int r = threadIdx.x; r < here; r += NW * 64) {
    if (from[r] == first + r) stays = true;
    else comes = true;
  }
  if (!__syncthreads_or(comes)) return;
  stays = __syncthreads_or(stays);
  const bool is_v = blockIdx.z != 0;
  uint8_t* head = (is_v ? pl.v : pl.k) + b * pl.sb + h * pl.sh;
  float* scale = (is_v ? pl.v_scale : pl.k_scale) + b * pl.ssb + h * pl.ssh;
  const int cut = K >> pl.block_shift;
  const float cut_scale = is_v ? cut_scales[bh].y : cut_scales[bh].x;
  const bool is_cut = block == cut;
  put_rows<NW, NC>(
      head + (int64_t)first * pl.st, pl.st, scale + block, is_cut ? cut_scale : scale[block], stays, here, pl.d,
      [&](int r) { return from[r] == first + r ? kStays : kComes; },
      [&](int r, int column, float(&x)[16]) {
        const int f = from[r], fb = f >> pl.block_shift;
        decode16(*reinterpret_cast<const uint4*>(head + (int64_t)f * pl.st + column), x, fb == cut ? cut_scale : scale[fb]);
      });
}

// The shape of a workgroup that holds a block's chunks in registers, four per thread before waves are added: f(waves, chunks).
template <typename F>
void with_block_shape(const Kv8Plan& pl, F f) {
  const int chunks = (pl.d >> 4) << pl.block_shift;
  using std::integral_constant;
  if (chunks <= 64) f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (chunks <= 128) f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else if (chunks <= 256) f(integral_constant<int, 1>{}, integral_constant<int, 4>{});
  else if (chunks <= 512) f(integral_constant<int, 2>{}, integral_constant<int, 4>{});
  else if (chunks <= 1024) f(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  else f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

hipError_t launch_kv8_append(const Kv8Plan& pl, const void* k_new, const void* v_new, const int32_t* first_position,
                             hipStream_t stream) {
  // where all heads hold n_cached rows the touched blocks are known
  const int T = 1 << pl.block_shift, into = pl.n_ctx ? T - 1 : pl.n_cached & (T - 1);
  const dim3 grid((unsigned)((into + pl.n_block + T - 1) / T), pl.nb * pl.Hkv, 2);
  with_block_shape(pl, [&](auto nw, auto nc) {
    constexpr int NW = decltype(nw)::value, NC = decltype(nc)::value;
    if (pl.dtype == EPICACHE_DTYPE_BF16)
      hipLaunchKernelGGL((kv8_append<__hip_bfloat16, NW, NC>), grid, dim3(NW * 64), 0, stream, pl,
                         static_cast<const __hip_bfloat16*>(k_new), static_cast<const __hip_bfloat16*>(v_new), first_position);
    else
      hipLaunchKernelGGL((kv8_append<float, NW, NC>), grid, dim3(NW * 64), 0, stream, pl, static_cast<const float*>(k_new),
                         static_cast<const float*>(v_new), first_position);
  });
  return hipGetLastError();
}

// Workspace: the sources of every head, row_from where the caller has no room for it, the cut blocks' scales.
size_t kv8_evict_workspace(const Kv8Plan& pl) {
  const size_t heads = (size_t)pl.nb * pl.Hkv;
  return 2 * align256(heads * kv8_most_kept(pl) * sizeof(int32_t)) + align256(heads * sizeof(float2));
}

hipError_t launch_kv8_evict(const Kv8Plan& pl, const int32_t* budgets, int32_t* n_kept, int32_t* row_from, void* workspace,
                            hipStream_t stream) {
  const int heads = pl.nb * pl.Hkv, pitch = kv8_most_kept(pl), T = 1 << pl.block_shift;
  char* ws = static_cast<char*>(workspace);
  int32_t* sources = reinterpret_cast<int32_t*>(ws);
  ws += align256((size_t)heads * pitch * sizeof(int32_t));
  if (!row_from) row_from = reinterpret_cast<int32_t*>(ws);
  ws += align256((size_t)heads * pitch * sizeof(int32_t));
  float2* cut_scales = reinterpret_cast<float2*>(ws);
  hipLaunchKernelGGL(kv8_choose, dim3(heads), dim3(1024), 0, stream, pl, budgets, n_kept, row_from, pitch, sources, cut_scales);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  with_block_shape(pl, [&](auto nw, auto nc) {
    constexpr int NW = decltype(nw)::value, NC = decltype(nc)::value;
    hipLaunchKernelGGL((kv8_move<NW, NC>), dim3((pitch + T - 1) / T, heads, 2), dim3(NW * 64), 0, stream, pl, n_kept, row_from,
                       pitch, cut_scales);
  });
  return hipGetLastError();
}

}  // namespace epicache
