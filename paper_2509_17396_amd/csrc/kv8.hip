// Rows into the 8-bit cache (epicache_kv8_append) and its eviction by accumulated attention weight (epicache_kv8_evict).
//
// Both write rows into blocks that share a scale, with one rule: the scale of a block is the smallest power of two that
// brings its new values to at most 448, and at least what it was while older rows stay in it (those are rounded again where it
// has grown).  A workgroup owns a block of K or of V, so the scale has one writer: it reads the new rows into registers, takes the
// largest magnitude, and writes codes.  One pass over the data.
// append is bound by memory: 32 x 8 heads of 4096 rows of 128 bf16 (537 MB in, 269 MB out) take 143 us, 5.7 TB/s.  A wave holds a block of 32
// rows of 128 by itself, so that it waits for nobody.
// evict moves a row for every one that goes and no other, instead of closing the gaps: 16 x 8 heads, a third of 24576 rows gone, move 358 MB and
// take 128 us, kv8_choose 22 of them and kv8_move 106 (4.2 TB/s of what the counters see, scattered rows of 128 bytes).
#include <hip/hip_bf16.h>

#include <type_traits>

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

// The largest magnitude among those of 16 codes that are numbers, as a code.
__device__ __forceinline__ uint32_t largest_code(uint4 u) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
  u16x2 most = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    uint32_t x = w[i] & 0x7f7f7f7fu;
    const uint32_t nan = (x + 0x01010101u) & 0x80808080u;
    x &= ~(nan | (nan - (nan >> 7)));
    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x & 0x00ff00ffu));
    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, (x >> 8) & 0x00ff00ffu));
  }
  return most[0] > most[1] ? most[0] : most[1];
}
__device__ __forceinline__ float code_value(uint32_t code) {
  float x[4];
  decode4(code, x);
  return x[0];
}

// What a head's eviction leaves for its moves: row holes[j] gets what row sources[j] holds; starts[i]: the moves into blocks before
// block i.
struct Moves {
  int32_t* holes;    // [heads][pitch]
  int32_t* sources;  // [heads][pitch]
  int32_t* starts;   // [heads][blocks + 1]
  float2* cut;       // [heads]: the scales of the block that K cuts, as they were
  int pitch, blocks;
};

// By one wave: the moves first .. end - 1 of head (b, h), all into block `block`, of K and V and of the rows' weight and position.
// K: rows that stay in the cache.  The block that K cuts may both take and give rows, so its scales as they were come from the caller.
__device__ __forceinline__ void move_block(const Kv8Plan& pl, int b, int h, const int32_t* holes, const int32_t* sources, int first,
                                           int end, int block, int K, float2 cut_scale, int lane) {
  constexpr int kHeld = 2;  // chunks of 16 codes of K and of V per lane that stay in registers between the two looks at them
  const int d = pl.d, shift = pl.block_shift;
  const int64_t pitch = pl.st;
  uint8_t* const codes[2] = {pl.k + b * pl.sb + h * pl.sh, pl.v + b * pl.sb + h * pl.sh};
  float* const scale[2] = {pl.k_scale + b * pl.ssb + h * pl.ssh, pl.v_scale + b * pl.ssb + h * pl.ssh};
  const int per_row = d >> 4, chunks = (end - first) * per_row, cut = K >> shift;
  const float inv = 1.f / (float)per_row;
  const int here = min(1 << shift, K - (block << shift));
  const bool any_stays = end - first < here;
  const float was[2] = {block == cut ? cut_scale.x : scale[0][block], block == cut ? cut_scale.y : scale[1][block]};
  struct Look {
    uint4 u[2];
    float s[2];
    int64_t to;
  };
  auto look = [&](int at, Look& x) {
    const int row = (int)(((float)at + 0.5f) * inv);  // at / per_row: at < 2048, per_row <= 16
    const int from = sources[first + row], column = (at - row * per_row) * 16, block_of = from >> shift;
    x.to = (int64_t)holes[first + row] * pitch + column;
#pragma unroll
    for (int v = 0; v < 2; v++) {
      x.u[v] = *reinterpret_cast<const uint4*>(codes[v] + (int64_t)from * pitch + column);
      x.s[v] = scale[v][block_of];
    }
    if (block_of == cut) x.s[0] = cut_scale.x, x.s[1] = cut_scale.y;
  };
  Look held[kHeld];
  float amax[2] = {0.f, 0.f};
#pragma unroll
  for (int c = 0; c < kHeld; c++)
    if (lane + c * 64 < chunks) look(lane + c * 64, held[c]);
  for (int j = first + lane; j < end; j += 64) {  // rows from K on are not written, so what is read here is what was there
    const int64_t of = b * pl.rsb + h * pl.rsh;
    const int to = holes[j], from = sources[j];
    pl.weight[of + to] = pl.weight[of + from];
    if (pl.position) pl.position[of + to] = pl.position[of + from];
  }
#pragma unroll
  for (int c = 0; c < kHeld; c++)
    if (lane + c * 64 < chunks) {
#pragma unroll
      for (int v = 0; v < 2; v++) amax[v] = fmaxf(amax[v], code_value(largest_code(held[c].u[v])) * held[c].s[v]);
    }
  for (int at = lane + kHeld * 64; at < chunks; at += 64) {
    Look x;
    look(at, x);
#pragma unroll
    for (int v = 0; v < 2; v++) amax[v] = fmaxf(amax[v], code_value(largest_code(x.u[v])) * x.s[v]);
  }
  float now[2];
#pragma unroll
  for (int v = 0; v < 2; v++) {
    amax[v] = __uint_as_float(wave_reduce(__float_as_uint(amax[v]), [](uint32_t x, uint32_t y) { return x > y ? x : y; }));
    now[v] = scale_for(amax[v]);
    if (any_stays) now[v] = fmaxf(now[v], was[v]);
  }
  auto again = [&](uint4 u, float from, float to) {
    if (from == to) return u;
    float x[16];
    decode16(u, x, from);
    return encode16(x, to);
  };
  auto put = [&](const Look& x) {
#pragma unroll
    for (int v = 0; v < 2; v++) *reinterpret_cast<uint4*>(codes[v] + x.to) = again(x.u[v], x.s[v], now[v]);
  };
#pragma unroll
  for (int c = 0; c < kHeld; c++)
    if (lane + c * 64 < chunks) put(held[c]);
  for (int at = lane + kHeld * 64; at < chunks; at += 64) {
    Look x;
    look(at, x);
    put(x);
  }
#pragma unroll
  for (int v = 0; v < 2; v++) {  // the rows that stay, where their scale has grown
    if (!(any_stays && now[v] > was[v])) continue;
    for (int at = lane; at < here * per_row; at += 64) {
      const int row = (int)(((float)at + 0.5f) * inv), i = (block << shift) + row;
      bool moved = false;
      for (int j = first; j < end; j++) moved = moved || holes[j] == i;
      uint4* p = reinterpret_cast<uint4*>(codes[v] + (int64_t)i * pitch + (at - row * per_row) * 16);
      if (!moved) *p = again(*p, was[v], now[v]);
    }
  }
  if (lane == 0) scale[0][block] = now[0], scale[1][block] = now[1];
}

// Which rows stay, and which row takes the place of one that goes.  One workgroup of NW waves per head; VPT keys per thread in
// registers, or (VPT = 0) made again in every sweep where the rows are too many.
// Leaves the moves and n_kept.  FUSED, for at most kFewMoves moves: makes them as well, a wave per block, and row_from_opt.
constexpr int kFewMoves = 64;  // a lane for each
template <int VPT, int NW, bool FUSED>
__global__ __launch_bounds__(NW * 64) void kv8_choose(Kv8Plan pl, const int32_t* __restrict__ budgets, int32_t* n_kept,
                                                      int32_t* row_from_opt, Moves mv) {
  constexpr bool kHeld = VPT > 0;
  constexpr int kRegs = kHeld ? VPT : 4;
  __shared__ SelectLds<NW> sm;
  __shared__ uint32_t hist_rep[kHeld ? 1 : 256 * kHistCopies];
  __shared__ uint32_t hist[kHeld ? 1 : 256];
  __shared__ uint32_t wave_a[NW], wave_b[NW];
  __shared__ int wave_latest[NW];
  __shared__ int32_t near_holes[FUSED ? kFewMoves : 1], near_sources[FUSED ? kFewMoves : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int n = kv8_old_rows(pl, bh) + pl.n_block, shift = pl.block_shift;
  int M = pl.budget;
  if (budgets) M = max(0, min(M, budgets[b]));
  const int K = min(M, n);
  float* weight = pl.weight + b * pl.rsb + h * pl.rsh;
  int32_t* position = pl.position ? pl.position + b * pl.rsb + h * pl.rsh : nullptr;
  float* k_scale = pl.k_scale + b * pl.ssb + h * pl.ssh;
  float* v_scale = pl.v_scale + b * pl.ssb + h * pl.ssh;
  int32_t* out = FUSED && row_from_opt ? row_from_opt + (size_t)bh * mv.pitch : nullptr;
  int32_t* holes_of = mv.holes + (size_t)bh * mv.pitch;
  int32_t* sources_of = mv.sources + (size_t)bh * mv.pitch;
  int32_t* starts = mv.starts + (size_t)bh * (mv.blocks + 1);
  const int kept_blocks = (K + (1 << shift) - 1) >> shift;
  if (K == n || K == 0) {  // all stay, or none
    if (out)
      for (int i = tid; i < mv.pitch; i += NW * 64) out[i] = i < K ? i : -1;
    if (!FUSED)
      for (int i = tid; i <= mv.blocks; i += NW * 64) starts[i] = 0;
    if (tid == 0) n_kept[bh] = K;
    return;
  }
  const float2 cut = make_float2(k_scale[K >> shift], v_scale[K >> shift]);
  if (!FUSED && tid == 0) mv.cut[bh] = cut;

  const int groups = kHeld ? VPT : (n + NW * 64 - 1) / (NW * 64);  // 64-wide groups per wave
  const int base = wave * groups * 64 + lane;
  const bool by_position = pl.n_recent > 0 && position != nullptr;
  int latest = n - 1;
  float w[kRegs];
  int pos[kRegs];
  if constexpr (kHeld) {
#pragma unroll
    for (int j = 0; j < kRegs; j++) w[j] = weight[min(base + j * 64, n - 1)];
    if (by_position) {
#pragma unroll
      for (int j = 0; j < kRegs; j++) pos[j] = position[min(base + j * 64, n - 1)];
    } else {
#pragma unroll
      for (int j = 0; j < kRegs; j++) pos[j] = base + j * 64;
    }
  }
  if (by_position) {
    latest = INT32_MIN;
    if constexpr (kHeld) {
#pragma unroll
      for (int j = 0; j < kRegs; j++) latest = max(latest, pos[j]);
    } else {
      for (int i = tid; i < n; i += NW * 64) latest = max(latest, position[i]);
    }
    latest = (int)(wave_reduce((uint32_t)latest ^ 0x80000000u, [](uint32_t x, uint32_t y) { return x > y ? x : y; }) ^ 0x80000000u);
    if (lane == 0) wave_latest[wave] = latest;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NW; x++) latest = max(latest, wave_latest[x]);
  }
  auto key_at = [&](int i) -> uint32_t {
    return i < n ? evict_key(weight[i], by_position ? position[i] : i, latest, pl.n_recent) : 0u;
  };

  uint32_t keys[kRegs];
  uint32_t thr, need_eq;
  bool cut_ties = true;
  if constexpr (kHeld) {
    uint32_t least = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < kRegs; j++) {
      const uint32_t key = evict_key(w[j], pos[j], latest, pl.n_recent);
      keys[j] = base + j * 64 < n ? key : 0u;
      if (base + j * 64 < n) least = min(least, key);
    }
    const Threshold t = select_threshold<kRegs, NW>(keys, least, n, (uint32_t)K, wave, lane, sm);
    thr = t.thr, need_eq = t.need_eq, cut_ties = t.cut;
  } else {
    for (int i = tid; i < 256 * kHistCopies; i += NW * 64) hist_rep[i] = 0;
    __syncthreads();
    uint32_t prefix = 0, mask = 0, kth = (uint32_t)K;
#pragma unroll 1
    for (int pass = 0; pass < 4; pass++) {
      const int digit = 24 - 8 * pass;
      for (int j = 0; j < groups; j++) {
        const uint32_t key = key_at(base + j * 64);
        if (key != 0 && (key & mask) == prefix) hist_count(hist_rep, (key >> digit) & 255u, lane);
      }
      __syncthreads();
      hist_fold(hist_rep, hist, tid);
      __syncthreads();
      uint32_t bin, above;
      locate_digit(hist, kth, lane, bin, above);
      prefix |= bin << digit;
      mask |= 255u << digit;
      kth -= above;
    }
    thr = prefix, need_eq = kth;
  }
  auto each_key = [&](auto f) {
    if constexpr (kHeld) {
#pragma unroll
      for (int j = 0; j < kRegs; j++) {
        one_group_at_a_time();
        f(base + j * 64, keys[j]);
      }
    } else {
      for (int j = 0; j < groups; j++) f(base + j * 64, key_at(base + j * 64));
    }
  };
  thr = __builtin_amdgcn_readfirstlane(thr);
  uint32_t eq_first = 0;  // ties before this wave, where not all of them stay
  if (cut_ties) {
    uint32_t ceq = 0;
    each_key([&](int, uint32_t key) { ceq += __popcll(__ballot(key == thr)); });
    if (lane == 0) wave_a[wave] = ceq;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NW; x++) eq_first += x < wave ? wave_a[x] : 0;
    __syncthreads();  // wave_a has been read
  }
  // f(row, stays): holes are rows below K that go, sources rows from K on that stay
  auto each_row = [&](auto f) {
    uint32_t eq = eq_first, t = thr;
    asm volatile("" : "+s"(t));  // the masks are made again, not kept in scalar registers from one sweep to the next
    if (cut_ties) {
      each_key([&](int i, uint32_t key) {
        const uint64_t beq = __ballot(key == t);
        f(i, key > t || (key == t && eq + lanes_below(beq) < need_eq));
        eq += __popcll(beq);
      });
    } else {
      each_key([&](int i, uint32_t key) { f(i, key >= t); });
    }
  };
  uint32_t holes = 0, sources = 0;
  each_row([&](int i, bool stays) {
    holes += i < K && !stays;
    sources += i >= K && stays;
  });
  auto add = [](uint32_t x, uint32_t y) { return x + y; };
  holes = wave_reduce(holes, add), sources = wave_reduce(sources, add);
  if (lane == 0) wave_a[wave] = holes, wave_b[wave] = sources;
  __syncthreads();
  holes = 0, sources = 0;
  uint32_t moves = 0;
#pragma unroll
  for (int x = 0; x < NW; x++) {
    if (x < wave) holes += wave_a[x], sources += wave_b[x];
    moves += wave_a[x];
  }
  const uint32_t holes_first = holes;
  if (FUSED) holes_of = near_holes, sources_of = near_sources;
  each_row([&](int i, bool stays) {
    const int first = i - lane;  // rows first .. first + 63 here: all on one side of K, but for the ones around it
    if (first < K) {
      const bool hole = i < K && !stays;
      const uint64_t mask = __ballot(hole);
      const uint32_t before = holes + lanes_below(mask);
      if (hole) holes_of[before] = i;
      if (!FUSED && i < K && (i & ((1 << shift) - 1)) == 0) starts[i >> shift] = (int32_t)before;
      holes += __popcll(mask);
    }
    if (first + 64 > K) {
      const bool source = i >= K && stays;
      const uint64_t mask = __ballot(source);
      if (source) sources_of[sources + lanes_below(mask)] = i;
      sources += __popcll(mask);
    }
  });
  if (!FUSED)
    for (int i = kept_blocks + tid; i <= mv.blocks; i += NW * 64) starts[i] = (int32_t)moves;
  if (tid == 0) n_kept[bh] = K;
  if constexpr (FUSED) {
    __syncthreads();
    if (out) {
      uint32_t before = holes_first;
      each_row([&](int i, bool stays) {
        const bool hole = i < K && !stays;
        const uint64_t mask = __ballot(hole);
        if (i < K) out[i] = hole ? sources_of[before + lanes_below(mask)] : i;
        before += __popcll(mask);
      });
      for (int i = K + tid; i < mv.pitch; i += NW * 64) out[i] = -1;
    }
    if (!kHeld) __syncthreads();  // the keys have been made for the last time: weights may change
    // a wave per block that takes rows in
    const int block_of = lane < (int)moves ? near_holes[lane] >> shift : -1;
    const int before = lane == 0 ? -2 : near_holes[max(lane - 1, 0)] >> shift;
    uint64_t firsts = __ballot(lane < (int)moves && block_of != before);
    for (int x = 0; firsts != 0; x++) {
      const int first = __ffsll((unsigned long long)firsts) - 1;
      firsts &= firsts - 1;
      if (x % NW != wave) continue;
      const int end = firsts ? __ffsll((unsigned long long)firsts) - 1 : (int)moves;
      move_block(pl, b, h, near_holes, near_sources, first, end, __builtin_amdgcn_readlane(block_of, first), K, cut, lane);
    }
  }
}

// The moves, a wave per block, and row_from_opt.
constexpr int kMoveWaves = 4;
__global__ __launch_bounds__(kMoveWaves * 64) void kv8_move(Kv8Plan pl, const int32_t* __restrict__ n_kept, int32_t* row_from_opt,
                                                            Moves mv) {
  __shared__ int32_t row_of[kMoveWaves][128];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.y, b = kv8_batch_of(pl, bh), h = bh - b * pl.Hkv;
  const int block = blockIdx.x * kMoveWaves + wave;
  if (block >= mv.blocks) return;
  const int32_t* starts = mv.starts + (size_t)bh * (mv.blocks + 1);
  const int32_t* holes = mv.holes + (size_t)bh * mv.pitch;
  const int32_t* sources = mv.sources + (size_t)bh * mv.pitch;
  const int first = starts[block], end = starts[block + 1], K = n_kept[bh];
  if (first != end) move_block(pl, b, h, holes, sources, first, end, block, K, mv.cut[bh], lane);
  if (row_from_opt) {
    const int row0 = block << pl.block_shift, rows = min(1 << pl.block_shift, mv.pitch - row0);
    for (int r = lane; r < rows; r += 64) row_of[wave][r] = row0 + r < K ? row0 + r : -1;
    for (int j = first + lane; j < end; j += 64) row_of[wave][holes[j] - row0] = sources[j];
    int32_t* out = row_from_opt + (size_t)bh * mv.pitch + row0;
    for (int r = lane; r < rows; r += 64) out[r] = row_of[wave][r];
  }
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

// Workspace: holes, sources and starts of every head, the cut blocks' scales.
static Moves moves_in(const Kv8Plan& pl, void* workspace, size_t* bytes) {
  const size_t heads = (size_t)pl.nb * pl.Hkv;
  const int T = 1 << pl.block_shift, pitch = kv8_most_kept(pl), blocks = (pitch + T - 1) / T;
  char* ws = static_cast<char*>(workspace);
  size_t at = 0;
  auto take = [&](size_t n) {
    char* p = ws ? ws + at : nullptr;
    at += align256(n);
    return reinterpret_cast<int32_t*>(p);
  };
  Moves mv;
  mv.pitch = pitch, mv.blocks = blocks;
  mv.holes = take(heads * pitch * sizeof(int32_t));
  mv.sources = take(heads * pitch * sizeof(int32_t));
  mv.starts = take(heads * (blocks + 1) * sizeof(int32_t));
  mv.cut = reinterpret_cast<float2*>(take(heads * sizeof(float2)));
  *bytes = at;
  return mv;
}

size_t kv8_evict_workspace(const Kv8Plan& pl) {
  size_t bytes;
  moves_in(pl, nullptr, &bytes);
  return bytes;
}

hipError_t launch_kv8_evict(const Kv8Plan& pl, const int32_t* budgets, int32_t* n_kept, int32_t* row_from, void* workspace,
                            hipStream_t stream) {
  size_t bytes;
  const Moves mv = moves_in(pl, workspace, &bytes);
  const int heads = pl.nb * pl.Hkv, rows = pl.n_cached + pl.n_block;
  // A few moves per head (a decoding step's: 32 heads of 2049 rows 14 us, 22 with a launch of their own) are made by the workgroup that
  // chose them.  Budgets in device memory may ask for many (64 heads of 4067 rows, a quarter of them gone: 60 us so).
  const bool fused = !budgets && rows - mv.pitch <= kFewMoves;
  auto go = [&](auto vpt, auto nw) {
    constexpr int VPT = decltype(vpt)::value, NW = decltype(nw)::value;
    if (fused) hipLaunchKernelGGL((kv8_choose<VPT, NW, true>), dim3(heads), dim3(NW * 64), 0, stream, pl, budgets, n_kept, row_from, mv);
    else hipLaunchKernelGGL((kv8_choose<VPT, NW, false>), dim3(heads), dim3(NW * 64), 0, stream, pl, budgets, n_kept, row_from, mv);
  };
  using std::integral_constant;
  if (rows <= 1024) go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  else if (rows <= 4096) go(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  else if (rows <= 8192) go(integral_constant<int, 8>{}, integral_constant<int, 16>{});
  else if (rows <= 16384) go(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  else if (rows <= 24576) go(integral_constant<int, 24>{}, integral_constant<int, 16>{});
  else if (rows <= 32768) go(integral_constant<int, 32>{}, integral_constant<int, 16>{});
  else go(integral_constant<int, 0>{}, integral_constant<int, 16>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || fused) return e;
  hipLaunchKernelGGL(kv8_move, dim3((mv.blocks + kMoveWaves - 1) / kMoveWaves, heads), dim3(kMoveWaves * 64), 0, stream, pl, n_kept,
                     row_from, mv);
  return hipGetLastError();
}

}  // namespace epicache
