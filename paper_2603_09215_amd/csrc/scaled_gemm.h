// Products of 8-bit rows and packed weights.  Two instructions do them:
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 weight rows x 128 with 128 x 16 rows of activations, takes both
// operands' powers of two from a byte per lane, and adds to fp32 sums.  Before it adds, it brings the products of eight
// neighbouring codes to the exponent of the largest and cuts them 13 bits below it (measured: 2^16 and 2^3 add up, 2^2 is
// lost; across eights nothing is), at most 2^-10 of their magnitudes and 1.4e-5 of the result for normal data.  Outputs
// of 16 bits, rounded at 2^-8, take it.
//
// v_mfma_f32_16x16x32_f16, at half the rate, on the codes as fp16, the weights' times their power relative to their row's
// largest: fp16 holds that exactly down to 2^-15 of that power and to 2^-25 of it (2^-32 of the row's largest weight)
// below.  Four of them are a block of 128, whose sum is multiplied by the activations' power and added in fp32; the weights'
// largest power multiplies the whole.  Outputs in fp32 and pairs take it: 1e-7 of the result.
//
// Operand lane l holds 32 codes of row l mod 16; which 32 of the 128 does not matter as long as both operands agree, so
// the lanes hold what loads well (scaled_rows.h, packed weights).  Of the result, lane l holds weight rows
// 4 (l / 16) .. + 3 of activation row l mod 16: four neighbouring outputs of one row.
#pragma once
#include <type_traits>

#include "scaled_rows.h"

namespace spark {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct GemmArgs {
  const uint8_t *codes, *powers;          // of the rows
  const uint8_t *weights, *weight_powers, *weight_tops;
  int m, n, k;
  int row_blocks;                         // of the weights
  void *out;                              // [m][n], or the codes of 8-bit rows
  uint8_t *out_powers;
  long long out_stride;
};

// A number that is the same for the whole wave, into a scalar register: quotients are worked out in vector registers, and a
// buffer descriptor made of one is otherwise sorted out lane by lane, load by load.
__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
// where part i of n of the groups begins (groups: 8192 at most, parts: 8192)
__device__ __forceinline__ int part_begin(int groups, int i, int n) { return scalar((unsigned)groups * i / n); }

// Loads by buffer descriptor: what lies behind its end reads as zero and asks memory for nothing.
typedef __amdgpu_buffer_rsrc_t buffer_t;
__device__ __forceinline__ buffer_t buffer_of(const void *p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, 0x00027000);
}
constexpr int ONCE = 2;   // read once on this chip
// (all of an offset in the lane's part, which the check against the end covers for certain)
template <int HINT> __device__ __forceinline__ i32x8 buffer_operand(const buffer_t &b, unsigned at, int apart) {
  const i32x4 u = __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, 0, HINT), v = __builtin_amdgcn_raw_buffer_load_b128(b, (int)(at + apart), 0, HINT);
  return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ uint32_t buffer_word(const buffer_t &b, unsigned at) { return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(b, (int)at, 0, 0); }

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <typename CODES, int N> __device__ __forceinline__ void scaled_f16(const CODES &c, float s, f16x8 (&v)[N]) {   // 8 N codes times s
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * q], s, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * q], s, true);
    const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * q + 1], s, false), e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c[2 * q + 1], s, true);
    v[q] = f16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
  }
}
__device__ __forceinline__ uint32_t byte_of(uint32_t bytes, int j) { return bytes >> (8 * j) & 255u; }
// 2^(byte - top), byte <= top; far down: 0
__device__ __forceinline__ float power_below(uint32_t byte, uint32_t top) { return __uint_as_float((uint32_t)max((int)byte - (int)top + 127, 0) << 23); }
// The sums are without the weights' largest power until the end, and times 2^-ROOM: of numbers that fp32 holds times weights of 448
// at most, 2^22 of them, every sum is then less than 2^(128 + 8.9 + 22 - 32), finite.  fp32's smallest step makes them multiples of
// 2^(ROOM - 149) of that largest power; the activations' power itself is exact down to 2^(ROOM - 149).
constexpr int ROOM = 32;
__device__ __forceinline__ float power_with_room(uint32_t byte) { return __uint_as_float(byte << 23) * (1.0f / (float)(1ll << ROOM)); }
// at the end the sums times 2^(top - 127 + ROOM), rounded once; that may be no fp32 number, so it is added to their exponents
__device__ __forceinline__ f32x4 with_tops(const f32x4 &v, uint32_t tops) {
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_ldexpf(v[i], (int)byte_of(tops, i) + (ROOM - 127));
  return r;
}

// four neighbouring outputs of a row
template <typename OUT> __device__ __forceinline__ void store_four(OUT *row, int o, int n, bool vec, const f32x4 &v) {
  if constexpr (sizeof(OUT) == 4) {
    if (vec && o + 3 < n) { *(f32x4 *)(row + o) = v; return; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (o + i < n) row[o + i] = v[i];
  } else {
    if (vec && o + 3 < n) {
      *(uint2 *)(row + o) = make_uint2(f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16), f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16));
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (o + i < n) row[o + i] = f32_to_bf16(v[i]);
  }
}

__device__ __forceinline__ float silu_times(float g, float u) { return g / (1.0f + expf(-g)) * u; }

// ------------------------------------------------------------------ few rows: the weights stream through registers

// What bounds it: the weights' way from memory.  A wave holds a group of four k blocks (8 KiB) of a row block in registers
// and asks for its successor block by block as it uses it, so that about that much is always on its way.
// All of these loads are unconditional (a load that may be skipped makes the next wait one for everything); behind the
// range they read zeros from nowhere, and zeros add nothing.

// The weights' side of a wave: row block nb, groups [g0, g1) of four k blocks
template <bool FP32> struct WeightStream {
  buffer_t codes, powers;
  unsigned end, powers_end;
  uint32_t top;   // (of the lane's row)
  i32x8 c[4];
  uint32_t p;
  __device__ __forceinline__ WeightStream(const GemmArgs &a, int nb, int g0, int g1) {
    const int blocks = sr_blocks(a.k), groups = sr_pitch(a.k) / 4;
    end = (unsigned)min(g1 * 4, blocks) * SW_TILE;
    powers_end = g1;
    codes = buffer_of(a.weights + (long long)nb * blocks * SW_TILE, end);
    powers = buffer_of(a.weight_powers + (long long)nb * groups * 64, powers_end * 64);
    ask_powers(g0);
    if (FP32) top = a.weight_tops[(long long)nb * 16 + (threadIdx.x & 15)];
#pragma unroll
    for (int j = 0; j < 4; ++j) ask(g0, j);
  }
  __device__ __forceinline__ void ask(int g, int j) {
    c[j] = buffer_operand<ONCE>(codes, (threadIdx.x & 63) * 16 + min((unsigned)(g * 4 + j) * SW_TILE, end), 1024);
  }
  __device__ __forceinline__ void ask_powers(int g) { p = buffer_word(powers, (threadIdx.x & 15) * 4 + min((unsigned)g, powers_end) * 64); }
};

// acc += a block's products; wp, xp: the rows' bytes of its group, j its number in it
template <bool FP32> __device__ __forceinline__ void add_block(f32x4 &acc, const i32x8 &w, const f16x8 (&wf)[4], const i32x8 &x, uint32_t wp, uint32_t xp, int j) {
  if constexpr (FP32) {
    f16x8 xf[4];
    scaled_f16(x, 1.0f, xf);
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) t = __builtin_amdgcn_mfma_f32_16x16x32_f16(wf[q], xf[q], t, 0, 0, 0);
    const float power = power_with_room(byte_of(xp, j));
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = fmaf(t[i], power, acc[i]);
  } else {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, 0, (int)(wp >> (8 * j)), 0, (int)(xp >> (8 * j)));
  }
}

// out = X W^T, up to 16 rows.  A workgroup has nw row blocks, kw waves each, which share k; their sums meet in
// LDS, added in order.  IN_LDS: the rows' codes lie in LDS, fetched once for all waves, rows 16 bytes apart beyond their length
// so that sixteen of them read side by side meet in no bank; otherwise (long rows) each wave reads its part of them itself, a
// byte beside every byte of the weights.  4608 x 3584: 6.7 us with one row, 9.2 with 16 (floor 2.5, a plain read in the same
// pieces 4.7); 3584 x 18944: 14.5 us with one (4.7 TB/s; 224 of 256 CUs have a row block), 18.5 with 16.
template <bool IN_LDS, typename OUT>
__global__ void __launch_bounds__(1024) scaled_stream_k(GemmArgs a, int nw, int kw) {
  constexpr bool FP32 = sizeof(OUT) == 4;
  extern __shared__ i32x4 lds[];   // [m][kp + 16 bytes], [m][pitch / 4 words]; then the sums [wave][64]
  const int wave = scalar(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15;
  const int first = blockIdx.x * nw, mine = scalar(wave / kw), part = wave - mine * kw;
  const int blocks = sr_blocks(a.k), pitch = sr_pitch(a.k), groups = pitch / 4, kp = blocks * SR_BLOCK;
  const int g0 = part_begin(groups, part, kw), g1 = part_begin(groups, part + 1, kw);   // (kw <= groups)
  const int wide = kp / 16, total = a.m * wide, words = a.m * groups;   // of the rows' codes sixteens, of their powers words, the rows one behind the other
  // (asked for before the weights, so that the rows lie in LDS by the time those come)
  i32x4 x_first;
  uint32_t xp_first;
  if constexpr (IN_LDS) {
    x_first = ((const i32x4 *)a.codes)[min((int)threadIdx.x, total - 1)];
    xp_first = ((const uint32_t *)a.powers)[min((int)threadIdx.x, words - 1)];
  }
  uint32_t tops = 0u;   // of the four outputs that this thread adds up at the end
  if constexpr (FP32) tops = ((const uint32_t *)a.weight_tops)[(long long)min(first + (int)(threadIdx.x >> 6), a.row_blocks - 1) * 4 + (lane >> 4)];
  WeightStream<FP32> ws(a, min(first + mine, a.row_blocks - 1), g0, g1);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  i32x8 c[4];
  uint32_t p = 0u;
  const buffer_t xb = buffer_of(a.codes, (unsigned)a.m * kp), xpb = buffer_of(a.powers, (unsigned)a.m * pitch);
  const int row = min(col, a.m - 1);   // (columns behind the last row repeat it, and are not stored)
  uint32_t *xpl = (uint32_t *)(lds + a.m * (wide + 1));
  auto ask = [&](int g, int j) { c[j] = buffer_operand<0>(xb, (unsigned)row * kp + (lane >> 4) * 16 + min(g * 4 + j, blocks - 1) * SR_BLOCK, 64); };
  auto ask_power = [&](int g) { p = buffer_word(xpb, (unsigned)row * pitch + g * 4); };
  if constexpr (IN_LDS) {
    if ((int)threadIdx.x < total) lds[threadIdx.x + threadIdx.x / wide] = x_first;
    if ((int)threadIdx.x < words) xpl[threadIdx.x] = xp_first;
    constexpr int AHEAD = 4;
    for (int i0 = threadIdx.x + blockDim.x; i0 < total; i0 += AHEAD * blockDim.x) {
      i32x4 v[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) v[u] = ((const i32x4 *)a.codes)[min(i0 + u * (int)blockDim.x, total - 1)];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u * (int)blockDim.x;
        if (i < total) lds[i + i / wide] = v[u];
      }
    }
    for (int i = threadIdx.x + blockDim.x; i < words; i += blockDim.x) xpl[i] = ((const uint32_t *)a.powers)[i];
    __syncthreads();
  } else {
    ask_power(g0);
#pragma unroll
    for (int j = 0; j < 4; ++j) ask(g0, j);
  }
  auto turn = [&](int g, auto more) {
    constexpr bool MORE = decltype(more)::value;
    const uint32_t wp = ws.p, xp = IN_LDS ? xpl[row * groups + g] : p;
    if constexpr (MORE) {
      ws.ask_powers(g + 1);
      if constexpr (!IN_LDS) ask_power(g + 1);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int kb = min(g * 4 + j, blocks - 1);   // (behind the last block: the last, times zeros)
      f16x8 wf[4];
      if constexpr (FP32) scaled_f16(ws.c[j], power_below(byte_of(wp, j), ws.top), wf);
      i32x8 x;
      if constexpr (IN_LDS) {
        const i32x4 *at = lds + row * (wide + 1) + (lane >> 4) + kb * 8;
        x = __builtin_shufflevector(at[0], at[4], 0, 1, 2, 3, 4, 5, 6, 7);
      } else {
        x = c[j];
      }
      add_block<FP32>(acc, ws.c[j], wf, x, wp, xp, j);
      if constexpr (MORE) {
        ws.ask(g + 1, j);
        if constexpr (!IN_LDS) ask(g + 1, j);
      }
    }
  };
  for (int g = g0; g + 1 < g1; ++g) turn(g, std::true_type());
  turn(g1 - 1, std::false_type());
  f32x4 *sums = (f32x4 *)lds;
  if constexpr (IN_LDS) __syncthreads();
  sums[wave * 64 + lane] = acc;
  __syncthreads();
  if (threadIdx.x >= nw * 64) return;
  const int b = threadIdx.x >> 6, r = col;
  if (r >= a.m || first + b >= a.row_blocks) return;
  const bool vec = a.out_stride % 4 == 0 && ((uintptr_t)a.out & (4 * sizeof(OUT) - 1)) == 0;
  f32x4 v = sums[b * kw * 64 + lane];
  for (int w = 1; w < kw; ++w) v += sums[(b * kw + w) * 64 + lane];
  if constexpr (FP32) v = with_tops(v, tops);
  store_four((OUT *)a.out + r * a.out_stride, (first + b) * 16 + (lane >> 4) * 4, a.n, vec, v);
}

// ------------------------------------------------------------------ tiles

__device__ __forceinline__ void tile_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Where a workgroup's tile lies: workgroups come to the eight XCDs in turn, and each XCD has a run of the tiles, those of
// one part of the weights next to each other, so that its L2 has that part once.
struct TilePlace { int n, m, split; };
__device__ __forceinline__ TilePlace tile_place(int n_tiles, int m_tiles) {
  const int total = gridDim.x, xcd = blockIdx.x & 7, each = total >> 3, rest = total & 7;
  const int id = xcd * each + min(xcd, rest) + (blockIdx.x >> 3);
  const int q = scalar(id / m_tiles), split = scalar(q / n_tiles);
  return TilePlace{q - split * n_tiles, id - q * m_tiles, split};
}

// What a tile's sums become: outputs of the type OUT, the 8-bit rows of a pair (`gated`), or, where k is cut (`parts`), fp32
// sums for a finishing launch, [split][row][16 row blocks].
enum TileEnd { TILE_OUT, TILE_GATED, TILE_PARTS };

// Eight waves of NT row blocks each, 16 MT rows.  The weights go from memory into registers, RB k blocks ahead, each to one
// wave; the rows' codes, which all waves share, through LDS in operand order, two buffers, a barrier per k block.  For
// outputs in fp32 they lie there as fp16, converted once instead of by every wave: twice the LDS, 70 % fewer conversions (2048 rows,
// a pair of 13696 x 4096: 452 -> 436 us).
// What it reaches: 2048 x 8192 x 8192 in 146 us with outputs in bf16 (1.88 PFLOP/s), 246 in fp32 (1.12); 1023 x 4096 x 13696
// 77 and 115 us.  The matrix units are busy 45 % of the time at the 2.0 GHz the chip then runs at;
// the rest goes to the tiles' way from L2 through the vector cache (weights fetched by two waves each, four row blocks a
// wave: bf16 162 -> 197 us) and from LDS.  Two k blocks per barrier and conversions
// placed between the matrix instructions by hand were all within 2 %.
// RB = 2: 32 x 3584 x 18944 in 19.1 us, pairs of 24 rows 26.8 and 64 rows 33.9; four blocks ahead 22.0, 27.7 and 36.2, one 20.4, 27.1 and 35.8.
// Few rows are bound by the weights' way: a pair of 18944 x 3584 with one row 26.0 us, 136 MB (a plain read: 20.4).
constexpr int TILE_WAVES = 8;
template <int NT, int MT, bool FP32, TileEnd END, typename OUT>
__global__ void __launch_bounds__(64 * TILE_WAVES) scaled_tile_k(GemmArgs a, int n_tiles, int m_tiles, int splits) {
  constexpr int WAVES = TILE_WAVES, RB = 2;
  constexpr int UNITS = 2 * MT, UN = (UNITS + WAVES - 1) / WAVES;   // units of the rows: 1 KiB of codes
  constexpr int UNIT = FP32 ? 128 : 64;   // sixteens of one in LDS
  constexpr int WORDS = 64 * WAVES;   // a thread has a word of the powers of either operand, wanted or not: a branch in the loop lets the compiler gather the products of several blocks behind it
  static_assert(END != TILE_GATED || (NT % 2 == 0 && NT * WAVES == 16), "a block of 128 outputs of both matrices");
  extern __shared__ i32x4 lds[];   // [2][MT][half][64] codes (FP32: [2][MT][quarter][64] fp16), [2][2][WORDS] words of powers; gated: then [16 MT][OUT_PITCH] floats
  constexpr int OUT_PITCH = SR_BLOCK + 4, XROWS = 16 * MT, WROWS = 16 * NT * WAVES;
  uint32_t *words = (uint32_t *)(lds + 2 * UNITS * UNIT);
  const int wave = scalar(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, part = lane >> 4;
  const TilePlace at = tile_place(n_tiles, m_tiles);
  const int blocks = sr_blocks(a.k), pitch = sr_pitch(a.k), groups = pitch / 4, kp = blocks * SR_BLOCK;
  const int g0 = part_begin(groups, at.split, splits), g1 = part_begin(groups, at.split + 1, splits);
  const int kb0 = g0 * 4, kb1 = min(g1 * 4, blocks);
  const int r0 = at.m * XROWS, rows = min(a.m - r0, XROWS);
  const unsigned x_end = (unsigned)rows * kp, xp_end = (unsigned)rows * pitch;
  const buffer_t xb = buffer_of(a.codes + (long long)r0 * kp, x_end), xpb = buffer_of(a.powers + (long long)r0 * pitch, xp_end);
  // NT row blocks one after the other; those behind the last read as zeros
  const int tile_nb = at.n * WAVES * NT, nb = tile_nb + wave * NT, have = max(0, min(NT, a.row_blocks - nb));
  const unsigned w_end = (unsigned)have * blocks * SW_TILE;
  const buffer_t wb = buffer_of(a.weights + (long long)(have ? nb : 0) * blocks * SW_TILE, w_end);
  const unsigned wp_end = (unsigned)min(WAVES * NT, a.row_blocks - tile_nb) * groups * 64;
  const buffer_t wpb = buffer_of(a.weight_powers + (long long)tile_nb * groups * 64, wp_end);

  // (loads come back in the order they were asked for: rows and powers fetched closer to their use than the weights would
  // make the wait for them one for the weights behind)
  i32x4 xs[RB][UN];
  i32x8 w[RB][NT];
  uint32_t xp_next, wp_next;
  auto ask_x = [&](int kb, i32x4 (&to)[UN]) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int unit = (u * WAVES + wave) % UNITS;   // (fewer units than waves: some fetch the same)
      to[u] = __builtin_amdgcn_raw_buffer_load_b128(xb, (int)((unsigned)((unit >> 1) * 16 + col) * kp + (unit & 1) * 64 + part * 16 +
                                                                (kb < kb1 ? (unsigned)kb * SR_BLOCK : x_end)), 0, 0);
    }
  };
  auto put_x = [&](int buffer, const i32x4 (&from)[UN]) {
#pragma unroll
    for (int u = 0; u < UN; ++u) {
      const int unit = (u * WAVES + wave) % UNITS;
      if constexpr (FP32) {
        f16x8 v[2];
        scaled_f16(from[u], 1.0f, v);
        lds[(buffer * UNITS + unit) * 128 + lane] = __builtin_bit_cast(i32x4, v[0]);
        lds[(buffer * UNITS + unit) * 128 + 64 + lane] = __builtin_bit_cast(i32x4, v[1]);
      } else {
        lds[(buffer * UNITS + unit) * 64 + lane] = from[u];
      }
    }
  };
  auto ask_w = [&](int kb, int nt, i32x8 &to) {
    to = buffer_operand<MT <= 4 ? ONCE : 0>(wb, lane * 16 + (kb < kb1 ? (unsigned)(nt * blocks + kb) * SW_TILE : w_end), 1024);
  };
  const unsigned xp_at = threadIdx.x < XROWS ? threadIdx.x * pitch : xp_end, wp_at = threadIdx.x < WROWS ? ((threadIdx.x >> 4) * groups * 16 + (threadIdx.x & 15)) * 4 : wp_end;
  auto ask_powers = [&](int g) {   // a row's word of the group
    xp_next = buffer_word(xpb, xp_at + (g < g1 ? (unsigned)g * 4 : xp_end));
    wp_next = buffer_word(wpb, wp_at + (g < g1 ? (unsigned)g * 64 : wp_end));
  };
  int row_top = 0;
  if constexpr (FP32) row_top = a.weight_tops[(long long)min(tile_nb + (int)(threadIdx.x >> 4), a.row_blocks - 1) * 16 + (threadIdx.x & 15)];
  auto put_powers = [&](int buffer) {
    words[buffer * 2 * WORDS + threadIdx.x] = xp_next;
    uint32_t v = wp_next;
    if constexpr (FP32) {   // relative to the row's largest, as the exponents of fp32 numbers
      v = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) v |= (uint32_t)max((int)byte_of(wp_next, j) - row_top + 127, 0) << (8 * j);
    }
    words[buffer * 2 * WORDS + WORDS + threadIdx.x] = v;
  };
  static_assert(XROWS <= 64 * WAVES && WROWS <= 64 * WAVES, "a thread has a row's word");
  f32x4 acc[NT][MT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t four[FP32 ? NT : 1];   // the largest powers of the rows of the lane's sums
  if constexpr (FP32) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) four[nt] = ((const uint32_t *)a.weight_tops)[(long long)min(nb + nt, a.row_blocks - 1) * 4 + part];
  }
  ask_powers(g0);
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    ask_x(kb0 + b, xs[b]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) ask_w(kb0 + b, nt, w[b][nt]);
  }
  put_powers(g0 & 1);
  put_x(0, xs[0]);
  ask_x(kb0 + RB, xs[0]);
  ask_powers(g0 + 1);
  for (int g = g0; g < g1; ++g) {
    const uint32_t *xw = words + (g & 1) * 2 * WORDS + col, *ww = words + (g & 1) * 2 * WORDS + WORDS + wave * NT * 16 + col;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int kb = g * 4 + j;
      __builtin_amdgcn_sched_barrier(0);   // (blocks worked on side by side take more registers than there are)
      tile_barrier();
      put_x((j + 1) & 1, xs[(j + 1) % RB]);
      ask_x(kb + 1 + RB, xs[(j + 1) % RB]);
      if (j == 3) {
        put_powers((g + 1) & 1);
        ask_powers(g + 2);
      }
      const i32x4 *xl = lds + (j & 1) * UNITS * UNIT + lane;
      if constexpr (FP32) {
        f16x8 wf[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          scaled_f16(w[j % RB][nt], __uint_as_float(byte_of(ww[nt * 16], j) << 23), wf[nt]);
          ask_w(kb + RB, nt, w[j % RB][nt]);
        }
        // the rows' operands come one ahead of their use, and no further: they are 16 registers each
        f16x8 xf[2][4];
        uint32_t xw_of[2];
        auto take_x = [&](int t) {
#pragma unroll
          for (int q = 0; q < 4; ++q) xf[t % 2][q] = __builtin_bit_cast(f16x8, xl[(t * 4 + q) * 64]);
          xw_of[t % 2] = xw[t * 16];
        };
        take_x(0);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          f32x4 sum[NT];
          if (t + 1 < MT) take_x(t + 1);
          const float power = power_with_room(byte_of(xw_of[t % 2], j));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) sum[nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wf[nt][0], xf[t % 2][0], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int q = 1; q < 4; ++q)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sum[nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wf[nt][q], xf[t % 2][q], sum[nt], 0, 0, 0);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nt][t][i] = fmaf(sum[nt][i], power, acc[nt][t][i]);
          if constexpr (NT * MT >= 16) __builtin_amdgcn_sched_barrier(0x7f);
        }
      } else {
        uint32_t wp[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) wp[nt] = ww[nt * 16] >> (8 * j);
        i32x8 x[2];
        uint32_t xp[2];
        auto take_x = [&](int t) {
          x[t % 2] = __builtin_shufflevector(xl[t * 128], xl[t * 128 + 64], 0, 1, 2, 3, 4, 5, 6, 7);
          xp[t % 2] = xw[t * 16] >> (8 * j);
        };
        take_x(0);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          if (t + 1 < MT) take_x(t + 1);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            acc[nt][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[j % RB][nt], x[t % 2], acc[nt][t], 0, 0, 0, (int)wp[nt], 0, (int)xp[t % 2]);
          if constexpr (NT * MT >= 16) __builtin_amdgcn_sched_barrier(0);   // (all of LDS's reads first, then the products: 158 us, not 147)
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) ask_w(kb + RB, nt, w[j % RB][nt]);
      }
    }
  }
  if constexpr (FP32) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int t = 0; t < MT; ++t) acc[nt][t] = with_tops(acc[nt][t], four[nt]);
  }
  if constexpr (END == TILE_GATED) {
    float *outs = (float *)lds;
    tile_barrier();
#pragma unroll
    for (int nt = 0; nt < NT; nt += 2)
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = silu_times(acc[nt][t][i], acc[nt + 1][t][i]);
        *(f32x4 *)(outs + (t * 16 + col) * OUT_PITCH + (wave * NT / 2 + nt / 2) * 16 + part * 4) = v;
      }
    tile_barrier();
    const int sub = threadIdx.x & 15, o = at.n * SR_BLOCK + sub * 8, nblocks = sr_blocks(a.n), npitch = sr_pitch(a.n);
    for (int row = threadIdx.x >> 4; row < XROWS; row += 4 * WAVES) {
      if (row >= rows) break;   // (the same for a row's sixteen lanes)
      const long long r = r0 + row;
      const f32x4 p = *(const f32x4 *)(outs + row * OUT_PITCH + sub * 8), q = *(const f32x4 *)(outs + row * OUT_PITCH + sub * 8 + 4);
      float v[8] = {p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (o + i >= a.n) v[i] = 0.f;
      uint32_t byte;
      const uint2 c = block_codes(v, byte);
      *(uint2 *)((uint8_t *)a.out + (r * nblocks + at.n) * SR_BLOCK + sub * 8) = c;
      uint8_t *powers = a.out_powers + r * npitch;
      if (sub == 0) powers[at.n] = (uint8_t)byte;
      if (at.n == nblocks - 1 && nblocks + sub < npitch) powers[nblocks + sub] = 127;
    }
  } else {
    const bool vec = END == TILE_PARTS || (a.out_stride % 4 == 0 && ((uintptr_t)a.out & (4 * sizeof(OUT) - 1)) == 0);
    const int n = END == TILE_PARTS ? a.row_blocks * 16 : a.n;
    OUT *out = (OUT *)a.out + (END == TILE_PARTS ? (long long)at.split * a.m * a.out_stride : 0);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int row = t * 16 + col;
      if (row < rows) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          if (nt < have) store_four(out + (r0 + row) * a.out_stride, (int)(nb + nt) * 16 + part * 4, n, vec, acc[nt][t]);
      }
    }
  }
}

// N fours of a part, all parts added in order; eight parts are asked for at a time, or their ways from memory follow each other
template <int N> __device__ __forceinline__ void add_parts(const float *p, int splits, long long apart, const int (&at)[N], f32x4 (&v)[N]) {
  constexpr int AHEAD = 8 / N > 2 ? 8 / N : 2;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += AHEAD) {
    f32x4 w[AHEAD][N];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) w[u][i] = *(const f32x4 *)(p + min(s0 + u, splits - 1) * apart + at[i]);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (s0 + u < splits) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += w[u][i];
      }
  }
}

// The parts of a cut k, added in order.  parts [split][m][pitch]; four outputs a thread.  With few rows a launch's own time and one way
// from memory (2 to 4 us), with 1023 x 4096 in two parts 9 us
template <typename OUT>
__global__ void __launch_bounds__(256) scaled_join_k(const float *__restrict__ parts, int splits, int m, int n, int pitch, OUT *__restrict__ out,
                                                     long long out_stride) {
  const int fours = (n + 3) / 4;
  const bool vec = out_stride % 4 == 0 && ((uintptr_t)out & (4 * sizeof(OUT) - 1)) == 0;
  const long long total = (long long)m * fours, apart = (long long)m * pitch;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long r = i / fours;
    const int o = (int)(i - r * fours) * 4;
    const int at[1] = {0};
    f32x4 v[1];
    add_parts<1>(parts + r * pitch + o, splits, apart, at, v);
    store_four(out + r * out_stride, o, n, vec, v[0]);
  }
}
// ... of a pair: sixteen lanes a block of 128 outputs of a row
__global__ void __launch_bounds__(256) scaled_join_gated_k(const float *__restrict__ parts, int splits, int m, int n, int pitch, uint8_t *__restrict__ codes,
                                                           uint8_t *__restrict__ powers) {
  const int blocks = sr_blocks(n), npitch = sr_pitch(n), sub = threadIdx.x & 15;
  const long long total = (long long)m * npitch, apart = (long long)m * pitch;
  for (long long b = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4; b < total; b += (long long)gridDim.x * 16) {
    const long long r = b / npitch;
    const int block = (int)(b - r * npitch), o = block * SR_BLOCK + sub * 8;
    if (block >= blocks) {
      if (sub == 0) powers[r * npitch + block] = 127;
      continue;
    }
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (o < n) {   // outputs o .. + 7 are half a row block of either matrix
      const int at[4] = {0, 4, 16, 20};
      f32x4 gu[4];
      add_parts<4>(parts + r * pitch + (o >> 4) * 32 + (o & 15), splits, apart, at, gu);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (o + i < n) v[i] = silu_times(gu[i >> 2][i & 3], gu[2 + (i >> 2)][i & 3]);
    }
    uint32_t byte;
    const uint2 c = block_codes(v, byte);
    *(uint2 *)(codes + (r * blocks + block) * SR_BLOCK + sub * 8) = c;
    if (sub == 0) powers[r * npitch + block] = (uint8_t)byte;
  }
}

}  // namespace spark
