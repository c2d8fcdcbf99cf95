// Attention of new rows over a paged cache (spark_cache_attend).
//
//   out = sum_t exp(s_t - M) v_t / L,  s_t = scale q . k_t,  M = max s_t,  L = sum_t exp(s_t - M),  lse = M + log L
//
// over the slots t that a row sees, in one pass with a running maximum and sum.  The (row, query head) pairs of a sequence and kv
// head share its keys and values; they are counted through, pair p being row p / group and head p mod group, and cut into tiles.
//
//   cached_stream_k  16 pairs: bound by the cache's way through memory.  Each wave has its own tokens.
//   cached_tile_k    128 or 256 pairs, bf16: bound by the matrix units.  A tile of keys and values in LDS serves all waves.
//   cached_join_k    where too few tiles would leave compute units idle, their tokens are cut into `splits` parts, whose
//                    unfinished sums come through the workspace; this adds them up in order.
//
// In all: scores transposed, S^T [token][pair] = K Q^T, so a lane holds scores of one pair and finds their maximum and sum
// by itself; and since a sum over tokens may go in any order, those registers are the operand of O^T = V^T P^T as
// they are, with a bf16 cache as two parts of bf16 (one would be 2^-8 off, as much as the result's own rounding).  Exponentials are of base 2, the
// scores' factor is scale log2 e.
//
// Slots that a row does not see: their scores are replaced, not added to.  Their values meet zeros, and zero times infinity is
// NaN, so behind the first row's last slot values that are no numbers go in as zeros, and what the rows that do see
// them get from them is added at the end (a probability is positive: infinity stays, NaN too).  Slots that all rows see are not
// looked at: if sums that are no numbers come of them, the tile is worked on AGAIN, and takes them all so.  Sums of large values may
// have left fp32's range before they were divided by L: the second time all probabilities are 2^32 smaller (2^23 slots of up to 2^8 each have room), which
// changes no bit of what was in range (but for products below 2^-94, which come close to the smallest numbers); parts say so by a negative sum.
#pragma once
#include "cached_format.h"
#include "cached_plan.h"

namespace spark {

struct AttendArgs {
  CacheView cache;
  BatchView batch;
  const void *q;
  void *out;
  float *lse;     // or nullptr
  float *part;    // splits > 1: sums [split][m][n_q_heads][head_dim], then (maximum, sum) of each
  float2 *part_ml;
  long long q_stride, out_stride;
  int n_q_heads, group, causal, splits;
  bool by_row;    // how tiles are numbered
  float factor;   // |scale| log2 e
  uint32_t flip;  // the sign of scale, put on the queries
};

typedef __attribute__((ext_vector_type(8))) __bf16 ca_bf16x8;
typedef __attribute__((ext_vector_type(4))) uint32_t ca_u32x4;
typedef __attribute__((ext_vector_type(4))) short ca_s16x4;
typedef __attribute__((ext_vector_type(4))) float ca_f32x4;
typedef __attribute__((ext_vector_type(16))) float ca_f32x16;
__device__ __forceinline__ ca_bf16x8 ca_operand(const ca_u32x4 &v) { return __builtin_bit_cast(ca_bf16x8, v); }
template <typename T> __device__ __forceinline__ ca_u32x4 ca_signed(ca_u32x4 v, uint32_t flip) {
  const uint32_t x = sizeof(T) == 4 ? flip : flip | (flip >> 16);
  return ca_u32x4{v.x ^ x, v.y ^ x, v.z ^ x, v.w ^ x};
}
// elements that are no numbers to zero; true if there was one
template <typename T> __device__ __forceinline__ bool ca_only_numbers(ca_u32x4 &v) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      if ((w[i] & 0x7f800000u) == 0x7f800000u) { w[i] = 0u; bad = true; }
    } else {
      if ((w[i] & 0x7f800000u) == 0x7f800000u) { w[i] &= 0xffffu; bad = true; }
      if ((w[i] & 0x7f80u) == 0x7f80u) { w[i] &= 0xffff0000u; bad = true; }
    }
  }
  v = ca_u32x4{w[0], w[1], w[2], w[3]};
  return bad;
}
// The slots of a tile whose values went in as zeros lie in first .. last.  Some of its sums are no numbers: again.
struct BadSlots { int first, last, again; };
__device__ __forceinline__ void note_bad(BadSlots &b, int slot) {
  atomicMin(&b.first, slot);
  atomicMax(&b.last, slot);
}
// (the second time nothing of the first is to be kept for it in registers)
template <bool AGAIN> __device__ __forceinline__ int this_thread() {
  int i = threadIdx.x;
  if constexpr (AGAIN) asm volatile("" : "+v"(i));
  return i;
}
template <bool AGAIN> __device__ __forceinline__ int this_block() {
  int i = blockIdx.x;
  if constexpr (AGAIN) asm volatile("" : "+s"(i));
  return i;
}
__device__ __forceinline__ float ca_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// a value of the other half of the wave, and this one
__device__ __forceinline__ float ca_max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float ca_sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Where the 16-byte piece c of row `row` of a tile lies in LDS: pieces of a row are turned so that the lanes of a read, 16 rows of
// one piece (keys) or four rows of four neighbouring pieces (values), meet different banks.
template <typename T, int HD> __device__ __forceinline__ int ca_turn(int row) {
  if constexpr (HD * sizeof(T) == 128) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
  return ((row & 3) << 2) | ((row >> 2) & 3);
}

// The tile of pairs that a workgroup takes: its sequence, tile in it and tiles of it, or false where there is none.  A sequence's tiles are
// numbered from a place that its first row gives: that row times a row's tiles, or its pairs before, in tiles, and one for every
// sequence before, each of which may leave a tile unfilled.  (Which: attend_tiles_by_row.)  So some numbers are nobody's, and the sequence
// is the last one whose place is not behind the tile: found in steps of 64, one up to 64 sequences, where a count over all
// of them takes a step for each 64 (a step's attention of 2048 dialogues of up to 250 slots: 279 us with the count, 174 with this; 180 since probabilities have two parts).
// Called by whole waves.
__device__ __forceinline__ bool find_tile(const BatchView &b, int page_tokens, int group, int per_tile, bool by_row, int tile, Sequence &q, int &t, int &count) {
  const int lane = threadIdx.x & 63, each = (group + per_tile - 1) / per_tile;
  for (int lo = 0, hi = b.n;;) {
    const int stride = (hi - lo + 63) / 64, s = lo + lane * stride;
    int first = 0, row0 = 0, rows = 0, length = 0;
    if (s < hi) {
      length = b.lengths[s];
      row0 = cut(b.starts[s], 0, b.m);
      rows = cut(b.starts[s + 1], row0, b.m) - row0;
      first = by_row ? row0 * each : row0 * group / per_tile + s;
    }
    const unsigned long long begun = __ballot(s < hi && first <= tile);
    if (!begun) return false;
    const int l = 63 - __clzll(begun);
    if (stride > 1) {
      lo += l * stride;
      hi = min(hi, lo + stride);
      continue;
    }
    q.row0 = __builtin_amdgcn_readlane(row0, l);
    q.rows = __builtin_amdgcn_readlane(rows, l);
    q.length = cut(__builtin_amdgcn_readlane(length, l), 0, b.max_pages * page_tokens);
    q.pages = b.table + (long long)(lo + l) * b.max_pages;
    t = tile - __builtin_amdgcn_readlane(first, l);
    count = (q.rows * group + per_tile - 1) / per_tile;
    return t < count;
  }
}

// the last slot that a row sees, -1: none
__device__ __forceinline__ int last_seen(const Sequence &q, int row, int causal) {
  const int slot = q.slot(row);
  return slot < 0 ? -1 : causal ? slot : q.length - 1;
}

// Where sixteen slots of a sequence lie, in a lane of their own: asked for some steps ahead of their use, so what comes of the table
// is looked at only then.
struct Asked { int page, token; };      // as the table has it, -1 past `end`
struct Found { int there, low, high; };   // is there a page, and their bytes from the first page's start on (of the first page where there is none)
__device__ __forceinline__ Asked ask(const Sequence &q, const CacheView &c, int sixteen, int end) {
  Asked r{-1, 0};
  if (sixteen * 16 < end) {
    int index;
    place_of(c, sixteen, index, r.token);
    r.page = q.pages[index];
  }
  return r;
}
template <int ROW> __device__ __forceinline__ Found find(const Asked &a, const CacheView &c, int type_bytes) {
  Found f;
  f.there = (unsigned)a.page < (unsigned)c.n_pages;
  const unsigned long long at = (unsigned long long)(f.there ? a.page : 0) * (unsigned long long)(c.page_stride * type_bytes) + (unsigned)(a.token * ROW);
  f.low = (int)(uint32_t)at;
  f.high = (int)(uint32_t)(at >> 32);
  return f;
}
// the start of the sixteen that lane i found, in the plane that begins at `plane` in the first page
__device__ __forceinline__ const char *at_lane(const char *plane, const Found &f, int i) {
  return plane + ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane(f.high, i) << 32 | (uint32_t)__builtin_amdgcn_readlane(f.low, i));
}

template <typename T, int HD>
__device__ __forceinline__ void write_result(const AttendArgs &a, int r, int h, int e0, ca_f32x4 y, float m, float l, float scale) {   // y: of sums as many times smaller
  y *= l == 0.f ? 0.f : scale / l;
  T *out = (T *)a.out + r * a.out_stride + (long long)h * HD + e0;
  if constexpr (sizeof(T) == 2) *(uint2 *)out = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
  else *(ca_f32x4 *)out = y;
  if (a.lse && e0 == 0) a.lse[(long long)r * a.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}
// four elements of a row and head: the result, or with more parts than one what it is joined from (m: maximum, l: sum; SMALL: y is 2^32 smaller).
// Every part of a row that is somebody's comes here, an empty one with zeros.
template <typename T, int HD, bool SMALL>
__device__ __forceinline__ void finish(const AttendArgs &a, int split, int r, int h, int e0, ca_f32x4 y, float m, float l) {
  const long long i = (long long)r * a.n_q_heads + h;
  if (a.splits > 1) {
    const long long at = (long long)split * a.batch.m * a.n_q_heads + i;
    *(ca_f32x4 *)(a.part + at * HD + e0) = y;
    if (e0 == 0) a.part_ml[at] = make_float2(m, SMALL ? -l : l);
    return;
  }
  write_result<T, HD>(a, r, h, e0, y, m, l, SMALL ? 0x1p32f : 1.f);
}

// ------------------------------------------------------------------ few pairs

// Tiles of 16 pairs; four waves, each with every fourth piece of TOKENS tokens of the workgroup's.  Matrix instructions of 16 x 16:
//   A of the scores: a lane's token is l mod 16, its k values come straight from the cache, 16 bytes a load;
//   A of the values: bf16 through LDS of the wave's own, read transposed; fp32 straight from the cache.
// The next piece's loads are on their way while a piece is worked on.  32 steps over up to 8191 slots, 32 + 2 heads of 128: 45 us, 4.5 TB/s.
template <typename T, int HD> struct Stream {
  static constexpr int PAIRS = 16, WAVES = 4, TOKENS = sizeof(T) == 2 ? 32 : 16, BLOCKS = TOKENS / 16;
  static constexpr int STEPS = HD * (int)sizeof(T) / 64;                        // 16-byte loads of a lane for 16 tokens' keys
  static constexpr int V_LOADS = HD * TOKENS * (int)sizeof(T) / 1024;           // of a lane for a piece's values, 16 bytes in all
  static constexpr int V_BYTES = sizeof(T) == 2 ? TOKENS * HD * 2 : 0;          // of LDS, a wave's
  static constexpr int O_PITCH = HD + 4;
  static constexpr size_t LDS = sizeof(float) * WAVES * PAIRS * O_PITCH;
  static_assert(LDS >= (size_t)WAVES * V_BYTES, "values and sums share it");
};

// false, with nothing written: sums that are no numbers (AGAIN takes no value that is none into its sums)
template <typename T, int HD, bool AGAIN>
__device__ __forceinline__ bool stream_tile(const AttendArgs &a, BadSlots &s_bad) {
  using S = Stream<T, HD>;
  constexpr bool BF = sizeof(T) == 2;
  extern __shared__ uint4 ca_smem[];
  const int thread = this_thread<AGAIN>(), block = this_block<AGAIN>();
  __shared__ float s_max[S::WAVES][S::PAIRS], s_sum[S::WAVES][S::PAIRS];
  const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), col = lane & 15, quad = lane >> 4;
  const int nkv = a.cache.n_kv_heads, kvh = block % nkv, split = block / nkv % a.splits;
  Sequence seq;
  int tile, count;
  if (!find_tile(a.batch, a.cache.page_tokens, a.group, S::PAIRS, a.by_row, block / nkv / a.splits, seq, tile, count)) return true;
  const int pair0 = tile * S::PAIRS, pairs = min(S::PAIRS, seq.rows * a.group - pair0);
  const int end = last_seen(seq, (pair0 + pairs - 1) / a.group, a.causal) + 1, least = last_seen(seq, pair0 / a.group, a.causal);
  const int all = (end + S::TOKENS - 1) / S::TOKENS, share = (all + a.splits - 1) / a.splits;
  const int first = split * share, stop = min(all, first + share);   // pieces
  const int sure = AGAIN ? -1 : least;   // values up to this slot go in as they are
  constexpr float SMALL = AGAIN ? 0x1p-32f : 1.f;

  // (waiting for a load waits for all before it: a piece's pages are asked for ahead of the last piece's keys and values)
  auto ask_piece = [&](int piece) { return ask(seq, a.cache, piece * S::BLOCKS + (lane & (S::BLOCKS - 1)), piece < stop ? end : 0); };
  constexpr int ROW = HD * (int)sizeof(T);
  const char *keys = (const char *)a.cache.plane<T>(0, 0, kvh), *values = (const char *)a.cache.plane<T>(0, 1, kvh);
  int piece = first + wave;
  Found found = find<ROW>(ask_piece(piece), a.cache, sizeof(T));
  Asked asked = ask_piece(piece + S::WAVES);
  const int mine = pair0 + min(col, pairs - 1), my_row = mine / a.group;   // (pairs past the last: that one, not written)
  const int limit = last_seen(seq, my_row, a.causal);
  ca_u32x4 q[S::STEPS];
  {
    const T *at = (const T *)a.q + (seq.row0 + my_row) * a.q_stride + (long long)(kvh * a.group + mine % a.group) * HD;
#pragma unroll
    for (int i = 0; i < S::STEPS; ++i) q[i] = ca_signed<T>(((const ca_u32x4 *)at)[4 * i + quad], a.flip);
  }
  ca_f32x4 o[HD / 16];
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) o[d] = ca_f32x4{0.f, 0.f, 0.f, 0.f};
  ca_u32x4 kr[S::BLOCKS][S::STEPS], vr[S::V_LOADS];
  char *s_v = (char *)ca_smem + wave * S::V_BYTES;
  constexpr int LPT = HD / 8;   // bf16: lanes a token's values take
  auto load_keys = [&]() {
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i) {
      const char *k = at_lane(keys, found, i);
#pragma unroll
      for (int e = 0; e < S::STEPS; ++e) kr[i][e] = *(const ca_u32x4 *)(k + (unsigned)(col * ROW + 64 * e + 16 * quad));
    }
  };
  auto load_values = [&]() {
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i) {
      const char *v = at_lane(values, found, i);
      if constexpr (BF) {
        constexpr int EACH = S::V_LOADS / S::BLOCKS;
#pragma unroll
        for (int e = 0; e < EACH; ++e) vr[i * EACH + e] = *(const ca_u32x4 *)(v + (unsigned)(1024 * e + 16 * lane));
      } else {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) vr[d][e] = *(const uint32_t *)(v + (unsigned)((4 * quad + e) * ROW + 64 * d + 4 * col));
      }
    }
  };
  // values behind `sure`, and of no page
  auto clean = [&](int piece, unsigned here) {
    const int t0 = piece * S::TOKENS;
    if constexpr (BF) {
#pragma unroll
      for (int e = 0; e < S::V_LOADS; ++e) {
        const int in = (e * 64 + lane) / LPT;
        if (t0 + in >= end || !((here >> (in / 16)) & 1)) vr[e] = ca_u32x4{0, 0, 0, 0};
        else if (t0 + in > sure && ca_only_numbers<T>(vr[e])) note_bad(s_bad, t0 + in);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int t = t0 + 4 * quad + e;
        bool bad = false;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
          const bool none = (vr[d][e] & 0x7f800000u) == 0x7f800000u && t > sure;
          bad |= none;
          if (t >= end || !here || none) vr[d][e] = 0u;
        }
        if (bad && t < end && here) note_bad(s_bad, t);
      }
    }
  };

  float *s_o = (float *)ca_smem;
  auto most = [&](int c) {
    float m = s_max[0][c];
#pragma unroll
    for (int w = 1; w < S::WAVES; ++w) m = fmaxf(m, s_max[w][c]);
    return m;
  };
  if (piece < stop) {
    load_keys();
    load_values();
  }
  __syncthreads();   // (s_bad)
  for (; piece < stop; piece += S::WAVES) {
    const unsigned here = (unsigned)__ballot(found.there) & ((1u << S::BLOCKS) - 1);   // which 16s of the piece have a page
    const int t0 = piece * S::TOKENS;
    ca_f32x4 sc[S::BLOCKS];
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i) {
      sc[i] = ca_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < S::STEPS; ++e) {
        if constexpr (BF) {
          sc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ca_operand(kr[i][e]), ca_operand(q[e]), sc[i], 0, 0, 0);
        } else {
          const ca_f32x4 k = __builtin_bit_cast(ca_f32x4, kr[i][e]), x = __builtin_bit_cast(ca_f32x4, q[e]);
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[j], x[j], sc[i], 0, 0, 0);
        }
      }
    }
    if (piece + S::WAVES < stop) {
      found = find<ROW>(asked, a.cache, sizeof(T));
      asked = ask_piece(piece + 2 * S::WAVES);
      load_keys();
    }
    const bool masked = t0 + S::TOKENS - 1 > sure || here != (1u << S::BLOCKS) - 1;
    if (masked) {
      clean(piece, here);
#pragma unroll
      for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t0 + 16 * i + 4 * quad + e > limit || !((here >> i) & 1)) sc[i][e] = -INFINITY;
    }
    ca_f32x4 va[BF ? 1 : S::V_LOADS];
    if constexpr (BF) {
#pragma unroll
      for (int e = 0; e < S::V_LOADS; ++e) {
        const int t = (e * 64 + lane) / LPT, c = lane % LPT;
        *(ca_u32x4 *)(s_v + t * HD * 2 + ((c ^ ca_turn<T, HD>(t)) << 4)) = vr[e];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
#pragma unroll
      for (int d = 0; d < S::V_LOADS; ++d) va[d] = __builtin_bit_cast(ca_f32x4, vr[d]);
    }
    if (piece + S::WAVES < stop) load_values();

    float big = -INFINITY;
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) big = fmaxf(big, sc[i][e]);
    big = fmaxf(big, __shfl_xor(big, 16, 64));
    big = ca_max_halves(big) * a.factor;
    // a pair's maximum follows once it is 2^8 behind: sums in fp32 have room for that
    const bool behind = big > top + 8.f;
    if (__any(behind)) {
      const float up = behind ? big : top, f = ca_exp2(top - (up == -INFINITY ? 0.f : up));
      top = up;
      sum *= f;
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[d] *= f;
    }
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sc[i][e] = SMALL * ca_exp2(fmaf(sc[i][e], a.factor, -base));
        sum += sc[i][e];
      }
    if constexpr (BF) {
      uint32_t high[4], low[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) pack_bf16_parts(sc[i / 2][i % 2 * 2], sc[i / 2][i % 2 * 2 + 1], high[i], low[i]);
      const ca_bf16x8 p = ca_operand(ca_u32x4{high[0], high[1], high[2], high[3]}), rest = ca_operand(ca_u32x4{low[0], low[1], low[2], low[3]});
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) {
        union { ca_s16x4 h[2]; ca_bf16x8 v; } x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int t = 16 * i + 4 * quad + (col >> 2), c = 2 * d + ((col & 3) >> 1);
          x.h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) ca_s16x4 *)(s_v + t * HD * 2 + ((c ^ ca_turn<T, HD>(t)) << 4) + 8 * (col & 1)));
        }
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, p, o[d], 0, 0, 0);
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, rest, o[d], 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(va[d][j], sc[0][j], o[d], 0, 0, 0);
    }
  }

  // the waves' sums brought to one maximum and added in order
  sum += __shfl_xor(sum, 16, 64);
  sum = ca_sum_halves(sum) * (1.f / SMALL);
  if (quad == 0) { s_max[wave][col] = top; s_sum[wave][col] = sum; }
  __syncthreads();   // (and every wave is done with its values)
  {
    const float m = most(col), f = ca_exp2(top - (m == -INFINITY ? 0.f : m));
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) *(ca_f32x4 *)(s_o + (wave * S::PAIRS + col) * S::O_PITCH + 16 * d + 4 * quad) = o[d] * f;
  }
  __syncthreads();
  // a thread has four elements of ITEMS pairs
  constexpr int ITEMS = S::PAIRS * (HD / 4) / (64 * S::WAVES);
  float m[ITEMS], l[ITEMS];
  ca_f32x4 y[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = k * 64 * S::WAVES + thread, c = i / (HD / 4);
    m[k] = most(c);
    l[k] = 0.f;
    y[k] = ca_f32x4{0.f, 0.f, 0.f, 0.f};
    bool numbers = true;
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) {
      l[k] += s_sum[w][c] * ca_exp2(s_max[w][c] - (m[k] == -INFINITY ? 0.f : m[k]));
      y[k] += *(const ca_f32x4 *)(s_o + (w * S::PAIRS + c) * S::O_PITCH + i % (HD / 4) * 4);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) numbers &= fabsf(y[k][e]) < INFINITY;
    if (!AGAIN && !numbers) s_bad.again = 1;
  }
  if constexpr (!AGAIN) {
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(s_bad.again)) return false;
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = k * 64 * S::WAVES + thread, c = i / (HD / 4), e0 = i % (HD / 4) * 4, p = pair0 + c;
    if (c >= pairs) break;
    const int row = p / a.group, r = seq.row0 + row, h = kvh * a.group + p % a.group;
    if (s_bad.last >= 0) {
      const int last = min(last_seen(seq, row, a.causal), s_bad.last);
      for (int t = s_bad.first; t <= last; ++t) {
        const int page = page_of(seq, t, a.cache.page_tokens, a.cache.n_pages);
        if (page < 0) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = Elem<T>::widen(a.cache.plane<T>(page, 1, kvh)[t % a.cache.page_tokens * HD + e0 + e]);
          if (!(fabsf(v) < INFINITY)) y[k][e] += v;
        }
      }
    }
    finish<T, HD, AGAIN>(a, split, r, h, e0, y[k], m[k], l[k]);
  }
  return true;
}

template <typename T, int HD>
__global__ void __launch_bounds__(256, 2) cached_stream_k(AttendArgs a) {
  __shared__ BadSlots s_bad;
  if (threadIdx.x == 0) s_bad = BadSlots{1 << 30, -1, 0};
  if (stream_tile<T, HD, false>(a, s_bad)) return;   // (the same for all of a workgroup)
  __syncthreads();
  stream_tile<T, HD, true>(a, s_bad);
}

// ------------------------------------------------------------------ many pairs

// WAVES waves of 32 pairs each, bf16; tiles of 64 tokens' keys and values in LDS, two of them, so that the next one's loads run while one is
// worked on.  Matrix instructions of 32 x 32 (A: a lane's token or head element is l mod 32, its k those of l / 32); a lane
// holds 32 of a tile's 64 scores of its pair, the other half of the wave the others.  8191 rows of 28 heads of 128: 694 us, 1040 TFLOP/s with the second part's
// products (one part took 537), where a library's product reaches 1140.  (fp32's matrix instructions
// take so long that the stream keeps up: such a kernel took 339 us against 361 for 2000 rows of 28 heads, 106 against 101 for 16 heads of 64.)
template <int HD, int WAVES> struct Tile {
  static constexpr int TOKENS = 64, PAIRS = 32 * WAVES;
  static constexpr int ROW = HD * (int)sizeof(bf16_t), LPT = ROW / 16;                   // bytes of a token, lanes that they take
  static constexpr int PER = 64 * WAVES / LPT, LOADS = TOKENS / PER;                // tokens of a pass of loads, passes
  static constexpr int BYTES = TOKENS * ROW;
  static constexpr int AHEAD = HD == 128 ? 0 : 1;                                    // steps of 16 tokens' values read ahead
  static constexpr int O_PITCH = 36;                                                // floats of a pair, of 32 elements
  static constexpr size_t TILES = 4 * (size_t)BYTES, SUMS = sizeof(float) * PAIRS * (O_PITCH + 2);   // keys and values, two buffers; later results
  static constexpr size_t LDS = TILES > SUMS ? TILES : SUMS;
};

// As stream_tile, but that it says so in s_bad and goes on to the end without writing (to leave in the middle keeps the sums over the branch, in 68 registers).
template <int HD, int WAVES, bool AGAIN>
__device__ __forceinline__ void work_tile(const AttendArgs &a, BadSlots &s_bad) {
  using T = bf16_t;
  using S = Tile<HD, WAVES>;
  constexpr int STEPS = HD * (int)sizeof(T) / 32;   // 16-byte pieces of a query that a lane holds
  extern __shared__ uint4 ca_smem[];
  const int thread = this_thread<AGAIN>(), block = this_block<AGAIN>();
  const int lane = thread & 63, wave = __builtin_amdgcn_readfirstlane(thread >> 6), col = lane & 31, half = lane >> 5;
  const int nkv = a.cache.n_kv_heads, kvh = block % nkv, split = block / nkv % a.splits;
  Sequence seq;
  int tile, count;
  if (!find_tile(a.batch, a.cache.page_tokens, a.group, S::PAIRS, a.by_row, block / nkv / a.splits, seq, tile, count)) return;
  tile = count - 1 - tile;   // the longest first
  const int pair0 = tile * S::PAIRS, pairs = min(S::PAIRS, seq.rows * a.group - pair0);
  const int end = last_seen(seq, (pair0 + pairs - 1) / a.group, a.causal) + 1, least = last_seen(seq, pair0 / a.group, a.causal);
  const int all = (end + S::TOKENS - 1) / S::TOKENS, share = (all + a.splits - 1) / a.splits;
  const int first = split * share, stop = min(all, first + share);   // tiles of tokens
  const int sure = AGAIN ? -1 : least;   // values up to this slot go in as they are
  constexpr float SMALL = AGAIN ? 0x1p-32f : 1.f;

  const int p = pair0 + min(wave * 32 + col, pairs - 1), row = p / a.group;
  const bool works = wave * 32 < pairs;
  const int limit = last_seen(seq, row, a.causal);
  const int wave_least = last_seen(seq, (pair0 + min(wave * 32, pairs - 1)) / a.group, a.causal);
  const int wave_most = last_seen(seq, (pair0 + min(wave * 32 + 31, pairs - 1)) / a.group, a.causal);
  ca_u32x4 q[STEPS];
  {
    const T *at = (const T *)a.q + (seq.row0 + row) * a.q_stride + (long long)(kvh * a.group + p % a.group) * HD;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = ca_signed<T>(((const ca_u32x4 *)at)[2 * i + half], a.flip);
  }

  char *lds = (char *)ca_smem;
  const int st = thread / S::LPT, sc16 = thread % S::LPT;   // this thread's token in a pass, and 16 bytes of it
  ca_u32x4 kr[S::LOADS], vr[S::LOADS];
  // a tile's four 16s are found by lanes 0..3; a wave's tokens of a pass lie in one of them
  auto ask_tile = [&](int t) { return ask(seq, a.cache, 4 * t + (lane & 3), t < stop ? end : 0); };
  const char *planes[2] = {(const char *)a.cache.plane<T>(0, 0, kvh), (const char *)a.cache.plane<T>(0, 1, kvh)};
  const unsigned in_sixteen = (st & 15) * S::ROW + 16 * sc16;
  const int sixteen = __builtin_amdgcn_readfirstlane(st >> 4);
  auto load = [&](const Found &f, int which, ca_u32x4 (&to)[S::LOADS]) {
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      static_assert(S::PER % 16 == 0, "whole 16s a pass");
      to[i] = *(const ca_u32x4 *)(at_lane(planes[which], f, i * (S::PER / 16) + sixteen) + in_sixteen);
    }
  };
  auto clean = [&](int t, unsigned here) {   // values behind `sure`, and of no page
    if (t * S::TOKENS + S::TOKENS - 1 <= sure && here == 15u) return;
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      const int in = i * S::PER + st, token = t * S::TOKENS + in;
      if (token >= end || !((here >> (in >> 4)) & 1)) vr[i] = ca_u32x4{0, 0, 0, 0};
      else if (token > sure && ca_only_numbers<T>(vr[i])) note_bad(s_bad, token);
    }
  };
  auto store = [&](char *to, const ca_u32x4 (&from)[S::LOADS]) {
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      const int token = i * S::PER + st;
      *(ca_u32x4 *)(to + token * S::ROW + ((sc16 ^ ca_turn<T, HD>(token)) << 4)) = from[i];
    }
  };
  auto keys_at = [&](int t) { return lds + ((t - first) & 1) * S::BYTES; };
  auto values_at = [&](int t) { return lds + (2 + ((t - first) & 1)) * S::BYTES; };

  ca_f32x16 o[HD / 32], sc[2];   // unfinished sums [head element][pair], scores [token][pair]
  uint32_t pr[2][16];            // probabilities: parts, two of bf16 a register
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float top = -INFINITY, sum = 0.f;   // the sum: of this lane's tokens

  auto scores = [&](int t) {
    const char *lk = keys_at(t) + col * S::ROW;
    auto key = [&](int b, int i) { return *(const ca_u32x4 *)(lk + 32 * b * S::ROW + (((2 * i + half) ^ ca_turn<T, HD>(col)) << 4)); };
    // operands are read two steps ahead of their use (the barriers hold the order: without them each read is waited for at once)
    ca_u32x4 k[3][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < 2; ++b) k[i][b] = key(b, i);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[b][r] = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      if (i + 2 < STEPS)
#pragma unroll
        for (int b = 0; b < 2; ++b) k[(i + 2) % 3][b] = key(b, i + 2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < 2; ++b) sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ca_operand(k[i % 3][b]), ca_operand(q[i]), sc[b], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto softmax = [&](int t, unsigned here) {
    const int t0 = t * S::TOKENS;
    if (t0 + S::TOKENS - 1 > wave_least || here != 15u) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int token = 32 * b + 8 * (r >> 2) + 4 * half + (r & 3);
          if (t0 + token > limit || !((here >> (2 * b + (r >> 3))) & 1)) sc[b][r] = -INFINITY;
        }
    }
    float big = sc[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) big = fmaxf(big, sc[b][r]);
    big = ca_max_halves(big) * a.factor;
    // a pair's maximum follows once it is 2^8 behind: sums in fp32 have room for that
    const bool behind = big > top + 8.f;
    if (__any(behind)) {
      const float up = behind ? big : top, f = ca_exp2(top - (up == -INFINITY ? 0.f : up));
      top = up;
      sum *= f;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
    }
    const float base = top == -INFINITY ? 0.f : top;
    float s2[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        sc[b][r] = SMALL * ca_exp2(fmaf(sc[b][r], a.factor, -base));
        s2[b] += sc[b][r];
        if (r & 1) pack_bf16_parts(sc[b][r - 1], sc[b][r], pr[0][8 * b + (r >> 1)], pr[1][8 * b + (r >> 1)]);
      }
    sum += s2[0] + s2[1];
  };
  auto values = [&](int t) {
    const char *lv = values_at(t);
    auto value = [&](int step, int d) {   // 16 tokens a step
      union { ca_s16x4 h[2]; ca_bf16x8 v; } x;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int token = 16 * step + 8 * i + 4 * half + ((lane >> 2) & 3), c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        x.h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) ca_s16x4 *)(lv + token * S::ROW + ((c ^ ca_turn<T, HD>(token)) << 4) + 8 * (lane & 1)));
      }
      return x.v;
    };
    // Operands are used for both parts of the probabilities.  They are read 16 tokens ahead; of heads of 128, for which registers do not reach, two blocks of
    // the head as soon as the last tokens' are done with (tiles of eight waves, which have them for either: 711 us so, 716).  The barriers hold the order.
    constexpr int AHEAD = S::AHEAD;
    ca_bf16x8 v[1 + AHEAD][HD / 32];
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) v[0][d] = value(0, d);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (AHEAD && j < 3)
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) v[(j + 1) & AHEAD][d] = value(j + 1, d);
      const ca_bf16x8 p[2] = {ca_operand(ca_u32x4{pr[0][4 * j], pr[0][4 * j + 1], pr[0][4 * j + 2], pr[0][4 * j + 3]}),
                              ca_operand(ca_u32x4{pr[1][4 * j], pr[1][4 * j + 1], pr[1][4 * j + 2], pr[1][4 * j + 3]})};
#pragma unroll
      for (int d0 = 0; d0 < HD / 32; d0 += 2) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int d = d0; d < d0 + 2; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[j & AHEAD][d], p[i], o[d], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (!AHEAD && j < 3)
#pragma unroll
          for (int d = d0; d < d0 + 2; ++d) v[0][d] = value(j + 1, d);
      }
    }
  };

  // A tile's values are followed by the next one's scores, so keys come one tile ahead of values: during tile t the buffers hold keys of t + 1
  // (and take those of t + 2) and values of t (and take those of t + 1).
  Asked asked[3] = {ask_tile(first), ask_tile(first + 1), ask_tile(first + 2)};
  Found found = find<S::ROW>(asked[0], a.cache, sizeof(T)), found_keys = find<S::ROW>(asked[1], a.cache, sizeof(T));
  unsigned here = (unsigned)__ballot(found.there) & 15u;
  __syncthreads();   // (s_bad)
  if (first < stop) {
    ca_u32x4 second[S::LOADS];
    load(found, 0, kr);
    load(found, 1, vr);
    load(found_keys, 0, second);
    store(keys_at(first), kr);
    clean(first, here);
    store(values_at(first), vr);
    store(keys_at(first + 1), second);
    __syncthreads();
    scores(first);
  }
  __syncthreads();   // (the first tile's keys are done with)
  for (int t = first; t < stop; ++t) {
    found = found_keys;
    found_keys = find<S::ROW>(asked[2], a.cache, sizeof(T));
    const unsigned here_next = (unsigned)__ballot(found.there) & 15u;
    if (t + 1 < stop) {
      asked[2] = ask_tile(t + 3);
      load(found_keys, 0, kr);   // of t + 2
      load(found, 1, vr);        // of t + 1
    }
    if (works && t * S::TOKENS <= wave_most) {
      softmax(t, here);
      __builtin_amdgcn_s_setprio(1);   // (the other wave's exponentials give way to these matrix instructions)
      values(t);
      scores(t + 1);
      __builtin_amdgcn_s_setprio(0);
    }
    here = here_next;
    if (t + 1 < stop) {
      clean(t + 1, here);
      store(keys_at(t + 2), kr);
      store(values_at(t + 1), vr);
    }
    __syncthreads();
  }
  if constexpr (!AGAIN) {
    bool numbers = true;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) numbers &= fabsf(o[d][r]) < INFINITY;
    if (!numbers) s_bad.again = 1;
    __syncthreads();
  }
  const bool writes = AGAIN || !s_bad.again;
  sum = ca_sum_halves(sum) * (1.f / SMALL);
  if (s_bad.last >= 0) {   // (the last store lies before the last barrier)
    for (int t = s_bad.first; t <= s_bad.last; ++t) {
      const int page = page_of(seq, t, a.cache.page_tokens, a.cache.n_pages);
      if (page < 0 || t > limit) continue;
      const T *v = a.cache.plane<T>(page, 1, kvh) + t % a.cache.page_tokens * HD + 4 * half;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = Elem<T>::widen(v[32 * d + 8 * (r >> 2) + (r & 3)]);
          if (!(fabsf(x) < INFINITY)) o[d][r] += x;
        }
    }
  }
  // Through LDS, 32 elements at a time, so that eight lanes write 32 elements of a pair next to each other (straight from the registers, where a
  // store's lanes are 16 bytes of 64 rows: 19 us more for 8191 rows).
  float *s_o = (float *)ca_smem + wave * 32 * S::O_PITCH;
  float2 *s_ml = (float2 *)((float *)ca_smem + S::PAIRS * S::O_PITCH) + wave * 32;
  if (half == 0) s_ml[col] = make_float2(top, sum);
  int out_row[4], out_head[4];   // -1: no pair
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = wave * 32 + 8 * i + (lane >> 3), pc = pair0 + c;
    out_row[i] = writes && c < pairs ? seq.row0 + pc / a.group : -1;
    out_head[i] = kvh * a.group + pc % a.group;
  }
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(ca_f32x4 *)(s_o + col * S::O_PITCH + 8 * i + 4 * half) = ca_f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 8 * i + (lane >> 3);
      const float2 ml = s_ml[c];
      if (out_row[i] >= 0)
        finish<T, HD, AGAIN>(a, split, out_row[i], out_head[i], 32 * d + 4 * (lane & 7), *(const ca_f32x4 *)(s_o + c * S::O_PITCH + 4 * (lane & 7)), ml.x, ml.y);
    }
  }
}

template <int HD, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2) cached_tile_k(AttendArgs a) {
  __shared__ BadSlots s_bad;
  if (threadIdx.x == 0) s_bad = BadSlots{1 << 30, -1, 0};
  work_tile<HD, WAVES, false>(a, s_bad);
  __syncthreads();
  if (!__builtin_amdgcn_readfirstlane(s_bad.again)) return;
  __syncthreads();
  work_tile<HD, WAVES, true>(a, s_bad);
}

// ------------------------------------------------------------------ the parts together

constexpr int JOIN_AHEAD = 4;   // parts on their way (both launches, a group of lanes to a vector, probabilities of one part: one step of 28 heads in 13 parts, one 12.7 us, four 10.9, eight 10.5, sixteen 10.3;
                                // 511 rows in 4 parts 39.8, 40.1, 40.5, 44.3)

// GROUPS of lanes to a vector, each with every GROUPS-th part, whose sums are added in their order.
template <typename T, int HD, int GROUPS>
__global__ void __launch_bounds__(256) cached_join_k(AttendArgs a) {
  constexpr int LANES = HD / 4;
  static_assert(GROUPS == 1 || GROUPS * LANES == 256, "several groups are a workgroup");
  const long long i = (long long)blockIdx.x * (256 / LANES / GROUPS) + threadIdx.x / (LANES * GROUPS);
  if (i >= (long long)a.batch.m * a.n_q_heads) return;   // (several groups: of all of a workgroup)
  const int r = (int)(i / a.n_q_heads), e0 = threadIdx.x % LANES * 4;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES % GROUPS;
  const long long step = (long long)a.batch.m * a.n_q_heads;
  // the first parts are on their way while all maxima and sums are looked at
  const float *part = a.part + i * HD + e0;
  ca_f32x4 v[JOIN_AHEAD];
  float2 ml[JOIN_AHEAD];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k) {
      const int s = min(s0 + k * GROUPS, a.splits - 1);
      v[k] = *(const ca_f32x4 *)(part + s * step * HD);
      ml[k] = a.part_ml[s * step + i];
    }
  };
  fetch(group);
  constexpr int OURS = 1, SMALL = 2;   // somebody's row; some of its parts are 2^32 smaller
  int is = 0;
  for (int s = lane; s < a.batch.n; s += LANES) is |= a.batch.starts[s] <= r && r < a.batch.starts[s + 1] ? OURS : 0;
  float l = 0.f, m = -INFINITY;
  for (int s = lane; s < a.splits; s += LANES) {
    float2 x = a.part_ml[s * step + i];
    is |= x.y < 0.f ? SMALL : 0;
    x.y = fabsf(x.y);
    const float top = fmaxf(m, x.x), base = top == -INFINITY ? 0.f : top;
    l = (l == 0.f ? 0.f : l * ca_exp2(m - base)) + (x.y == 0.f ? 0.f : x.y * ca_exp2(x.x - base));
    m = top;
  }
  const float mine = m;
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor(m, o, LANES));
    is |= __shfl_xor(is, o, LANES);
  }
  if (!(is & OURS)) return;
  const float base = m == -INFINITY ? 0.f : m;
  l = l == 0.f ? 0.f : l * ca_exp2(mine - base);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) l += __shfl_xor(l, o, LANES);
  static_assert(MOST_SPLITS <= 256, "sums that fp32 holds, 2^8 smaller, have room");
  const float scale = is & SMALL ? 0x1p-32f : 0x1p-8f;
  ca_f32x4 y = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = group; s0 < a.splits; s0 += JOIN_AHEAD * GROUPS) {
    if (s0 > group) fetch(s0);
#pragma unroll
    for (int k = 0; k < JOIN_AHEAD; ++k) {
      const bool none = s0 + k * GROUPS >= a.splits;
      const float g = none ? 0.f : ca_exp2(ml[k].x - base) * (ml[k].y < 0.f ? 1.f : scale);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += none ? 0.f : g == 0.f && !(fabsf(v[k][e]) < INFINITY) ? v[k][e] : v[k][e] * g;   // (an infinity stays one)
    }
  }
  if constexpr (GROUPS > 1) {
    __shared__ ca_f32x4 s_y[GROUPS][LANES];
    s_y[group][lane] = y;
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int j = 1; j < GROUPS; ++j) y += s_y[j][lane];
  }
  write_result<T, HD>(a, r, (int)(i % a.n_q_heads), e0, y, m, l, 1.f / scale);
}

}  // namespace spark
