// Attention of new rows over a paged cache (spark_cache_attend).
//
//   out = sum_t exp(s_t - M) v_t / L,  s_t = scale q . k_t,  M = max s_t,  L = sum_t exp(s_t - M),  lse = M + log L
//
// over the slots t that a row sees, in one pass with a running maximum and sum.  The (row, query head) pairs of a sequence and kv
// head share its keys and values; they are counted through, pair p being row p / group and head p mod group, and cut into tiles.
//
//   cached_stream_k  up to 16 or 32 pairs: bound by the cache's way through memory.  Each wave has its own tokens.
//   cached_tile_k    128 or 256 pairs: bound by the matrix units.  A tile of keys and values in LDS serves all waves.
//   cached_join_k    where too few tiles would leave compute units idle, their tokens are cut into `splits` parts, whose
//                    unfinished sums come through the workspace; this adds them up in order.
//
// In all: scores transposed, S^T [token][pair] = K Q^T, so a lane holds scores of one pair and finds their maximum and sum
// by itself; and since a sum over tokens may go in any order, those registers are, rounded, the operand of O^T = V^T P^T as
// they are.  Exponentials are of base 2, the scores' factor is scale log2 e.
//
// Slots that a row does not see: their scores are replaced, not added to.  Their values meet zeros, and zero times infinity is
// NaN, so behind the first row's last slot values that are no numbers go in as zeros, and what the rows that do see
// them get from them is added at the end (a probability is positive: infinity stays, NaN too).
#pragma once
#include "cached_format.h"

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
  float factor;   // |scale| log2 e
  uint32_t flip;  // the sign of scale, put on the queries
};

typedef __attribute__((ext_vector_type(8))) __bf16 ca_bf16x8;
typedef __attribute__((ext_vector_type(4))) short ca_s16x4;
typedef __attribute__((ext_vector_type(4))) float ca_f32x4;
typedef __attribute__((ext_vector_type(16))) float ca_f32x16;
__device__ __forceinline__ ca_bf16x8 ca_operand(const uint4 &v) { return __builtin_bit_cast(ca_bf16x8, v); }
template <typename T> __device__ __forceinline__ uint4 ca_signed(uint4 v, uint32_t flip) {
  const uint32_t x = sizeof(T) == 4 ? flip : flip | (flip >> 16);
  return make_uint4(v.x ^ x, v.y ^ x, v.z ^ x, v.w ^ x);
}
// elements that are no numbers to zero; true if there was one
template <typename T> __device__ __forceinline__ bool ca_only_numbers(uint4 &v) {
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
  v = make_uint4(w[0], w[1], w[2], w[3]);
  return bad;
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

// The tile of pairs that a workgroup takes, from a count over all sequences: its sequence, tile in it and tiles of it, or false.
// Called by whole waves.
__device__ __forceinline__ bool find_tile(const BatchView &b, int page_tokens, int group, int per_tile, int tile, Sequence &q, int &t, int &count) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < b.n; s0 += 64) {
    int c = 0, row0 = 0, rows = 0, length = 0;
    if (s0 + lane < b.n) {
      length = b.lengths[s0 + lane];
      row0 = cut(b.starts[s0 + lane], 0, b.m);
      rows = cut(b.starts[s0 + lane + 1], row0, b.m) - row0;
      c = (rows * group + per_tile - 1) / per_tile;
    }
    int incl = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(incl, o, 64);
      if (lane >= o) incl += up;
    }
    const unsigned long long past = __ballot(incl > tile);
    if (past) {
      const int l = __ffsll(past) - 1;
      q.row0 = __builtin_amdgcn_readlane(row0, l);
      q.rows = __builtin_amdgcn_readlane(rows, l);
      q.length = cut(__builtin_amdgcn_readlane(length, l), 0, b.max_pages * page_tokens);
      q.pages = b.table + (long long)(s0 + l) * b.max_pages;
      count = __builtin_amdgcn_readlane(c, l);
      t = tile - (__builtin_amdgcn_readlane(incl, l) - count);
      return true;
    }
    tile -= __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// the last slot that a row sees, -1: none
__device__ __forceinline__ int last_seen(const Sequence &q, int row, int causal) {
  const int slot = q.slot(row);
  return slot < 0 ? -1 : causal ? slot : q.length - 1;
}

// the page of each 16 slots from slot 16 (first + i) on in lane i; -1 past `end` or where there is none
__device__ __forceinline__ int pages_of(const Sequence &q, const CacheView &c, int sixteen, int end) {
  return sixteen * 16 < end ? page_of(q, sixteen * 16, c.page_tokens, c.n_pages) : -1;
}

// ------------------------------------------------------------------ few pairs

// NB blocks of 16 pairs; four waves, each with every fourth piece of TOKENS tokens of the workgroup's.  Matrix instructions of 16 x 16:
//   A of the scores: a lane's token is l mod 16, its k values come straight from the cache, 16 bytes a load;
//   A of the values: bf16 through LDS of the wave's own, read transposed; fp32 straight from the cache.
// The next piece's loads are on their way while a piece is worked on.
template <typename T, int HD, int NB> struct Stream {
  static constexpr int WAVES = 4, TOKENS = sizeof(T) == 2 ? 32 : 16, BLOCKS = TOKENS / 16;
  static constexpr int STEPS = HD * (int)sizeof(T) / 64;           // 16-byte loads of a lane for 16 tokens' keys
  static constexpr int V_LOADS = sizeof(T) == 2 ? TOKENS * HD / 512 : HD / 4;   // of a lane: 16 bytes, fp32: four
  static constexpr int V_BYTES = sizeof(T) == 2 ? TOKENS * HD * 2 : 0;          // of LDS, a wave's
  static constexpr int O_PITCH = HD + 4;
  static constexpr size_t LDS = WAVES * V_BYTES > (int)sizeof(float) * WAVES * 16 * O_PITCH ? WAVES * V_BYTES : sizeof(float) * WAVES * 16 * O_PITCH;
};

template <typename T, int HD, int NB>
__global__ void __launch_bounds__(256) cached_stream_k(AttendArgs a) {
  using S = Stream<T, HD, NB>;
  constexpr bool BF = sizeof(T) == 2;
  extern __shared__ uint4 ca_smem[];
  __shared__ float s_max[S::WAVES][NB * 16], s_sum[S::WAVES][NB * 16];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
  const int nkv = a.cache.n_kv_heads, kvh = blockIdx.x % nkv, split = blockIdx.x / nkv % a.splits;
  Sequence seq;
  int tile, count;
  if (!find_tile(a.batch, a.cache.page_tokens, a.group, NB * 16, blockIdx.x / nkv / a.splits, seq, tile, count)) return;
  const int pair0 = tile * NB * 16, pairs = min(NB * 16, seq.rows * a.group - pair0);
  const int end = last_seen(seq, (pair0 + pairs - 1) / a.group, a.causal) + 1, least = last_seen(seq, pair0 / a.group, a.causal);
  const int all = (end + S::TOKENS - 1) / S::TOKENS, share = (all + a.splits - 1) / a.splits;
  const int first = split * share, stop = min(all, first + share);   // pieces
  if (threadIdx.x == 0) s_bad = 0;

  uint4 q[NB][S::STEPS];
  int limit[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int p = pair0 + min(b * 16 + col, pairs - 1), row = p / a.group;   // (pairs past the last: that one, not written)
    limit[b] = last_seen(seq, row, a.causal);
    const T *at = (const T *)a.q + (seq.row0 + row) * a.q_stride + (long long)(kvh * a.group + p % a.group) * HD;
#pragma unroll
    for (int i = 0; i < S::STEPS; ++i) q[b][i] = ca_signed<T>(((const uint4 *)at)[4 * i + quad], a.flip);
  }
  ca_f32x4 o[NB][HD / 16];
  float top[NB], sum[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    top[b] = -INFINITY;
    sum[b] = 0.f;
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) o[b][d] = ca_f32x4{0.f, 0.f, 0.f, 0.f};
  }

  uint4 kr[S::BLOCKS][S::STEPS];
  uint4 vr[BF ? S::V_LOADS : S::V_LOADS / 4];
  char *s_v = (char *)ca_smem + wave * S::V_BYTES;
  constexpr int LPT = HD / 8;   // bf16: lanes a token's values take
  auto load_keys = [&](int piece, int pages) {
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i) {
      const int page = __builtin_amdgcn_readlane(pages, i), in = (piece * S::TOKENS + 16 * i) % a.cache.page_tokens;
      if (page >= 0) {
        const uint4 *k = (const uint4 *)(a.cache.plane<T>(page, 0, kvh) + (in + col) * HD) + quad;
#pragma unroll
        for (int e = 0; e < S::STEPS; ++e) kr[i][e] = k[4 * e];
      } else {
#pragma unroll
        for (int e = 0; e < S::STEPS; ++e) kr[i][e] = make_uint4(0, 0, 0, 0);
      }
    }
  };
  auto load_values = [&](int piece, int pages) {
#pragma unroll
    for (int i = 0; i < S::BLOCKS; ++i) {
      const int page = __builtin_amdgcn_readlane(pages, i), in = (piece * S::TOKENS + 16 * i) % a.cache.page_tokens;
      const T *v = a.cache.plane<T>(max(page, 0), 1, kvh) + in * HD;
      if constexpr (BF) {
        constexpr int EACH = S::V_LOADS / S::BLOCKS;
#pragma unroll
        for (int e = 0; e < EACH; ++e) vr[i * EACH + e] = page >= 0 ? ((const uint4 *)v)[e * 64 + lane] : make_uint4(0, 0, 0, 0);
      } else {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = page >= 0 ? ((const uint32_t *)v)[(4 * quad + e) * HD + 16 * d + col] : 0u;
          vr[d] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
  };
  // values behind `least`
  auto clean = [&](int piece) {
    const int t0 = piece * S::TOKENS;
    bool bad = false;
    if constexpr (BF) {
#pragma unroll
      for (int e = 0; e < S::V_LOADS; ++e) {
        const int t = t0 + (e * 64 + lane) / LPT;
        if (t >= end) vr[e] = make_uint4(0, 0, 0, 0);
        else if (t > least) bad |= ca_only_numbers<T>(vr[e]);
      }
    } else {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) {
        uint32_t w[4] = {vr[d].x, vr[d].y, vr[d].z, vr[d].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int t = t0 + 4 * quad + e;
          const bool none = (w[e] & 0x7f800000u) == 0x7f800000u;
          bad |= none && t > least && t < end;
          if (t >= end || (none && t > least)) w[e] = 0u;
        }
        vr[d] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    if (bad) s_bad = 1;
  };

  constexpr int PER16 = S::TOKENS / 16;
  // (waiting for a load waits for all before it: a piece's pages are asked for ahead of the last piece's keys and values)
  auto pages_at = [&](int piece) { return pages_of(seq, a.cache, piece * PER16 + (lane & (S::BLOCKS - 1)), piece < stop ? end : 0); };
  int piece = first + wave;
  int pages = pages_at(piece), next_pages = pages_at(piece + S::WAVES);
  if (piece < stop) {
    load_keys(piece, pages);
    load_values(piece, pages);
  }
  __syncthreads();   // (s_bad)
  for (; piece < stop; piece += S::WAVES) {
    const unsigned now = (unsigned)__ballot(pages >= 0) & ((1u << S::BLOCKS) - 1);   // which 16s of the piece have a page
    const int t0 = piece * S::TOKENS;
    ca_f32x4 sc[NB][S::BLOCKS];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < S::BLOCKS; ++i) {
        sc[b][i] = ca_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < S::STEPS; ++e) {
          if constexpr (BF) {
            sc[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ca_operand(kr[i][e]), ca_operand(q[b][e]), sc[b][i], 0, 0, 0);
          } else {
            const float4 k = __builtin_bit_cast(float4, kr[i][e]), x = __builtin_bit_cast(float4, q[b][e]);
            sc[b][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x, x.x, sc[b][i], 0, 0, 0);
            sc[b][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.y, x.y, sc[b][i], 0, 0, 0);
            sc[b][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.z, x.z, sc[b][i], 0, 0, 0);
            sc[b][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(k.w, x.w, sc[b][i], 0, 0, 0);
          }
        }
      }
    pages = next_pages;
    if (piece + S::WAVES < stop) {
      next_pages = pages_at(piece + 2 * S::WAVES);
      load_keys(piece + S::WAVES, pages);
    }
    if (t0 + S::TOKENS - 1 > least) clean(piece);
    uint4 va[BF ? 1 : HD / 16];
    if constexpr (BF) {
#pragma unroll
      for (int e = 0; e < S::V_LOADS; ++e) {
        const int t = (e * 64 + lane) / LPT, c = lane % LPT;
        *(uint4 *)(s_v + t * HD * 2 + ((c ^ ca_turn<T, HD>(t)) << 4)) = vr[e];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) va[d] = vr[d];
    }
    if (piece + S::WAVES < stop) load_values(piece + S::WAVES, pages);
    const bool masked = t0 + S::TOKENS - 1 > least || now != (1u << S::BLOCKS) - 1;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (masked) {
#pragma unroll
        for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + 16 * i + 4 * quad + e > limit[b] || !((now >> i) & 1)) sc[b][i][e] = -INFINITY;
      }
      float big = -INFINITY;
#pragma unroll
      for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) big = fmaxf(big, sc[b][i][e]);
      big = fmaxf(big, __shfl_xor(big, 16, 64));
      big = ca_max_halves(big) * a.factor;
      // a pair's maximum follows once it is 2^8 behind: sums in fp32 have room for that
      const bool behind = big > top[b] + 8.f;
      if (__any(behind)) {
        const float up = behind ? big : top[b], f = ca_exp2(top[b] - (up == -INFINITY ? 0.f : up));
        top[b] = up;
        sum[b] *= f;
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[b][d][e] *= f;
      }
      const float base = top[b] == -INFINITY ? 0.f : top[b];
#pragma unroll
      for (int i = 0; i < S::BLOCKS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sc[b][i][e] = ca_exp2(fmaf(sc[b][i][e], a.factor, -base));
          sum[b] += sc[b][i][e];
        }
    }
    if constexpr (BF) {
      ca_bf16x8 p[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
        p[b] = ca_operand(make_uint4(pack_bf16(sc[b][0][0], sc[b][0][1]), pack_bf16(sc[b][0][2], sc[b][0][3]), pack_bf16(sc[b][1][0], sc[b][1][1]),
                                     pack_bf16(sc[b][1][2], sc[b][1][3])));
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) {
        union { ca_s16x4 h[2]; ca_bf16x8 v; } x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int t = 16 * i + 4 * quad + (col >> 2), c = 2 * d + ((col & 3) >> 1);
          x.h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) ca_s16x4 *)(s_v + t * HD * 2 + ((c ^ ca_turn<T, HD>(t)) << 4) + 8 * (col & 1)));
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, p[b], o[b][d], 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) {
        const float4 v = __builtin_bit_cast(float4, va[d]);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          o[b][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x, sc[b][0][0], o[b][d], 0, 0, 0);
          o[b][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.y, sc[b][0][1], o[b][d], 0, 0, 0);
          o[b][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.z, sc[b][0][2], o[b][d], 0, 0, 0);
          o[b][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.w, sc[b][0][3], o[b][d], 0, 0, 0);
        }
      }
    }
  }

  // the waves' sums brought to one maximum and added in order
  float *s_o = (float *)ca_smem;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    sum[b] += __shfl_xor(sum[b], 16, 64);
    sum[b] = ca_sum_halves(sum[b]);
    if (quad == 0) { s_max[wave][b * 16 + col] = top[b]; s_sum[wave][b * 16 + col] = sum[b]; }
  }
  __syncthreads();   // (and every wave is done with its values)
  const bool bad = s_bad != 0;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    float most = -INFINITY;
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) most = fmaxf(most, s_max[w][b * 16 + col]);
    const float f = ca_exp2(top[b] - (most == -INFINITY ? 0.f : most));
#pragma unroll
    for (int d = 0; d < HD / 16; ++d) *(ca_f32x4 *)(s_o + (wave * 16 + col) * S::O_PITCH + 16 * d + 4 * quad) = o[b][d] * f;
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * HD / 4; i += 64 * S::WAVES) {
      const int c = i / (HD / 4), e0 = i % (HD / 4) * 4, p = pair0 + b * 16 + c;
      if (b * 16 + c >= pairs) break;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < S::WAVES; ++w) m = fmaxf(m, s_max[w][b * 16 + c]);
      ca_f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < S::WAVES; ++w) {
        l += s_sum[w][b * 16 + c] * ca_exp2(s_max[w][b * 16 + c] - (m == -INFINITY ? 0.f : m));
        y += *(const ca_f32x4 *)(s_o + (w * 16 + c) * S::O_PITCH + e0);
      }
      const int row = p / a.group, r = seq.row0 + row, h = kvh * a.group + p % a.group;
      if (bad) {
        const int last = last_seen(seq, row, a.causal);
        for (int t = max(first * S::TOKENS, least + 1); t <= min(last, stop * S::TOKENS - 1); ++t) {
          const int page = page_of(seq, t, a.cache.page_tokens, a.cache.n_pages);
          if (page < 0) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = Elem<T>::widen(a.cache.plane<T>(page, 1, kvh)[t % a.cache.page_tokens * HD + e0 + e]);
            if (!(fabsf(v) < INFINITY)) y[e] += v;
          }
        }
      }
      if (a.splits > 1) {
        const long long at = ((long long)split * a.batch.m + r) * a.n_q_heads + h;
        *(ca_f32x4 *)(a.part + at * HD + e0) = y;
        if (e0 == 0) a.part_ml[at] = make_float2(m, l);
      } else {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        T *out = (T *)a.out + r * a.out_stride + (long long)h * HD + e0;
        if constexpr (BF) *(uint2 *)out = make_uint2(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv));
        else *(float4 *)out = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
        if (a.lse && e0 == 0) a.lse[(long long)r * a.n_q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ many pairs

// WAVES waves of 32 pairs each; tiles of 64 tokens' keys and values in LDS, two of them, so that the next one's loads run while one is
// worked on.  Matrix instructions of 32 x 32 (A: a lane's token or head element is l mod 32, its k those of l / 32); a lane
// holds 32 of a tile's 64 scores of its pair, the other half of the wave the others.
template <typename T, int HD, int WAVES> struct Tile {
  static constexpr int TOKENS = 64, PAIRS = 32 * WAVES;
  static constexpr int ROW = HD * (int)sizeof(T), LPT = ROW / 16;                   // bytes of a token, lanes that they take
  static constexpr int PER = 64 * WAVES / LPT, LOADS = TOKENS / PER;                // tokens of a pass of loads, passes
  static constexpr int BYTES = TOKENS * ROW;
  static constexpr size_t LDS = 4 * (size_t)BYTES;                                  // keys and values, two buffers
};

template <typename T, int HD, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, WAVES == 4 && HD * sizeof(T) == 512 ? 1 : 2) cached_tile_k(AttendArgs a) {
  using S = Tile<T, HD, WAVES>;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int STEPS = HD * (int)sizeof(T) / 32;   // 16-byte pieces of a query that a lane holds
  extern __shared__ uint4 ca_smem[];
  __shared__ int s_bad;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int nkv = a.cache.n_kv_heads, kvh = blockIdx.x % nkv, split = blockIdx.x / nkv % a.splits;
  Sequence seq;
  int tile, count;
  if (!find_tile(a.batch, a.cache.page_tokens, a.group, S::PAIRS, blockIdx.x / nkv / a.splits, seq, tile, count)) return;
  tile = count - 1 - tile;   // the longest first
  const int pair0 = tile * S::PAIRS, pairs = min(S::PAIRS, seq.rows * a.group - pair0);
  const int end = last_seen(seq, (pair0 + pairs - 1) / a.group, a.causal) + 1, least = last_seen(seq, pair0 / a.group, a.causal);
  const int all = (end + S::TOKENS - 1) / S::TOKENS, share = (all + a.splits - 1) / a.splits;
  const int first = split * share, stop = min(all, first + share);   // tiles of tokens
  if (threadIdx.x == 0) s_bad = 0;

  const int p = pair0 + min(wave * 32 + col, pairs - 1), row = p / a.group;
  const bool live = wave * 32 + col < pairs, works = wave * 32 < pairs;
  const int limit = last_seen(seq, row, a.causal);
  const int wave_least = last_seen(seq, (pair0 + min(wave * 32, pairs - 1)) / a.group, a.causal);
  const int wave_most = last_seen(seq, (pair0 + min(wave * 32 + 31, pairs - 1)) / a.group, a.causal);
  uint4 q[STEPS];
  {
    const T *at = (const T *)a.q + (seq.row0 + row) * a.q_stride + (long long)(kvh * a.group + p % a.group) * HD;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = ca_signed<T>(((const uint4 *)at)[2 * i + half], a.flip);
  }

  char *lds = (char *)ca_smem;
  const int st = threadIdx.x / S::LPT, sc16 = threadIdx.x % S::LPT;   // this thread's token in a pass, and 16 bytes of it
  uint4 kr[S::LOADS], vr[S::LOADS];
  // the pages of a tile's four 16s in lanes 0..3
  auto pages_at = [&](int t) { return pages_of(seq, a.cache, 4 * t + (lane & 3), t < stop ? end : 0); };
  auto load = [&](int t, int pages) {
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      const int token = i * S::PER + st, sixteen = __builtin_amdgcn_readfirstlane(token >> 4);   // (a wave's tokens of a pass share theirs)
      const int page = __builtin_amdgcn_readlane(pages, sixteen), in = (t * S::TOKENS + 16 * sixteen) % a.cache.page_tokens + (token & 15);
      if (page >= 0) {
        kr[i] = ((const uint4 *)(a.cache.plane<T>(page, 0, kvh) + in * HD))[sc16];
        vr[i] = ((const uint4 *)(a.cache.plane<T>(page, 1, kvh) + in * HD))[sc16];
      } else {
        kr[i] = make_uint4(0, 0, 0, 0);
        vr[i] = make_uint4(0, 0, 0, 0);
      }
    }
  };
  auto store = [&](int t, int buf) {
    if (t * S::TOKENS + S::TOKENS - 1 > least) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < S::LOADS; ++i) {
        const int token = t * S::TOKENS + i * S::PER + st;
        if (token >= end) vr[i] = make_uint4(0, 0, 0, 0);
        else if (token > least) bad |= ca_only_numbers<T>(vr[i]);
      }
      if (bad) s_bad = 1;
    }
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
      const int token = i * S::PER + st, at = token * S::ROW + ((sc16 ^ ca_turn<T, HD>(token)) << 4);
      *(uint4 *)(lds + 2 * buf * S::BYTES + at) = kr[i];
      *(uint4 *)(lds + (2 * buf + 1) * S::BYTES + at) = vr[i];
    }
  };

  ca_f32x16 o[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float top = -INFINITY, sum = 0.f;   // the sum: of this lane's tokens

  int pages = pages_at(first), next_pages = pages_at(first + 1);
  __syncthreads();   // (s_bad)
  if (first < stop) {
    load(first, pages);
    store(first, 0);
  }
  __syncthreads();
  for (int t = first; t < stop; ++t) {
    const int buf = (t - first) & 1, t0 = t * S::TOKENS;
    const unsigned here = (unsigned)__ballot(pages >= 0) & 15u;
    pages = next_pages;
    if (t + 1 < stop) {
      load(t + 1, pages);
      next_pages = pages_at(t + 2);
    }
    if (works && t0 <= wave_most) {
      const char *lk = lds + 2 * buf * S::BYTES, *lv = lk + S::BYTES;
      ca_f32x16 sc[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[b][r] = 0.f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const uint4 k = *(const uint4 *)(lk + (32 * b + col) * S::ROW + (((2 * i + half) ^ ca_turn<T, HD>(col)) << 4));
          if constexpr (BF) {
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ca_operand(k), ca_operand(q[i]), sc[b], 0, 0, 0);
          } else {
            const float4 x = __builtin_bit_cast(float4, k), y = __builtin_bit_cast(float4, q[i]);
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, y.x, sc[b], 0, 0, 0);
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, y.y, sc[b], 0, 0, 0);
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, y.z, sc[b], 0, 0, 0);
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, y.w, sc[b], 0, 0, 0);
          }
        }
      }
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
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sc[b][r] = ca_exp2(fmaf(sc[b][r], a.factor, -base));
          sum += sc[b][r];
        }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        if constexpr (BF) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {   // 16 tokens
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack_bf16(sc[b][8 * j + 2 * e], sc[b][8 * j + 2 * e + 1]);
            const ca_bf16x8 pr = ca_operand(make_uint4(w[0], w[1], w[2], w[3]));
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
              union { ca_s16x4 h[2]; ca_bf16x8 v; } x;
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int token = 32 * b + 16 * j + 8 * i + 4 * half + ((lane >> 2) & 3), c = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                x.h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) ca_s16x4 *)(lv + token * S::ROW + ((c ^ ca_turn<T, HD>(token)) << 4) + 8 * (lane & 1)));
              }
              o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v, pr, o[d], 0, 0, 0);
            }
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int token = 32 * b + 8 * (r >> 2) + 4 * half + (r & 3);
#pragma unroll
            for (int d = 0; d < HD / 32; ++d) {
              const int c = 8 * d + (col >> 2);
              const float v = *(const float *)(lv + token * S::ROW + ((c ^ ca_turn<T, HD>(token)) << 4) + 4 * (col & 3));
              o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, sc[b][r], o[d], 0, 0, 0);
            }
          }
        }
      }
    }
    if (t + 1 < stop) store(t + 1, buf ^ 1);
    __syncthreads();
  }

  sum = ca_sum_halves(sum);
  const int r0 = seq.row0 + row, h = kvh * a.group + p % a.group;
  if (s_bad) {   // (the last store lies before the last barrier)
    for (int t = max(first * S::TOKENS, least + 1); t < min(end, stop * S::TOKENS); ++t) {
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
  if (!live) return;
  const long long at = ((long long)split * a.batch.m + r0) * a.n_q_heads + h;
  const float inv = a.splits > 1 ? 1.f : sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e0 = 32 * d + 8 * i + 4 * half;
      const float4 y = make_float4(o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv);
      if (a.splits > 1) *(float4 *)(a.part + at * HD + e0) = y;
      else if constexpr (BF) *(uint2 *)((T *)a.out + r0 * a.out_stride + (long long)h * HD + e0) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
      else *(float4 *)((T *)a.out + r0 * a.out_stride + (long long)h * HD + e0) = y;
    }
  if (half == 0) {
    if (a.splits > 1) a.part_ml[at] = make_float2(top, sum);
    else if (a.lse) a.lse[(long long)r0 * a.n_q_heads + h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994530942f;
  }
}

// ------------------------------------------------------------------ the parts together

constexpr int MOST_SPLITS = 64;

template <typename T, int HD>
__global__ void __launch_bounds__(256) cached_join_k(AttendArgs a) {
  constexpr int LANES = HD / 4;
  const long long i = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (i >= (long long)a.batch.m * a.n_q_heads) return;
  const int r = (int)(i / a.n_q_heads), e0 = threadIdx.x % LANES * 4;
  const int lane = threadIdx.x % LANES;
  bool ours = false;   // somebody's row
  for (int s = lane; s < a.batch.n; s += LANES) ours |= a.batch.starts[s] <= r && r < a.batch.starts[s + 1];
  const long long step = (long long)a.batch.m * a.n_q_heads;
  // the parts' maxima and sums, one or a few a lane
  constexpr int EACH = MOST_SPLITS / LANES;
  float f[EACH], l = 0.f, m = -INFINITY;
  float2 ml[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int s = j * LANES + lane;
    ml[j] = s < a.splits ? a.part_ml[s * step + i] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, ml[j].x);
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor(m, o, LANES));
    ours |= __shfl_xor((int)ours, o, LANES) != 0;
  }
  if (!ours) return;
  const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    f[j] = ml[j].y == 0.f ? -1.f : ca_exp2(ml[j].x - base);   // (-1: its sums were not written)
    l += ml[j].y == 0.f ? 0.f : ml[j].y * f[j];
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) l += __shfl_xor(l, o, LANES);
  ca_f32x4 y = {0.f, 0.f, 0.f, 0.f};
  const float *part = a.part + i * HD + e0;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
#pragma unroll 8
    for (int s = 0; s < min(LANES, a.splits - j * LANES); ++s) {
      const float g = __shfl(f[j], s, LANES);
      const ca_f32x4 v = *(const ca_f32x4 *)(part + (j * LANES + s) * step * HD);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += g < 0.f ? 0.f : g == 0.f && !(fabsf(v[e]) < INFINITY) ? v[e] : v[e] * g;   // (an infinity stays one)
    }
  }
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  T *out = (T *)a.out + r * a.out_stride + i % a.n_q_heads * HD + e0;
  if constexpr (sizeof(T) == 2) *(uint2 *)out = make_uint2(pack_bf16(y[0] * inv, y[1] * inv), pack_bf16(y[2] * inv, y[3] * inv));
  else *(float4 *)out = make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
  if (a.lse && e0 == 0) a.lse[i] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}

}  // namespace spark
