// The attention weight that each slot of a cache gets from a batch's rows (spark_cache_weigh).
//
//   out[t] = decay before[t] + sum over rows r that see t, heads h of the group: exp(scale q_rh . k_t - lse_rh)
//
// With few rows bound by the keys' way through memory, with many by the exponentials and the queries' way out of L2.  A wave takes 32 tokens, whose keys
// stay in registers, and goes through the (row, head) pairs in blocks of 32: scores S [pair][token] = Q K^T, so that a lane has 16 scores of one
// token and its sum is one register.  Many pairs: the eight waves of a workgroup share their tokens, each loading an eighth of their keys, deal out the
// blocks, the next one's queries on their way while one is worked on, and add up their sums in order.  1024 pairs of 8191 slots and two heads, bf16: 12.4 us.
// On the way there: one piece of 32 tokens instead of two, so twice the queries out of L2 (134 MB), 20; two 16.2 (3.2 of it exponentials, 2.5 queries); keys
// loaded once 14.1 (sixteen waves 14.8); operands of queries read from LDS as they are used 12.3.  Few: each wave has its own tokens, the next ones' keys are on
// their way while they are worked on, and a single block's queries stay: 32 steps of up to 4095 slots, 4 heads, 25 us, 4.1 TB/s.
// Nothing is added by atomics.  What a wave's blocks lose in their additions is carried along, so the error does not grow with the rows.
#pragma once
#include "cached_attend.h"

namespace spark {

struct WeighArgs {
  CacheView cache;
  BatchView batch;
  const void *q;
  const float *lse, *before;   // before: or nullptr
  float *out;
  long long q_stride;
  int n_q_heads, group, causal;
  uint32_t reciprocal;         // 2^32 / group rounded up, 0 for one
  float factor, decay;         // factor and flip as in AttendArgs
  uint32_t flip;
};

template <typename T, bool MANY> struct Weigh {
  static constexpr int WAVES = MANY ? 8 : 4, WAY = MANY ? 8 : 1;            // of a workgroup; that share tokens
  static constexpr int TB = MANY && sizeof(T) == 2 ? 2 : 1;                  // pieces of 32 tokens that a wave works on at a time
  static constexpr int PIECES = WAVES / WAY * TB;                            // that a workgroup works on at a time
  static constexpr size_t lds(int hd) { return MANY ? (WAVES + TB) * 32 * hd * sizeof(T) : 0; }   // a block of queries a wave, the keys
};

template <typename T, int HD, bool MANY>
__global__ void __launch_bounds__(MANY ? 512 : 256) cached_weigh_k(WeighArgs a) {
  using W = Weigh<T, MANY>;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int STEPS = HD * (int)sizeof(T) / 32, TB = W::TB;   // 16-byte pieces of a key or query that a lane holds
  __shared__ float4 s_bias[W::WAVES][8];   // of a wave's block of pairs: -lse log2 e,
  __shared__ int4 s_limit[W::WAVES][8];    // and the last slot seen
  __shared__ float s_sum[W::WAVES][TB][32];
  extern __shared__ __attribute__((aligned(16))) char s_dyn[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int s = blockIdx.x / a.cache.n_kv_heads, kvh = blockIdx.x % a.cache.n_kv_heads;
  const Sequence seq = sequence(a.batch, s, a.cache.page_tokens);
  const int pairs = seq.rows * a.group, blocks = (pairs + 31) / 32, pieces = (seq.length + 31) / 32;

  // the 16s of TB pieces are found by the first lanes
  auto ask_piece = [&](int piece) { return ask(seq, a.cache, 2 * piece + (lane & (2 * TB - 1)), seq.length); };
  constexpr int ROW = HD * (int)sizeof(T);
  const char *keys = (const char *)a.cache.plane<T>(0, 0, kvh);
  auto load_keys = [&](const Found &f, ca_u32x4 (&k)[TB][STEPS]) {
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const char *lower = at_lane(keys, f, 2 * j), *upper = at_lane(keys, f, 2 * j + 1);
      const char *at = (col >> 4 ? upper : lower) + ((col & 15) * ROW + 16 * half);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) k[j][i] = *(const ca_u32x4 *)(at + 32 * i);
    }
  };
  // Queries of block b and their lse.  As operands (few pairs), or whole rows in the lanes' order (many: 0.7 us
  // less, of 16.9 at the time, than with 32 bytes of each of 32 rows a load) that go to LDS.
  constexpr int VECS = 2 * STEPS;   // of a query
  auto load_queries = [&](int b, ca_u32x4 (&q)[STEPS], float &lse) {
    const int first = b * 32 / a.group, past = b * 32 - first * a.group, most = pairs - 1 - b * 32;   // (pairs past the last: that one, left out)
    auto place = [&](int pair, int &h) {   // its row; (numbers below 2^13 by one of at most 2^12: exact)
      const int n = past + min(pair, most), r = a.reciprocal ? (int)__umulhi((uint32_t)n, a.reciprocal) : n;
      h = kvh * a.group + n - r * a.group;
      return seq.row0 + first + r;
    };
    int h;
    const long long row = place(col, h);
    lse = a.lse[row * a.n_q_heads + h];
    if constexpr (MANY) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const long long r = place(i * (64 / VECS) + lane / VECS, h);
        q[i] = ((const ca_u32x4 *)((const T *)a.q + r * a.q_stride + (long long)h * HD))[lane % VECS];
      }
    } else {
      const ca_u32x4 *at = (const ca_u32x4 *)((const T *)a.q + row * a.q_stride + (long long)h * HD);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) q[i] = at[2 * i + half];
    }
  };
  auto turn = [&](const ca_u32x4 (&in)[STEPS]) {   // to LDS, a row's pieces turned by its number
    ca_u32x4 *block = (ca_u32x4 *)s_dyn + wave * 32 * VECS;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const int row = i * (64 / VECS) + lane / VECS;
      block[row * VECS + ((lane ^ row) & (VECS - 1))] = in[i];
    }
  };
  auto turned = [&](int row, int i) { return ((const ca_u32x4 *)s_dyn)[row * VECS + ((2 * i + half) ^ (col & (VECS - 1)))]; };   // (row mod 32 is col)
  bool some_out = false;   // of the block in LDS: a pair that gives nothing
  auto place_block = [&](int b, float lse) {
    const bool none = b * 32 + col >= pairs || lse == -INFINITY;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (half == 0) {
      ((float *)s_bias[wave])[col] = none ? 0.f : lse * -1.44269504088896340736f;
      ((int *)s_limit[wave])[col] = none ? -1 : last_seen(seq, (b * 32 + col) / a.group, a.causal);
    }
    some_out = __any(none);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  float total[TB], lost[TB];   // of this wave's blocks so far, and what their additions have lost: rows may be many
  // what a block's pairs give tokens t0 + 32 j + col
  auto add_block = [&](int b, int t0, const ca_u32x4 (&k)[TB][STEPS], const ca_u32x4 (&q)[STEPS]) {
    const bool masked = some_out || t0 + 32 * TB - 1 > last_seen(seq, b * 32 / a.group, a.causal);
    ca_f32x16 sc[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[j][r] = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
      const ca_u32x4 qs = ca_signed<T>(MANY ? turned(wave * 32 + col, i) : q[i], a.flip);
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        if constexpr (BF) {
          sc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ca_operand(qs), ca_operand(k[j][i]), sc[j], 0, 0, 0);
        } else {
          const ca_f32x4 x = __builtin_bit_cast(ca_f32x4, qs), z = __builtin_bit_cast(ca_f32x4, k[j][i]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], z[e], sc[j], 0, 0, 0);
        }
      }
    }
    float sum[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) sum[j] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // pairs 8 i + 4 half + 0..3
      const float4 bias = s_bias[wave][2 * i + half];
      const float bs[4] = {bias.x, bias.y, bias.z, bias.w};
      float x[TB][4];
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = ca_exp2(fmaf(sc[j][4 * i + e], a.factor, bs[e]));
      if (masked) {
        const int4 limit = s_limit[wave][2 * i + half];
        const int lim[4] = {limit.x, limit.y, limit.z, limit.w};
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j][e] = t0 + 32 * j + col <= lim[e] ? x[j][e] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j] += x[j][e];
    }
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      const float more = sum[j] - lost[j], now = total[j] + more;
      lost[j] = now < INFINITY ? now - total[j] - more : 0.f;   // (an infinity stays one)
      total[j] = now;
    }
  };
  auto begin = [&]() {
#pragma unroll
    for (int j = 0; j < TB; ++j) total[j] = lost[j] = 0.f;
  };
  auto last_of = [&](int b) { return last_seen(seq, min(b * 32 + 31, pairs - 1) / a.group, a.causal); };   // what block b sees
  auto write = [&](int piece, bool has_page, float sum) {
    const int t = piece * 32 + col;
    if (half || t >= seq.length) return;
    const long long at = (long long)blockIdx.x * a.batch.max_pages * a.cache.page_tokens + t;
    sum = has_page ? sum : 0.f;   // (slots of no page: whatever came of the first page's keys)
    a.out[at] = a.before ? a.decay * a.before[at] + sum : sum;
  };

  const int step = gridDim.y * W::PIECES;
  int piece = blockIdx.y * W::PIECES + wave / W::WAY * TB;
  ca_u32x4 k[TB][STEPS], q[STEPS];
  float lse = 0.f;
  if constexpr (MANY) {
    for (; piece < pieces; piece += step) {   // (the same for all of a workgroup)
      const Asked asked = ask_piece(piece);
      const int t0 = piece * 32;
      int b = wave;
      while (b < blocks && t0 > last_of(b)) b += W::WAY;
      ca_u32x4 ahead[STEPS];
      float next_lse = 0.f;
      if (b < blocks) load_queries(b, ahead, next_lse);
      const Found found = find<ROW>(asked, a.cache, sizeof(T));
      const unsigned here = (unsigned)__ballot(found.there);
      // each wave loads its share of the keys; through LDS all have them all
      constexpr int TOKENS = 64 / VECS;
      ca_u32x4 share[32 * TB / (W::WAVES * TOKENS)];
#pragma unroll
      for (int j = 0; j < 32 * TB / (W::WAVES * TOKENS); ++j) {
        const int token = (j * W::WAVES + wave) * TOKENS;
        share[j] = ((const ca_u32x4 *)(at_lane(keys, found, token / 16) + (token % 16 + lane / VECS) * ROW))[lane % VECS];
      }
      ca_u32x4 *block = (ca_u32x4 *)s_dyn + W::WAVES * 32 * VECS;
#pragma unroll
      for (int j = 0; j < 32 * TB / (W::WAVES * TOKENS); ++j) {
        const int token = (j * W::WAVES + wave) * TOKENS + lane / VECS;
        block[token * VECS + ((lane ^ token) & (VECS - 1))] = share[j];
      }
      __syncthreads();
      begin();
#pragma unroll
      for (int j = 0; j < TB; ++j) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) k[j][i] = turned((W::WAVES + j) * 32 + col, i);
      }
      for (; b < blocks; b += W::WAY) {
        turn(ahead);
        lse = next_lse;
        if (b + W::WAY < blocks) load_queries(b + W::WAY, ahead, next_lse);
        place_block(b, lse);
        add_block(b, t0, k, q);
      }
#pragma unroll
      for (int j = 0; j < TB; ++j) {
        total[j] = ca_sum_halves(total[j]);
        if (half == 0) s_sum[wave][j][col] = total[j];
      }
      __syncthreads();
      if (wave < TB) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < W::WAVES; ++w) sum += s_sum[w][wave][col];
        write(piece + wave, (here >> (2 * wave + (col >> 4))) & 1, sum);
      }
      __syncthreads();
    }
  } else {
    ca_u32x4 ahead[TB][STEPS];
    Found found = find<ROW>(ask_piece(piece), a.cache, sizeof(T));
    Asked asked = ask_piece(piece + step);
    int held = -1;
    if (piece < pieces) load_keys(found, ahead);
    for (; piece < pieces; piece += step) {   // (a wave by itself)
      const bool has_page = ((unsigned)__ballot(found.there) >> (col >> 4)) & 1;
      const int t0 = piece * 32;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) k[0][i] = ahead[0][i];
      if (piece + step < pieces) {
        found = find<ROW>(asked, a.cache, sizeof(T));
        asked = ask_piece(piece + 2 * step);
        load_keys(found, ahead);
      }
      begin();
      for (int b = 0; b < blocks; ++b) {
        if (t0 > last_of(b)) continue;
        if (b != held) {
          load_queries(b, q, lse);
          place_block(b, lse);
          held = b;
        }
        add_block(b, t0, k, q);
      }
      write(piece, has_page, ca_sum_halves(total[0]));
    }
  }
}

}  // namespace spark
