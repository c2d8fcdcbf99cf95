// The attention weight that each slot of a cache gets from a batch's rows (spark_cache_weigh).
//
//   out[t] = decay before[t] + sum over rows r that see t, heads h of the group: exp(scale q_rh . k_t - lse_rh)
//
// With few rows bound by the keys' way through memory, with many by the exponentials.  A wave takes 32 tokens, whose keys stay in registers, and
// goes through the (row, head) pairs in blocks of 32: scores S [pair][token] = Q K^T, so that a lane has 16 scores of one token and
// its sum is one register.  With many pairs the four waves of a workgroup share the tokens and deal out the
// blocks, and add up their sums in order; with few each has its own tokens.  Nothing is added by atomics.
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
  int n_q_heads, group, causal, way;   // way: waves that share their tokens, 1 or 4
  float factor, decay;                 // factor and flip as in AttendArgs
  uint32_t flip;
};

template <typename T, int HD>
__global__ void __launch_bounds__(256) cached_weigh_k(WeighArgs a) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int STEPS = HD * (int)sizeof(T) / 32;   // 16-byte pieces of a key or query that a lane holds
  __shared__ float4 s_bias[4][8];   // of a wave's block of pairs: -lse log2 e,
  __shared__ int4 s_limit[4][8];    // and the last slot seen
  __shared__ float s_sum[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int s = blockIdx.x / a.cache.n_kv_heads, kvh = blockIdx.x % a.cache.n_kv_heads;
  const Sequence seq = sequence(a.batch, s, a.cache.page_tokens);
  const int pairs = seq.rows * a.group, blocks = (pairs + 31) / 32, own = 4 / a.way;
  const int pieces = (seq.length + 31) / 32;
  for (int y = blockIdx.y * own; y < pieces; y += gridDim.y * own) {
    const int t0 = (y + wave / a.way) * 32, t = t0 + col;
    // (a wave past the length works on nothing, and comes to the barriers)
    const int pages = pages_of(seq, a.cache, t0 / 16 + (lane & 1), seq.length);
    const unsigned here = (unsigned)__ballot(pages >= 0) & 3u;
    ca_u32x4 k[STEPS];
    {
      int index, in;
      place_of(a.cache, t0 / 16 + (col >> 4), index, in);
      const ca_u32x4 *at = (const ca_u32x4 *)(a.cache.plane<T>(max(__shfl(pages, col >> 4, 64), 0), 0, kvh) + (in + (col & 15)) * HD);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) k[i] = here ? at[2 * i + half] : ca_u32x4{0, 0, 0, 0};
    }
    float total = 0.f;
    for (int b = wave % a.way; b < blocks; b += a.way) {
      const int first = last_seen(seq, b * 32 / a.group, a.causal), last = last_seen(seq, min(b * 32 + 31, pairs - 1) / a.group, a.causal);
      if (t0 > last || !here) continue;
      const int p = min(b * 32 + col, pairs - 1), row = p / a.group, h = kvh * a.group + p % a.group;
      const T *at = (const T *)a.q + (seq.row0 + row) * a.q_stride + (long long)h * HD;
      ca_u32x4 q[STEPS];
#pragma unroll
      for (int i = 0; i < STEPS; ++i) q[i] = ca_signed<T>(((const ca_u32x4 *)at)[2 * i + half], a.flip);
      const float lse = a.lse[(long long)(seq.row0 + row) * a.n_q_heads + h];
      const bool none = b * 32 + col >= pairs || lse == -INFINITY;
      if (half == 0) {
        ((float *)s_bias[wave])[col] = none ? 0.f : lse * -1.44269504088896340736f;
        ((int *)s_limit[wave])[col] = none ? -1 : last_seen(seq, row, a.causal);
      }
      const bool masked = __any(none) || t0 + 31 > first || here != 3u;
      ca_f32x16 sc;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        if constexpr (BF) {
          sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ca_operand(q[i]), ca_operand(k[i]), sc, 0, 0, 0);
        } else {
          const float4 x = __builtin_bit_cast(float4, q[i]), z = __builtin_bit_cast(float4, k[i]);
          sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, z.x, sc, 0, 0, 0);
          sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, z.y, sc, 0, 0, 0);
          sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, z.z, sc, 0, 0, 0);
          sc = __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, z.w, sc, 0, 0, 0);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // pairs 8 i + 4 half + 0..3
        const float4 bias = s_bias[wave][2 * i + half];
        const float bs[4] = {bias.x, bias.y, bias.z, bias.w};
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ca_exp2(fmaf(sc[4 * i + e], a.factor, bs[e]));
        if (masked) {
          const int4 limit = s_limit[wave][2 * i + half];
          const int lim[4] = {limit.x, limit.y, limit.z, limit.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = t <= lim[e] ? x[e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) total += x[e];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
    total = ca_sum_halves(total);
    if (!((here >> (col >> 4)) & 1)) total = 0.f;
    if (a.way > 1) {
      if (half == 0) s_sum[wave][col] = total;
      __syncthreads();
      total = s_sum[0][col] + s_sum[1][col] + s_sum[2][col] + s_sum[3][col];
      __syncthreads();
    }
    if (half == 0 && wave % a.way == 0 && t < seq.length) {
      const long long at = (long long)blockIdx.x * a.batch.max_pages * a.cache.page_tokens + t;
      a.out[at] = a.before ? a.decay * a.before[at] + total : total;
    }
  }
}

}  // namespace spark
