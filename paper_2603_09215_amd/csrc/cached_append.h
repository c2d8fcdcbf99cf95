// Queries and keys normed and turned, keys and values into the cache (spark_cache_append).
//
//   x' = x / sqrt(mean x^2 + eps) * gain;  (a, b) -> amplitude * (a cos t - b sin t, b cos t + a sin t),  t = position * freqs[j]
//
// Bound by memory: every value is read once and written once, some twenty operations each.  A workgroup takes `rows` rows and a
// share of their heads: it works out the rows' sines and cosines once, into LDS, for all of those heads.
#pragma once
#include "cached_format.h"

namespace spark {

struct AppendArgs {
  CacheView cache;
  BatchView batch;
  const void *q, *k, *v;
  void *q_out;
  long long q_stride, k_stride, v_stride, out_stride;
  int n_q_heads, rotary, interleaved, rows, heads_per_wg;
  float amplitude;
  double eps;
  const double *freqs;
  const int *positions;
  const float *q_gain, *k_gain;
};

// cos and sin of a 64-bit angle in fp32: the angle in quarter turns, its whole part taken away in 64 bits (exact up to 2^52
// of them), the rest, at most an eighth of a turn, to 32 bits; there the series end below 2^-28 of the result
__device__ __forceinline__ void cos_sin(double angle, float &c, float &s) {
  const double turns = angle * 0.63661977236758134308, whole = rint(turns);
  const float x = (float)((turns - whole) * 1.57079632679489661923);
  const float y = x * x;
  const float sn = x + x * y * (-1.f / 6 + y * (1.f / 120 + y * (-1.f / 5040 + y * (1.f / 362880))));
  const float cs = 1.f + y * (-0.5f + y * (1.f / 24 + y * (-1.f / 720 + y * (1.f / 40320 + y * (-1.f / 3628800)))));
  const int quarter = (int)((long long)whole & 3);
  c = quarter == 0 ? cs : quarter == 1 ? -sn : quarter == 2 ? -cs : sn;
  s = quarter == 0 ? sn : quarter == 1 ? cs : quarter == 2 ? -sn : -cs;
}

template <typename T> __device__ __forceinline__ void load4(const T *p, float *f) {
  if constexpr (sizeof(T) == 4) {
    const float4 v = *(const float4 *)p;
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  } else {
    const uint2 v = *(const uint2 *)p;
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
}
template <typename T> __device__ __forceinline__ void store_four(T *p, const float *f) {
  if constexpr (sizeof(T) == 4) *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
  else *(uint2 *)p = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
}

// A head's vector takes HD / 8 lanes of eight values each, as four pairs: (a, b) of pair p are values (p, p + rotary / 2),
// interleaved (2 p, 2 p + 1), and past the rotary part (which stays) neighbours.  A group of such lanes has one row and goes through its share of
// the heads, so angles, gains and the row's place are found once for all of them.  VEC: rotary a multiple of eight
// and everything aligned for vectors of four values; then a lane's pairs are all turned or none.
template <typename S, typename T, int HD, bool VEC>
__global__ void __launch_bounds__(256) cached_append_k(AppendArgs a) {
  extern __shared__ float2 s_trig[];   // [rows][rotary / 2] cosine and sine
  __shared__ int s_seq[4];
  constexpr int LANES = HD / 8;
  const int half = a.rotary / 2, row_first = blockIdx.x * a.rows, row_end = min(row_first + a.rows, a.batch.m);
  // each row's sequence: the first that ends behind it, if it has begun (rows outside all of them: -1)
  if ((int)threadIdx.x < row_end - row_first) {
    const int r = row_first + threadIdx.x;
    int lo = 0, hi = a.batch.n;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (a.batch.starts[mid + 1] > r) hi = mid;
      else lo = mid + 1;
    }
    s_seq[threadIdx.x] = lo < a.batch.n && a.batch.starts[lo] <= r ? lo : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < (row_end - row_first) * half; i += blockDim.x) {
    const int r = row_first + i / half, s = s_seq[i / half];
    if (s < 0) continue;
    int position;
    if (a.positions) {
      position = a.positions[r];
    } else {
      const Sequence q = sequence(a.batch, s, a.cache.page_tokens);
      position = q.slot(r - q.row0);
    }
    float c, sn;
    cos_sin((double)position * a.freqs[i % half], c, sn);
    s_trig[i] = make_float2(c * a.amplitude, sn * a.amplitude);
  }
  __syncthreads();

  const int groups = blockDim.x / LANES / a.rows, group = threadIdx.x / LANES, i = group / groups, r = row_first + i;
  if (r >= row_end || s_seq[i] < 0) return;
  const Sequence seq = sequence(a.batch, s_seq[i], a.cache.page_tokens);
  const int slot = seq.slot(r - seq.row0), page = slot < 0 ? -1 : page_of(seq, slot, a.cache.page_tokens, a.cache.n_pages);
  const int token = slot < 0 ? 0 : slot % a.cache.page_tokens;
  const int c = threadIdx.x % LANES, p0 = 4 * c, nq = a.n_q_heads, nkv = a.cache.n_kv_heads;
  // where a lane's eight values lie: VEC two fours, else pairs
  const bool turned = p0 < half, apart = turned && !a.interleaved;
  int at[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (VEC) {
      at[e] = apart ? p0 + (e & 3) + (e >> 2) * half : (turned ? 2 * p0 : a.rotary + 2 * (p0 - half)) + e;
    } else {   // the first of four pairs, the second of them
      const int p = p0 + (e & 3);
      at[e] = p < half ? (a.interleaved ? 2 * p + (e >> 2) : p + (e >> 2) * half) : a.rotary + 2 * (p - half) + (e >> 2);
    }
  }
  float cs[4], sn[4], gain[2][8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 v = p0 + e < half ? s_trig[i * half + p0 + e] : make_float2(1.f, 0.f);
    cs[e] = v.x;
    sn[e] = v.y;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    gain[0][e] = a.q_gain ? a.q_gain[at[e]] : 1.f;
    gain[1][e] = a.k_gain ? a.k_gain[at[e]] : 1.f;
  }
  const int head0 = blockIdx.y * a.heads_per_wg, head_end = min(head0 + a.heads_per_wg, nq + 2 * nkv);
  const S *q = (const S *)a.q + r * a.q_stride, *k = (const S *)a.k + r * a.k_stride, *v = (const S *)a.v + r * a.v_stride;
  T *out = (T *)a.q_out + r * a.out_stride, *place = a.cache.plane<T>(max(page, 0), 0, 0) + token * HD;
  const long long plane = (long long)a.cache.page_tokens * HD;
#pragma unroll 2
  for (int h = head0 + group % groups; h < head_end; h += groups) {
    const int which = h < nq ? 0 : h < nq + nkv ? 1 : 2;
    const S *src = which == 0 ? q + h * HD : which == 1 ? k + (h - nq) * HD : v + (h - nq - nkv) * HD;
    float x[8];
    if constexpr (VEC) {
      load4(src + at[0], x);
      load4(src + at[4], x + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = Elem<S>::widen(src[at[e]]);
    }
    if (which == 0 ? a.q_gain != nullptr : which == 1 && a.k_gain != nullptr) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if (sum > 1e-30f && sum < 1e37f) {
        const float f = 1.0f / sqrtf(sum * (1.0f / HD) + (float)a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= f * (which == 0 ? gain[0][e] : gain[1][e]);
      } else {   // squares that leave fp32's range (the same lanes for all of a head)
        double wide = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) wide += (double)x[e] * x[e];
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) wide += __shfl_xor(wide, o, 64);
        const double f = 1.0 / sqrt(wide * (1.0 / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)(x[e] * f * (which == 0 ? gain[0][e] : gain[1][e]));
      }
    }
    if (which < 2 && a.rotary) {
      if (!VEC || apart) {
        if (turned) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (!VEC && p0 + e >= half) continue;
            const float t = x[e] * cs[e] - x[4 + e] * sn[e];
            x[4 + e] = x[4 + e] * cs[e] + x[e] * sn[e];
            x[e] = t;
          }
        }
      } else if (turned) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float t = x[2 * e] * cs[e] - x[2 * e + 1] * sn[e];
          x[2 * e + 1] = x[2 * e + 1] * cs[e] + x[2 * e] * sn[e];
          x[2 * e] = t;
        }
      }
    }
    if (which > 0 && page < 0) continue;
    T *dst = which == 0 ? out + h * HD : place + (which - 1) * nkv * plane + (h - nq - (which - 1) * nkv) * plane;
    if constexpr (VEC) {
      store_four(dst + at[0], x);
      store_four(dst + at[4], x + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) dst[at[e]] = Elem<T>::narrow(x[e]);
    }
  }
}

}  // namespace spark
