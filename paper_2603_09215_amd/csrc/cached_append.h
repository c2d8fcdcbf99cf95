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
template <typename T> __device__ __forceinline__ void store4(T *p, const float *f) {
  if constexpr (sizeof(T) == 4) {
    *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
  } else {
    *(uint2 *)p = make_uint2(f32_to_bf16(f[0]) | ((uint32_t)f32_to_bf16(f[1]) << 16), f32_to_bf16(f[2]) | ((uint32_t)f32_to_bf16(f[3]) << 16));
  }
}

// A head's vector takes HD / 8 lanes of eight values each, as four pairs: (a, b) of pair p are values (p, p + rotary / 2),
// interleaved (2 p, 2 p + 1), and past the rotary part (which stays) its neighbours.  VEC: rotary a multiple of
// eight and everything aligned for vectors of four values; then a lane's pairs are all turned or none.
template <typename S, typename T, int HD, bool VEC>
__global__ void __launch_bounds__(256) cached_append_k(AppendArgs a) {
  extern __shared__ float s_trig[];   // [rows][rotary / 2] cosines and sines
  constexpr int LANES = HD / 8;
  const int half = a.rotary / 2, row_first = blockIdx.x * a.rows, row_end = min(row_first + a.rows, a.batch.m);
  __shared__ int s_seq[64];
  // each row's sequence: the last that starts at it or before (rows outside all of them: -1)
  if ((int)threadIdx.x < row_end - row_first) {
    const int r = row_first + threadIdx.x;
    int lo = 0, hi = a.batch.n;   // the first start past r lies in lo .. hi + 1
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (a.batch.starts[mid + 1] > r) hi = mid;
      else lo = mid + 1;
    }
    s_seq[threadIdx.x] = lo < a.batch.n && a.batch.starts[lo] <= r ? lo : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < (row_end - row_first) * half; i += blockDim.x) {
    const int r = row_first + i / half, j = i % half, s = s_seq[i / half];
    if (s < 0) continue;
    const Sequence q = sequence(a.batch, s, a.cache.page_tokens);
    const int position = a.positions ? a.positions[r] : q.slot(r - q.row0);
    float c, sn;
    cos_sin((double)position * a.freqs[j], c, sn);
    s_trig[2 * i] = c * a.amplitude;
    s_trig[2 * i + 1] = sn * a.amplitude;
  }
  __syncthreads();
  const int heads = a.n_q_heads + 2 * a.cache.n_kv_heads, head0 = blockIdx.y * a.heads_per_wg, share = min(a.heads_per_wg, heads - head0);
  const int c = threadIdx.x % LANES, p0 = 4 * c;
  for (int u = threadIdx.x / LANES; u < (row_end - row_first) * share; u += blockDim.x / LANES) {
    const int i = u / share, r = row_first + i, h = head0 + u % share, s = s_seq[i];
    if (s < 0) continue;   // (the same for all lanes of a head)
    const int which = h < a.n_q_heads ? 0 : h < a.n_q_heads + a.cache.n_kv_heads ? 1 : 2;
    const int kvh = h - a.n_q_heads - (which == 2 ? a.cache.n_kv_heads : 0);
    const S *src = which == 0 ? (const S *)a.q + r * a.q_stride + (long long)h * HD
                 : which == 1 ? (const S *)a.k + r * a.k_stride + (long long)kvh * HD
                              : (const S *)a.v + r * a.v_stride + (long long)kvh * HD;
    const bool turn = which < 2;
    // where pair p lies
    auto first = [&](int p) { return p < half ? (a.interleaved ? 2 * p : p) : a.rotary + 2 * (p - half); };
    auto second = [&](int p) { return p < half ? (a.interleaved ? 2 * p + 1 : p + half) : a.rotary + 2 * (p - half) + 1; };
    const bool apart = !a.interleaved && p0 < half;   // (VEC)
    float x[4], y[4];
    if constexpr (VEC) {
      float lo[4], hi[4];
      load4(src + (apart ? p0 : first(p0)), lo);
      load4(src + (apart ? p0 + half : first(p0) + 4), hi);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = apart ? lo[e] : e < 2 ? lo[2 * (e & 1)] : hi[2 * (e & 1)];
        y[e] = apart ? hi[e] : e < 2 ? lo[2 * (e & 1) + 1] : hi[2 * (e & 1) + 1];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = Elem<S>::widen(src[first(p0 + e)]);
        y[e] = Elem<S>::widen(src[second(p0 + e)]);
      }
    }
    const float *gain = which == 0 ? a.q_gain : which == 1 ? a.k_gain : nullptr;
    if (gain) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += x[e] * x[e] + y[e] * y[e];
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if (sum > 1e-30f && sum < 1e37f) {
        const float f = 1.0f / sqrtf(sum * (1.0f / HD) + (float)a.eps);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] *= f * gain[first(p0 + e)];
          y[e] *= f * gain[second(p0 + e)];
        }
      } else {   // squares that leave fp32's range (the same lanes for all of a head)
        double wide = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) wide += (double)x[e] * x[e] + (double)y[e] * y[e];
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) wide += __shfl_xor(wide, o, 64);
        const double f = 1.0 / sqrt(wide * (1.0 / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = (float)(x[e] * f * gain[first(p0 + e)]);
          y[e] = (float)(y[e] * f * gain[second(p0 + e)]);
        }
      }
    }
    if (turn) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (p0 + e < half) {
          const float cs = s_trig[2 * (i * half + p0 + e)], sn = s_trig[2 * (i * half + p0 + e) + 1];
          const float t = x[e] * cs - y[e] * sn;
          y[e] = y[e] * cs + x[e] * sn;
          x[e] = t;
        }
      }
    }
    T *dst;
    if (which == 0) {
      dst = (T *)a.q_out + r * a.out_stride + (long long)h * HD;
    } else {
      const Sequence q = sequence(a.batch, s, a.cache.page_tokens);
      const int slot = q.slot(r - q.row0);
      if (slot < 0) continue;
      const int page = page_of(q, slot, a.cache.page_tokens, a.cache.n_pages);
      if (page < 0) continue;
      dst = a.cache.plane<T>(page, which - 1, kvh) + slot % a.cache.page_tokens * HD;
    }
    if constexpr (VEC) {
      float lo[4], hi[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] = apart ? x[e] : (e & 1) ? y[e >> 1] : x[e >> 1];
        hi[e] = apart ? y[e] : (e & 1) ? y[2 + (e >> 1)] : x[2 + (e >> 1)];
      }
      store4(dst + (apart ? p0 : first(p0)), lo);
      store4(dst + (apart ? p0 + half : first(p0) + 4), hi);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dst[first(p0 + e)] = Elem<T>::narrow(x[e]);
        dst[second(p0 + e)] = Elem<T>::narrow(y[e]);
      }
    }
  }
}

}  // namespace spark
