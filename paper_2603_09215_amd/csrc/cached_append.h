// Queries and keys normed and turned, keys and values into the cache (spark_cache_append).
//
//   x' = x / sqrt(mean x^2 + eps) * gain;  (a, b) -> amplitude * (a cos t - b sin t, b cos t + a sin t),  t = position * freqs[j]
//
// Bound by memory: every value is read once and written once, some twenty operations each.  A workgroup takes `rows` rows and a
// share of their heads: it works out the rows' sines and cosines once, into LDS, for all of those heads.  8191 rows of 36 heads of 128, bf16, norms, half of
// each head turned: 42 us, 3.6 TB/s (a copy of as many bytes 29); one row 3.7 us.
#pragma once
#include "cached_format.h"

namespace spark {

constexpr int APPEND_ROWS = 16;   // of a workgroup, at most
constexpr int APPEND_AHEAD = 2;   // heads whose values are on their way (8191 rows of 36 heads, in graphs: one 45.7 us, two 42.0, four 44.0)

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

// a lane's eight values as they lie: two fours, or (not aligned for that) one by one
template <typename S, bool VEC> struct Eight;
template <> struct Eight<float, true> {
  float4 v[2];
  __device__ __forceinline__ void load(const float *p, const int (&at)[8]) { v[0] = *(const float4 *)(p + at[0]); v[1] = *(const float4 *)(p + at[4]); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) { x[4 * i] = v[i].x; x[4 * i + 1] = v[i].y; x[4 * i + 2] = v[i].z; x[4 * i + 3] = v[i].w; }
  }
};
template <> struct Eight<bf16_t, true> {
  uint2 v[2];
  __device__ __forceinline__ void load(const bf16_t *p, const int (&at)[8]) { v[0] = *(const uint2 *)(p + at[0]); v[1] = *(const uint2 *)(p + at[4]); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[4 * i] = __uint_as_float(v[i].x << 16); x[4 * i + 1] = __uint_as_float(v[i].x & 0xffff0000u);
      x[4 * i + 2] = __uint_as_float(v[i].y << 16); x[4 * i + 3] = __uint_as_float(v[i].y & 0xffff0000u);
    }
  }
};
template <typename S> struct Eight<S, false> {
  S v[8];
  __device__ __forceinline__ void load(const S *p, const int (&at)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = p[at[e]];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = Elem<S>::widen(v[e]);
  }
};
// sum over the LANES (8 or 16) lanes of a head, the same bits in each
template <int CTRL> __device__ __forceinline__ float add_lane(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int LANES> __device__ __forceinline__ float head_sum(float v) {
  v = add_lane<0xb1>(v);    // neighbours,
  v = add_lane<0x4e>(v);    // pairs of them,
  v = add_lane<0x141>(v);   // fours (mirrored within eight)
  if constexpr (LANES == 16) v = add_lane<0x140>(v);   // eights (mirrored within sixteen)
  return v;
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
  __shared__ int s_seq[APPEND_ROWS];
  constexpr int LANES = HD / 8;
  const int half = a.rotary / 2, row_first = blockIdx.x * a.rows, row_end = min(row_first + a.rows, a.batch.m);
  const int groups = blockDim.x / LANES / a.rows, group = threadIdx.x / LANES, i = group / groups, r = min(row_first + i, a.batch.m - 1);
  const int c = threadIdx.x % LANES, p0 = 4 * c, nq = a.n_q_heads, nkv = a.cache.n_kv_heads;
  // where a lane's eight values lie: VEC two fours, else the first of four pairs and the second of them
  const bool turned = p0 < half, apart = turned && !a.interleaved;
  int at[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (VEC) {
      at[e] = apart ? p0 + (e & 3) + (e >> 2) * half : (turned ? 2 * p0 : a.rotary + 2 * (p0 - half)) + e;
    } else {
      const int p = p0 + (e & 3);
      at[e] = p < half ? (a.interleaved ? 2 * p + (e >> 2) : p + (e >> 2) * half) : a.rotary + 2 * (p - half) + (e >> 2);
    }
  }
  const S *q = (const S *)a.q + r * a.q_stride, *k = (const S *)a.k + r * a.k_stride, *v = (const S *)a.v + r * a.v_stride;
  auto source = [&](int h) { return h < nq ? q + h * HD : h < nq + nkv ? k + (h - nq) * HD : v + (h - nq - nkv) * HD; };
  // the first heads' values are on their way while the row's place and angles are found, the next ones' while one is worked on
  const int head_end = min((int)(blockIdx.y + 1) * a.heads_per_wg, nq + 2 * nkv);
  int h = blockIdx.y * a.heads_per_wg + group % groups;
  Eight<S, VEC> ahead[APPEND_AHEAD];
#pragma unroll
  for (int d = 0; d < APPEND_AHEAD; ++d)
    if (h + d * groups < head_end) ahead[d].load(source(h + d * groups), at);

  // each row's sequence: the first that ends behind it, if it has begun (rows outside all of them: -1)
  if ((int)threadIdx.x < row_end - row_first) {
    const int row = row_first + threadIdx.x;
    int lo = 0, hi = a.batch.n;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (a.batch.starts[mid + 1] > row) hi = mid;
      else lo = mid + 1;
    }
    s_seq[threadIdx.x] = lo < a.batch.n && a.batch.starts[lo] <= row ? lo : -1;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < (row_end - row_first) * half; j += blockDim.x) {
    const int row = row_first + j / half, s = s_seq[j / half];
    if (s < 0) continue;
    int position;
    if (a.positions) {
      position = a.positions[row];
    } else {
      const Sequence seq = sequence(a.batch, s, a.cache.page_tokens);
      position = seq.slot(row - seq.row0);
    }
    float cosine, sine;
    cos_sin((double)position * a.freqs[j % half], cosine, sine);
    s_trig[j] = make_float2(cosine * a.amplitude, sine * a.amplitude);
  }
  __syncthreads();
  if (row_first + i >= row_end || s_seq[i] < 0) return;
  const Sequence seq = sequence(a.batch, s_seq[i], a.cache.page_tokens);
  const int slot = seq.slot(r - seq.row0), page = slot < 0 ? -1 : page_of(seq, slot, a.cache.page_tokens, a.cache.n_pages);
  const int token = slot < 0 ? 0 : slot % a.cache.page_tokens;
  float cs[4], sn[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 t = p0 + e < half ? s_trig[i * half + p0 + e] : make_float2(1.f, 0.f);
    cs[e] = t.x;
    sn[e] = t.y;
  }
  T *out = (T *)a.q_out + r * a.out_stride, *place = a.cache.plane<T>(max(page, 0), 0, 0) + token * HD;
  const long long plane = (long long)a.cache.page_tokens * HD;
  int known = -1;
  const float *gain_at = nullptr;
  float gain[8];   // of queries, then of keys
  auto head = [&](Eight<S, VEC> &values) {
    const int which = h < nq ? 0 : h < nq + nkv ? 1 : 2;
    float x[8];
    values.get(x);
    if (h + APPEND_AHEAD * groups < head_end) values.load(source(h + APPEND_AHEAD * groups), at);
    if (which != known) {
      known = which;
      gain_at = which == 0 ? a.q_gain : which == 1 ? a.k_gain : nullptr;
#pragma unroll
      for (int e = 0; e < 8; ++e) gain[e] = gain_at ? gain_at[at[e]] : 1.f;
    }
    if (gain_at) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
      sum = head_sum<LANES>(sum);
      if (sum > 1e-30f && sum < 1e37f && a.eps < 1e37) {
        const float f = __builtin_amdgcn_rsqf(sum * (1.0f / HD) + (float)a.eps);   // (off by a last bit)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * f * gain[e];   // (the factor times the gain might leave fp32's range)
      } else {   // squares, or eps, that leave fp32's range (the same lanes for all of a head)
        double wide = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) wide += (double)x[e] * x[e];
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) wide += __shfl_xor(wide, o, 64);
        const double f = 1.0 / sqrt(wide * (1.0 / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)(x[e] * f * gain[e]);
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
    if (which > 0 && page < 0) return;
    T *dst = which == 0 ? out + h * HD : place + (which - 1) * nkv * plane + (h - nq - (which - 1) * nkv) * plane;
    if constexpr (VEC) {
      store_four(dst + at[0], x);
      store_four(dst + at[4], x + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) dst[at[e]] = Elem<T>::narrow(x[e]);
    }
  };
  while (h < head_end) {
#pragma unroll
    for (int d = 0; d < APPEND_AHEAD; ++d) {
      if (h < head_end) head(ahead[d]);
      h += groups;
    }
  }
}

}  // namespace spark
