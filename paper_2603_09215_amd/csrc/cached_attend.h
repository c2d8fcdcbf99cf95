// Attention of new rows over a paged cache (spark_cache_attend).
//
//   out = sum_t exp(s_t - M) v_t / L,  s_t = scale q . k_t,  M = max s_t,  L = sum_t exp(s_t - M),  lse = M + log L
//
// over the slots t that a row sees, in one pass with a running maximum and sum.
#pragma once
#include "cached_format.h"

namespace spark {

struct AttendArgs {
  CacheView cache;
  BatchView batch;
  const void *q;
  void *out;
  float *lse;   // or nullptr
  long long q_stride, out_stride;
  int n_q_heads, group, causal;
  float scale;
};

// a wave per row and query head
template <typename T, int HD>
__global__ void __launch_bounds__(64) cached_attend_k(AttendArgs a) {
  const int r = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
  int s = 0;
  while (s < a.batch.n && a.batch.starts[s + 1] <= r) ++s;
  if (s == a.batch.n || a.batch.starts[s] > r) return;
  const Sequence seq = sequence(a.batch, s, a.cache.page_tokens);
  const int end = a.causal || seq.slot(r - seq.row0) < 0 ? seq.slot(r - seq.row0) + 1 : seq.length;
  constexpr int E = HD / 64;
  float q[E], o[E] = {}, top = -INFINITY, sum = 0.f;
  for (int e = 0; e < E; ++e) q[e] = Elem<T>::widen(((const T *)a.q)[r * a.q_stride + h * HD + 64 * e + lane]) * a.scale;
  for (int t = 0; t < end; ++t) {
    const int page = page_of(seq, t, a.cache.page_tokens, a.cache.n_pages);
    if (page < 0) continue;
    const T *k = a.cache.plane<T>(page, 0, h / a.group) + t % a.cache.page_tokens * HD, *v = a.cache.plane<T>(page, 1, h / a.group) + t % a.cache.page_tokens * HD;
    float x = 0.f;
    for (int e = 0; e < E; ++e) x += q[e] * Elem<T>::widen(k[64 * e + lane]);
    x = wave_sum(x);
    const float now = fmaxf(top, x), base = now == -INFINITY ? 0.f : now, f = expf(top - base), p = expf(x - base);
    sum = sum * f + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * Elem<T>::widen(v[64 * e + lane]);
    top = now;
  }
  for (int e = 0; e < E; ++e) ((T *)a.out)[r * a.out_stride + h * HD + 64 * e + lane] = Elem<T>::narrow(sum > 0.f || sum != sum ? o[e] / sum : 0.f);
  if (a.lse && lane == 0) a.lse[(long long)r * a.n_q_heads + h] = sum > 0.f || sum != sum ? top + logf(sum) : -INFINITY;
}

}  // namespace spark
