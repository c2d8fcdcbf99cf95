// The attention weight that each slot of a cache gets from a batch's rows (spark_cache_weigh).
//
//   out[t] = decay before[t] + sum over rows r that see t, heads h of the group: exp(scale q_rh . k_t - lse_rh)
#pragma once
#include "cached_format.h"

namespace spark {

struct WeighArgs {
  CacheView cache;
  BatchView batch;
  const void *q;
  const float *lse, *before;   // before: or nullptr
  float *out;
  long long q_stride;
  int n_q_heads, group, causal;
  float scale, decay;
};

// a thread per slot
template <typename T, int HD>
__global__ void __launch_bounds__(256) cached_weigh_k(WeighArgs a) {
  const int s = blockIdx.x / a.cache.n_kv_heads, kvh = blockIdx.x % a.cache.n_kv_heads;
  const Sequence seq = sequence(a.batch, s, a.cache.page_tokens);
  for (int t = blockIdx.y * blockDim.x + threadIdx.x; t < seq.length; t += gridDim.y * blockDim.x) {
  const long long at = (long long)blockIdx.x * a.batch.max_pages * a.cache.page_tokens + t;
  float total = a.before ? a.decay * a.before[at] : 0.f;
  const int page = page_of(seq, t, a.cache.page_tokens, a.cache.n_pages);
  if (page >= 0) {
    const T *k = a.cache.plane<T>(page, 0, kvh) + t % a.cache.page_tokens * HD;
    for (int i = 0; i < seq.rows; ++i) {
      const int slot = seq.slot(i);
      if (slot < 0 || (a.causal && t > slot)) continue;
      for (int h = kvh * a.group; h < (kvh + 1) * a.group; ++h) {
        const T *q = (const T *)a.q + (seq.row0 + i) * a.q_stride + (long long)h * HD;
        const float lse = a.lse[(long long)(seq.row0 + i) * a.n_q_heads + h];
        float x = 0.f;
        for (int e = 0; e < HD; ++e) x += Elem<T>::widen(q[e]) * Elem<T>::widen(k[e]);
        if (lse != -INFINITY) total += expf(x * a.scale - lse);
      }
    }
  }
  a.out[at] = total;
  }
}

}  // namespace spark
