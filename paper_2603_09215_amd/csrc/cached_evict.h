// Eviction from a paged cache by weight (spark_cache_evict): which slots stay, and the move of their keys and values.
#pragma once
#include "cached_format.h"

namespace spark {

struct EvictArgs {
  CacheView cache;
  BatchView batch;
  const float *weights;
  float *weights_out;
  int *kept, *lengths_out;
  const int *table_out;   // of the batch itself: in place
  int out_pages, keep, first, recent;
};

constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / 64;

// larger weight, larger key; -0 as +0; every NaN above all numbers
__device__ __forceinline__ uint32_t weight_key(float w) { return float_order_key(w + 0.f); }

// What is kept, one workgroup a sequence and head.  The `need` heaviest of the slots between the first and the recent ones: the
// key of the last of them by four digits of eight bits from the top, counted in LDS, each over the slots that
// share the digits found so far; then one pass in slot order writes the slots above that key and the
// first of those that have it.  Places are counts of what stays before them, so nothing depends on the order of threads.
__global__ void __launch_bounds__(EVICT_THREADS) cached_choose_k(EvictArgs a) {
  __shared__ unsigned s_count[256], s_wave[EVICT_WAVES], s_wave_ties[EVICT_WAVES], s_digit, s_before;
  const int s = blockIdx.x / a.cache.n_kv_heads, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slots = a.batch.max_pages * a.cache.page_tokens, length = cut(a.batch.lengths[s], 0, slots);
  const float *w = a.weights + (long long)blockIdx.x * slots;
  float *w_out = a.weights_out + (long long)blockIdx.x * slots;
  int *kept = a.kept + (long long)blockIdx.x * a.keep;
  const int left = min(length, a.keep);
  if (blockIdx.x % a.cache.n_kv_heads == 0 && tid == 0) a.lengths_out[s] = left;
  const bool all = length <= a.keep;
  const int lo = all ? 0 : a.first, hi = all ? 0 : length - a.recent;   // what is chosen from
  unsigned need = all ? 0u : (unsigned)(a.keep - a.first - a.recent), prefix = 0;
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_count[tid] = 0;
      __syncthreads();
      for (int t = lo + tid; t < hi; t += EVICT_THREADS) {
        const uint32_t key = weight_key(w[t]);
        if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_count[(key >> shift) & 255], 1u);
      }
      __syncthreads();
      if (wave == 0) {   // lane l: the digits 255 - 4 l and the three below it
        unsigned c[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += c[e] = s_count[255 - 4 * lane - e];
        unsigned incl = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const unsigned up = __shfl_up(incl, o, 64);
          if (lane >= o) incl += up;
        }
        unsigned before = incl - sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (before < need && need <= before + c[e]) { s_digit = 255 - 4 * lane - e; s_before = before; }
          before += c[e];
        }
      }
      __syncthreads();
      prefix |= s_digit << shift;
      need -= s_before;   // of those with this key so far
      __syncthreads();
    }
  }
  // in slot order; `need` of the slots whose key is `prefix`
  const bool some = !all && a.keep > a.first + a.recent;
  unsigned base = 0, base_ties = 0;   // what stays, and slots with the key, before this round
  for (int t0 = 0; t0 < length; t0 += EVICT_THREADS) {
    const int t = t0 + tid;
    const float x = t < length ? w[t] : 0.f;
    const uint32_t key = weight_key(x);
    const bool middle = t >= lo && t < hi, tie = some && middle && key == prefix;
    const bool above = t < length && (!middle || (some && key > prefix));
    const unsigned long long b_above = __ballot(above), b_tie = __ballot(tie), below = (1ull << lane) - 1;
    if (lane == 0) { s_wave[wave] = __popcll(b_above); s_wave_ties[wave] = __popcll(b_tie); }
    __syncthreads();
    unsigned place = base + __popcll(b_above & below), ties = base_ties + __popcll(b_tie & below);
    for (int v = 0; v < EVICT_WAVES; ++v) {
      const unsigned n = s_wave[v], nt = s_wave_ties[v];
      if (v < wave) { place += n; ties += nt; }
      base += n;
      base_ties += nt;
    }
    place += min(ties, need);
    if (above || (tie && ties < need)) {
      kept[place] = t;
      w_out[place] = x;   // (place <= t, and all threads have read their slot)
    }
    __syncthreads();
  }
  for (int t = left + tid; t < a.keep; t += EVICT_THREADS) kept[t] = -1;
  for (int t = left + tid; t < length; t += EVICT_THREADS) w_out[t] = 0.f;
}

// The move.  A vector is PIECES of 16 bytes; a workgroup takes of one sequence and head the keys or values, COLS pieces of each, and
// goes through its share of the kept slots in rounds.  In place one workgroup has all of them: a round's entries are all
// read before any is written, and it writes no slot past those that it has read, so nothing is lost.
template <typename T, int HD, int COLS>
__global__ void __launch_bounds__(1024) cached_move_k(EvictArgs a) {
  constexpr int SHARES = HD * (int)sizeof(T) / 16 / COLS;
  const int col = blockIdx.x % SHARES, which = blockIdx.x / SHARES % 2, sh = blockIdx.x / SHARES / 2;
  const int s = sh / a.cache.n_kv_heads, head = sh % a.cache.n_kv_heads, pt = a.cache.page_tokens;
  const int length = cut(a.batch.lengths[s], 0, a.batch.max_pages * pt), left = min(length, a.keep);
  const bool in_place = a.table_out == a.batch.table;
  if (in_place && left == length) return;
  const int *kept = a.kept + (long long)sh * a.keep, *in = a.batch.table + (long long)s * a.batch.max_pages, *out = a.table_out + (long long)s * a.out_pages;
  const int piece = col * COLS + threadIdx.x % COLS, entries = blockDim.x / COLS;
  for (int i0 = blockIdx.y * entries; i0 < left; i0 += gridDim.y * entries) {
    const int i = i0 + threadIdx.x / COLS;
    uint4 v = make_uint4(0, 0, 0, 0), *dst = nullptr;
    if (i < left) {
      const int t = cut(kept[i], 0, length - 1), from = in[t / pt], to = out[i / pt];
      if ((unsigned)from < (unsigned)a.cache.n_pages) v = ((const uint4 *)(a.cache.plane<T>(from, which, head) + t % pt * HD))[piece];
      if ((unsigned)to < (unsigned)a.cache.n_pages && !(in_place && t == i)) dst = (uint4 *)(a.cache.plane<T>(to, which, head) + i % pt * HD) + piece;
    }
    if (in_place) {
      wait_memory_ops();
      __syncthreads();
    }
    if (dst) *dst = v;
  }
}

}  // namespace spark
