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

typedef __attribute__((ext_vector_type(4))) uint32_t move_u32x4;

// larger weight, larger key; -0 as +0; every NaN above all numbers
__device__ __forceinline__ uint32_t weight_key(float w) { return float_order_key(w + 0.f); }

// What is kept, one workgroup a sequence and head, up to eight slots in a row to a thread.  The `need` heaviest of the slots between the first
// and the recent ones: the key of the last of them by digits of 11, 11 and 10 bits from the top, counted in LDS, each over the slots that share
// the digits found so far; then the slots above that key and the first of those that have it are written in slot
// order.  Places are counts of what stays before them, so nothing depends on the order of threads.  Up to eight slots a thread are read once.
// Bound by its barriers and, with many slots, by one compute unit's instructions a head: four heads of 4097 slots take 10 us, 64 of up to 8191 15, four of 60000 142.
constexpr int EVICT_EACH = 8, EVICT_BINS = 2048;

template <int CTRL, int ROWS> __device__ __forceinline__ unsigned add_from(unsigned v) {   // a lane's value from another one's, of some rows of 16
  return v + (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true);
}
// inclusive sum over a wave's lanes
__device__ __forceinline__ unsigned wave_scan(unsigned v) {
  v = add_from<0x111, 0xf>(v);   // 1, 2, 4 and 8 to the right within sixteen
  v = add_from<0x112, 0xf>(v);
  v = add_from<0x114, 0xf>(v);
  v = add_from<0x118, 0xf>(v);
  v = add_from<0x142, 0xa>(v);   // the last of sixteen to the next sixteen,
  return add_from<0x143, 0xc>(v);   // of 32 to the upper 32
}
// sum over the threads before this one in the workgroup, and over all of them
template <int WAVES> __device__ __forceinline__ unsigned evict_scan(unsigned v, unsigned *s_wave, unsigned &total) {
  static_assert(WAVES <= 16, "waves fit a row of lanes");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned incl = wave_scan(v);
  __syncthreads();
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  unsigned w = (lane & 15) < WAVES ? s_wave[lane & 15] : 0u;
  w = add_from<0x111, 0xf>(w);
  w = add_from<0x112, 0xf>(w);
  w = add_from<0x114, 0xf>(w);
  w = add_from<0x118, 0xf>(w);
  total = (unsigned)__builtin_amdgcn_readlane((int)w, 15);
  return incl - v + (wave ? (unsigned)__builtin_amdgcn_readlane((int)w, wave - 1) : 0u);
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) cached_choose_k(EvictArgs a) {
  constexpr int WAVES = THREADS / 64, DIGITS = EVICT_BINS / THREADS;   // DIGITS: a thread's
  __shared__ unsigned s_count[EVICT_BINS], s_wave[WAVES], s_digit, s_before;
  const int s = blockIdx.x / a.cache.n_kv_heads, tid = threadIdx.x;
  const int slots = a.batch.max_pages * a.cache.page_tokens, length = cut(a.batch.lengths[s], 0, slots);
  const float *w = a.weights + (long long)blockIdx.x * slots;
  float *w_out = a.weights_out + (long long)blockIdx.x * slots;
  int *kept = a.kept + (long long)blockIdx.x * a.keep;
  const int left = min(length, a.keep);
  if (blockIdx.x % a.cache.n_kv_heads == 0 && tid == 0) a.lengths_out[s] = left;
  const bool all = length <= a.keep;
  const int lo = all ? 0 : a.first, hi = all ? 0 : length - a.recent;   // what is chosen from
  unsigned need = all ? 0u : (unsigned)(a.keep - a.first - a.recent), prefix = 0;
  const bool some = need > 0;
  const int each = cut((length + THREADS - 1) / THREADS, 1, EVICT_EACH), chunk = each * THREADS;
  float x[EVICT_EACH];
  uint32_t key[EVICT_EACH];   // 0, which no weight has, for what is not chosen from: in the lowest place, never reached
  int held = -1;              // which chunk they are of
  auto fetch = [&](int c0) {
    if (c0 == held) return;
    held = c0;
#pragma unroll
    for (int e = 0; e < EVICT_EACH; ++e) {
      const int t = c0 + tid * each + e;
      x[e] = e < each && t < length ? w[t] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < EVICT_EACH; ++e) {
      const int t = c0 + tid * each + e;
      key[e] = e < each && t >= lo && t < hi ? weight_key(x[e]) : 0u;
    }
  };
  if (some) {
    constexpr uint32_t ZERO = 0x80000000u;   // the key of nothing, which many slots may have: counted by waves
#pragma unroll 1
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0;
      const unsigned mask = digit == 2 ? 1023u : 2047u, span = digit == 0 ? ~0u : digit == 1 ? (1u << 21) - 1 : (1u << 10) - 1;   // keys with this prefix
#pragma unroll
      for (int j = 0; j < DIGITS; ++j) s_count[j * THREADS + tid] = 0;
      __syncthreads();
      for (int c0 = 0; c0 < length; c0 += chunk) {
        fetch(c0);
        unsigned zeros = 0;
#pragma unroll
        for (int e = 0; e < EVICT_EACH; ++e) {
          if (e < each) {
            const bool zero = key[e] == ZERO, counts = (key[e] ^ prefix) <= span;
            zeros += __popcll(__ballot(zero));
            if (counts && (key[e] & 0x7fffffffu)) atomicAdd(&s_count[(key[e] >> shift) & mask], 1u);
          }
        }
        if (zeros && (ZERO ^ prefix) <= span && (tid & 63) == 0) atomicAdd(&s_count[(ZERO >> shift) & mask], zeros);
      }
      __syncthreads();
      // from the highest digit down, DIGITS a thread
      unsigned n[DIGITS], sum = 0, total;
#pragma unroll
      for (int j = 0; j < DIGITS; ++j) sum += n[j] = s_count[EVICT_BINS - 1 - DIGITS * tid - j];
      unsigned before = evict_scan<WAVES>(sum, s_wave, total);
#pragma unroll
      for (int j = 0; j < DIGITS; ++j) {
        if (before < need && need <= before + n[j]) {
          s_digit = EVICT_BINS - 1 - DIGITS * tid - j;
          s_before = before;
        }
        before += n[j];
      }
      __syncthreads();
      prefix |= s_digit << shift;
      need -= s_before;   // of those with this key so far
    }
  }
  // in slot order; `need` of the slots whose key is `prefix`
  unsigned base = 0, base_ties = 0;   // what stays for sure, and slots with the key, before this chunk
  for (int c0 = 0; c0 < length; c0 += chunk) {
    fetch(c0);
    unsigned above = 0, tie = 0;   // bits
#pragma unroll
    for (int e = 0; e < EVICT_EACH; ++e) {
      const int t = c0 + tid * each + e;
      const bool middle = t >= lo && t < hi, there = e < each && t < length;
      if (there && (!middle || (some && key[e] > prefix))) above |= 1u << e;
      if (there && some && middle && key[e] == prefix) tie |= 1u << e;
    }
    unsigned total;
    const unsigned before = evict_scan<WAVES>(__popc(above) | __popc(tie) << 16, s_wave, total);   // (8192 at most of each)
    unsigned ties = base_ties + (before >> 16), place = base + (before & 0xffffu) + min(ties, need);
#pragma unroll
    for (int e = 0; e < EVICT_EACH; ++e) {
      const bool is_tie = (tie >> e) & 1;
      if (((above >> e) & 1) || (is_tie && ties < need)) {
        kept[place] = c0 + tid * each + e;
        w_out[place] = x[e];   // (place is at most the slot, and all threads have read theirs)
        ++place;
      }
      ties += is_tie;
    }
    base += total & 0xffffu;
    base_ties += total >> 16;
  }
  for (int t = left + tid; t < a.keep; t += THREADS) kept[t] = -1;
  __syncthreads();
  for (int t = left + tid; t < length; t += THREADS) w_out[t] = 0.f;
}

// The move.  A vector is PIECES of 16 bytes; a workgroup takes of one sequence and head the keys or values, COLS pieces of each, and
// goes through its share of the kept slots in rounds, MOVE_BATCH entries a thread on their way at a time (67 MB moved: 33 us one by
// one, 27 in fours).  In place one workgroup has all of them: a round's entries are all read before any is
// written, and it writes no slot past those that it has read, so nothing is lost.
constexpr int MOVE_BATCH = 4;

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
  for (int i0 = blockIdx.y * MOVE_BATCH * entries; i0 < left; i0 += gridDim.y * MOVE_BATCH * entries) {
    int t[MOVE_BATCH], from[MOVE_BATCH], to[MOVE_BATCH];
    move_u32x4 v[MOVE_BATCH];
#pragma unroll
    for (int j = 0; j < MOVE_BATCH; ++j) t[j] = cut(kept[min(i0 + j * entries + (int)threadIdx.x / COLS, left - 1)], 0, length - 1);
#pragma unroll
    for (int j = 0; j < MOVE_BATCH; ++j) {
      from[j] = in[t[j] / pt];
      to[j] = out[min(i0 + j * entries + (int)threadIdx.x / COLS, left - 1) / pt];
    }
#pragma unroll
    for (int j = 0; j < MOVE_BATCH; ++j) {
      const bool there = (unsigned)from[j] < (unsigned)a.cache.n_pages;
      const move_u32x4 x = ((const move_u32x4 *)(a.cache.plane<T>(there ? from[j] : 0, which, head) + t[j] % pt * HD))[piece];
      v[j] = there ? x : move_u32x4{0, 0, 0, 0};
    }
    if (in_place) {
      wait_memory_ops();
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < MOVE_BATCH; ++j) {
      const int i = i0 + j * entries + (int)threadIdx.x / COLS;
      if (i < left && (unsigned)to[j] < (unsigned)a.cache.n_pages && !(in_place && t[j] == i))
        ((move_u32x4 *)(a.cache.plane<T>(to[j], which, head) + i % pt * HD))[piece] = v[j];
    }
  }
}

}  // namespace spark
