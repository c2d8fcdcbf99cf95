// A paged cache and the batch of sequences that a call works on, as the kernels see them (include/spark.h, "Operators on a
// paged cache").  What the device tensors hold is cut to its range here, so no value in them leads out of a buffer.
#pragma once
#include "device_common.h"

namespace spark {

struct CacheView {
  void *pool;             // of the layer: its first page's keys of head 0
  long long page_stride;  // elements
  int n_pages, n_kv_heads, page_tokens, head_dim;
  int sixteens;           // page_tokens / 16
  uint32_t reciprocal;    // 2^32 / sixteens rounded up, 0 for one
  // keys (which 0) or values (1) of a head in a page: [page_tokens][head_dim]
  template <typename T> __device__ __forceinline__ T *plane(int page, int which, int head) const {
    return (T *)pool + page * page_stride + (long long)(which * n_kv_heads + head) * page_tokens * head_dim;
  }
};

struct BatchView {
  const int *starts, *lengths, *table;
  int m, n, max_pages;
};

struct Sequence {
  int row0, rows, length;
  const int *pages;
  __device__ __forceinline__ int slot(int row) const { return length - rows + row; }   // negative: none
};

typedef __attribute__((ext_vector_type(2))) __bf16 ca_bf16x2;
typedef __attribute__((ext_vector_type(2))) float ca_f32x2;
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {   // half to even, one instruction
  const ca_f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, ca_bf16x2));
}

// two parts that add up to a and b but for 2^-16 of them: what each is rounded to, and what that leaves
__device__ __forceinline__ void pack_bf16_parts(float a, float b, uint32_t &high, uint32_t &low) {
  high = pack_bf16(a, b);
  low = pack_bf16(a - __uint_as_float(high << 16), b - __uint_as_float(high & 0xffff0000u));
}

__device__ __forceinline__ int cut(int v, int lo, int hi) { return min(max(v, lo), hi); }

__device__ __forceinline__ Sequence sequence(const BatchView &b, int s, int page_tokens) {
  Sequence q;
  q.row0 = cut(b.starts[s], 0, b.m);
  q.rows = cut(b.starts[s + 1], q.row0, b.m) - q.row0;
  q.length = cut(b.lengths[s], 0, b.max_pages * page_tokens);
  q.pages = b.table + (long long)s * b.max_pages;
  return q;
}

// Which of a sequence's pages holds its slots 16 n .. 16 n + 15, and from which of the page's tokens on.  n stays below 2^20 (2^19
// sixteens of a sequence, and the few that are asked for ahead) and a page has at most 2^12, so the product with the rounded
// reciprocal, off by less than n / 2^32 of 2^12 parts, is exact when cut.
__device__ __forceinline__ void place_of(const CacheView &c, int n, int &index, int &token) {
  index = c.reciprocal ? (int)__umulhi((uint32_t)n, c.reciprocal) : n;
  token = (n - index * c.sixteens) * 16;
}

// the page of a slot, -1 where there is none
__device__ __forceinline__ int page_of(const Sequence &q, int slot, int page_tokens, int n_pages) {
  const int p = q.pages[slot / page_tokens];
  return (unsigned)p < (unsigned)n_pages ? p : -1;
}

}  // namespace spark
