// The operators on a paged cache: launches and C ABI (include/spark.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "../../include/spark.h"
#include "cached_append.h"
#include "cached_attend.h"
#include "cached_evict.h"
#include "cached_weigh.h"

namespace spark {
namespace {

bool aligned(const void *p, size_t a) { return p && ((uintptr_t)p & (a - 1)) == 0; }
size_t type_bytes(int dtype) { return dtype == SPARK_DTYPE_BF16 ? 2 : 4; }
bool dtype_ok(int32_t d) { return d == SPARK_DTYPE_FP32 || d == SPARK_DTYPE_BF16; }
bool within(int64_t v, int64_t lo, int64_t hi) { return v >= lo && v <= hi; }

// sizes alone
bool sizes_ok(const spark_cache *c, const spark_cache_batch *b) {
  return c && b && c->size == sizeof(spark_cache) && b->size == sizeof(spark_cache_batch) && dtype_ok(c->dtype) && within(c->n_pages, 1, 1 << 24) &&
         within(c->n_layers, 1, 1 << 16) && within(c->n_kv_heads, 1, 1 << 12) && within(c->page_tokens, 16, 1 << 16) && c->page_tokens % 16 == 0 &&
         (c->head_dim == 64 || c->head_dim == 128) && within(c->layer, 0, c->n_layers - 1) && within(b->m, 0, 1 << 22) && within(b->n, 0, 1 << 16) &&
         (int64_t)b->n * c->n_kv_heads <= 1 << 20 &&
         within(b->max_pages, 1, 1 << 24) && (int64_t)b->max_pages * c->page_tokens <= 1 << 23;
}
bool heads_ok(const spark_cache *c, const spark_cache_batch *b, int32_t n_q_heads) {
  return within(n_q_heads, 1, 1 << 12) && n_q_heads % c->n_kv_heads == 0 && (int64_t)b->m * n_q_heads <= 1 << 26;
}
bool batch_ok(const spark_cache *c, const spark_cache_batch *b) {
  return sizes_ok(c, b) && aligned(c->pool, 16) && aligned(b->starts, 4) && aligned(b->lengths, 4) && aligned(b->table, 4);
}
bool scale_ok(float scale) { return scale != 0.f && std::fabs(scale) <= 0x1p127f; }   // (times log2 e it is a number still)
// rows of `heads` vectors
bool rows_ok(const void *p, size_t align, int64_t stride, int64_t heads, const spark_cache *c) {
  return aligned(p, align) && within(stride, heads * c->head_dim, (int64_t)1 << 40);
}

CacheView view(const spark_cache *c) {
  const long long layer = 2ll * c->n_kv_heads * c->page_tokens * c->head_dim;
  const uint32_t sixteens = c->page_tokens / 16;
  return CacheView{(char *)c->pool + c->layer * layer * type_bytes(c->dtype), layer * c->n_layers, c->n_pages, c->n_kv_heads, c->page_tokens, c->head_dim,
                   (int)sixteens, sixteens == 1 ? 0u : (uint32_t)(((1ull << 32) + sixteens - 1) / sixteens)};
}
BatchView view(const spark_cache_batch *b) { return BatchView{b->starts, b->lengths, b->table, b->m, b->n, b->max_pages}; }
int status() { return hipGetLastError() == hipSuccess ? SPARK_OK : SPARK_EHIP; }

// calls f(T{}, std::integral_constant<int, HD>{})
template <typename F> void by_cache(int dtype, int head_dim, F f) {
  using H64 = std::integral_constant<int, 64>;
  using H128 = std::integral_constant<int, 128>;
  if (dtype == SPARK_DTYPE_FP32) head_dim == 64 ? f(float{}, H64{}) : f(float{}, H128{});
  else head_dim == 64 ? f(bf16_t{}, H64{}) : f(bf16_t{}, H128{});
}

AttendPlan plan_of(const spark_cache *c, const spark_cache_batch *b, int32_t n_q_heads, int n_cu) {
  return attend_plan(c->dtype == SPARK_DTYPE_FP32, c->head_dim, c->n_kv_heads, n_q_heads / c->n_kv_heads, b->m, b->n, (long long)b->max_pages * c->page_tokens, n_cu);
}
size_t attend_workspace(const spark_cache *c, const spark_cache_batch *b, int32_t n_q_heads, const AttendPlan &p) {
  return p.splits == 1 ? 0 : (size_t)p.splits * b->m * n_q_heads * (c->head_dim + 2) * sizeof(float);
}

// compute units of the current device; looked up once per device
int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// more LDS than 64 KiB has to be asked for, once a kernel and device
template <auto KERN> bool allow_lds(size_t bytes) {
  static std::atomic<uint64_t> asked{0};
  if (bytes <= 60 << 10) return true;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return false;
  if (dev < 64 && (asked.load(std::memory_order_relaxed) >> dev & 1)) return true;
  if (hipFuncSetAttribute((const void *)KERN, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) return false;
  if (dev < 64) asked.fetch_or(1ull << dev, std::memory_order_relaxed);
  return true;
}

}  // namespace
}  // namespace spark

using namespace spark;

extern "C" {

int spark_cache_append(const spark_cache *cache, const spark_cache_batch *batch, const spark_rotation *rotation, int32_t n_q_heads, int32_t src_dtype,
                       const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
                       int64_t out_stride, void *hip_stream) {
  if (!batch_ok(cache, batch) || !heads_ok(cache, batch, n_q_heads) || !dtype_ok(src_dtype) || !rotation || rotation->size != sizeof(spark_rotation))
    return SPARK_EINVAL;
  const size_t sb = type_bytes(src_dtype), cb = type_bytes(cache->dtype);
  if (!rows_ok(q, sb, q_stride, n_q_heads, cache) || !rows_ok(k, sb, k_stride, cache->n_kv_heads, cache) ||
      !rows_ok(v, sb, v_stride, cache->n_kv_heads, cache) || !rows_ok(q_out, cb, out_stride, n_q_heads, cache) ||
      (q_out == q && (src_dtype != cache->dtype || (out_stride != q_stride && batch->m > 1))))
    return SPARK_EINVAL;
  if (!within(rotation->rotary, 0, cache->head_dim) || rotation->rotary % 2 || !std::isfinite(rotation->amplitude) || !(rotation->eps >= 0.0) ||
      (rotation->rotary > 0 && !aligned(rotation->freqs, 8)) || ((uintptr_t)rotation->positions & 3) || ((uintptr_t)rotation->q_gain & 3) ||
      ((uintptr_t)rotation->k_gain & 3))
    return SPARK_EINVAL;
  if (batch->m == 0 || batch->n == 0) return SPARK_OK;
  AppendArgs a{};
  a.cache = view(cache); a.batch = view(batch);
  a.q = q; a.k = k; a.v = v; a.q_out = q_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride;
  a.n_q_heads = n_q_heads; a.rotary = rotation->rotary; a.interleaved = rotation->interleaved != 0;
  a.amplitude = rotation->amplitude; a.eps = rotation->eps;
  a.freqs = rotation->freqs; a.positions = rotation->positions; a.q_gain = rotation->q_gain; a.k_gain = rotation->k_gain;
  auto vec = [](const void *p, size_t bytes, int64_t stride) { return aligned(p, 4 * bytes) && stride % 4 == 0; };
  const bool wide = a.rotary % 8 == 0 && vec(q, sb, q_stride) && vec(k, sb, k_stride) && vec(v, sb, v_stride) && vec(q_out, cb, out_stride);
  const int heads = n_q_heads + 2 * cache->n_kv_heads;
  // A workgroup's start (its rows' places and angles) takes some 3 us: about a thousand of them where there are rows enough, each with all
  // of its rows' heads, and the heads dealt out where there are few.  (32 + 2 x 2 heads, normed: 8191 rows 44.5 us in eights, 49 in fours, 56
  // in twos; 2000 rows 19 one by one, 14.4 in twos, 15.4 in fours; 512 rows 5.5 with half of the heads a workgroup, 7.1 with 16; one row 3.7 with 16, 4.5 with 40.)
  a.rows = 1;
  while (a.rows < APPEND_ROWS && batch->m / (2 * a.rows) >= 1000) a.rows *= 2;
  a.heads_per_wg = batch->m >= 1000 ? heads : batch->m >= 256 ? std::max(16, (heads + 1) / 2) : 16;
  const dim3 grid((batch->m + a.rows - 1) / a.rows, (heads + a.heads_per_wg - 1) / a.heads_per_wg);
  const size_t lds = sizeof(float) * a.rows * a.rotary;
  by_cache(cache->dtype, cache->head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    auto go = [&](auto kern) { kern<<<grid, 256, lds, (hipStream_t)hip_stream>>>(a); };
    if (src_dtype == SPARK_DTYPE_FP32) wide ? go(cached_append_k<float, T, HD, true>) : go(cached_append_k<float, T, HD, false>);
    else wide ? go(cached_append_k<bf16_t, T, HD, true>) : go(cached_append_k<bf16_t, T, HD, false>);
  });
  return status();
}

int spark_cache_workspace_bytes(const spark_cache *cache, const spark_cache_batch *batch, int32_t n_q_heads, size_t *bytes) {
  if (!sizes_ok(cache, batch) || !heads_ok(cache, batch, n_q_heads) || !bytes) return SPARK_EINVAL;
  *bytes = 0;
  if (batch->m == 0 || batch->n == 0) return SPARK_OK;
  const int n_cu = compute_units();
  if (n_cu <= 0) return SPARK_EHIP;
  *bytes = attend_workspace(cache, batch, n_q_heads, plan_of(cache, batch, n_q_heads, n_cu));
  return SPARK_OK;
}

int spark_cache_attend(const spark_cache *cache, const spark_cache_batch *batch, int32_t n_q_heads, const void *q, int64_t q_stride, float scale,
                       int32_t causal, void *out, int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  if (!batch_ok(cache, batch) || !heads_ok(cache, batch, n_q_heads) || !rows_ok(q, 16, q_stride, n_q_heads, cache) || q_stride % 8 ||
      !rows_ok(out, 16, out_stride, n_q_heads, cache) || out_stride % 8 || ((uintptr_t)lse & 3) || !scale_ok(scale))
    return SPARK_EINVAL;
  if (batch->m == 0 || batch->n == 0) return SPARK_OK;
  const int n_cu = compute_units();
  if (n_cu <= 0) return SPARK_EHIP;
  const AttendPlan plan = plan_of(cache, batch, n_q_heads, n_cu);
  const size_t need = attend_workspace(cache, batch, n_q_heads, plan);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SPARK_ENOMEM;
  if (need > 0 && !aligned(workspace, 16)) return SPARK_EINVAL;
  AttendArgs a{};
  a.cache = view(cache); a.batch = view(batch);
  a.q = q; a.out = out; a.lse = lse; a.q_stride = q_stride; a.out_stride = out_stride;
  a.n_q_heads = n_q_heads; a.group = n_q_heads / cache->n_kv_heads; a.causal = causal != 0;
  a.factor = std::fabs(scale) * 1.44269504088896340736f;
  a.flip = scale < 0.f ? 0x80000000u : 0u;
  a.splits = plan.splits;
  a.by_row = attend_tiles_by_row(plan.pairs, a.group, batch->m, batch->n);
  a.part = (float *)workspace;
  a.part_ml = (float2 *)(a.part + (size_t)plan.splits * batch->m * n_q_heads * cache->head_dim);
  hipStream_t stream = (hipStream_t)hip_stream;
  const unsigned grid = (unsigned)(plan.tiles * cache->n_kv_heads * plan.splits);
  bool ok = true;
  by_cache(cache->dtype, cache->head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    auto go = [&](auto kern, int threads, size_t lds, bool allowed) {
      if ((ok = allowed)) kern<<<grid, threads, lds, stream>>>(a);
    };
    if constexpr (sizeof(T) == 2) {   // (fp32 has no tiles)
      if (plan.pairs == 128) go(cached_tile_k<HD, 4>, 256, Tile<HD, 4>::LDS, allow_lds<cached_tile_k<HD, 4>>(Tile<HD, 4>::LDS));
      if constexpr (HD == 128)
        if (plan.pairs == 256) go(cached_tile_k<HD, 8>, 512, Tile<HD, 8>::LDS, allow_lds<cached_tile_k<HD, 8>>(Tile<HD, 8>::LDS));
    }
    if (plan.pairs == 16) go(cached_stream_k<T, HD>, 256, Stream<T, HD>::LDS, true);
    if (ok && plan.splits > 1) {
      const long long vectors = (long long)batch->m * n_q_heads, each = 256 / (HD / 4);
      if (join_by_workgroups(vectors)) cached_join_k<T, HD, 256 / (HD / 4)><<<(unsigned)vectors, 256, 0, stream>>>(a);
      else cached_join_k<T, HD, 1><<<(unsigned)((vectors + each - 1) / each), 256, 0, stream>>>(a);
    }
  });
  return ok ? status() : SPARK_EHIP;
}

int spark_cache_weigh(const spark_cache *cache, const spark_cache_batch *batch, int32_t n_q_heads, const void *q, int64_t q_stride, float scale,
                      int32_t causal, const float *lse, const float *before, float decay, float *out, void *hip_stream) {
  if (!batch_ok(cache, batch) || !heads_ok(cache, batch, n_q_heads) || (batch->m > 0 && (!rows_ok(q, 16, q_stride, n_q_heads, cache) || q_stride % 8 || !aligned(lse, 4))) ||
      ((uintptr_t)before & 3) || !aligned(out, 4) || !scale_ok(scale) || !std::isfinite(decay))
    return SPARK_EINVAL;
  if (batch->n == 0) return SPARK_OK;
  const int n_cu = compute_units();
  if (n_cu <= 0) return SPARK_EHIP;
  WeighArgs a{};
  a.cache = view(cache); a.batch = view(batch);
  a.q = q; a.lse = lse; a.before = decay != 0.f ? before : nullptr; a.out = out; a.q_stride = q_stride;
  a.n_q_heads = n_q_heads; a.group = n_q_heads / cache->n_kv_heads; a.causal = causal != 0;
  a.factor = std::fabs(scale) * 1.44269504088896340736f;
  a.flip = scale < 0.f ? 0x80000000u : 0u;
  a.decay = decay;
  a.reciprocal = a.group == 1 ? 0u : (uint32_t)(((1ull << 32) + a.group - 1) / a.group);
  // Many pairs from a block for each of eight waves on (32 + 2 heads, bf16, 64 rows over 8191 slots: 13.9 us, a wave by itself 33), and in bf16 from two
  // blocks on where a round of workgroups does it (8 rows 5.0 and 7.4; 2 rows 4.6 and 4.5; of two sequences, so in two rounds, 8.5 and 7.6; of 16 over 4095
  // slots 31 and 22; fp32 8 rows 19 and 18, of two sequences 34 and 19).  Few: workgroups that stay for several pieces, as many as a compute unit
  // has registers for (32 steps of 4095 slots, 28 + 4 heads: three 24.6 us, two 28, four 31; fp32 two 64, three 77).
  const int heads = batch->n * cache->n_kv_heads, pieces = (batch->max_pages * cache->page_tokens + 31) / 32;
  const long long pairs = (long long)batch->m * a.group / batch->n;   // of a sequence and head, on average
  const bool round = cache->dtype == SPARK_DTYPE_BF16 && (long long)heads * ((pieces + 1) / 2) <= n_cu;
  const bool many = pairs >= 256 || (round && pairs > 32);
  bool ok = true;
  by_cache(cache->dtype, cache->head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value;
    auto go = [&](auto kern, int each, int waves, int most, size_t lds = 0) {
      kern<<<dim3(heads, std::min((pieces + each - 1) / each, most)), 64 * waves, lds, (hipStream_t)hip_stream>>>(a);
    };
    if (many) {
      constexpr size_t lds = Weigh<T, true>::lds(HD);
      if ((ok = allow_lds<cached_weigh_k<T, HD, true>>(lds))) go(cached_weigh_k<T, HD, true>, Weigh<T, true>::PIECES, Weigh<T, true>::WAVES, std::max(1, (1 << 16) / heads), lds);
    } else go(cached_weigh_k<T, HD, false>, Weigh<T, false>::PIECES, Weigh<T, false>::WAVES, std::max(1, (sizeof(T) * HD == 512 ? 2 : 3) * n_cu / heads));
  });
  return ok ? status() : SPARK_EHIP;
}

int spark_cache_evict(const spark_cache *cache, const spark_cache_batch *batch, const float *weights, int32_t keep, int32_t first, int32_t recent,
                      const int32_t *table_out, int32_t out_pages, float *weights_out, int32_t *kept, int32_t *lengths_out, void *hip_stream) {
  if (!sizes_ok(cache, batch) || !aligned(cache->pool, 16) || !aligned(batch->lengths, 4) || !aligned(batch->table, 4) || !aligned(weights, 4) ||
      !aligned(weights_out, 4) || !aligned(kept, 4) || !aligned(lengths_out, 4) || ((uintptr_t)table_out & 3) || lengths_out == batch->lengths)
    return SPARK_EINVAL;
  const int64_t slots = (int64_t)batch->max_pages * cache->page_tokens;
  if (first < 0 || recent < 0 || !within(keep, 1, slots) || (int64_t)first + recent > keep ||
      (table_out && (!within(out_pages, 1, 1 << 24) || (int64_t)out_pages * cache->page_tokens < keep)) ||
      (table_out && table_out == batch->table && out_pages != batch->max_pages && batch->n > 1))
    return SPARK_EINVAL;
  if (batch->n == 0) return SPARK_OK;
  EvictArgs a{};
  a.cache = view(cache); a.batch = view(batch);
  a.weights = weights; a.weights_out = weights_out; a.kept = kept; a.lengths_out = lengths_out;
  a.table_out = table_out ? table_out : batch->table;
  a.out_pages = table_out ? out_pages : batch->max_pages;
  a.keep = keep; a.first = first; a.recent = recent;
  const int heads = batch->n * cache->n_kv_heads;
  hipStream_t stream = (hipStream_t)hip_stream;
  // (small workgroups where each thread's slots stay in registers: 8192 heads of up to 250 slots with the move 220 us, large ones 400; 1024 of up to 2000 230 and 248;
  // four of 2000 12 and 12; but four of 4097 25 and 14)
  if (slots <= 256 * EVICT_EACH) cached_choose_k<256><<<heads, 256, 0, stream>>>(a);
  else cached_choose_k<1024><<<heads, 1024, 0, stream>>>(a);
  by_cache(cache->dtype, cache->head_dim, [&](auto t, auto hd) {
    using T = decltype(t);
    constexpr int HD = decltype(hd)::value, PIECES = HD * sizeof(T) / 16;
    if (a.table_out == batch->table) {
      cached_move_k<T, HD, 8><<<heads * 2 * (PIECES / 8), heads > 1 << 18 ? 256 : 1024, 0, stream>>>(a);   // (a launch takes less than 2^32 threads)
    } else {
      const int rounds = (keep * PIECES + 256 * MOVE_BATCH - 1) / (256 * MOVE_BATCH);
      cached_move_k<T, HD, PIECES><<<dim3(heads * 2, std::min(rounds, std::max(1, std::min(256, (1 << 20) / heads)))), 256, 0, stream>>>(a);
    }
  });
  return status();
}

}  // extern "C"
