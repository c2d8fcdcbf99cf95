// The operators on 8-bit rows: launches and C ABI (include/spark.h).
#include "scaled_ops.h"

#include <algorithm>
#include <atomic>

#include "../../include/spark.h"
#include "scaled_gemm.h"
#include "scaled_plan.h"

namespace spark {
namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
size_t type_bytes(int dtype) { return dtype == SR_BF16 ? 2 : 4; }
bool rows_vector(const void *p, int dtype, long long stride, int k) {
  return k % 8 == 0 && aligned16(p) && stride * (long long)type_bytes(dtype) % 16 == 0;
}

template <typename T, typename Y, bool HAS_Y, bool VEC>
void norm_shape(const NormArgs &a, hipStream_t stream) {
  const int eights = sr_blocks(a.k) * 16;   // threads' worth of a row
  auto threads = [&](int s) { return (eights + 64 * s - 1) / (64 * s) * 64; };
  if (eights <= 512) scaled_norm_k<T, Y, HAS_Y, VEC, 512, 1><<<a.m, threads(1), 0, stream>>>(a);
  else if (eights <= 2048) scaled_norm_k<T, Y, HAS_Y, VEC, 1024, 2><<<a.m, threads(2), 0, stream>>>(a);
  else scaled_norm_k<T, Y, HAS_Y, VEC, 1024, 0><<<a.m, 1024, 0, stream>>>(a);
}
template <typename T, typename Y, bool HAS_Y> void norm_vec(const NormArgs &a, bool vec, hipStream_t stream) {
  if (vec) norm_shape<T, Y, HAS_Y, true>(a, stream);
  else norm_shape<T, Y, HAS_Y, false>(a, stream);
}
template <typename T> void norm_y(const NormArgs &a, int y_dtype, bool vec, hipStream_t stream) {
  if (y_dtype == SR_NONE) norm_vec<T, float, false>(a, vec, stream);
  else if (y_dtype == SR_FP32) norm_vec<T, float, true>(a, vec, stream);
  else norm_vec<T, bf16_t, true>(a, vec, stream);
}

GemmArgs gemm_args(const ScaledProduct &p, int pair) {
  GemmArgs a{};
  a.codes = p.codes; a.powers = p.powers;
  a.weights = p.weights;
  a.row_blocks = (int)sw_row_blocks(p.n, pair);
  a.weight_powers = a.weights + sw_code_bytes(a.row_blocks, p.k);
  a.weight_tops = a.weight_powers + sw_power_bytes(a.row_blocks, p.k);
  a.m = p.m; a.n = p.n; a.k = p.k;
  return a;
}

constexpr int STREAM_ROWS = 16;
constexpr size_t STREAM_LDS = 64 << 10;   // two workgroups a CU

template <typename OUT> void stream_launch(const GemmArgs &a, hipStream_t stream) {
  const int groups = sr_pitch(a.k) / 4, turns = (groups + 15) / 16, kw = (groups + turns - 1) / turns, nw = std::max(1, 4 / kw);
  const unsigned grid = (unsigned)((a.row_blocks + nw - 1) / nw);
  const size_t rows = (size_t)a.m * (sr_blocks(a.k) * SR_BLOCK + 16 + sr_pitch(a.k)), sums = sizeof(f32x4) * 64 * nw * kw;
  if (rows <= STREAM_LDS) scaled_stream_k<true, OUT><<<grid, 64 * nw * kw, std::max(rows, sums), stream>>>(a, nw, kw);
  else scaled_stream_k<false, OUT><<<grid, 64 * nw * kw, sums, stream>>>(a, nw, kw);
}

constexpr int TILES_MOST = 1 << 20;   // of a launch
size_t lds_of(int tm, bool fp32, bool gated) {
  return std::max((size_t)(fp32 ? 4 : 2) * tm * SW_TILE + 4 * 512 * sizeof(uint32_t), gated ? sizeof(float) * 16 * tm * (SR_BLOCK + 4) : 0);
}

template <bool FP32, TileEnd END, typename OUT> void tile_launch(GemmArgs a, const TilePlan &p, hipStream_t stream) {
  const TileShape &t = TILE_SHAPES[p.shape];
  const int nt = (a.row_blocks + t.nt * TILE_WAVES - 1) / (t.nt * TILE_WAVES);
  if constexpr (END != TILE_PARTS) {   // (a launch's threads are counted in 32 bits; where k is cut there are 512 workgroups at most)
    const int most = std::max(1, TILES_MOST / nt) * 16 * t.mt;
    if (a.m > most) {
      GemmArgs b = a;
      for (int r = 0; r < a.m; r += b.m) {   // (b.m <= a.m - r)
        b.m = std::min(most, a.m - r);
        tile_launch<FP32, END, OUT>(b, p, stream);
        b.codes += (long long)b.m * sr_blocks(a.k) * SR_BLOCK;
        b.powers += (long long)b.m * sr_pitch(a.k);
        if constexpr (END == TILE_GATED) {
          b.out = (uint8_t *)b.out + (long long)b.m * sr_blocks(a.n) * SR_BLOCK;
          b.out_powers += (long long)b.m * sr_pitch(a.n);
        } else {
          b.out = (OUT *)b.out + b.m * a.out_stride;
        }
      }
      return;
    }
  }
  const int mt = (a.m - 1) / (16 * t.mt) + 1;
  const unsigned grid = (unsigned)nt * mt * p.splits;
  const size_t lds = lds_of(t.mt, FP32, END == TILE_GATED);
  auto go = [&](auto kern) { kern<<<grid, 64 * TILE_WAVES, lds, stream>>>(a, nt, mt, p.splits); };
  if constexpr (END != TILE_GATED) {
    if (p.shape == 0) return go(scaled_tile_k<1, 2, FP32, END, OUT>);
    if (p.shape == 1) return go(scaled_tile_k<1, 4, FP32, END, OUT>);
  }
  if constexpr (END == TILE_GATED || (END == TILE_PARTS && FP32)) {
    if (p.shape == 2) return go(scaled_tile_k<2, 1, FP32, END, OUT>);
  }
  if (p.shape == 3) go(scaled_tile_k<2, 2, FP32, END, OUT>);
  else if (p.shape == 4) go(scaled_tile_k<2, 4, FP32, END, OUT>);
  else go(scaled_tile_k<2, 8, FP32, END, OUT>);
}

template <typename OUT> void matmul_launch(GemmArgs a, void *workspace, int n_cu, hipStream_t stream) {
  if (a.m <= STREAM_ROWS) return stream_launch<OUT>(a, stream);
  constexpr bool FP32 = sizeof(OUT) == 4;
  const TilePlan p = tile_plan(a.m, a.row_blocks, a.k, false, FP32, n_cu);
  if (p.splits == 1) return tile_launch<FP32, TILE_OUT, OUT>(a, p, stream);
  GemmArgs b = a;
  b.out = workspace;
  b.out_stride = (long long)a.row_blocks * 16;
  tile_launch<FP32, TILE_PARTS, float>(b, p, stream);
  const long long fours = (long long)a.m * ((a.n + 3) / 4);
  scaled_join_k<OUT><<<(unsigned)std::min<long long>((fours + 255) / 256, 1 << 16), 256, 0, stream>>>((const float *)workspace, p.splits, a.m, a.n,
                                                                                                    a.row_blocks * 16, (OUT *)a.out, a.out_stride);
}

}  // namespace

namespace {
template <typename T, bool VEC> void rows_launch(const T *x, long long stride, int m, int k, uint8_t *codes, uint8_t *powers, hipStream_t stream) {
  const unsigned pitch = sr_pitch(k);
  const long long most = (1ll << 27) / pitch;   // rows of a launch, whose threads, sixteen a block, are counted in 32 bits
  for (long long r0 = 0; r0 < m; r0 += most) {
    const unsigned total = (unsigned)std::min(m - r0, most) * pitch, groups = (total + 15) / 16;
    const T *xr = x + r0 * stride;
    uint8_t *cr = codes + r0 * sr_blocks(k) * SR_BLOCK, *pr = powers + r0 * pitch;
    // (two blocks at a time once that leaves eight workgroups a CU)
    if (groups < 4096) scaled_rows_k<T, VEC, 1><<<groups, 256, 0, stream>>>(xr, stride, total, k, cr, pr);
    else scaled_rows_k<T, VEC, 2><<<(groups + 1) / 2, 256, 0, stream>>>(xr, stride, total, k, cr, pr);
  }
}
}  // namespace

hipError_t launch_scaled_rows(const void *x, int dtype, long long stride, int m, int k, uint8_t *codes, uint8_t *powers, hipStream_t stream) {
  const bool vec = rows_vector(x, dtype, stride, k);
  if (dtype == SR_FP32) {
    if (vec) rows_launch<float, true>((const float *)x, stride, m, k, codes, powers, stream);
    else rows_launch<float, false>((const float *)x, stride, m, k, codes, powers, stream);
  } else {
    if (vec) rows_launch<bf16_t, true>((const bf16_t *)x, stride, m, k, codes, powers, stream);
    else rows_launch<bf16_t, false>((const bf16_t *)x, stride, m, k, codes, powers, stream);
  }
  return hipGetLastError();
}

hipError_t launch_scaled_norm(const NormArgs &a, int h_dtype, int y_dtype, hipStream_t stream) {
  const bool vec = rows_vector(a.h, h_dtype, a.h_stride, a.k) && rows_vector(a.h_out, h_dtype, a.out_stride, a.k) && aligned16(a.gain) &&
                   (y_dtype == SR_NONE || rows_vector(a.y, y_dtype, a.y_stride, a.k));
  constexpr int MOST_ROWS = 1 << 20;   // of a launch, whose threads are counted in 32 bits
  NormArgs b = a;
  b.one_over_k = 1.0 / a.k;
  while (b.m > 0) {
    const int left = b.m - MOST_ROWS;
    b.m = std::min(b.m, MOST_ROWS);
    if (h_dtype == SR_FP32) norm_y<float>(b, y_dtype, vec, stream);
    else norm_y<bf16_t>(b, y_dtype, vec, stream);
    const size_t hb = type_bytes(h_dtype), done = (size_t)b.m;
    if (b.rows) {
      b.rows += done;
    } else {
      b.h = (const char *)b.h + done * b.h_stride * hb;
      b.h_out = (char *)b.h_out + done * b.out_stride * hb;
    }
    if (b.y) b.y = (const char *)b.y + done * b.y_stride * type_bytes(y_dtype);
    b.codes += done * sr_blocks(b.k) * SR_BLOCK;
    b.powers += done * sr_pitch(b.k);
    b.m = left;
  }
  return hipGetLastError();
}

hipError_t launch_scaled_pack(const void *w, int dtype, long long stride, int n, int k, void *packed, long long blocks, int step, int first, hipStream_t stream) {
  const bool vec = rows_vector(w, dtype, stride, k);
  uint8_t *codes = (uint8_t *)packed, *powers = codes + sw_code_bytes(blocks, k);
  const long long groups = sw_row_blocks(n, 0);
  for (long long r0 = 0; r0 < groups; r0 += 32768) {   // (a grid's second side ends at 65535)
    const dim3 grid(sr_pitch(k), (unsigned)std::min<long long>(groups - r0, 32768));
    if (dtype == SR_FP32) {
      if (vec) scaled_pack_k<float, true><<<grid, 256, 0, stream>>>((const float *)w, stride, n, k, codes, powers, step, first, (int)r0);
      else scaled_pack_k<float, false><<<grid, 256, 0, stream>>>((const float *)w, stride, n, k, codes, powers, step, first, (int)r0);
    } else {
      if (vec) scaled_pack_k<bf16_t, true><<<grid, 256, 0, stream>>>((const bf16_t *)w, stride, n, k, codes, powers, step, first, (int)r0);
      else scaled_pack_k<bf16_t, false><<<grid, 256, 0, stream>>>((const bf16_t *)w, stride, n, k, codes, powers, step, first, (int)r0);
    }
  }
  return hipGetLastError();
}

hipError_t launch_scaled_tops(void *packed, long long blocks, int k, hipStream_t stream) {
  uint8_t *powers = (uint8_t *)packed + sw_code_bytes(blocks, k);
  scaled_tops_k<<<(unsigned)((blocks * 16 + 255) / 256), 256, 0, stream>>>(powers, blocks * 16, sr_pitch(k) / 4, powers + sw_power_bytes(blocks, k));
  return hipGetLastError();
}

hipError_t launch_scaled_add(float *h, const RowDesc *rows, const void *y, int y_dtype, int m, int k, hipStream_t stream) {
  const unsigned grid = (unsigned)std::min<long long>(((long long)m * (k / 4) + 255) / 256, 4096);
  if (y_dtype == SR_FP32) scaled_add_k<float><<<grid, 256, 0, stream>>>(h, rows, (const float *)y, m, k);
  else scaled_add_k<bf16_t><<<grid, 256, 0, stream>>>(h, rows, (const bf16_t *)y, m, k);
  return hipGetLastError();
}

size_t scaled_workspace_bytes(int m, int n, int k, int pair, int n_cu) {
  if (m == 0 || (m <= STREAM_ROWS && !pair)) return 0;
  const int row_blocks = (int)sw_row_blocks(n, pair);
  int splits = 1;
  for (int fp32 = pair; fp32 < 2; ++fp32) {   // (outputs of either type)
    const int s = tile_plan(m, row_blocks, k, pair, fp32, n_cu).splits;
    splits = std::max(splits, s);
  }
  return splits == 1 ? 0 : sizeof(float) * splits * m * row_blocks * 16;
}

hipError_t launch_scaled_matmul(const ScaledProduct &p, void *out, int out_dtype, long long out_stride, void *workspace, int n_cu, hipStream_t stream) {
  GemmArgs a = gemm_args(p, 0);
  a.out = out;
  a.out_stride = out_stride;
  if (out_dtype == SR_FP32) matmul_launch<float>(a, workspace, n_cu, stream);
  else matmul_launch<bf16_t>(a, workspace, n_cu, stream);
  return hipGetLastError();
}

hipError_t launch_scaled_gated(const ScaledProduct &p, uint8_t *codes, uint8_t *powers, void *workspace, int n_cu, hipStream_t stream) {
  GemmArgs a = gemm_args(p, 1);
  a.out = codes;
  a.out_powers = powers;
  const TilePlan plan = tile_plan(a.m, a.row_blocks, a.k, true, true, n_cu);
  if (plan.splits == 1) {
    tile_launch<true, TILE_GATED, float>(a, plan, stream);
    return hipGetLastError();
  }
  GemmArgs sums = a;
  sums.out = workspace;
  sums.out_stride = (long long)a.row_blocks * 16;
  tile_launch<true, TILE_PARTS, float>(sums, plan, stream);
  const long long groups = (long long)a.m * sr_pitch(a.n);
  scaled_join_gated_k<<<(unsigned)std::min<long long>((groups + 15) / 16, 1 << 16), 256, 0, stream>>>((const float *)workspace, plan.splits, a.m, a.n,
                                                                                                    a.row_blocks * 16, codes, powers);
  return hipGetLastError();
}

}  // namespace spark

// ------------------------------------------------------------------ C ABI

namespace {

using namespace spark;

constexpr int32_t MOST = 1 << 22;   // of n and k: offsets inside a tile stay in 32 bits

bool dtype_ok(int32_t d) { return d == SPARK_DTYPE_FP32 || d == SPARK_DTYPE_BF16; }
bool aligned(const void *p, size_t a) { return p && ((uintptr_t)p & (a - 1)) == 0; }
bool matrix_ok(const void *p, int32_t dtype, int64_t stride, int32_t k) {
  return dtype_ok(dtype) && aligned(p, type_bytes(dtype)) && stride >= k && stride <= (int64_t)1 << 40;
}
bool size_ok(int32_t v) { return v >= 1 && v <= MOST; }
int status(hipError_t e) { return e == hipSuccess ? SPARK_OK : SPARK_EHIP; }

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

int product_ok(const void *codes, const void *powers, int32_t m, const void *packed, int32_t n, int32_t k, int pair, const void *workspace,
               size_t workspace_bytes, int &n_cu) {
  if (!aligned(codes, 16) || !aligned(powers, 4) || !aligned(packed, 16) || m < 0 || !size_ok(n) || !size_ok(k)) return SPARK_EINVAL;
  if ((n_cu = compute_units()) <= 0) return SPARK_EHIP;
  const size_t need = scaled_workspace_bytes(m, n, k, pair, n_cu);
  if (need > 0 && (!workspace || workspace_bytes < need)) return SPARK_ENOMEM;
  return need > 0 && !aligned(workspace, 16) ? SPARK_EINVAL : SPARK_OK;
}

}  // namespace

extern "C" {

int spark_scaled_rows(const void *x, int32_t dtype, int64_t stride, int32_t m, int32_t k, void *codes, void *powers, void *hip_stream) {
  if (m < 0 || !size_ok(k) || !matrix_ok(x, dtype, stride, k) || !aligned(codes, 16) || !aligned(powers, 4)) return SPARK_EINVAL;
  if (m == 0) return SPARK_OK;
  return status(launch_scaled_rows(x, dtype, stride, m, k, (uint8_t *)codes, (uint8_t *)powers, (hipStream_t)hip_stream));
}

int spark_scaled_norm(const void *h, int32_t h_dtype, int64_t h_stride, const void *y, int32_t y_dtype, int64_t y_stride, void *h_out,
                      int64_t out_stride, const float *gain, double eps, int32_t m, int32_t k, void *codes, void *powers, void *hip_stream) {
  if (m < 0 || !size_ok(k) || !matrix_ok(h, h_dtype, h_stride, k) || !matrix_ok(h_out, h_dtype, out_stride, k) || !aligned(gain, 4) ||
      (y && !matrix_ok(y, y_dtype, y_stride, k)) || !(eps >= 0.0) || (h_out == h && out_stride != h_stride && m > 1) || !aligned(codes, 16) ||
      !aligned(powers, 4))
    return SPARK_EINVAL;
  if (m == 0) return SPARK_OK;
  NormArgs a{};
  a.h = h; a.y = y; a.h_out = h_out; a.gain = gain;
  a.h_stride = h_stride; a.y_stride = y_stride; a.out_stride = out_stride;
  a.m = m; a.k = k; a.eps = eps;
  a.codes = (uint8_t *)codes; a.powers = (uint8_t *)powers;
  return status(launch_scaled_norm(a, h_dtype, y ? y_dtype : SR_NONE, (hipStream_t)hip_stream));
}

int spark_scaled_weight_bytes(int32_t n, int32_t k, int32_t pair, size_t *bytes) {
  if (!size_ok(n) || !size_ok(k) || !bytes) return SPARK_EINVAL;
  *bytes = sw_bytes(n, k, pair != 0);
  return SPARK_OK;
}

int spark_scaled_pack(const void *w, const void *up, int32_t dtype, int64_t stride, int32_t n, int32_t k, void *packed, size_t packed_bytes,
                      void *hip_stream) {
  if (!size_ok(n) || !size_ok(k) || !matrix_ok(w, dtype, stride, k) || (up && !matrix_ok(up, dtype, stride, k)) || !aligned(packed, 16))
    return SPARK_EINVAL;
  if (packed_bytes < sw_bytes(n, k, up != nullptr)) return SPARK_ENOMEM;
  const long long blocks = sw_row_blocks(n, up != nullptr);
  hipError_t e = launch_scaled_pack(w, dtype, stride, n, k, packed, blocks, up ? 2 : 1, 0, (hipStream_t)hip_stream);
  if (e == hipSuccess && up) e = launch_scaled_pack(up, dtype, stride, n, k, packed, blocks, 2, 1, (hipStream_t)hip_stream);
  if (e == hipSuccess) e = launch_scaled_tops(packed, blocks, k, (hipStream_t)hip_stream);
  return status(e);
}

int spark_scaled_workspace_bytes(int32_t m, int32_t n, int32_t k, int32_t pair, size_t *bytes) {
  if (m < 0 || !size_ok(n) || !size_ok(k) || !bytes) return SPARK_EINVAL;
  const int n_cu = compute_units();
  if (n_cu <= 0) return SPARK_EHIP;
  *bytes = scaled_workspace_bytes(m, n, k, pair != 0, n_cu);
  return SPARK_OK;
}

int spark_scaled_matmul(const void *codes, const void *powers, int32_t m, const void *packed, int32_t n, int32_t k, void *out,
                        int32_t out_dtype, int64_t out_stride, void *workspace, size_t workspace_bytes, void *hip_stream) {
  int n_cu = 0;
  if (!matrix_ok(out, out_dtype, out_stride, n)) return SPARK_EINVAL;
  if (int rc = product_ok(codes, powers, m, packed, n, k, 0, workspace, workspace_bytes, n_cu)) return rc;
  if (m == 0) return SPARK_OK;
  const ScaledProduct p{(const uint8_t *)codes, (const uint8_t *)powers, (const uint8_t *)packed, m, n, k};
  return status(launch_scaled_matmul(p, out, out_dtype, out_stride, workspace, n_cu, (hipStream_t)hip_stream));
}

int spark_scaled_gated(const void *codes, const void *powers, int32_t m, const void *packed, int32_t n, int32_t k, void *out_codes,
                       void *out_powers, void *workspace, size_t workspace_bytes, void *hip_stream) {
  int n_cu = 0;
  if (!aligned(out_codes, 16) || !aligned(out_powers, 4)) return SPARK_EINVAL;
  if (int rc = product_ok(codes, powers, m, packed, n, k, 1, workspace, workspace_bytes, n_cu)) return rc;
  if (m == 0) return SPARK_OK;
  const ScaledProduct p{(const uint8_t *)codes, (const uint8_t *)powers, (const uint8_t *)packed, m, n, k};
  return status(launch_scaled_gated(p, (uint8_t *)out_codes, (uint8_t *)out_powers, workspace, n_cu, (hipStream_t)hip_stream));
}

}  // extern "C"
