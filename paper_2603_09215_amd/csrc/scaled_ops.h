// Launches of the operators on 8-bit rows (scaled_ops.hip), for the C ABI and for the layers of a context.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "scaled_format.h"

namespace spark {

hipError_t launch_scaled_rows(const void *x, int dtype, long long stride, int m, int k, uint8_t *codes, uint8_t *powers, hipStream_t stream);
hipError_t launch_scaled_norm(const NormArgs &a, int h_dtype, int y_dtype, hipStream_t stream);
// n rows of w to every `step`-th row block from `first` on of packed weights of `blocks` row blocks; when all are there,
// launch_scaled_tops adds the rows' largest powers
hipError_t launch_scaled_pack(const void *w, int dtype, long long stride, int n, int k, void *packed, long long blocks, int step, int first, hipStream_t stream);
hipError_t launch_scaled_tops(void *packed, long long blocks, int k, hipStream_t stream);

// a product's operands: 8-bit rows and packed weights
struct ScaledProduct {
  const uint8_t *codes, *powers;   // of the rows
  const uint8_t *weights;
  int m, n, k;
};
size_t scaled_workspace_bytes(int m, int n, int k, int pair, int n_cu);
hipError_t launch_scaled_matmul(const ScaledProduct &p, void *out, int out_dtype, long long out_stride, void *workspace, int n_cu, hipStream_t stream);
// h[rows[r].x_slot] += y[r], fp32; y of y_dtype; k a multiple of four
hipError_t launch_scaled_add(float *h, const RowDesc *rows, const void *y, int y_dtype, int m, int k, hipStream_t stream);
hipError_t launch_scaled_gated(const ScaledProduct &p, uint8_t *codes, uint8_t *powers, void *workspace, int n_cu, hipStream_t stream);

}  // namespace spark
