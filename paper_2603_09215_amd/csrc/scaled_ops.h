// Launches of the operators on 8-bit rows (scaled_ops.hip), for the C ABI and for the layers of a context.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "scaled_rows.h"

namespace spark {

hipError_t launch_scaled_rows(const void *x, int dtype, long long stride, int m, int k, uint8_t *codes, uint8_t *powers, hipStream_t stream);
hipError_t launch_scaled_norm(const NormArgs &a, int h_dtype, int y_dtype, hipStream_t stream);
hipError_t launch_scaled_pack(const void *w, int dtype, long long stride, int n, int k, void *packed, int pair_rows, int first, hipStream_t stream);

// a product's operands: 8-bit rows and packed weights
struct ScaledProduct {
  const uint8_t *codes, *powers;   // of the rows
  const uint8_t *weights;
  int m, n, k;
};
size_t scaled_workspace_bytes(int m, int n, int k, int pair, int n_cu);
hipError_t launch_scaled_matmul(const ScaledProduct &p, void *out, int out_dtype, long long out_stride, void *workspace, int n_cu, hipStream_t stream);
hipError_t launch_scaled_gated(const ScaledProduct &p, uint8_t *codes, uint8_t *powers, void *workspace, int n_cu, hipStream_t stream);

}  // namespace spark
