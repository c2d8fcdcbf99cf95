// 8-bit rows: e4m3 codes with a power of two for every 128 values of a row, and weights packed in them: the formats, and
// what the launches of scaled_ops.h take.
//
// A row of k values is kp codes (kp = k rounded up to 128s, zeros behind k) and `pitch` bytes b (one per 128 codes,
// padded to a multiple of four with 127); a code c of a block stands for c * 2^(b - 127).  The power is the smallest for
// which no magnitude of the block passes 448, e4m3's largest: with the block's largest = f 2^x, f in [0.5, 1), and
// 448 = 0.875 * 2^9, it is 2^(x - 9), or the next one where f > 0.875.  A power of two and not any fp32 number, because
// the 8-bit matrix instructions of this chip multiply by it themselves (an exponent byte per lane) and the conversions to
// 16 bits do, so that a product needs little arithmetic besides them; what it costs is nothing in precision (e4m3 keeps 4 significant bits over 2^15 whatever the
// power), and at most one of those 15 binades.  NaN and infinities become e4m3's NaN and have no part in the power.
#pragma once
#include "device_common.h"

namespace spark {

constexpr int SR_BLOCK = 128;   // codes per power of two
constexpr int SR_NONE = -1, SR_FP32 = 0, SR_BF16 = 1;   // (SPARK_DTYPE_*)

__host__ __device__ __forceinline__ int sr_blocks(int k) { return (int)(((long long)k + SR_BLOCK - 1) / SR_BLOCK); }
__host__ __device__ __forceinline__ int sr_pitch(int k) { return (sr_blocks(k) + 3) & ~3; }   // bytes of powers per row

// Packed weights: tiles of 16 rows x 128 k as the matrix instructions take them, [row block][k block][half][lane][16 codes]:
// lane l of half h holds row l mod 16, k = 64 h + 16 (l / 16) .. + 15, so that a wave reads a tile with two contiguous
// instructions.  Behind them the powers, [row block][k block / 4][row][4], of blocks of zeros and behind the last the lowest,
// and behind those each row's largest power, [row block][16].  Rows behind n are zeros.  A pair of matrices (gated)
// alternates its row blocks: even ones of the gate, odd ones of the other.
constexpr int SW_TILE = 2048;
__host__ __device__ __forceinline__ long long sw_row_blocks(int n, int pair) { return (((long long)n + 15) / 16) * (pair ? 2 : 1); }
__host__ __device__ __forceinline__ size_t sw_code_bytes(long long blocks, int k) { return (size_t)blocks * sr_blocks(k) * SW_TILE; }
__host__ __device__ __forceinline__ size_t sw_power_bytes(long long blocks, int k) { return (size_t)blocks * sr_pitch(k) * 16; }
__host__ __device__ __forceinline__ size_t sw_bytes(int n, int k, int pair) {
  const long long blocks = sw_row_blocks(n, pair);
  return sw_code_bytes(blocks, k) + sw_power_bytes(blocks, k) + (size_t)blocks * 16;
}

// Arguments of the residual's addition and norm (scaled_rows.h)
struct NormArgs {
  const void *h, *y;
  void *h_out;
  const float *gain;
  long long h_stride, y_stride, out_stride;
  const RowDesc *rows;   // nullable: row r of h and h_out is rows[r].x_slot
  int m, k;
  double eps, one_over_k;   // (the launch's)
  uint8_t *codes, *powers;
};

}  // namespace spark
