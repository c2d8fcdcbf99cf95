// The kernels that make 8-bit rows (scaled_format.h): of plain rows, behind the residual's addition and the norm, of weights.
#pragma once
#include "scaled_format.h"

namespace spark {

// ------------------------------------------------------------------ eight values, a sixteenth of a block, per thread

// The fp32 number that rounds like d to anything of 22 bits and fewer: cut toward zero, the last bit set if something was
// cut off.  (Rounded to the nearest fp32 first, one value in 2^20 would fall on the middle between two codes and then be
// rounded to the wrong one.)
__device__ __forceinline__ float cut_odd(double d) {
  const float f = (float)d;
  uint32_t u = __float_as_uint(f);
  const double back = (double)f;
  if (fabs(back) > fabs(d)) u -= 1u;          // (an infinity becomes the largest finite number: too large for any code either way)
  if (back != d && d == d) u |= 1u;
  return __uint_as_float(u);
}

__device__ __forceinline__ uint32_t finite_magnitude(float f) {
  const uint32_t u = __float_as_uint(f) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}

// the byte of a block whose largest magnitude has these bits
__device__ __forceinline__ uint32_t power_byte(uint32_t top) {
  const int b = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return top == 0u ? 127u : (uint32_t)max(b, 1);
}
__device__ __forceinline__ float power_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// eight values times `inv` as codes (to the nearest, half to even; |v * inv| <= 448 where v is finite)
__device__ __forceinline__ uint2 eight_codes(const float (&v)[8], float inv) {
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = fabsf(v[i]) < INFINITY ? v[i] * inv : __uint_as_float(0x7fc00000u);
  uint32_t lo = 0u, hi = 0u;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(s[4], s[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(s[6], s[7], hi, true);
  return make_uint2(lo, hi);
}

// The 16 lanes of a block (neighbours) bring eight values each; returns their codes, `byte` the block's.
__device__ __forceinline__ uint2 block_codes(const float (&v)[8], uint32_t &byte) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[i]));
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  byte = power_byte(top);
  return eight_codes(v, power_inverse(byte));
}

// elements c0 .. c0+7 of a row of k; VEC: rows are 16-byte aligned and k is a multiple of eight
template <typename T, bool VEC>
__device__ __forceinline__ void load_eight(const T *row, long long c0, int k, float (&v)[8]) {
  if constexpr (VEC) {
    if (c0 < k) {
      if constexpr (sizeof(T) == 2) {
        Elem<T>::unpack(*(const uint4 *)(row + c0), v);
      } else {
        Elem<T>::unpack(*(const uint4 *)(row + c0), *(float (*)[4]) & v[0]);
        Elem<T>::unpack(*(const uint4 *)(row + c0 + 4), *(float (*)[4]) & v[4]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c0 + i < k ? Elem<T>::widen(row[c0 + i]) : 0.f;
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_eight(T *row, long long c0, int k, const float (&v)[8]) {   // v: values of T
  if constexpr (VEC) {
    if (c0 >= k) return;
    if constexpr (sizeof(T) == 2) {
      uint4 r;
      r.x = (__float_as_uint(v[0]) >> 16) | (__float_as_uint(v[1]) & 0xffff0000u);
      r.y = (__float_as_uint(v[2]) >> 16) | (__float_as_uint(v[3]) & 0xffff0000u);
      r.z = (__float_as_uint(v[4]) >> 16) | (__float_as_uint(v[5]) & 0xffff0000u);
      r.w = (__float_as_uint(v[6]) >> 16) | (__float_as_uint(v[7]) & 0xffff0000u);
      *(uint4 *)(row + c0) = r;
    } else {
      *(float4 *)(row + c0) = make_float4(v[0], v[1], v[2], v[3]);
      *(float4 *)(row + c0 + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i < k) row[c0 + i] = sizeof(T) == 2 ? (T)(__float_as_uint(v[i]) >> 16) : (T)v[i];
  }
}

// ------------------------------------------------------------------ rows

// x [m][k] -> 8-bit rows.  Sixteen lanes a block, blocks of all rows in one sequence.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
scaled_rows_k(const T *__restrict__ x, long long stride, int m, int k, uint8_t *__restrict__ codes, uint8_t *__restrict__ powers) {
  const int pitch = sr_pitch(k), blocks = sr_blocks(k), sub = threadIdx.x & 15;
  const long long total = (long long)m * pitch;
  for (long long b = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4; b < total; b += (long long)gridDim.x * 16) {
    const long long r = b / pitch;
    const int kb = (int)(b - r * pitch);
    if (kb >= blocks) {   // (the same for the sixteen lanes)
      if (sub == 0) powers[r * pitch + kb] = 127;
      continue;
    }
    float v[8];
    load_eight<T, VEC>(x + r * stride, (long long)kb * SR_BLOCK + sub * 8, k, v);
    uint32_t byte;
    const uint2 c = block_codes(v, byte);
    *(uint2 *)(codes + (r * blocks + kb) * SR_BLOCK + sub * 8) = c;
    if (sub == 0) powers[r * pitch + kb] = (uint8_t)byte;
  }
}

// ------------------------------------------------------------------ the residual's addition and the norm

// h' = h + y (rounded to h's type; y absent: h' = h), v = h' / sqrt(mean h'^2 + eps) * gain -> 8-bit rows.
// In 64 bits from the sum of squares to the code: that is what makes every code the one that the formula gives, whatever
// the order of the sum, and a memory-bound kernel has the time for it.
// One workgroup of NT threads a row; a thread has S times eight values in registers.  S == 0: a row of any length, read a
// second time for the codes.
template <typename T, typename Y, bool HAS_Y, bool VEC, int NT, int S>
__global__ void __launch_bounds__(NT) scaled_norm_k(NormArgs a) {
  __shared__ double sums[NT / 64];
  const int k = a.k, pitch = sr_pitch(k), blocks = sr_blocks(k);
  const long long kp = (long long)blocks * SR_BLOCK;
  const long long r = blockIdx.x, slot = a.rows ? a.rows[r].x_slot : r;
  const T *h = (const T *)a.h + slot * a.h_stride;
  const Y *y = (const Y *)a.y + r * a.y_stride;
  T *out = (T *)a.h_out + slot * a.out_stride;
  auto take = [&](long long c0, float (&v)[8]) {
    load_eight<T, VEC>(h, c0, k, v);
    if constexpr (HAS_Y) {
      float w[8];
      load_eight<Y, VEC>(y, c0, k, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = v[i] + w[i];   // (one rounding, whatever y's type)
        else v[i] = bf16_to_f32(f32_to_bf16(cut_odd((double)v[i] + (double)w[i])));
      }
    }
  };
  constexpr int KEEP = S > 0 ? S : 1;
  float v[KEEP][8];
  double ss = 0.0;
  if constexpr (S > 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const long long c0 = ((long long)s * NT + threadIdx.x) * 8;
      take(c0, v[s]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += (double)v[s][i] * (double)v[s][i];
    }
    if (HAS_Y || out != h) {
#pragma unroll
      for (int s = 0; s < S; ++s) store_eight<T, VEC>(out, ((long long)s * NT + threadIdx.x) * 8, k, v[s]);
    }
  } else {
    for (long long c0 = threadIdx.x * 8; c0 < kp; c0 += NT * 8) {
      take(c0, v[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += (double)v[0][i] * (double)v[0][i];
      if (HAS_Y || out != h) store_eight<T, VEC>(out, c0, k, v[0]);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) ss += sums[w];
  const double inv = 1.0 / sqrt(ss / (double)k + a.eps);
  auto give = [&](long long c0, const float (&vv)[8]) {
    float g[8], n[8];
    load_eight<float, VEC>(a.gain, c0, k, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] = cut_odd((double)vv[i] * inv * (double)g[i]);
    uint32_t byte;
    const uint2 c = block_codes(n, byte);   // (a block's sixteen lanes are all inside the padded row, or none)
    if (c0 < kp) {
      *(uint2 *)(a.codes + r * kp + c0) = c;
      if ((threadIdx.x & 15) == 0) a.powers[r * pitch + c0 / SR_BLOCK] = (uint8_t)byte;
    }
  };
  if constexpr (S > 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) give(((long long)s * NT + threadIdx.x) * 8, v[s]);
  } else {
    for (long long c0 = threadIdx.x * 8; c0 < kp; c0 += NT * 8) {   // (what this thread has written itself)
      load_eight<T, VEC>(out, c0, k, v[0]);
      give(c0, v[0]);
    }
  }
  if (threadIdx.x < pitch - blocks) a.powers[r * pitch + blocks + threadIdx.x] = 127;
}

// h[row] += y[row] where no norm follows (behind the last layer of a run); four values a thread
template <typename Y>
__global__ void __launch_bounds__(256) scaled_add_k(float *__restrict__ h, const RowDesc *__restrict__ rows, const Y *__restrict__ y, int m, int k) {
  const int fours = k / 4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)m * fours; i += (long long)gridDim.x * 256) {
    const int r = (int)(i / fours), c = (int)(i - (long long)r * fours) * 4;
    float4 *at = (float4 *)(h + (long long)rows[r].x_slot * k + c);
    const Y *v = y + (long long)r * k + c;
    float4 s = *at;
    s.x += Elem<Y>::widen(v[0]); s.y += Elem<Y>::widen(v[1]); s.z += Elem<Y>::widen(v[2]); s.w += Elem<Y>::widen(v[3]);
    *at = s;
  }
}

// ------------------------------------------------------------------ weights

// grid: (k blocks padded to pitch, row blocks); sixteen lanes quantise a row's block
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
scaled_pack_k(const T *__restrict__ w, long long stride, int n, int k, uint8_t *__restrict__ codes, uint8_t *__restrict__ powers,
              int step, int first, int row0) {
  const int kb = blockIdx.x, blocks = sr_blocks(k), row = threadIdx.x >> 4, sub = threadIdx.x & 15;
  const long long group = blockIdx.y + row0, block = group * step + first;   // of the rows, of the packed matrix
  uint8_t *at = powers + ((block * (sr_pitch(k) / 4) + kb / 4) * 16 + row) * 4 + kb % 4;
  if (kb >= blocks) {
    if (sub == 0) *at = 1;
    return;
  }
  float v[8];
  const long long r = group * 16 + row;
  if (r < n) {
    load_eight<T, VEC>(w + r * stride, (long long)kb * SR_BLOCK + sub * 8, k, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
  uint32_t byte;
  const uint2 c = block_codes(v, byte);
  uint32_t any = (c.x | c.y) & 0x7f7f7f7fu;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) any |= (uint32_t)__shfl_xor((int)any, o, 64);
  // k = 8 sub: half sub / 8, lane group (sub mod 8) / 2, codes 8 (sub mod 2) .. of the lane's sixteen
  *(uint2 *)(codes + (block * blocks + kb) * SW_TILE + (sub >> 3) * 1024 + (((sub & 7) >> 1) * 16 + row) * 16 + (sub & 1) * 8) = c;
  if (sub == 0) *at = any ? (uint8_t)byte : 1;
}

// each row's largest power: a thread a row
__global__ void __launch_bounds__(256)
scaled_tops_k(const uint8_t *__restrict__ powers, long long rows, int groups, uint8_t *__restrict__ tops) {
  const long long r = (long long)blockIdx.x * 256 + threadIdx.x;
  if (r >= rows) return;
  const uint32_t *p = (const uint32_t *)powers + (r >> 4) * groups * 16 + (r & 15);
  uint32_t top = 0u;
  for (int g = 0; g < groups; ++g) {
    const uint32_t v = p[(long long)g * 16];
    top = max(max(max(v & 255u, v >> 8 & 255u), max(v >> 16 & 255u, v >> 24)), top);
  }
  tops[r] = (uint8_t)top;
}

}  // namespace spark
