// The kernels that make 8-bit rows (scaled_format.h): of plain rows, behind the residual's addition and the norm, of weights.
#pragma once
#include "scaled_format.h"

namespace spark {

// ------------------------------------------------------------------ eight values, a sixteenth of a block, per thread

// The fp32 number that rounds like d to anything of 22 bits and fewer.  d rounded to the nearest fp32 does, but where that
// lies on the middle between two such numbers, which d itself may lie beside (one value in 2^20 would be rounded to the wrong
// code): all those middles, and the borders between two powers, end in 13 zeros at least (19 where fp32 has 24 bits).  There
// d is cut toward zero and the last bit set if something was cut off.
__device__ __forceinline__ float for_rounding(double d) {
  const float f = (float)d;
  uint32_t u = __float_as_uint(f);
  if ((u & 0x1fffu) == 0u) {
    const double back = (double)f;
    if (fabs(back) > fabs(d)) u -= 1u;          // (an infinity becomes the largest finite number: too large for any code either way)
    if (back != d && d == d) u |= 1u;
  }
  return __uint_as_float(u);
}
// v + w to the nearest bf16, half to even, as fp32 numbers; v from bf16, w from Y.  The fp32 sum lies on the same side of every
// middle as v + w itself unless it is one.  With w from bf16 it then is v + w: of 8 bits each, they do not fit into 24 only where
// one is under 2^-16 of the other, which is a bf16 number and no middle near it.  With w from fp32 a sum that was rounded (the
// other way round it does not lead back) is worked out in 64 bits.
template <typename Y> __device__ __forceinline__ void add_bf16(float (&v)[8], const float (&w)[8]) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = v[i] + w[i];
  if constexpr (sizeof(Y) == 4) {
    bool unsure = false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      unsure |= ((__float_as_uint(s[i]) & 0xffffu) == 0x8000u) & ((s[i] - v[i] != w[i]) | (s[i] - w[i] != v[i]));   // (no short cuts: a branch each)
    if (__any(unsure)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double d = (double)v[i] + (double)w[i];
        uint32_t u = __float_as_uint(s[i]);
        if ((u & 0xffffu) == 0x8000u && (double)s[i] != d) u += fabs(d) > fabs((double)s[i]) ? 1u : ~0u;   // off the middle, to d's side
        s[i] = __uint_as_float(u);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t r = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{s[i], s[i + 1]}, b2));
    v[i] = __uint_as_float(r << 16);
    v[i + 1] = __uint_as_float(r & 0xffff0000u);
  }
}

// the byte of a block whose largest magnitude has these bits
__device__ __forceinline__ uint32_t power_byte(uint32_t top) {
  const int b = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return top == 0u ? 127u : (uint32_t)max(b, 1);
}
__device__ __forceinline__ float power_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// eight numbers of magnitude 448 at most as codes, to the nearest, half to even
__device__ __forceinline__ uint2 eight_codes(const float (&s)[8]) {
  uint32_t lo = 0u, hi = 0u;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(s[4], s[5], hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(s[6], s[7], hi, true);
  return make_uint2(lo, hi);
}

// the largest of sixteen neighbouring lanes, in all of them
__device__ __forceinline__ uint32_t max_of_16(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, false));    // the other of two
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, false));    // the other two of four
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // mirrored in eight
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, false));   // and in sixteen
}

// The 16 lanes of a block (neighbours) bring eight values each; returns their codes, `byte` the block's.
__device__ __forceinline__ uint2 block_codes(const float (&v)[8], uint32_t &byte) {
  constexpr uint32_t INF = 0x7f800000u;
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max_of_16(top);
  float s[8];
  if (top >= INF) {   // some are no numbers (the same for the sixteen lanes): they are NaN, and have no part in the power
    top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = __float_as_uint(v[i]) & 0x7fffffffu;
      top = max(top, u < INF ? u : 0u);
    }
    top = max_of_16(top);
    byte = power_byte(top);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = (__float_as_uint(v[i]) & 0x7fffffffu) < INF ? v[i] * power_inverse(byte) : __uint_as_float(0x7fc00000u);
  } else {
    byte = power_byte(top);
    const float inv = power_inverse(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = v[i] * inv;
  }
  return eight_codes(s);
}

// Elements c0 .. c0+7 of a row of k, zeros behind its end; asked for, and settled once they are there.  VEC: rows are 16-byte
// aligned and k is a multiple of eight.  Otherwise eight are fetched from wherever they lie (the hardware's vector loads need
// no alignment), at a row's end the last eight of it, which are then moved into place: no branch stands between the loads.
// (4099 rows of 2500 bf16 values: element by element 66 us, only the last ones so 29, this 22.5, now 19.6.)
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) AnyEight { T v[8]; };
template <typename T> struct Eight { uint4 r[sizeof(T) / 2]; };   // as they lie in memory
template <typename T, bool VEC>
__device__ __forceinline__ Eight<T> ask_eight(const T *row, long long c0, int k) {
  Eight<T> e{};
  if constexpr (VEC) {
    if (c0 < k) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) e.r[i] = ((const uint4 *)(row + c0))[i];
    }
  } else if (k >= 8) {
    __builtin_memcpy(e.r, (const AnyEight<T> *)(row + min(c0, k - 8LL)), sizeof(e.r));
  } else if (k > 0) {
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = row[min(i, k - 1)];
    __builtin_memcpy(e.r, v, sizeof(e.r));
  }
  return e;
}
template <typename T, bool VEC>
__device__ __forceinline__ void settle_eight(const Eight<T> &e, long long c0, int k, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    Elem<T>::unpack(e.r[0], v);
  } else {
    Elem<T>::unpack(e.r[0], *(float (*)[4]) & v[0]);
    Elem<T>::unpack(e.r[1], *(float (*)[4]) & v[4]);
  }
  if (!VEC && __any(c0 + 8 > k)) {
    const int left = (int)max(min(k - c0, 8LL), 0LL), off = k >= 8 ? 8 - left : 0;   // of the eight, the last `left` (the first, in a row of fewer)
#pragma unroll
    for (int by = 4; by > 0; by >>= 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = off & by ? (i + by < 8 ? v[i + by] : 0.f) : v[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? v[i] : 0.f;
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void load_eight(const T *row, long long c0, int k, float (&v)[8]) {
  settle_eight<T, VEC>(ask_eight<T, VEC>(row, c0, k), c0, k, v);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_eight(T *row, long long c0, int k, const float (&v)[8]) {   // v: values of T
  uint32_t r[2 * sizeof(T)];
#pragma unroll
  for (int i = 0; i < 2 * (int)sizeof(T); ++i)
    r[i] = sizeof(T) == 2 ? (__float_as_uint(v[2 * i & 7]) >> 16) | (__float_as_uint(v[2 * i + 1 & 7]) & 0xffff0000u) : __float_as_uint(v[i & 7]);
  if (VEC ? c0 < k : c0 + 8 <= k) {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4 *)(row + c0))[i] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
    } else {
      __builtin_memcpy((AnyEight<T> *)(row + c0), r, sizeof(r));
    }
  } else if constexpr (!VEC) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i < k) row[c0 + i] = sizeof(T) == 2 ? (T)(__float_as_uint(v[i]) >> 16) : (T)v[i];
  }
}

// ------------------------------------------------------------------ rows

// 1 / sqrt(x) in 64 bits, x >= 0 or NaN; 0 and infinity give infinity and 0.  The hardware's estimate (2^-23 and better) and two steps of
// Newton's: the root and two divisions by the library are 60 instructions of every wave, an eighth of the norm's.
__device__ __forceinline__ double inverse_root(double x) {
  const double r = __builtin_amdgcn_rsq(x);
  double y = r;
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-x * y, y, 1.0), y);
  return x > 0.0 && x < __builtin_inf() ? y : r;
}

// x [m][k] -> 8-bit rows.  Sixteen lanes a block, U blocks at a time; blocks of all rows in one sequence (2^27 at most).
// Bound by memory: 8191 x 4096 bf16 in 22.2 us, 4.5 TB/s (a copy: 5.2); 32 x 3584 fp32 in 2.4 us, a launch's own time.
template <typename T, bool VEC, int U>
__global__ void __launch_bounds__(256)
scaled_rows_k(const T *__restrict__ x, long long stride, unsigned total, int k, uint8_t *__restrict__ codes, uint8_t *__restrict__ powers) {
  const unsigned pitch = sr_pitch(k), blocks = sr_blocks(k), sub = threadIdx.x & 15;
  const unsigned apart = gridDim.x * 16, first = (blockIdx.x * 256 + threadIdx.x) >> 4;
  float v[U][8];
  unsigned row[U], block[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const unsigned b = first + u * apart;
    row[u] = b / pitch;
    block[u] = b - row[u] * pitch;
    load_eight<T, VEC>(x + (long long)row[u] * stride, (long long)block[u] * SR_BLOCK + sub * 8, b < total ? k : 0, v[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (first + u * apart >= total) break;   // (the same for the sixteen lanes)
    uint8_t *power = powers + (long long)row[u] * pitch + block[u];
    if (block[u] >= blocks) {
      if (sub == 0) *power = 127;
      continue;
    }
    uint32_t byte;
    const uint2 c = block_codes(v[u], byte);
    *(uint2 *)(codes + ((long long)row[u] * blocks + block[u]) * SR_BLOCK + sub * 8) = c;
    if (sub == 0) *power = (uint8_t)byte;
  }
}

// ------------------------------------------------------------------ the residual's addition and the norm

// h' = h + y (rounded to h's type; y absent: h' = h), v = h' / sqrt(mean h'^2 + eps) * gain -> 8-bit rows.
// In 64 bits from the sum of squares to the code: that is what makes every code the one that the formula gives, whatever
// the order of the sum; where fp32 settles the code (below) it stands in.  4096 x 4096 bf16 takes 25 us (4.7 TB/s; instructions
// and memory about level), fp32 with y in bf16 37 us (5.0 TB/s); with both in fp32 1023 x 4096 14 us, 2048 x 18944 112 us
// (4.5 TB/s), one row 3.0 us.
// One workgroup a row, of MOST threads at most; a thread has S times eight values in registers.  S == 0: a row of any length,
// read a second time for the codes (from L2: 2048 x 18944 in 112 us; four times eight a thread, 640 threads: 121).  Workgroups that
// stay and fetch their next row ahead take as long (4096 x 4096 bf16 31 us, 1023 rows 15), and so do rows dealt to the XCDs in runs.
template <typename T, typename Y, bool HAS_Y, bool VEC, int MOST, int S>
__global__ void __launch_bounds__(MOST) scaled_norm_k(NormArgs a) {
  __shared__ double sums[MOST / 64];
  const int NT = blockDim.x;
  const int k = a.k, pitch = sr_pitch(k), blocks = sr_blocks(k);
  const long long kp = (long long)blocks * SR_BLOCK;
  const long long r = blockIdx.x, slot = a.rows ? a.rows[r].x_slot : r;
  const T *h = (const T *)a.h + slot * a.h_stride;
  const Y *y = (const Y *)a.y + r * a.y_stride;
  T *out = (T *)a.h_out + slot * a.out_stride;
  auto take = [&](long long c0, float (&v)[8], float *g) {
    const Eight<T> h8 = ask_eight<T, VEC>(h, c0, k);
    Eight<Y> y8;
    if constexpr (HAS_Y) y8 = ask_eight<Y, VEC>(y, c0, k);
    if constexpr (S > 0) load_eight<float, VEC>(a.gain, c0, k, *(float (*)[8])g);
    settle_eight<T, VEC>(h8, c0, k, v);
    if constexpr (HAS_Y) {
      float w[8];
      settle_eight<Y, VEC>(y8, c0, k, w);
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w[i];   // (one rounding, whatever y's type)
      } else {
        add_bf16<Y>(v, w);
      }
    }
  };
  constexpr int KEEP = S > 0 ? S : 1;
  float v[KEEP][8], gain[KEEP][8];
  double ss = 0.0;
  if constexpr (S > 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const long long c0 = ((long long)s * NT + threadIdx.x) * 8;
      take(c0, v[s], gain[s]);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += (double)v[s][i] * (double)v[s][i];
    }
    if (HAS_Y || out != h) {
#pragma unroll
      for (int s = 0; s < S; ++s) store_eight<T, VEC>(out, ((long long)s * NT + threadIdx.x) * 8, k, v[s]);
    }
  } else {
    for (long long c0 = threadIdx.x * 8; c0 < kp; c0 += NT * 8) {
      take(c0, v[0], nullptr);
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
  for (int w = 0; w < NT / 64; ++w) ss += sums[w];
  const double inv = inverse_root(ss * a.one_over_k + a.eps);
  // The product in fp32, three roundings, is at most 3 units of its last place off: enough to tell which code is nearest
  // unless it lies within 8 of a middle between two (whose last 19 bits are zeros), or may leave fp32's range: it does not with the
  // root's inverse in [2^-30, 2^60], gains in [2^-20, 2^40] or zero, and sums of 2^-60 and more or zero (one too large is flagged as a
  // middle).  Otherwise, for one wave of 60, the products are taken in 64 bits.  (All of them in 64 bits: a pass of 4096 x 4096 bf16 took 35 us, bound by instructions.)
  const float inv32 = (float)inv;
  const bool odd = !(inv32 >= 0x1p-30f && inv32 <= 0x1p60f);
  auto give = [&](long long c0, const float (&vv)[8], const float (&g)[8]) {
    float n[8];
    uint32_t middle = ~0u, small = ~0u, low = ~0u, high = 0u;   // (smallest and largest of the eight; zeros, less one, are in none)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      n[i] = vv[i] * (inv32 * g[i]);
      const uint32_t u = __float_as_uint(n[i]), less = (__float_as_uint(vv[i]) & 0x7fffffffu) - 1u, size = __float_as_uint(g[i]) & 0x7fffffffu;
      middle = min(middle, ((u + 8u) & 0x7ffffu) | (less & 0x80000000u));
      small = min(small, less);
      low = min(low, size - 1u);
      high = max(high, size);
    }
    const bool unsure = odd | (middle < 16u) | (small < 0x217fffffu) | (low < 0x357fffffu) | (high > 0x53800000u);
    uint32_t lift = 0u;   // of the block's power
    if (__any(unsure)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) n[i] = for_rounding((double)vv[i] * inv * (double)g[i]);
      // (a norm is at most sqrt(k) times its gain, and k 2^22)
      if (__builtin_expect(__any(high >= 0x79800000u), 0)) {   // blocks that pass fp32's range: 2^-64 of them, of the format's largest number at most
        double d[8];
        bool far = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          d[i] = (double)vv[i] * inv * (double)g[i];
          far |= fabs(d[i]) >= 0x1p127 && fabs(d[i]) < __builtin_inf();
        }
        lift = max_of_16(far) ? 64u : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (lift) n[i] = for_rounding((fabs(d[i]) < __builtin_inf() ? fmin(fmax(d[i], -0x1.cp135), 0x1.cp135) : d[i]) * 0x1p-64);
      }
      if (__builtin_expect(odd, 0)) {   // a root that is no number: zeros behind the row's end all the same
#pragma unroll
        for (int i = 0; i < 8; ++i) n[i] = c0 + i < k ? n[i] : 0.f;
      }
    }
    uint32_t byte;
    const uint2 c = block_codes(n, byte);   // (a block's sixteen lanes are all inside the padded row, or none)
    if (c0 < kp) {
      *(uint2 *)(a.codes + r * kp + c0) = c;
      if ((threadIdx.x & 15) == 0) a.powers[r * pitch + c0 / SR_BLOCK] = (uint8_t)(byte + lift);
    }
  };
  if constexpr (S > 0) {
#pragma unroll
    for (int s = 0; s < S; ++s) give(((long long)s * NT + threadIdx.x) * 8, v[s], gain[s]);
  } else {
    for (long long c0 = threadIdx.x * 8; c0 < kp; c0 += NT * 8) {   // (what this thread has written itself)
      load_eight<T, VEC>(out, c0, k, v[0]);
      load_eight<float, VEC>(a.gain, c0, k, gain[0]);
      give(c0, v[0], gain[0]);
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
  any = max_of_16(any);
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
