// Rows to 8-bit integers: q = the integer nearest to 127 x / a, a the row's largest magnitude, and the row's scale a / 127.
//
// Bound by memory: a row is read once, held in registers while its largest magnitude is found, and written once (rows that
// do not fit are read again).  A wavefront has a row, a workgroup a long one.
#pragma once

#include "t3_device.h"

namespace t3k {

constexpr int kQuantPieces = 8;        // pieces of 8 elements a lane holds

// 127 x / a to the nearest integer, ties to even, as if the quotient were not rounded before.  In fp32, x times 127 / a is off by less
// than 2^-15 (two roundings of half a step of numbers up to 127); where that could decide, the quotient is taken in fp64, whose rounding cannot: 127 x is exact
// there, and a quotient that is no odd multiple of 1/2 is at least 2^-33 away from all of them (twice 127 x and an odd multiple of a are
// multiples of 2^-7 of a's last place where they are that near).
__device__ __forceinline__ int quantised(float x, float a, float inv, bool tiny) {
  const float f = x * inv;
  float n = __builtin_rintf(f);
  if (tiny || __builtin_fabsf(f - n) > 0.5f - 0x1p-15f) n = (float)__builtin_rint((double)x * 127.0 / (double)a);
  return (int)n;
}

template <int TEAM, bool F32>
__global__ __launch_bounds__(256) void quant_rows_kernel(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int32_t rows,
                                                         int32_t cols) {
  __shared__ uint32_t tops[4];
  const int lane = (int)threadIdx.x % TEAM;
  const int64_t row = (int64_t)blockIdx.x * (256 / TEAM) + threadIdx.x / TEAM;
  if (row >= rows) return;                       // (whole wavefronts; a workgroup of one row stays together)
  const char *from = (const char *)x + row * ldx * (F32 ? 4 : 2);
  const int pieces = cols >> 3;
  float v[kQuantPieces][8];
  auto load = [&](int base) {
#pragma unroll
    for (int u = 0; u < kQuantPieces; ++u) {
      const int at = base + u * TEAM + lane;
      u32x4 lo{0, 0, 0, 0}, hi{0, 0, 0, 0};
      if (at < pieces) {
        if (F32) {
          lo = ((const u32x4 *)from)[2 * at];
          hi = ((const u32x4 *)from)[2 * at + 1];
        } else {
          lo = ((const u32x4 *)from)[at];
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t bits = F32 ? (e < 4 ? lo[e & 3] : hi[e & 3]) : (e & 1 ? lo[e >> 1] & 0xFFFF0000u : lo[e >> 1] << 16);
        v[u][e] = __builtin_bit_cast(float, bits);
      }
    }
  };
  // the largest magnitude by its bits: a NaN's and infinity's are larger than any number's
  uint32_t top = 0;
  constexpr int kHeld = TEAM * kQuantPieces;
  for (int base = 0; base == 0 || base < pieces; base += kHeld) {
    load(base);
#pragma unroll
    for (int u = 0; u < kQuantPieces; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(uint32_t, v[u][e]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  if (TEAM == 256) {
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  }
  const bool finite = top < 0x7F800000u, any = top != 0u && finite;
  const float a = __builtin_bit_cast(float, top), inv = __fdiv_rn(127.0f, a);
  const bool tiny = a < 0x1p-100f;               // (127 / a might be infinite)
  if (lane == 0) scale[row] = finite ? __fdiv_rn(a, 127.0f) : __builtin_nanf("");
  int8_t *to = q + row * ldq;
  for (int base = 0; base == 0 || base < pieces; base += kHeld) {
    if (pieces > kHeld) load(base);
#pragma unroll
    for (int u = 0; u < kQuantPieces; ++u) {
      const int at = base + u * TEAM + lane;
      u32x2 w{0, 0};
      if (any) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)quantised(v[u][e], a, inv, tiny) & 0xFFu) << (8 * (e & 3));
      }
      if (at < pieces) ((u32x2 *)to)[at] = w;
    }
  }
}

}  // namespace t3k
