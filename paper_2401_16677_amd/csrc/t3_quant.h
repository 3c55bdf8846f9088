// Rows to 8-bit integers: q = the integer nearest to 127 x / a, a the row's largest magnitude, and the row's scale a / 127.
//
// Bound by memory: a row is read once, held in registers while its largest magnitude is found, and written once (rows that
// do not fit are read again).  A wavefront has a row, a workgroup a long one.  From memory: bfloat16 4096 x 6144 16 to 18 us, 4.2 to 4.7 TB/s, the rate of a copy, float32
// 25 us, 5.0; 4096 x 12288 31 and 48 us, 4.9 and 5.3; bfloat16 37 x 6144 4 us and 1 x 1536 2.4 us, a launch and two round trips.
#pragma once

#include "t3_device.h"

namespace t3k {

constexpr int kQuantPieces = 8;        // pieces of 8 elements a lane holds at most

// 127 x / a to the nearest integer, ties to even, as if the quotient were not rounded before: eight of them, in the bytes of two words.
// by_a = 1 / a, rounded.  127 x is a number p, of fp32 x with a rest; f = p by_a + (what p by_a misses, an exact remainder) by_a is the quotient with one
// rounding but for 2^-46 of it, so it is on the quotient's side of every k + 1/2, or at k + 1/2 itself; 1.5 2^23 + f has the integer nearest to f in
// its low bits.  Where f is k + 1/2 the remainder's sign decides.  (That is one number in 10^5, and behind a branch.)
template <bool F32>
__device__ __forceinline__ u32x2 quantised(const float (&x)[8], float a, float by_a) {
  constexpr float kWhole = 12582912.0f;
  float m[8], f[8], off = 0.0f;
  auto remainder = [&](int e, float f) {
    const float p = 127.0f * x[e], r = __builtin_fmaf(-f, a, p);
    return F32 ? r + __builtin_fmaf(127.0f, x[e], -p) : r;
  };
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float f0 = 127.0f * x[e] * by_a;
    f[e] = __builtin_fmaf(remainder(e, f0), by_a, f0);
    m[e] = f[e] + kWhole;
    off = fmaxf(off, __builtin_fabsf(f[e] - (m[e] - kWhole)));
  }
  if (off == 0.5f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = f[e] - (m[e] - kWhole);
      if (__builtin_fabsf(d) == 0.5f && remainder(e, f[e]) * d > 0.0f) m[e] += 2.0f * d;
    }
  }
  auto four = [&](int e) {                       // low bytes together
    auto b = [&](int i) { return __builtin_bit_cast(uint32_t, m[e + i]); };
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b(3), b(2), 0x0c0c0400u), __builtin_amdgcn_perm(b(1), b(0), 0x0c0c0400u), 0x05040100u);
  };
  return u32x2{four(0), four(4)};
}

// PIECES: of 8 elements that a lane holds at a time.
template <int TEAM, int PIECES, bool F32>
__global__ __launch_bounds__(256) void quant_rows_kernel(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int32_t rows,
                                                         int32_t cols) {
  __shared__ uint32_t tops[4];
  const int lane = (int)threadIdx.x % TEAM;
  const int64_t row = (int64_t)blockIdx.x * (256 / TEAM) + threadIdx.x / TEAM;
  if (row >= rows) return;                       // (whole wavefronts; a workgroup of one row stays together)
  const char *from = (const char *)x + row * ldx * (F32 ? 4 : 2);
  const int pieces = cols >> 3;
  float v[PIECES][8];
  auto load = [&](int base) {
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
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
  constexpr int kHeld = TEAM * PIECES;
  for (int base = 0; base == 0 || base < pieces; base += kHeld) {
    load(base);
#pragma unroll
    for (int u = 0; u < PIECES; ++u)
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
  const float largest = __builtin_bit_cast(float, top);
  if (lane == 0) scale[row] = finite ? __fdiv_rn(largest, 127.0f) : __builtin_nanf("");
  // (rows whose 1 / a or 127 x might not be a float, or whose remainders might be too small for one, are taken at another power of two, which
  // changes no quotient; elements that would fall below the smallest float are nowhere near 1/2)
  const float by = largest < 0x1p-40f ? 0x1p100f : (largest > 0x1p100f ? 0x1p-20f : 1.0f), a = largest * by, by_a = __fdiv_rn(1.0f, a);
  int8_t *to = q + row * ldq;
  for (int base = 0; base == 0 || base < pieces; base += kHeld) {
    if (pieces > kHeld) load(base);
    if (by != 1.0f) {
#pragma unroll
      for (int u = 0; u < PIECES; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] *= by;
    }
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
      const int at = base + u * TEAM + lane;
      if (at < pieces) ((u32x2 *)to)[at] = any ? quantised<F32>(v[u], a, by_a) : u32x2{0, 0};
    }
  }
}

}  // namespace t3k
