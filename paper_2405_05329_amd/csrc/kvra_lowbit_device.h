// The 8- and 4-bit formats, for the kernels that read and write them (not installed).
#ifndef KVRA_LOWBIT_DEVICE_H
#define KVRA_LOWBIT_DEVICE_H

#include "kvra_internal.h"

namespace kvra {

// Scales are powers of two, held as their exponent + 127 (e8m0).  A block's is the smallest with which nothing that is finite
// overflows, kept within bounds that leave every value it can stand for a normal bf16 number.
constexpr int kScaleMin = -100, kScaleMax = 120;

// The top 16 bits of 240 * 2^kScaleMax (as of every fp32 number above it): the largest finite value of the cache.  The next code with that
// scale, 256, stands for 2^128, which is infinity in bf16 and would reach even queries that do not see it (a weight of zero times infinity).
constexpr unsigned kCacheMost = 0x7F70;

// The smallest e with amax <= HIGH * 2^e, HIGH = 448 = 0.875 * 2^9 (e4m3) or 6 = 0.75 * 2^3 (e2m1); amax finite, >= 0.
template <int HIGH>
__device__ __forceinline__ int scale_exponent(float amax) {
  static_assert(HIGH == 448 || HIGH == 6, "");
  const unsigned u = __float_as_uint(amax);                  // (a subnormal amax counts as 2^-127: below the bound anyway)
  const int e = static_cast<int>(u >> 23) - (HIGH == 448 ? 127 + 8 : 127 + 2);
  const unsigned mant = u & 0x7FFFFFu, most = HIGH == 448 ? 0x600000u : 0x400000u;   // 448 = 1.75 * 2^8, 6 = 1.5 * 2^2
  return min(max(e + (mant > most ? 1 : 0), kScaleMin), kScaleMax);
}

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }   // |e| <= 126

// The factor a scale byte stands for, as the conversion instructions take it (255, "not a number", makes every value one).
__device__ __forceinline__ float scale_factor(unsigned byte) { return __uint_as_float(byte << 23); }

// 0x80 in every byte of four e4m3 codes that is NaN (0x7F or 0xFF).
__device__ __forceinline__ unsigned nan_bytes(unsigned codes) { return ((codes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

}  // namespace kvra

#endif
