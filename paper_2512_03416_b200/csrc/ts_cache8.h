// The 8-bit KV cache's number format, shared by the kernels that write it and those that read it.
#pragma once
#include <stdint.h>

namespace ts {

// values: e4m3 codes [page][K, V][KV head][slot][D]; scales: one byte per row of these, E + 127, or 255 for a row with a NaN.
struct Cache8 {
  uint8_t* values;
  uint8_t* scales;
};
constexpr int kCache8MaxExp = 62;      // |E| at most: 2^(E of a row - E of another) then stays a normal fp32 number

#ifdef __CUDACC__
// Smallest E with m <= 448 * 2^E, for m > 0 the magnitude whose bf16 bits are `bits` (infinity counts as the largest):
// 448 = 1.75 * 2^8, and m = f * 2^e with f = 1 + (bits & 127) / 128.
__device__ __forceinline__ int cache8_exponent(uint32_t bits) {
  if (bits == 0) return 0;
  const int e = (int)(bits >> 7) - 127, above = (bits & 0x7f) > 0x60;      // a subnormal m has e = -127 here: below the clamp
  return min(max(e - 8 + above, -kCache8MaxExp), kCache8MaxExp);
}
// E of a scale byte (not of 255). A byte that no row was written with is taken to the nearest that one could have been.
__device__ __forceinline__ int cache8_exp_of(uint8_t byte) { return min(max((int)byte - 127, -kCache8MaxExp), kCache8MaxExp); }
// 2^E, or NaN
__device__ __forceinline__ float cache8_power(uint8_t byte) { return byte == 255 ? __int_as_float(0x7fc00000) : __int_as_float((cache8_exp_of(byte) + 127) << 23); }
#endif

}  // namespace ts
