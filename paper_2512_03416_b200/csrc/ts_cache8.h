// The 8-bit KV cache's number format, shared by the kernels that write it and those that read it.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

namespace ts {

// values: e4m3 codes [page][K, V][KV head][slot][D]; scales: one byte per row of these, E + 127, or 255 for a row with a NaN.
struct Cache8 {
  uint8_t* values;
  uint8_t* scales;
};
constexpr int kCache8MaxExp = 62;      // |E| at most: 2^(E of a row - E of another) then stays a normal fp32 number
// Scale byte of a row of zeros. Other rows have it only if their largest magnitude is in (224, 448], so readers to whom a V row's exponent is its
// size look at the codes of rows with this byte: zeros are smaller than any row.
constexpr uint8_t kCache8ZeroByte = 127;

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
__device__ __forceinline__ uint32_t cache8_magnitudes(const uint4& codes) { return (codes.x | codes.y | codes.z | codes.w) & 0x7f7f7f7fu; }
// 2^E, or NaN
__device__ __forceinline__ float cache8_power(uint8_t byte) { return byte == 255 ? __int_as_float(0x7fc00000) : __int_as_float((cache8_exp_of(byte) + 127) << 23); }
// Four e4m3 codes as f16 pairs (0, 2) and (1, 3), times 2^-8: a code shifted to the sign and to bits 13..7 is the f16 number 2^-8 times
// its value, subnormal ones too (the formats differ in the bias alone).
// Seven integer instructions; with two conversion instructions instead 37 rows of 8192 keys, one token each, took 163 us, not 145.
__device__ __forceinline__ void cache8_widen(uint32_t w, uint32_t& even, uint32_t& odd) {
  even = ((w << 7) & 0x3f803f80u) | ((w << 8) & 0x80008000u);
  odd = ((w >> 1) & 0x3f803f80u) | (w & 0x80008000u);
}
// Four bf16 (a, b: two each), times `by`, as two e4m3 addends: hi + lo. Exact where lo is a normal code or hi alone will do.
__device__ __forceinline__ void cache8_split(uint32_t a, uint32_t b, float by, uint32_t& hi, uint32_t& lo) {
  const uint32_t x[2] = {a, b};
  uint32_t h[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 f = make_float2(__uint_as_float(x[i] << 16) * by, __uint_as_float(x[i] & 0xffff0000u) * by);
    h[i] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)h[i], __NV_E4M3);
    const float2 g = __half22float2(__half2(r));
    l[i] = __nv_cvt_float2_to_fp8x2(make_float2(f.x - g.x, f.y - g.y), __NV_SATFINITE, __NV_E4M3);
  }
  hi = h[0] | h[1] << 16;
  lo = l[0] | l[1] << 16;
}
#endif

}  // namespace ts
