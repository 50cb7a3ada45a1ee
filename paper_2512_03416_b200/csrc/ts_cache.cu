// The KV cache written and read back (sm_100a): bf16 pages, or the 8-bit cache.
//
// 8-bit cache: the D elements of a (token, KV head, K or V) row are e4m3 codes of x * 2^-E, where E is the smallest
// whole number with max|x| <= 448 * 2^E (0 for a row of zeros, clamped to [-62, 62]). A row with a NaN is one of NaN: its scale says so. A power of two costs no precision: e4m3
// has the same four significant bits in every binade, so it loses nothing against a scale of max|x| / 448, the codes are the
// bf16 value rounded once, and code * 2^E is exact in bf16. It is one byte per row (E + 127) instead of four.
//
// Both directions are bound by memory: 4 D Hkv bytes of a token in bf16, 2 (D + 1) Hkv in 8 bits. One warp per token at a time:
// a lane moves 16 bytes of bf16 (8 bytes of codes), the D / 8 lanes of a row find its largest magnitude with shuffles,
// and eight rows' loads per lane are in flight before the first is used.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "../../include/tokenscale.h"
#include "ts_cache8.h"
#include "ts_internal.h"

namespace ts {
namespace {

constexpr int kThreads = 256, kInFlight = 8;

// Position of a token: its row, its place in the row's request, and the page that holds it (-1: none, reported).
struct Place {
  int page, slot;
};
__device__ __forceinline__ Place place_of(const StepDevice& s, const int32_t* rows, int tok) {
  const int n = s.n_rows + 1;
  int lo = 0, hi = s.n_rows;                    // last row whose first token is <= tok
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (rows[mid] <= tok) lo = mid; else hi = mid;
  }
  const int t = rows[n + lo] + (tok - rows[lo]), slot = rows[2 * n + lo];
  Place p = {-1, t & (kPageSize - 1)};
  if ((unsigned)slot >= (unsigned)s.max_requests || (unsigned)(t >> 4) >= (unsigned)s.max_pages_per_req) {
    if ((threadIdx.x & 31) == 0) atomicOr(s.status, TS_DEV_BAD_INDEX);
    return p;
  }
  const int page = s.table[(size_t)slot * s.max_pages_per_req + (t >> 4)];
  if ((unsigned)page >= (unsigned)s.n_pages) {
    if ((threadIdx.x & 31) == 0) atomicOr(s.status, TS_DEV_BAD_PAGE);
    return p;
  }
  p.page = page;
  return p;
}

// Eight bf16 of one row in a lane, LPR lanes per row -> the row's codes in place and its scale byte.
template <int LPR>
__device__ __forceinline__ uint2 quantise(const uint4& v, uint8_t& scale) {
  // magnitudes as integers are ordered as the numbers are, NaN behind infinity
  uint32_t most = 0;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
#pragma unroll
  for (int sh = 1; sh < LPR; sh <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, sh));
  const int E = cache8_exponent(most);
  scale = most > 0x7f80u ? 255 : (uint8_t)(E + 127);
  const float by = __int_as_float((127 - E) << 23);
  uint32_t out[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float x0 = __uint_as_float(w[2 * i] << 16), x1 = __uint_as_float(w[2 * i] & 0xffff0000u);
    const float x2 = __uint_as_float(w[2 * i + 1] << 16), x3 = __uint_as_float(w[2 * i + 1] & 0xffff0000u);
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x0 * by, x1 * by), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x2 * by, x3 * by), __NV_SATFINITE, __NV_E4M3);
    out[i] = lo | hi << 16;
  }
  return make_uint2(out[0], out[1]);
}
// Eight codes times 2^(byte - 127), as bf16 (exact; what leaves bf16's range becomes infinite).
__device__ __forceinline__ uint4 dequantise(const uint2& c, uint8_t scale) {
  const float by = cache8_power(scale);
  uint32_t out[4];
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * by, f.y * by);
    out[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

// WRITE: the step's K/V rows (or the tokens `source` names) into their pages. Else: pages into k, v.
template <bool WRITE, bool Q8, int D>
__global__ void __launch_bounds__(kThreads)
cache_kernel(const __grid_constant__ StepParams<kInlineWords> params, const Cache8 cache, const int32_t* __restrict__ source,
             const int n_source) {
  const StepDevice& s = params.s;
  extern __shared__ int32_t rows[];
  constexpr int LPR = D / 8;                     // lanes of a row
  pdl_launch_dependents();
  pdl_wait();
  stage_rows(s, rows, threadIdx.x, blockDim.x);
  __syncthreads();
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n_chunks = 2 * s.Hkv * LPR;          // 16-byte chunks of a token's K and V
  const int half = s.Hkv * LPR;
  uint16_t* const k = const_cast<uint16_t*>(s.k_new);
  uint16_t* const v = const_cast<uint16_t*>(s.v_new);
  for (int tok = blockIdx.x * warps + warp; tok < s.n_tokens; tok += gridDim.x * warps) {
    int wide_tok = tok;                          // the token's place in k and v
    if (WRITE && source) {
      wide_tok = source[tok];
      if ((unsigned)wide_tok >= (unsigned)n_source) {
        if (lane == 0) atomicOr(s.status, TS_DEV_BAD_INDEX);
        continue;
      }
    }
    const size_t wide0 = (size_t)wide_tok * s.Hkv * D;
    // the loads of the tokens' own rows need no page: they fly while it is looked up
    uint4 w[kInFlight];
    auto load_wide = [&](int base) {
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const int c = base + u * 32 + lane;
        w[u] = make_uint4(0, 0, 0, 0);
        if (c < n_chunks) w[u] = *reinterpret_cast<const uint4*>((c < half ? k + wide0 + c * 8 : v + wide0 + (c - half) * 8));
      }
    };
    if (WRITE) load_wide(0);
    const Place p = place_of(s, rows, tok);
    for (int base = 0; base < n_chunks; base += kInFlight * 32) {
      if (WRITE && base > 0) load_wide(base);
      // chunk c belongs to (K|V, head) c / LPR, counted through, and is the (c % LPR)-th of that row
      auto row_of = [&](int c) { return ((size_t)(p.page < 0 ? 0 : p.page) * 2 * s.Hkv + c / LPR) * kPageSize + p.slot; };
      if constexpr (WRITE) {
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
          const int c = base + u * 32 + lane;
          if (base + u * 32 >= n_chunks) break;  // whole warps: the shuffles below
          if constexpr (Q8) {
            uint8_t scale;
            const uint2 codes = quantise<LPR>(w[u], scale);
            if (c < n_chunks && p.page >= 0) {
              *reinterpret_cast<uint2*>(cache.values + row_of(c) * D + (c % LPR) * 8) = codes;
              if (c % LPR == 0) cache.scales[row_of(c)] = scale;
            }
          } else {
            if (c < n_chunks && p.page >= 0) *reinterpret_cast<uint4*>(s.pool + row_of(c) * D + (c % LPR) * 8) = w[u];
          }
        }
      } else {
        uint2 codes[kInFlight];
        uint8_t scale[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
          const int c = base + u * 32 + lane;
          if (c < n_chunks && p.page >= 0) {
            if constexpr (Q8) {
              codes[u] = *reinterpret_cast<const uint2*>(cache.values + row_of(c) * D + (c % LPR) * 8);
              scale[u] = cache.scales[row_of(c)];
            } else {
              w[u] = *reinterpret_cast<const uint4*>(s.pool + row_of(c) * D + (c % LPR) * 8);
            }
          }
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
          const int c = base + u * 32 + lane;
          if (c < n_chunks && p.page >= 0) {
            if constexpr (Q8) w[u] = dequantise(codes[u], scale[u]);
            *reinterpret_cast<uint4*>((c < half ? k + wide0 + c * 8 : v + wide0 + (c - half) * 8)) = w[u];
          }
        }
      }
    }
  }
}

template <bool WRITE, bool Q8, int D>
cudaError_t launch_t(const StepDevice& s, const Cache8& cache, const int32_t* source, int n_source, cudaStream_t stream) {
  const int per_block = kThreads / 32;
  const int blocks = (s.n_tokens + per_block - 1) / per_block;
  StepParams<kInlineWords> params;
  fill_params(s, &params);
  return launch_pdl(cache_kernel<WRITE, Q8, D>, dim3(blocks < 148 * 8 ? blocks : 148 * 8), dim3(kThreads), staged_rows_bytes(s.n_rows), stream,
                    params, cache, source, n_source);
}
template <bool WRITE>
cudaError_t launch(const StepDevice& s, const Cache8& cache, const int32_t* source, int n_source, cudaStream_t stream) {
  if (s.n_tokens <= 0) return cudaSuccess;
  if (cache.values)
    return s.D == 128 ? launch_t<WRITE, true, 128>(s, cache, source, n_source, stream) : launch_t<WRITE, true, 64>(s, cache, source, n_source, stream);
  return s.D == 128 ? launch_t<WRITE, false, 128>(s, cache, source, n_source, stream) : launch_t<WRITE, false, 64>(s, cache, source, n_source, stream);
}

}  // namespace

cudaError_t launch_cache_append(const StepDevice& s, const Cache8& cache, const int32_t* source, int n_source, cudaStream_t stream) {
  return launch<true>(s, cache, source, n_source, stream);
}
cudaError_t launch_cache_read(const StepDevice& s, const Cache8& cache, cudaStream_t stream) {
  return launch<false>(s, cache, nullptr, 0, stream);
}

}  // namespace ts
