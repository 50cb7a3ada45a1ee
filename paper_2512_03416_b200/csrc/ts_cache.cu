// The KV cache written and read back (sm_100a): bf16 pages, or the 8-bit cache.
//
// 8-bit cache: the D elements of a (token, KV head, K or V) row are e4m3 codes of x * 2^-E, where E is the smallest
// whole number with max|x| <= 448 * 2^E (0 for a row of zeros, clamped to [-62, 62]). A row with a NaN is one of NaN: its scale says
// so. A power of two costs no precision: e4m3 has the same four significant bits in every binade, so it loses nothing against a scale of
// max|x| / 448, the codes are the bf16 value rounded once, and code * 2^E is exact in bf16. It is one byte per row (E + 127) instead of four.
//
// Both directions are bound by memory: 4 D Hkv bytes of a token in bf16, 2 (D + 1) Hkv in 8 bits. One warp per token at a time:
// a lane moves 16 bytes of bf16 (8 bytes of codes), the D / 8 lanes of a row find its largest magnitude with shuffles,
// and eight rows' loads per lane are in flight before the first is used. 32768 tokens of eight heads of 128 (202 MB): written in 42 us (4.8 TB/s),
// read back in 37 (5.5), of 31 at the rate of a copy; of the writes' 42, the scattered scale bytes take 1.7. More loads in flight (the next
// token's while this one is written) took 45 to 49 us: what counts is that neighbouring tokens are written together.
#include <cuda_bf16.h>

#include "../../include/tokenscale.h"
#include "ts_cache8.h"
#include "ts_internal.h"

namespace ts {
namespace {

constexpr int kThreads = 256, kInFlight = 8;
// Thread blocks per SM at most, several times those that run at a time: neighbouring tokens are then written at the same time. 32768 tokens of
// eight heads of 128 in 8 bits, written / read back: 4 per SM 45.0 / 38.1 us, 8 43.8 / 38.9, 16 42.2 / 36.9, a warp per token 43.8 / 36.3.
constexpr int kBlocksPerSm = 16;
// Rows whose arrays every thread block copies to its shared memory (48 KB without asking for more). Of more rows they are looked up where they
// are: the search for a token's row is then a dozen round trips to L2, of calls that have thousands of rows.
constexpr int kStagedRows = 4095;

// Position of a token: its row, its place in the row's request, and the page that holds it (-1: none, reported).
struct Place {
  int page, slot;
};
template <bool STAGED>
__device__ __forceinline__ Place place_of(const StepDevice& s, const int32_t* rows, int tok) {
  const int n = s.n_rows + 1;
  auto first = [&](int r) { return STAGED ? rows[r] : s.row_tok0(r); };
  int lo = 0, hi = s.n_rows;                    // last row whose first token is <= tok
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first(mid) <= tok) lo = mid; else hi = mid;
  }
  const int t = (STAGED ? rows[n + lo] : s.row_ctx(lo)) + (tok - first(lo)), slot = STAGED ? rows[2 * n + lo] : s.row_slot(lo);
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

__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {       // two bf16
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Two bf16 as two codes, to nearest even, what is too large as the largest.
__device__ __forceinline__ uint16_t codes_of(uint32_t w) {
  uint16_t c;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(c) : "f"(__uint_as_float(w & 0xffff0000u)), "f"(__uint_as_float(w << 16)));
  return c;
}
__device__ __forceinline__ uint32_t join(uint16_t lo, uint16_t hi) {
  uint32_t d;
  asm("mov.b32 %0, {%1, %2};\n" : "=r"(d) : "h"(lo), "h"(hi));
  return d;
}
// 2^E twice, as bf16
__device__ __forceinline__ uint32_t power2(int E) { return (uint32_t)(E + 127) * 0x00800080u; }

// Eight bf16 of one row in a lane, LPR lanes per row -> the row's codes in place and its scale byte. x * 2^-E is exact in bf16: only
// what is 2^-125 and less of the row's largest is rounded, to a number whose code is 0.
template <int LPR>
__device__ __forceinline__ uint2 quantise(const uint4& v, uint8_t& scale) {
  // magnitudes as integers are ordered as the numbers are, NaN behind infinity
  uint32_t most = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
#pragma unroll
  for (int sh = 1; sh < LPR; sh <<= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, sh));
  most = max(most >> 16, most & 0xffffu);
  const int E = cache8_exponent(most);
  scale = most > 0x7f80u ? 255 : (uint8_t)(E + 127);
  const uint32_t by = power2(-E);
  return make_uint2(join(codes_of(mul2(v.x, by)), codes_of(mul2(v.y, by))), join(codes_of(mul2(v.z, by)), codes_of(mul2(v.w, by))));
}
// Eight codes times 2^(byte - 127), as bf16 (exact). A code's exponent and mantissa shifted to bits 10..4 are the bf16 number 2^-120 times its
// value, subnormal ones too.
__device__ __forceinline__ uint4 dequantise(const uint2& c, uint8_t scale) {
  const uint32_t by = scale == 255 ? 0x7fc07fc0u : power2(cache8_exp_of(scale));
  auto four = [&](uint32_t w, uint32_t& lo, uint32_t& hi) {
    uint32_t even = ((w << 4) & 0x07f007f0u) | ((w << 8) & 0x80008000u), odd = ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u);
    even = mul2(mul2(even, 0x7b807b80u), by);    // 2^120
    odd = mul2(mul2(odd, 0x7b807b80u), by);
    lo = __byte_perm(even, odd, 0x5410);
    hi = __byte_perm(even, odd, 0x7632);
  };
  uint4 out;
  four(c.x, out.x, out.y);
  four(c.y, out.z, out.w);
  return out;
}

// WRITE: the step's K/V rows (or the tokens `source` names) into their pages. Else: pages into k, v.
template <bool WRITE, bool Q8, int D, bool STAGED>
__global__ void __launch_bounds__(kThreads)
cache_kernel(const __grid_constant__ StepParams<kInlineWords> params, const Cache8 cache, const int32_t* __restrict__ source,
             const int n_source) {
  const StepDevice& s = params.s;
  extern __shared__ int32_t rows[];
  constexpr int LPR = D / 8;                     // lanes of a row
  pdl_launch_dependents();
  pdl_wait();
  if (STAGED) {
    stage_rows(s, rows, threadIdx.x, blockDim.x);
    __syncthreads();
  }
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // A lane has chunk j * 32 + lane (16 bytes of bf16) of a token's K, and of its V, for j = 0 .. per - 1: u counts K's and V's through.
  // Their places differ by multiples of that of j = 1, which spares the inner loops the address arithmetic.
  const int half = s.Hkv * LPR, per = (half + 31) / 32;
  const size_t lane_row = (size_t)(lane / LPR) * kPageSize, v_rows = (size_t)s.Hkv * kPageSize;
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
    const size_t wide0 = (size_t)wide_tok * s.Hkv * D + lane * 8;
    // the loads of the tokens' own rows need no page: they fly while it is looked up
    uint4 w[kInFlight];
    auto load_wide = [&](int base) {
#pragma unroll
      for (int i = 0; i < kInFlight; ++i) {
        const int u = base + i, j = u >= per ? u - per : u;
        w[i] = make_uint4(0, 0, 0, 0);
        if (u < 2 * per && j * 32 + lane < half) w[i] = *reinterpret_cast<const uint4*>((u >= per ? v : k) + wide0 + j * 256);
      }
    };
    if (WRITE) load_wide(0);
    const Place p = place_of<STAGED>(s, rows, tok);
    const bool placed = p.page >= 0;
    // the lane's first row in the page
    const size_t row0 = (size_t)(placed ? p.page : 0) * 2 * v_rows + lane_row + p.slot;
    for (int base = 0; base < 2 * per; base += kInFlight) {
      if (WRITE && base > 0) load_wide(base);
      uint2 codes[kInFlight];
      uint8_t scale[kInFlight];
#pragma unroll
      for (int i = 0; i < kInFlight; ++i) {
        const int u = base + i, j = u >= per ? u - per : u;
        if (u >= 2 * per) break;                 // whole warps: the shuffles below
        const bool mine = placed && j * 32 + lane < half;
        const size_t row = row0 + (u >= per ? v_rows : 0) + j * (32 / LPR * kPageSize);
        uint2* const at8 = reinterpret_cast<uint2*>(cache.values + row * D + lane % LPR * 8);
        uint4* const at16 = reinterpret_cast<uint4*>(s.pool + row * D + lane % LPR * 8);
        if constexpr (WRITE && Q8) {
          uint8_t b;
          const uint2 c = quantise<LPR>(w[i], b);
          if (mine) {
            *at8 = c;
            if (lane % LPR == 0) cache.scales[row] = b;
          }
        } else if constexpr (WRITE) {
          if (mine) *at16 = w[i];
        } else if (mine) {
          if constexpr (Q8) {
            codes[i] = *at8;
            scale[i] = cache.scales[row];
          } else {
            w[i] = *at16;
          }
        }
      }
      if constexpr (!WRITE) {
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
          const int u = base + i, j = u >= per ? u - per : u;
          if (u < 2 * per && placed && j * 32 + lane < half) {
            if constexpr (Q8) w[i] = dequantise(codes[i], scale[i]);
            *reinterpret_cast<uint4*>((u >= per ? v : k) + wide0 + j * 256) = w[i];
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
  const dim3 grid(blocks < 148 * kBlocksPerSm ? blocks : 148 * kBlocksPerSm);
  return s.n_rows <= kStagedRows
             ? launch_pdl(cache_kernel<WRITE, Q8, D, true>, grid, dim3(kThreads), staged_rows_bytes(s.n_rows), stream, params, cache, source, n_source)
             : launch_pdl(cache_kernel<WRITE, Q8, D, false>, grid, dim3(kThreads), 0, stream, params, cache, source, n_source);
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
