// Attention for trees of drafted tokens on the 5th-generation tensor cores (sm_100a, head_dim 128): rows whose nodes make more
// than a few dozen (node, head) pairs per KV head. The mathematics, work items and results are those of ts_tree.cu.
//
// One persistent CTA per SM. A work unit = (work item, KV head, one or two query tiles of 128 packed (node, head) rows); units
// come off a global queue, longest first. A unit's keys pass by in blocks of 128 (eight pages; the row's own nodes are a block
// of their own, the last one):
//     S = Q K^T   (tcgen05.mma, fp32 accumulator in TMEM)
//     online softmax, a thread per query row
//     O += P V    (tcgen05.mma, P from TMEM, O accumulates in TMEM)
// There are two slots, each with its S (128 TMEM columns, P over it), its O (128 columns) and four softmax warps, half a period apart,
// so that the tensor cores work for one while the other is in its softmax. A unit of two query tiles gives each slot a tile; both
// take every block. A unit of one tile gives the slots its blocks in turn, as two splits, which are added up in the epilogue.
//
// What bounds it: a tile of 128 rows takes 1024 cycles of MMAs and as many of exponentials per block; the block's K and V take
// 2850 cycles of an SM's share of HBM in bf16, 1430 in 8 bits. Units of one tile are HBM's, units of two tiles the chain's of a
// tile (scores, exponentials, P V, next scores).
//
// 8-bit cache: K goes to the tensor cores as it is (kind::f8f6f4). The queries are two e4m3 addends each, q = (q1 + q2) 2^e with
// a power of two per row: bf16's eight significant bits are twice e4m3's four, so the sum is exact down to 2^-9 of the row's
// largest element (and off by 2^-18 of that below). V is widened to f16 (exact) by four warps between its copy and the MMA, because P in
// 8 bits would lose what many small weights carry together. Exponents as in ts_tree.cu. The row's own K are two e4m3 addends as well: their 64
// rows at most are rows 0..63 and 64..127 of one K tile, and the scores are added in pairs; their V are f16 with a power of two.
//
// Warps: 0-3 / 4-7 softmax of slot A / B (thread = TMEM lane = query row), 8-11 transform (queries, V, the row's own nodes, the keys'
// exponents), 12 K loader (also takes the units), 13 V loader, 14 MMA issuer. Every wait is bounded; one that runs out raises
// TS_DEV_TIMEOUT, and the CTA ends: no new copies or MMAs, those in flight are waited for (with a limit).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math_constants.h>

#include "../../include/tokenscale.h"
#include "ts_ptx.h"
#include "ts_tc.h"
#include "ts_tma.h"
#include "ts_tree.h"

namespace ts {
namespace {

constexpr int kThreads = 512;
constexpr int kRegsSoftmax = 200, kRegsAux = 56, kRegsLaunch = 128;
static_assert(256 * kRegsSoftmax + 256 * kRegsAux <= kThreads * kRegsLaunch, "register split exceeds the launch's total");
constexpr int kWarpTransform = 8, kWarpK = 12, kWarpV = 13, kWarpMma = 14;
constexpr int kD = 128, kBlock = 128, kBlockPages = kBlock / kPageSize;
constexpr int kTile = 128 * kD * 2;              // 128 x 128 16-bit operand: two 64-column halves of 128 rows of 128 bytes
constexpr int kHalf = kTile / 2;
constexpr int kTile8 = 128 * kD;                 // 128 x 128 8-bit operand: 128 rows of 128 bytes
constexpr int kUnitRing = 4, kUnitReaders = 14;  // V loader, MMA issuer, 4 transform and 8 softmax warps
constexpr float kMoveBy = 8.f;                   // log2: how far a row's maximum may exceed its reference
constexpr float kShift16 = 7.f;                  // log2 of the factor on f16 weights: 2^(8 + 7) is within f16, 2^-21 a normal number
constexpr long long kDrainCycles = 20000000;

template <int NT, bool Q8>
struct Map {
  static constexpr int kKStages = Q8 ? (NT == 1 ? 4 : 3) : (NT == 1 ? 3 : 2);
  static constexpr int kRawStages = Q8 ? (NT == 1 ? 3 : 2) : 0;            // V codes as they are copied
  static constexpr int kVStages = Q8 ? 2 : 3;                             // V as the MMA reads it
  static constexpr int kKBytes = Q8 ? kTile8 : kTile;
  static constexpr int kOffQ = 0;                                         // Q8: q1, q2 of a tile
  static constexpr int kOffK = kOffQ + NT * kTile;
  static constexpr int kOffV = kOffK + kKStages * kKBytes;
  static constexpr int kOffRaw = kOffV + kVStages * kTile;
  static constexpr int kOffTab = kOffRaw + kRawStages * kTile8;           // Q8, per V stage: K power, V exponent, its inverse power [3][128]
  static constexpr int kOffQScale = kOffTab + (Q8 ? kVStages * 3 * kBlock * 4 : 0);   // Q8: [NT][128] power of two of a query
  static constexpr int kOffXchg = kOffQScale + (Q8 ? NT * 128 * 4 : 0);   // [slot][128] (maximum, sum)
  static constexpr int kOffBad = kOffXchg + 2 * 128 * 8;                  // per V stage: the row's own V rows that are not finite, 64 bits
  static constexpr int kOffUnits = kOffBad + 32;
  static constexpr int kOffBar = kOffUnits + kUnitRing * 64;
  enum {
    UNIT_FULL = 0, UNIT_EMPTY = UNIT_FULL + kUnitRing,
    Q_FULL = UNIT_EMPTY + kUnitRing, Q_EMPTY,
    K_FULL, K_EMPTY = K_FULL + kKStages,
    V_LANDED = K_EMPTY + kKStages,                                        // the copies of a V block (Q8: of its codes) are there
    RAW_EMPTY = V_LANDED + (Q8 ? kRawStages : kVStages),
    V_FULL = RAW_EMPTY + kRawStages, V_EMPTY = V_FULL + kVStages,
    TAB_FULL = V_EMPTY + kVStages,                                        // [kVStages] the keys' exponents of a block
    K_OWN = TAB_FULL + kVStages,                                          // K of the row's own nodes is there
    S_FULL, P_FULL = S_FULL + 2,                                          // [slot][half of the keys]
    O_FULL = P_FULL + 4, O_EMPTY = O_FULL + 2, XCHG, DRAIN = XCHG + 4, COUNT
  };
  static constexpr int kOffMisc = kOffBar + COUNT * 8;                    // TMEM address, failure flag
  static constexpr int kBytes = kOffMisc + 16;
};
static_assert(Map<1, false>::kBytes <= 232448 && Map<2, false>::kBytes <= 232448 && Map<1, true>::kBytes <= 232448 && Map<2, true>::kBytes <= 232448,
              "exceeds the shared memory one CTA can opt into");

struct Unit {
  int valid;                           // 0: there are no more units
  int tok0, T, ctx, head, table_slot;
  int t0, cnt_a, cnt_b;                // first node of tile A, nodes of the tiles
  int p_begin, n_pages;                // pages of cached tokens
  int n_cached, own;                   // blocks of cached tokens; 1 if the row's own nodes follow
  int partial_slot;
  int pad[2];
};
static_assert(sizeof(Unit) == 64, "a unit's record is four 16-byte chunks");

template <int N>
__device__ __forceinline__ void reg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void reg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(N)); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint64_t pack_f2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack_f2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;\n" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t widen(uint32_t w) {     // two e4m3 codes in the low half -> f16 pair
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffff), __NV_E4M3);
  return (uint32_t)h.x | (uint32_t)h.y << 16;
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ uint32_t max_magnitude(const uint4& w) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
  return most;
}
__device__ __forceinline__ bool not_finite(const uint4& w) {
  auto odd = [](uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; };
  return odd(w.x) || odd(w.y) || odd(w.z) || odd(w.w);
}
// x * 2^-e of eight bf16 as two e4m3 addends each: hi + lo
__device__ __forceinline__ void split8(const uint4& w, float down, uint2& hi, uint2& lo) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = make_float2(__uint_as_float(x[i] << 16) * down, __uint_as_float(x[i] & 0xffff0000u) * down);
    h[i] = __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3);
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)h[i], __NV_E4M3);
    const float2 g = __half22float2(__half2(r));
    l[i] = __nv_cvt_float2_to_fp8x2(make_float2(f.x - g.x, f.y - g.y), __NV_SATFINITE, __NV_E4M3);
  }
  hi = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
  lo = make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
}
// 16-byte chunk c (of eight 16-bit elements) of row r of a 16-bit operand tile; eight codes c of row r of an 8-bit one
__device__ __forceinline__ uint32_t at16(int r, int c) { return (uint32_t)((c >> 3) * kHalf + r * 128 + (((c ^ r) & 7) << 4)); }
__device__ __forceinline__ uint32_t at8(int r, int c) { return (uint32_t)(r * 128 + ((((c >> 1) ^ r) & 7) << 4) + (c & 1) * 8); }

// kind::f8f6f4: both operands e4m3
__device__ __forceinline__ void mma8_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t issue) {
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(issue)
      : "memory");
}
// fp32 accumulator, M = N = 128, formats 0 (f16 resp. e4m3)
__host__ __device__ constexpr uint32_t instr_desc0(bool b_mn_major) { return instr_desc(b_mn_major) & ~((1u << 7) | (1u << 10)); }

template <int NT, bool Q8>
__global__ void __launch_bounds__(kThreads, 1)
tree_tc_kernel(const __grid_constant__ StepParams<kInlineWords> params, const __grid_constant__ TreeArgs a, const __grid_constant__ CUtensorMap tile_map) {
  using L = Map<NT, Q8>;
  const StepDevice& s = params.s;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - smem_u32(smem_raw));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = s.Hq / s.Hkv;
  pdl_launch_dependents();
  if (base != smem_u32(smem_raw)) {              // never expected: the kernel has no static shared memory in front of its window
    if (tid == 0) atomicOr(s.status, TS_DEV_BAD_INDEX);
    return;
  }
  auto bar = [&](int i) { return base + (uint32_t)(L::kOffBar + i * 8); };
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(smem + L::kOffMisc);
  Unit* units = reinterpret_cast<Unit*>(smem + L::kOffUnits);

  if (tid == 0) {
    misc[1] = 0;
    for (int i = 0; i < L::COUNT; ++i) {
      int n = 1;
      if (i >= L::UNIT_EMPTY && i < L::UNIT_EMPTY + kUnitRing) n = kUnitReaders;
      if (i == L::Q_FULL || i == L::K_OWN || (i >= L::RAW_EMPTY && i < L::V_EMPTY) || (i >= L::TAB_FULL && i < L::K_OWN)) n = 4;   // transform warps
      if (i >= L::P_FULL && i < L::O_FULL) n = 4;             // softmax warps of the slot
      if (i == L::O_EMPTY) n = 8;
      if (i >= L::XCHG && i < L::DRAIN) n = 2;
      mbar_init(bar(i), n);
    }
    mbar_init_fence();
  }
  if (warp == kWarpMma) tmem_alloc(base + L::kOffMisc, 512);
  if (warp == kWarpK && lane == 0) tma_prefetch_desc(&tile_map);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  const uint32_t tmem = misc[0];

  auto failed = [&]() { return __any_sync(0xffffffffu, misc[1] != 0); };
  // Whole warps; false for all lanes when the wait ran out, here or somewhere else in the CTA.
  auto wait = [&](int i, uint32_t parity) -> bool {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar(i), parity))) return true;
    const long long t0 = clock64();
    for (;;) {
      if (__all_sync(0xffffffffu, mbar_try_wait(bar(i), parity))) return true;
      if (__any_sync(0xffffffffu, misc[1] != 0)) return false;
      if (__any_sync(0xffffffffu, clock64() - t0 > s.wait_cycles)) {
        if (lane == 0) {
          atomicOr(s.status, TS_DEV_TIMEOUT);
          misc[1] = 1;
        }
        __syncwarp();
        return false;
      }
    }
  };
  auto arrive = [&](int i) {                     // one arrival of the warp, behind everything its lanes did
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(i));
  };
  // Record of the k-th unit of this CTA; false when there is none.
  auto next_unit = [&](int k, Unit& u) -> bool {
    const int e = k % kUnitRing;
    if (!wait(L::UNIT_FULL + e, (k / kUnitRing) & 1)) return false;
    const int4* src = reinterpret_cast<const int4*>(units + e);
    int4* dst = reinterpret_cast<int4*>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = src[i];
    arrive(L::UNIT_EMPTY + e);
    return u.valid != 0;
  };
  // Which slots a unit uses, and for which blocks: two tiles: both, all blocks; one tile: in turn.
  auto slot_steps = [](const Unit& u, int x) {
    const int n = u.n_cached + u.own;
    return u.cnt_b > 0 ? n : (n + 1 - x) / 2;
  };

  if (warp < 8) {
    // ================================================================ softmax and epilogue, a thread per query row
    reg_inc<kRegsSoftmax>();
    const int x = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t tS = tmem + x * 128 + lanes;
    const uint32_t tO = tmem + 256 + lanes;      // of slot A; slot B's 128 columns on
    float2* xchg = reinterpret_cast<float2*>(smem + L::kOffXchg);
    const float scale = s.scale_log2;
    const uint64_t scale2 = pack_f2(scale, scale);
    const int row_node = row / G, row_head = row % G;
    int steps = 0;                               // of this slot so far
    int n_o[2] = {0, 0}, n_x = 0;                // units in which the slots had steps; units of one tile
    int v0 = 0;                                  // blocks of earlier units
    bool ok = true;
    for (int k = 0; ok; ++k) {
      Unit u;
      if (!next_unit(k, u)) break;
      const bool two = u.cnt_b > 0;
      const int cnt = two && x ? u.cnt_b : u.cnt_a;
      const int node = u.t0 + (two && x ? a.tile_tokens : 0) + row_node;
      const bool real = row_node < cnt;
      const bool idle = quarter * 32 >= cnt * G;           // no row of this warp is a query
      const int n = slot_steps(u, x), n_blocks = u.n_cached + u.own;
      float m = -CUDART_INF_F, l = 0.f;
      float q_scale = 1.f;
      for (int i = 0; i < n; ++i, ++steps) {
        const int j = two ? i : 2 * i + x;                 // block of the unit
        const int st = (v0 + j) % L::kVStages;
        ok = wait(L::S_FULL + x, steps & 1);
        ok = ok && wait(L::TAB_FULL + st, ((v0 + j) / L::kVStages) & 1);
        if (!ok) break;
        if (idle) {                                        // P of these rows may be anything: nobody reads their O
          arrive(L::P_FULL + 2 * x);
          arrive(L::P_FULL + 2 * x + 1);
          continue;
        }
        tc_fence_after();
        float v[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(&v[32 * c], tS + 32 * c);
        tmem_ld_wait();
        const bool own = j == u.n_cached;
        const float* tab = reinterpret_cast<const float*>(smem + L::kOffTab) + st * 3 * kBlock;
        if constexpr (Q8) {
          if (i == 0) q_scale = scale * reinterpret_cast<const float*>(smem + L::kOffQScale)[(two ? x : 0) * 128 + row];
          if (own) {
#pragma unroll
            for (int e = 0; e < 64; ++e) v[e] += v[64 + e];            // the two addends of K
          }
          const uint64_t row2 = pack_f2(q_scale, q_scale);
#pragma unroll
          for (int e = 0; e < 128; e += 4) {
            const ulonglong2 kp = *reinterpret_cast<const ulonglong2*>(tab + e), ve = *reinterpret_cast<const ulonglong2*>(tab + kBlock + e);
            unpack_f2(fma2(pack_f2(v[e], v[e + 1]), mul2(kp.x, row2), ve.x), v[e], v[e + 1]);
            unpack_f2(fma2(pack_f2(v[e + 2], v[e + 3]), mul2(kp.y, row2), ve.y), v[e + 2], v[e + 3]);
          }
        }
        // keys that this row does not see
        if (own) {
          uint64_t bits = 0;
          if (real) bits = a.mask ? a.mask[u.tok0 + node] : (2ull << node) - 1;
          if (u.T < 64) bits &= (1ull << u.T) - 1;
          const uint64_t bad = *reinterpret_cast<const uint64_t*>(smem + L::kOffBad + st * 8);
#pragma unroll
          for (int e = 0; e < 64; ++e) {
            v[e] = (bad >> e) & 1 ? CUDART_NAN_F : v[e];
            v[e] = (bits >> e) & 1 ? v[e] : -CUDART_INF_F;
            v[64 + e] = -CUDART_INF_F;
          }
        } else {
          const int valid = u.ctx - (u.p_begin * kPageSize + j * kBlock);
          const int end = min(valid, (u.n_pages - j * kBlockPages) * kPageSize);
          if (end < kBlock) {
#pragma unroll
            for (int e = 0; e < 128; ++e) v[e] = e < end ? v[e] : -CUDART_INF_F;
          }
        }
        float m0 = max3(v[0], v[1], v[2]), m1 = max3(v[3], v[4], v[5]), m2 = max3(v[6], v[7], v[8]), m3 = max3(v[9], v[10], v[11]);
#pragma unroll
        for (int e = 12; e < 124; e += 8) {
          m0 = max3(m0, v[e], v[e + 1]);
          m1 = max3(m1, v[e + 2], v[e + 3]);
          m2 = max3(m2, v[e + 4], v[e + 5]);
          m3 = max3(m3, v[e + 6], v[e + 7]);
        }
        m0 = max3(m0, v[124], v[125]);
        m1 = max3(m1, v[126], v[127]);
        float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
        if (!Q8) top *= scale;                             // the scale is positive
        const bool move = top > m + kMoveBy;               // the first key seen too: m is -inf before it
        if (__any_sync(0xffffffffu, move)) {
          const float keep = move ? ex2(m - top) : 1.f;    // 0 the first time
          if (move) m = top;
          l *= keep;
          if (i > 0) {                                     // O holds the steps in front: their P V was issued before these scores' product
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
              float ov[16];
              tmem_ld16(ov, tO + x * 128 + c * 16);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) ov[e] *= keep;
              tmem_st16(tO + x * 128 + c * 16, *reinterpret_cast<const uint32_t(*)[16]>(ov));
            }
          }
        }
        const float ref = (m == -CUDART_INF_F ? 0.f : m) - (Q8 ? kShift16 : 0.f);
        const uint64_t neg2 = pack_f2(-ref, -ref);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < 4; ++c) {                      // 32 keys at a time; half of the keys are announced when their P is in TMEM
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            float p[4];
            uint64_t x0 = pack_f2(v[32 * c + e], v[32 * c + e + 1]), x1 = pack_f2(v[32 * c + e + 2], v[32 * c + e + 3]);
            x0 = Q8 ? add2(x0, neg2) : fma2(x0, scale2, neg2);
            x1 = Q8 ? add2(x1, neg2) : fma2(x1, scale2, neg2);
            unpack_f2(x0, p[0], p[1]);
            unpack_f2(x1, p[2], p[3]);
#pragma unroll
            for (int t = 0; t < 4; ++t) p[t] = ex2(p[t]);
            if constexpr (Q8) {
              const ulonglong2 inv = *reinterpret_cast<const ulonglong2*>(tab + 2 * kBlock + 32 * c + e);
              sum[0] = fma2(pack_f2(p[0], p[1]), inv.x, sum[0]);
              sum[1] = fma2(pack_f2(p[2], p[3]), inv.y, sum[1]);
              pk[e / 2] = pack_f16(p[0], p[1]);
              pk[e / 2 + 1] = pack_f16(p[2], p[3]);
            } else {
              sum[0] = add2(sum[0], pack_f2(p[0], p[1]));
              sum[1] = add2(sum[1], pack_f2(p[2], p[3]));
              pk[e / 2] = pack_bf16(p[0], p[1]);
              pk[e / 2 + 1] = pack_bf16(p[2], p[3]);
            }
          }
          tmem_st16(tS + c * 16, pk);
          if (c & 1) {
            tmem_st_wait();
            tc_fence_before();
            arrive(L::P_FULL + 2 * x + (c >> 1));
          }
        }
        float s0, s1;
        unpack_f2(add2(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
      }
      if (!ok) break;
      v0 += n_blocks;
      // ------------------------------------------------------------------ epilogue
      // Two tiles: a slot's warps write their tile. One tile: both slots' warps know both sums, and each writes half of the columns.
      const int n_other = slot_steps(u, x ^ 1);
      float w_mine = 1.f, w_other = 0.f;
      if (!two) {
        if (k > 0) ok = wait(L::O_EMPTY, (k - 1) & 1);     // the other warp has read what the unit before left here
        if (!ok) break;
        xchg[x * 128 + row] = make_float2(m, l);
        arrive(L::XCHG + quarter);
        ok = wait(L::XCHG + quarter, n_x++ & 1);
        if (!ok) break;
        const float2 other = xchg[(x ^ 1) * 128 + row];
        const float mm = fmaxf(m, other.x), ref = mm == -CUDART_INF_F ? 0.f : mm;
        w_mine = ex2(m - ref);                             // 0 for a slot that saw no key
        w_other = ex2(other.x - ref);
        l = w_mine * l + w_other * other.y;
        m = mm;
      }
      if (n > 0) ok = wait(L::O_FULL + x, n_o[x] & 1);
      if (ok && !two && n_other > 0) ok = wait(L::O_FULL + (x ^ 1), n_o[x ^ 1] & 1);
      if (!ok) break;
      if (n > 0) ++n_o[x];
      if (n_other > 0) ++n_o[x ^ 1];
      tc_fence_after();
      if (!idle) {
        const bool split = u.partial_slot >= 0;
        const uint32_t out_row = real ? (uint32_t)((split ? u.partial_slot : u.tok0) + node) * s.Hq + u.head * G + row_head : 0xffffffffu;
        const float inv = split ? 1.f : l == 0.f ? 0.f : 1.f / l;      // no visible key: zeros
        w_mine *= inv;
        w_other *= inv;
        if (split && real && (two || x == 0)) *reinterpret_cast<float2*>(s.part_ml + (size_t)out_row * 2) = make_float2(m, l);
        const int c_begin = two ? 0 : x * 4, c_end = two ? 8 : x * 4 + 4;
#pragma unroll 1
        for (int c = c_begin; c < c_end; ++c) {            // sixteen columns at a time
          float ov[16];
          if (n > 0) {
            tmem_ld16(ov, tO + x * 128 + c * 16);
            tmem_ld_wait();
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) ov[e] = n > 0 ? ov[e] * w_mine : 0.f;
          if (!two && n_other > 0) {
            float o2[16];
            tmem_ld16(o2, tO + (x ^ 1) * 128 + c * 16);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) ov[e] = fmaf(o2[e], w_other, ov[e]);
          }
          // A row is one thread's; the four lanes of a quad swap pieces first, so that they write neighbouring bytes of a row
          // together: 16-byte pieces of fp32, 8-byte pieces of bf16.
          uint32_t w[4][4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              w[i][e] = split ? __float_as_uint(ov[4 * i + e]) : e < 2 ? pack_bf16(ov[4 * i + 2 * e], ov[4 * i + 2 * e + 1]) : 0u;
#pragma unroll
          for (int bit = 1; bit < 4; bit <<= 1) {          // 4 x 4 transpose over the quad: w[i] becomes piece lane % 4 of row i
            const bool up = lane & bit;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (i & bit) continue;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? w[i][e] : w[i | bit][e], bit);
                if (up) w[i][e] = got; else w[i | bit][e] = got;
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t r = __shfl_sync(0xffffffffu, out_row, (lane & ~3) + i);
            if (r != 0xffffffffu) {
              const size_t at = (size_t)r * kD + c * 16 + (lane & 3) * 4;
              if (split) *reinterpret_cast<uint4*>(s.part_acc + at) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
              else *reinterpret_cast<uint2*>(s.out + at) = make_uint2(w[i][0], w[i][1]);
            }
          }
        }
      }
      tc_fence_before();
      arrive(L::O_EMPTY);
    }
  } else {
    reg_dec<kRegsAux>();
    if (warp < kWarpK) {
      // ============================================================== transform
      const int w = warp - kWarpTransform, t = tid - kWarpTransform * 32;
      const int half = lane >> 4, ch = lane & 15;            // sixteen lanes per row, 16 bytes each
      int g = 0, raw = 0;                                    // blocks of earlier units; of cached tokens
      constexpr int kRaw = Q8 ? L::kRawStages : 1;
      bool ok = true;
      for (int k = 0; ok; ++k) {
        Unit u;
        if (!next_unit(k, u)) break;
        if (k > 0 && !(ok = wait(L::Q_EMPTY, (k - 1) & 1))) break;
        // ---- queries
#pragma unroll 1
        for (int tile = 0; tile < (u.cnt_b > 0 ? 2 : 1); ++tile) {
          const int cnt = tile ? u.cnt_b : u.cnt_a, q0 = u.t0 + tile * a.tile_tokens;
          unsigned char* dst = smem + L::kOffQ + tile * kTile;
#pragma unroll 1
          for (int i0 = 0; i0 < 16; i0 += 4) {
            if ((w * 32 + i0 * 2) / G >= cnt) break;   // the rest of the warp's rows are no queries: whatever the tile holds there stays
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = w * 32 + (i0 + i) * 2 + half;
              x[i] = make_uint4(0, 0, 0, 0);
              if (r / G < cnt)
                x[i] = *reinterpret_cast<const uint4*>(s.q + ((size_t)(u.tok0 + q0 + r / G) * s.Hq + u.head * G + r % G) * kD + ch * 8);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = w * 32 + (i0 + i) * 2 + half;
              if constexpr (Q8) {
                uint32_t most = max_magnitude(x[i]);
#pragma unroll
                for (int sh = 1; sh < 16; sh <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, sh));
                const int e = most == 0 ? 0 : min(max((int)(most >> 7) - 127 - 7, -118), 118);      // largest to 2^7 .. 2^8
                uint2 hi, lo;
                split8(x[i], power(-e), hi, lo);
                *reinterpret_cast<uint2*>(dst + at8(r, ch)) = hi;
                *reinterpret_cast<uint2*>(dst + kTile8 + at8(r, ch)) = lo;
                if (ch == 0) reinterpret_cast<float*>(smem + L::kOffQScale)[tile * 128 + r] = power(e);
              } else {
                *reinterpret_cast<uint4*>(dst + at16(r, ch)) = x[i];
              }
            }
          }
        }
        fence_proxy_async();
        arrive(L::Q_FULL);
        // ---- key blocks
        const int32_t* table_row = s.table + (size_t)u.table_slot * s.max_pages_per_req;
        // Q8: exponents of key t of cached block j
        int ek = 127, ev = 127;
        auto fetch_exps = [&](int j) {
          ek = ev = 127;
          const int p = j * kBlockPages + (t >> 4);
          if (p < u.n_pages) {
            const int page = table_row[u.p_begin + p];
            if ((unsigned)page < (unsigned)s.n_pages) {
              const uint8_t* src = a.cache.scales + ((size_t)page * 2 * s.Hkv + u.head) * kPageSize + (t & 15);
              ek = src[0];
              ev = src[(size_t)s.Hkv * kPageSize];
            }
          }
        };
        if (Q8 && u.n_cached > 0) fetch_exps(0);
        for (int j = 0; j < u.n_cached + u.own; ++j, ++g) {
          const int st = g % L::kVStages;
          const bool own = j == u.n_cached;
          unsigned char* vt = smem + L::kOffV + st * kTile;
          float* tab = reinterpret_cast<float*>(smem + L::kOffTab) + st * 3 * kBlock;
          const int end = own ? u.T : min(u.ctx - (u.p_begin * kPageSize + j * kBlock), (u.n_pages - j * kBlockPages) * kPageSize);   // keys of the block
          if constexpr (Q8) {
            if (g >= L::kVStages && !(ok = wait(L::V_EMPTY + st, ((g / L::kVStages) & 1) ^ 1))) break;
            if (!own) {
              const int e = cache8_exp_of((uint8_t)ev);
              tab[t] = power(cache8_exp_of((uint8_t)ek));
              tab[kBlock + t] = (float)e;
              tab[2 * kBlock + t] = power(-e);
              arrive(L::TAB_FULL + st);
              if (j + 1 < u.n_cached) fetch_exps(j + 1);
              if (!(ok = wait(L::V_LANDED + raw % kRaw, (raw / kRaw) & 1))) break;
              const unsigned char* codes = smem + L::kOffRaw + raw % kRaw * kTile8;
              // sixteen codes -> two pieces of eight f16; eight lanes take four pieces' worth of two neighbouring rows, so that their
              // stores fall into different banks
#pragma unroll 2
              for (int i = 0; i < 8; ++i) {
                const int r = w * 32 + (i >> 1) * 8 + (lane >> 3) * 2 + ((lane >> 2) & 1), c = (i & 1) * 4 + (lane & 3);
                uint4 x = *reinterpret_cast<const uint4*>(codes + r * 128 + (((c ^ r) & 7) << 4));
                if (r >= end) x = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(vt + at16(r, 2 * c)) = make_uint4(widen(x.x), widen(x.x >> 16), widen(x.y), widen(x.y >> 16));
                *reinterpret_cast<uint4*>(vt + at16(r, 2 * c + 1)) = make_uint4(widen(x.z), widen(x.z >> 16), widen(x.w), widen(x.w >> 16));
              }
              arrive(L::RAW_EMPTY + raw % kRaw);
              ++raw;
              fence_proxy_async();
              arrive(L::V_FULL + st);
              continue;
            }
          } else {
            if (!(ok = wait(L::V_LANDED + st, (g / L::kVStages) & 1))) break;
            if (!own) {
              // rows behind the block's last key may hold anything, and 0 * NaN is none
              for (int i = t; i < (kBlock - end) * 16; i += 128) *reinterpret_cast<uint4*>(vt + at16(end + (i >> 4), i & 15)) = make_uint4(0, 0, 0, 0);
              if (end < kBlock) fence_proxy_async();
              arrive(L::TAB_FULL + st);
              arrive(L::V_FULL + st);
              continue;
            }
          }
          // ---- the row's own nodes: warp w has nodes 16 w .. 16 w + 15
          const int kst = g % L::kKStages;
          if (!(ok = wait(L::K_FULL + kst, (g / L::kKStages) & 1))) break;        // the K loader has seen the stage empty
          unsigned char* kt = smem + L::kOffK + kst * L::kKBytes;
          uint32_t bad = 0;
#pragma unroll 1
          for (int i = 0; i < 8; ++i) {
            const int r = w * 16 + i * 2 + half;
            uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
            if (r < end) {
              const size_t at = ((size_t)(u.tok0 + r) * s.Hkv + u.head) * kD + ch * 8;
              kx = *reinterpret_cast<const uint4*>(s.k_new + at);
              vx = *reinterpret_cast<const uint4*>(s.v_new + at);
            }
            const uint32_t odd = __ballot_sync(0xffffffffu, not_finite(vx));
            if (odd & (0xffffu << (half * 16))) vx = make_uint4(0, 0, 0, 0);      // must not reach the nodes that do not see it; a NaN score for the others
            bad |= (odd & 0xffffu ? 1u : 0u) << (i * 2) | (odd >> 16 ? 2u : 0u) << (i * 2);
            if constexpr (Q8) {
              uint32_t mk = max_magnitude(kx), mv = max_magnitude(vx);
#pragma unroll
              for (int sh = 1; sh < 16; sh <<= 1) {
                mk = max(mk, __shfl_xor_sync(0xffffffffu, mk, sh));
                mv = max(mv, __shfl_xor_sync(0xffffffffu, mv, sh));
              }
              const int e_k = mk == 0 ? 0 : min(max((int)(mk >> 7) - 127 - 7, -kCache8MaxExp), kCache8MaxExp);
              const int e_v = mv == 0 ? 0 : min(max((int)(mv >> 7) - 127 - 14, -kCache8MaxExp), kCache8MaxExp);
              uint2 hi, lo;
              split8(kx, power(-e_k), hi, lo);
              *reinterpret_cast<uint2*>(kt + at8(r, ch)) = hi;
              *reinterpret_cast<uint2*>(kt + at8(64 + r, ch)) = lo;
              const float down = power(-e_v);
              auto f16 = [&](uint32_t x) { return pack_f16(__uint_as_float(x << 16) * down, __uint_as_float(x & 0xffff0000u) * down); };
              *reinterpret_cast<uint4*>(vt + at16(r, ch)) = make_uint4(f16(vx.x), f16(vx.y), f16(vx.z), f16(vx.w));
              if (ch == 0) {
                tab[r] = power(e_k);
                tab[kBlock + r] = (float)e_v;
                tab[2 * kBlock + r] = power(-e_v);
                tab[2 * kBlock + 64 + r] = 1.f;              // of keys that there are not: their weights are 0
              }
            } else {
              *reinterpret_cast<uint4*>(kt + at16(r, ch)) = kx;
              *reinterpret_cast<uint4*>(vt + at16(r, ch)) = vx;
            }
            *reinterpret_cast<uint4*>(vt + at16(64 + r, ch)) = make_uint4(0, 0, 0, 0);
          }
          if (lane == 0) reinterpret_cast<uint16_t*>(smem + L::kOffBad + st * 8)[w] = (uint16_t)bad;
          fence_proxy_async();
          arrive(L::TAB_FULL + st);
          arrive(L::K_OWN);
          arrive(L::V_FULL + st);
        }
      }
    } else if (warp == kWarpK || warp == kWarpV) {
      // ============================================================== K and V loaders: a page of a KV head is a copy (bf16: two, 64 columns each)
      const int kv = warp - kWarpK;
      constexpr int kCopies = Q8 ? kBlockPages : 2 * kBlockPages, kCopyBytes = kPageSize * 128;
      const int stages = kv == 0 ? L::kKStages : Q8 ? L::kRawStages : L::kVStages;
      const int landed = kv == 0 ? (int)L::K_FULL : (int)L::V_LANDED, empty = kv == 0 ? (int)L::K_EMPTY : Q8 ? (int)L::RAW_EMPTY : (int)L::V_EMPTY;
      const uint32_t ring = base + (kv == 0 ? L::kOffK : Q8 ? L::kOffRaw : L::kOffV);
      const int stage_bytes = kv == 0 ? L::kKBytes : Q8 ? kTile8 : kTile;
      const int n_tiles = a.n_tiles, n_units = s.n_items * s.Hkv * n_tiles;
      int fetched = -1;                                      // unit that the queue has handed out (K loader)
      int g = 0;                                             // blocks through this ring
      bool ok = true;
      for (int k = 0; ok; ++k) {
        Unit u;
        if (kv == 0) {
          if (k >= kUnitRing && !(ok = wait(L::UNIT_EMPTY + k % kUnitRing, ((k / kUnitRing) & 1) ^ 1))) break;
          int unit = 0;
          if (lane == 0) {
            unit = fetched >= 0 ? fetched : (int)blockIdx.x;
            for (;; unit = (int)gridDim.x + atomicAdd(s.pf_queue, 1)) {
              u = Unit{};
              if (unit >= n_units) break;
              const WorkItem it = s.item(unit / (n_tiles * s.Hkv));
              u.t0 = unit % n_tiles * NT * a.tile_tokens;
              u.T = it.q_count;
              u.cnt_a = min(a.tile_tokens, u.T - u.t0);
              u.cnt_b = NT == 2 ? max(0, min(a.tile_tokens, u.T - u.t0 - a.tile_tokens)) : 0;
              if (u.cnt_a <= 0) continue;                    // a row of fewer nodes than the longest one
              u.valid = 1;
              u.head = unit / n_tiles % s.Hkv;
              u.tok0 = s.row_tok0(it.row);
              u.ctx = s.row_ctx(it.row);
              u.table_slot = s.row_slot(it.row);
              u.partial_slot = it.partial_slot;
              u.p_begin = it.k_begin;
              const int cached = (u.ctx + kPageSize - 1) / kPageSize;
              u.n_pages = max(0, min(it.k_end, cached) - it.k_begin);
              u.own = it.k_end > cached;
              if ((unsigned)u.table_slot >= (unsigned)s.max_requests || cached > s.max_pages_per_req) {
                atomicOr(s.status, TS_DEV_BAD_INDEX);
                u.table_slot = u.n_pages = 0;
              }
              u.n_cached = (u.n_pages + kBlockPages - 1) / kBlockPages;
              break;
            }
            const int4* src = reinterpret_cast<const int4*>(&u);
            int4* dst = reinterpret_cast<int4*>(units + k % kUnitRing);
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = src[i];
            mbar_arrive(bar(L::UNIT_FULL + k % kUnitRing));
            // the next one: the round trip passes next to this unit's copies
            if (u.valid) fetched = (int)gridDim.x + atomicAdd(s.pf_queue, 1);
          }
          __syncwarp();
          int4* all = reinterpret_cast<int4*>(&u);
          const int4* src = reinterpret_cast<const int4*>(units + k % kUnitRing);
#pragma unroll
          for (int i = 0; i < 4; ++i) all[i] = src[i];
          if (!u.valid) break;
        } else if (!next_unit(k, u)) {
          break;
        }
        const int32_t* table_row = s.table + (size_t)u.table_slot * s.max_pages_per_req + u.p_begin;
        const int my_page = Q8 ? lane : lane >> 1;
        auto fetch_page = [&](int j) {
          const int p = j * kBlockPages + my_page;
          int page = s.n_pages;
          if (lane < kCopies && p < u.n_pages) {
            page = table_row[p];
            if ((unsigned)page >= (unsigned)s.n_pages) {
              atomicOr(s.status, TS_DEV_BAD_PAGE);
              page = s.n_pages;                              // out of range on purpose: the copy delivers zeros
            }
          }
          return page;
        };
        int page = fetch_page(0);
        const int n_blocks = u.n_cached + (kv == 0 || !Q8 ? u.own : 0);      // the nodes' V in 8-bit steps does not pass the ring of codes
        for (int j = 0; j < n_blocks; ++j, ++g) {
          const int st = g % stages;
          const int page_next = j + 1 < u.n_cached ? fetch_page(j + 1) : 0;
          if (g >= stages && !(ok = wait(empty + st, ((g / stages) & 1) ^ 1))) break;
          if (j == u.n_cached) {
            if (lane == 0) mbar_arrive(bar(landed + st));    // the transform warps fill the stage
          } else {
            const int n_pg = min(kBlockPages, u.n_pages - j * kBlockPages);
            if (lane == 0) mbar_expect_tx(bar(landed + st), n_pg * kCopyBytes * (kCopies / kBlockPages));
            __syncwarp();
            if (lane < kCopies && my_page < n_pg) {
              const uint32_t dst = ring + st * stage_bytes + my_page * kCopyBytes + (Q8 ? 0 : (lane & 1) * kHalf);
              tma_load_5d(dst, &tile_map, bar(landed + st), Q8 ? 0 : (lane & 1) * 64, 0, u.head, kv, page);
            }
          }
          __syncwarp();
          page = page_next;
        }
      }
      if (failed())
        for (int i = max(0, g - stages); i < g; ++i) mbar_wait(bar(landed + i % stages), (i / stages) & 1, kDrainCycles);
    } else if (warp == kWarpMma) {
      // ============================================================== MMA issuer
      const uint32_t issue = elect_one();
      constexpr uint32_t idesc_qk = Q8 ? instr_desc0(false) : instr_desc(false), idesc_pv = Q8 ? instr_desc0(true) : instr_desc(true);
      const uint64_t q_desc = smem_desc(base + L::kOffQ, 0, 1024), k_desc = smem_desc(base + L::kOffK, 0, 1024);
      const uint64_t v_desc = smem_desc(base + L::kOffV, kHalf, 1024);
      int g = 0, n_own = 0, steps[2] = {0, 0};               // blocks and steps of earlier units
      bool ok = true;
      for (int k = 0; ok; ++k) {
        Unit u;
        if (!next_unit(k, u)) break;
        if (!(ok = wait(L::Q_FULL, k & 1))) break;
        const bool two = u.cnt_b > 0;
        const int n_blocks = u.n_cached + u.own, n_steps = two ? 2 * n_blocks : n_blocks;
        auto block_of = [&](int i) { return two ? i >> 1 : i; };
        auto qk = [&](int i) {                               // S of step i's slot
          const int x = i & 1, j = block_of(i), st = (g + j) % L::kKStages;
          if (!two || x == 0) {
            if (!(ok = ok && wait(L::K_FULL + st, ((g + j) / L::kKStages) & 1))) return;
            if (j == u.n_cached && !(ok = wait(L::K_OWN, n_own & 1))) return;
          }
          tc_fence_after();
          const uint64_t kd = k_desc + (uint64_t)((st * L::kKBytes) >> 4), qd = q_desc + (uint64_t)(((two ? x : 0) * kTile) >> 4);
          if constexpr (Q8) {
#pragma unroll
            for (int piece = 0; piece < 2; ++piece)
#pragma unroll
              for (int c = 0; c < kD / 32; ++c)
                mma8_ss(tmem + x * 128, qd + (uint64_t)((piece * kTile8 + c * 32) >> 4), kd + (uint64_t)((c * 32) >> 4), idesc_qk, piece + c > 0, issue);
          } else {
#pragma unroll
            for (int c = 0; c < kD / 16; ++c) {
              const uint64_t off = (uint64_t)(((c >> 2) * kHalf + (c & 3) * 32) >> 4);
              mma_ss(tmem + x * 128, qd + off, kd + off, idesc_qk, c > 0, issue);
            }
          }
          tc_commit(bar(L::S_FULL + x), issue);
          if (!two || x == 1) tc_commit(bar(L::K_EMPTY + st), issue);
          if (i == n_steps - 1) tc_commit(bar(L::Q_EMPTY), issue);
        };
        auto pv = [&](int i) {                               // O of step i's slot (+)= P V
          const int x = i & 1, j = block_of(i), st = (g + j) % L::kVStages, n = i >> 1;   // n-th step of the slot in this unit
          if (i == 0 && k > 0 && !(ok = wait(L::O_EMPTY, (k - 1) & 1))) return;
          if (!two || x == 0)
            if (!(ok = wait(L::V_FULL + st, ((g + j) / L::kVStages) & 1))) return;
          const uint64_t vd = v_desc + (uint64_t)((st * kTile) >> 4);
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            if (!(ok = wait(L::P_FULL + 2 * x + part, (steps[x] + n) & 1))) return;
            tc_fence_after();
#pragma unroll
            for (int kk = part * 4; kk < part * 4 + 4; ++kk)
              mma_ts(tmem + 256 + x * 128, tmem + x * 128 + kk * 8, vd + (uint64_t)((kk * 2048) >> 4), idesc_pv, (n > 0 || kk > 0) ? 1u : 0u, issue);
          }
          if (!two || x == 1) tc_commit(bar(L::V_EMPTY + st), issue);
          if (i + 2 >= n_steps) tc_commit(bar(L::O_FULL + x), issue);
        };
        qk(0);
        if (ok && n_steps > 1) qk(1);
        for (int i = 0; ok && i < n_steps; ++i) {
          pv(i);
          if (ok && i + 2 < n_steps) qk(i + 2);
        }
        g += n_blocks;
        n_own += u.own;
        steps[0] += (n_steps + 1) / 2;
        steps[1] += n_steps / 2;
      }
      // no MMA, and no arrival of one, is left behind
      tc_commit(bar(L::DRAIN), issue);
      if (!mbar_wait(bar(L::DRAIN), 0, kDrainCycles) && lane == 0) atomicOr(s.status, TS_DEV_TIMEOUT);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kWarpMma) tmem_dealloc(tmem, 512);
  if (tid == 0) {                                            // the last CTA to leave puts the queue back
    __threadfence();
    if (atomicAdd(s.pf_queue + 2, 1) == (int)gridDim.x - 1) {
      s.pf_queue[0] = 0;
      s.pf_queue[2] = 0;
    }
  }
}

template <int NT, bool Q8>
cudaError_t launch_t(const StepDevice& s, const TreeArgs& a, const CUtensorMap& map, int n_ctas, cudaStream_t stream) {
  constexpr int smem = Map<NT, Q8>::kBytes;
  const cudaError_t e = cudaFuncSetAttribute(tree_tc_kernel<NT, Q8>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  StepParams<kInlineWords> params;
  fill_params(s, &params);
  return launch_pdl(tree_tc_kernel<NT, Q8>, dim3(n_ctas), dim3(kThreads), smem, stream, params, a, map);
}

}  // namespace

cudaError_t launch_tree_tc(const StepDevice& s, const TreeArgs& a, int tiles_per_unit, const CUtensorMap& map, int n_sms, cudaStream_t stream) {
  const long long units = (long long)s.n_items * s.Hkv * a.n_tiles;
  if (units <= 0) return cudaSuccess;
  const int n_ctas = (int)(units < n_sms ? units : n_sms);
  if (a.cache.values) return tiles_per_unit == 1 ? launch_t<1, true>(s, a, map, n_ctas, stream) : launch_t<2, true>(s, a, map, n_ctas, stream);
  return tiles_per_unit == 1 ? launch_t<1, false>(s, a, map, n_ctas, stream) : launch_t<2, false>(s, a, map, n_ctas, stream);
}

}  // namespace ts
