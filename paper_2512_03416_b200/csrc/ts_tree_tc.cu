// Attention for trees of drafted tokens on the 5th-generation tensor cores (sm_100a, head_dim 128): rows whose nodes make more
// than a few dozen (node, head) pairs per KV head. The mathematics, work items and results are those of ts_tree.cu.
//
// One persistent CTA per SM. A work unit = (work item, KV head, one or two query tiles of 128 packed (node, head) rows); units
// come off a global queue, longest first. A unit's keys pass by in blocks of 128 (eight pages; the row's own nodes are a block
// of their own, the last one):
//     S = Q K^T   (tcgen05.mma, fp32 accumulator in TMEM)
//     online softmax, four lanes per query row
//     O += P V    (tcgen05.mma, P from TMEM, O accumulates in TMEM)
// There are two slots, each with its S (128 TMEM columns, P over it), its O (128 columns) and eight softmax warps, half a period apart,
// so that the tensor cores work for one while the other is in its softmax. A unit of two query tiles gives each slot a tile; both
// take every block. A unit of one tile gives the slots its blocks in turn, as two splits, which are added up in the epilogue.
//
// What bounds it: a tile of 128 rows takes 1024 cycles of MMAs and as many of exponentials per block; the block's K and V take
// 2850 cycles of an SM's share of HBM in bf16, 1430 in 8 bits. Units of one tile are HBM's in bf16 (37 rows of 8192 keys x 16 nodes, 8 KV heads x 4
// query heads: 1.24 GB in 206 us, 6.0 TB/s = 0.93 of a copy). In 8 bits they are their own chain's (the same: 0.64 GB in 166 to 177 us, 3.8 TB/s):
// about 2600 cycles per block from P V over the widening of the next V to the next P V, with the looks at barriers of the one MMA issuer. There the roles' instructions
// together are more than the instruction cache holds (stalls for no instruction 1.2 per issue): code that is never reached can cost 30 %.
// Units of two tiles are the chain's of a tile (scores, exponentials, P V, next scores; 4100 to 4700 cycles per block; 37 rows of 4096 keys x
// 32 nodes, 8 KV heads x 8 query heads: 157 us, 0.59 of the MMAs' rate, in 8 bits 183). A change of units costs 5 us of latency where
// rows are short, because a unit's epilogue and the next one's first scores follow each other (64 rows of 500 keys x 8 nodes 47 us, of 22 for their bytes).
// It took 8 when four warps laid out a row's nodes two rows at a time; loads of the next unit's queries ahead of the wait for their place
// gained 0.5 % in bf16 and lost 7 in 8 bits (the widening then keeps fewer loads under way).
//
// 8-bit cache: K goes to the tensor cores as it is (kind::f8f6f4). The queries are two e4m3 addends each, q = (q1 + q2) 2^e with
// a power of two per row: bf16's eight significant bits are twice e4m3's four, so the sum is exact down to 2^-9 of the row's
// largest element (and off by 2^-18 of that below). V is widened to f16 (exact) by four warps between its copy and the MMA, because P in
// 8 bits would lose what many small weights carry together. A K row's exponent is multiplied to its score. The V rows of 32 keys are
// brought to the largest of their exponents, E, as they are widened (exact for rows up to 2^15 smaller, to 2^-8 of their largest element up to
// 2^22), so that the weights of these keys get E alone: 2^(s + E - m), m the running maximum of s + E, and the sum takes it out again. The
// row's own K are two e4m3 addends as well: their 64 rows at most are rows 0..63 and 64..127 of one K tile, and the scores are added in
// pairs; their V are f16 with an exponent per 32 nodes.
//
// Warps: 0-7 / 8-15 softmax of slot A / B (sixteen query rows each, four lanes per row), 16-23 transform (queries, V, the row's own nodes),
// 24 K loader (also takes the units), 25 V loader, 26 MMA issuer, 27 exponents of the cached keys. Every wait is bounded; one that runs out raises
// TS_DEV_TIMEOUT, and the CTA ends: no new copies or MMAs, those in flight are waited for (with a limit).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include <type_traits>

#include "../../include/tokenscale.h"
#include "ts_ptx.h"
#include "ts_tc.h"
#include "ts_tma.h"
#include "ts_tree.h"

namespace ts {
namespace {

constexpr int kThreads = 896;
// Register split (setmaxnreg works on whole warpgroups): four of softmax warps, two of transform warps, one of loaders and MMA issuer
constexpr int kRegsLaunch = 72, kRegsSoftmax = 88, kRegsTransform = 48, kRegsAux = 56;
static_assert(512 * kRegsSoftmax + 256 * kRegsTransform + 128 * kRegsAux <= kThreads * kRegsLaunch, "register split exceeds the launch's total");
constexpr int kWarpTransform = 16, kTransformWarps = 8, kWarpK = 24, kWarpV = 25, kWarpMma = 26, kWarpTables = 27;
constexpr int kD = 128, kBlock = 128, kBlockPages = kBlock / kPageSize;
constexpr int kTile = 128 * kD * 2;              // 128 x 128 16-bit operand: two 64-column halves of 128 rows of 128 bytes
constexpr int kHalf = kTile / 2;
constexpr int kTile8 = 128 * kD;                 // 128 x 128 8-bit operand: 128 rows of 128 bytes
constexpr int kUnitRing = 4, kUnitReaders = 26;  // V loader, MMA issuer, 8 transform and 16 softmax warps; in 8 bits the tables' warp
constexpr int kTabStages = 4;                    // blocks of cached tokens whose keys' exponents are held; two of nodes
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
  // Q8, of a block (cached ones take the first kTabStages places in turn, blocks of nodes the other two): [128] powers of two of the K rows;
  // exponents of the four groups of 32 V rows and two to minus these; of cached blocks [128] f16 factors that bring the V rows to them
  static constexpr int kOffTab = kOffRaw + kRawStages * kTile8;
  static constexpr int kOffExp = kOffTab + (Q8 ? (kTabStages + 2) * kBlock * 4 : 0);
  static constexpr int kOffBy = kOffExp + (Q8 ? (kTabStages + 2) * 32 : 0);
  // Q8: [2][NT][128] powers of two of the queries, of units of even and of odd number: Q_EMPTY of a unit says that its operand is free, and comes before
  // the softmax warps have looked at its powers where the unit is short (its scores are issued while they are still in the epilogue in
  // front of it). The next but one unit's powers are written behind Q_EMPTY of the unit in between, whose scores follow all P of this one.
  static constexpr int kOffQScale = kOffBy + (Q8 ? kTabStages * kBlock * 2 : 0);
  static constexpr int kOffXchg = kOffQScale + (Q8 ? 2 * NT * 128 * 4 : 0);           // [slot][warp][16] (maximum, sum)
  static constexpr int kOffBad = kOffXchg + 2 * 128 * 8;                  // two blocks of nodes: those whose V is not finite, 64 bits
  static constexpr int kOffUnits = kOffBad + 32;
  static constexpr int kOffBar = kOffUnits + kUnitRing * 64;
  enum {
    UNIT_FULL = 0, UNIT_EMPTY = UNIT_FULL + kUnitRing,
    Q_FULL = UNIT_EMPTY + kUnitRing, Q_EMPTY,
    K_FULL, K_EMPTY = K_FULL + kKStages,
    V_LANDED = K_EMPTY + kKStages,                                        // the copies of a V block (Q8: of its codes) are there
    RAW_EMPTY = V_LANDED + (Q8 ? kRawStages : kVStages),
    V_FULL = RAW_EMPTY + kRawStages, V_EMPTY = V_FULL + kVStages,
    TAB_FULL = V_EMPTY + kVStages, TAB_EMPTY = TAB_FULL + kTabStages,     // Q8: the exponents of a block of cached tokens
    OWN_TAB = TAB_EMPTY + kTabStages,                                     // [2] what there is to know of a block of nodes
    K_OWN = OWN_TAB + 2,                                          // K of the row's own nodes is there
    // [4] K's stage for a row's own nodes is theirs: as many as the ring has stages at most, since that barrier's phases are not followed by those who
    // fill the stage
    OWN_FREE, S_FULL = OWN_FREE + 4, P_FULL = S_FULL + 2,                                          // [slot][half of the keys]
    O_FULL = P_FULL + 4, O_EMPTY = O_FULL + 2, XCHG, DRAIN = XCHG + 4, COUNT
  };
  static_assert(kKStages <= 4, "OWN_FREE");
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
// Four e4m3 codes as f16 pairs (0, 2) and (1, 3), times 2^-8 `by`
__device__ __forceinline__ void widen4(uint32_t w, uint32_t by, uint32_t& even, uint32_t& odd) {
  cache8_widen(w, even, odd);
  const __half2 f = *reinterpret_cast<const __half2*>(&by);
  const __half2 a = __hmul2(*reinterpret_cast<const __half2*>(&even), f), b = __hmul2(*reinterpret_cast<const __half2*>(&odd), f);
  even = *reinterpret_cast<const uint32_t*>(&a);
  odd = *reinterpret_cast<const uint32_t*>(&b);
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
// eight bf16, times `by`, as two e4m3 addends each: hi + lo
__device__ __forceinline__ void split8(const uint4& w, float by, uint2& hi, uint2& lo) {
  cache8_split(w.x, w.y, by, hi.x, lo.x);
  cache8_split(w.z, w.w, by, hi.y, lo.y);
}
// Query q of a tile sits in this row of its operand and TMEM lane: sixteen at a time go to the four lane quarters in turn, each of which is one SM
// sub-partition's, so that few queries use all four. (Together with the second pair of transform
// warps, which came at the same time: 64 rows of up to 16 nodes x 4 heads in 8 bits 193 -> 163 us.)
__device__ __forceinline__ int row_of(int q) { return (q >> 4 & 3) * 32 + (q >> 6) * 16 + (q & 15); }
// 16-byte chunk c (of eight 16-bit elements) of row r of a 16-bit operand tile; eight codes c of row r of an 8-bit one
__device__ __forceinline__ uint32_t at16(int r, int c) { return (uint32_t)((c >> 3) * kHalf + r * 128 + (((c ^ r) & 7) << 4)); }
__device__ __forceinline__ uint32_t at8(int r, int c) { return (uint32_t)(r * 128 + ((((c >> 1) ^ r) & 7) << 4) + (c & 1) * 8); }

// shared memory by its 32-bit address (a generic pointer is two registers)
__device__ __forceinline__ int lds_i(uint32_t at) {
  int v;
  asm volatile("ld.shared.s32 %0, [%1];\n" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void lds_f4(uint32_t at, uint64_t& lo, uint64_t& hi) {      // four
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];\n" : "=l"(lo), "=l"(hi) : "r"(at) : "memory");
}
// (volatile: loads that follow each other are issued one behind the other, in front of what is done with them)
__device__ __forceinline__ uint4 lds_u4(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
// Place of key k's power in its table: the columns of a lane in two neighbouring eights lie together.
__device__ __forceinline__ int tab_at(int k) { return ((k >> 4) * 4 + (k >> 1 & 3)) * 4 + (k >> 3 & 1) * 2 + (k & 1); }
__device__ __forceinline__ uint64_t lds_f2(uint32_t at) {       // two floats
  uint64_t v;
  asm volatile("ld.shared.b64 %0, [%1];\n" : "=l"(v) : "r"(at) : "memory");
  return v;
}
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

// TMEM of sixteen rows, eight columns at a time: lane l gets columns 2 (l % 4), + 1 of rows l / 4 (v[4 i], v[4 i + 1]) and l / 4 + 8
// (v[4 i + 2], v[4 i + 3]) of the i-th eight, as in an accumulator fragment of mma.sync.
__device__ __forceinline__ void tmem_ld_rows32(float* v, uint32_t taddr) {            // 64 columns
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_rows8(float (&v)[8], uint32_t taddr) {        // 16 columns
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st_rows8(uint32_t taddr, const float (&v)[8]) {
  const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// 16-bit pairs of the same places: w[2 i], w[2 i + 1] = rows l / 4 and l / 4 + 8 of the i-th eight; 64 of them make 32 columns.
__device__ __forceinline__ void tmem_st_pairs(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(taddr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

template <int NT, bool Q8>
__global__ void __launch_bounds__(kThreads, 1)
tree_tc_kernel(const __grid_constant__ StepParams<kInlineWords> params, const __grid_constant__ TreeArgs a, const __grid_constant__ CUtensorMap tile_map) {
  using L = Map<NT, Q8>;
  const StepDevice& s = params.s;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - smem_u32(smem_raw));
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);      // known to be the same for a warp
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
      if (i >= L::UNIT_EMPTY && i < L::UNIT_EMPTY + kUnitRing) n = kUnitReaders + (Q8 ? 1 : 0);
      if (i == L::Q_FULL || (i >= L::RAW_EMPTY && i < L::V_EMPTY) || (i >= L::OWN_TAB && i < L::K_OWN)) n = kTransformWarps;
      if (i == L::K_OWN) n = kTransformWarps / 2;
      if (i >= L::P_FULL && i < L::O_FULL) n = 8;             // softmax warps of the slot
      if (i == L::O_EMPTY) n = 16;
      if (i >= L::XCHG && i < L::DRAIN) n = 4;                // the warps of a lane quarter, of both slots
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
  auto wait_both = [&](int i, uint32_t pi, int j, uint32_t pj) -> bool {
    const bool a0 = mbar_try_wait(bar(i), pi), b0 = mbar_try_wait(bar(j), pj);      // both looks are under way together
    if (__all_sync(0xffffffffu, a0 && b0)) return true;
    return wait(i, pi) && wait(j, pj);
  };
  auto arrive = [&](int i) {                     // one arrival of the warp, behind everything its lanes did
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(i));
  };
  if (warp < kWarpTransform) {
    // ================================================================ softmax and epilogue: sixteen rows of a slot per warp
    reg_inc<kRegsSoftmax>();
    const int x = warp >> 3, quarter = warp & 3, part = (warp >> 2) & 1, row0 = row_of((warp & 7) * 16);
    const int col = (lane & 3) * 2;              // this lane's rows are row0 + lane / 4 and the eighth behind it, its columns col, col + 1 of each eight
    const uint32_t tS = tmem + x * 128 + ((uint32_t)row0 << 16);
    const uint32_t tO = tmem + 256 + ((uint32_t)row0 << 16);      // of slot A; slot B's 128 columns on
    const float scale = s.scale_log2;
    // Counters, as far as barrier phases need them: the registers are the scores'. Units (modulo 8, the ring's place and phase) with a bit 3
    // once there was one; blocks of cached tokens modulo 8 and of nodes modulo 4 (their tables' place and phase); parities: bit 0 steps of this slot, 1 and 2 units in
    // which this and the other slot had steps, 3 units of one tile.
    int k8 = 0, c8 = 0, o4 = 0, par = 0;
    static_assert(kUnitRing == 4 && kTabStages == 4, "counted modulo 8");
    bool ok = true;
    while (ok) {
      // The unit's record stays in the ring until the unit is done, and what is seldom needed is read from there.
      if (!wait(L::UNIT_FULL + (k8 & 3), (k8 >> 2) & 1)) break;
      const uint32_t rec = base + L::kOffUnits + (k8 & 3) * 64;
      auto field = [&](size_t off) { return lds_i(rec + (uint32_t)off); };
#define UNIT(f) field(offsetof(Unit, f))
      if (!UNIT(valid)) break;
      const bool two = UNIT(cnt_b) > 0;
      const int n_cached = UNIT(n_cached), n_keys = min(UNIT(ctx) - UNIT(p_begin) * kPageSize, UNIT(n_pages) * kPageSize);
      const int n_q = (two && x ? UNIT(cnt_b) : UNIT(cnt_a)) * G;
      // A unit of one tile of up to 64 queries has them in its rows twice: the two warps of a lane quarter take 64 of a block's keys each.
      const bool half = !two && n_q <= 64;
      const int query0 = half ? quarter * 16 : (warp & 7) * 16;
      const bool idle = query0 >= n_q;                     // the warp has no query
      auto steps_of = [&](int slot) {                      // two tiles: all blocks; one tile: in turn
        const int blocks = n_cached + UNIT(own);
        return two ? blocks : (blocks + 1 - slot) / 2;
      };
      float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};      // running maximum; this lane's part of the sum
      float q_scale[2] = {scale, scale};
      // block j of the unit; the slot's first one and how many on is the next
      int j = two ? 0 : x;
      const int n_blocks = n_cached + UNIT(own), dj = two ? 1 : 2;
      bool first = true;
      for (; j < n_blocks; j += dj, par ^= 1, first = false) {
        const bool own = j == n_cached;
        const int tb = own ? kTabStages + (o4 & 1) : (c8 + j) & 3;         // place of the block's tables
        if (own) ok = wait_both(L::OWN_TAB + (o4 & 1), o4 >> 1, L::S_FULL + x, par & 1);
        else if (Q8) ok = wait_both(L::TAB_FULL + tb, ((c8 + j) >> 2) & 1, L::S_FULL + x, par & 1);
        else ok = wait(L::S_FULL + x, par & 1);
        if (!ok) break;
        if (idle) {                                        // P of these rows may be anything: nobody reads their O
          arrive(L::P_FULL + 2 * x);
          arrive(L::P_FULL + 2 * x + 1);
          continue;
        }
        tc_fence_after();
        if constexpr (Q8) {
          if (first) {                                     // the queries' powers of two
            const uint32_t qs = base + L::kOffQScale + (((k8 & 1) * NT + (two ? x : 0)) * 128 + query0 + (lane >> 2)) * 4;
            q_scale[0] = scale * lds_f(qs);
            q_scale[1] = scale * lds_f(qs + 32);
          }
        }
        auto step = [&](auto halves_tag) {
          constexpr int H = decltype(halves_tag)::value;   // how many halves of the block's keys the warp takes
          const int h0 = H == 2 ? 0 : part;                // the first of them
          float v[32 * H];
#pragma unroll
          for (int h = 0; h < H; ++h) tmem_ld_rows32(&v[32 * h], tS + 64 * (h0 + h));
          const int end = n_keys - j * kBlock - 64 * h0;
          [[maybe_unused]] const uint32_t tab = base + L::kOffTab + tb * kBlock * 4 + h0 * 256 + col * 8;
          [[maybe_unused]] uint64_t kp[4];                 // looked up while the scores come
          if constexpr (Q8) {
#pragma unroll
            for (int e = 0; e < 4; e += 2) lds_f4(tab + 32 * e, kp[e], kp[e + 1]);
          }
          tmem_ld_wait();
          if constexpr (Q8) {
            if (own) {                                     // the two addends of K
              if constexpr (H == 2) {
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] += v[32 + e];
              } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  float o2[8];
                  tmem_ld_rows8(o2, tS + 64 + 16 * c);
                  tmem_ld_wait();
#pragma unroll
                  for (int e = 0; e < 8; ++e) v[8 * c + e] += o2[e];
                }
              }
            }
            // scores that can be compared: times the K rows' powers
#pragma unroll
            for (int e = 0; e < 8 * H; ++e) {
              if (e >= 4 && e % 2 == 0) lds_f4(tab + 32 * e, kp[e & 3], kp[(e & 3) + 1]);
              unpack_f2(mul2(pack_f2(v[4 * e], v[4 * e + 1]), kp[e & 3]), v[4 * e], v[4 * e + 1]);
              unpack_f2(mul2(pack_f2(v[4 * e + 2], v[4 * e + 3]), kp[e & 3]), v[4 * e + 2], v[4 * e + 3]);
            }
          }
          // keys that a row does not see
          if (own) {
            const uint64_t bad = lds_f2(base + L::kOffBad + (o4 & 1) * 8) >> col;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int q = query0 + (lane >> 2) + 8 * r, node = UNIT(t0) + (two && x ? a.tile_tokens : 0) + q / G, T = UNIT(T);
              uint64_t bits = 0;
              if (q < n_q) bits = a.mask ? a.mask[UNIT(tok0) + node] : (2ull << node) - 1;
              if (T < 64) bits &= (1ull << T) - 1;
              bits = h0 == 0 ? bits >> col : 0;            // 64 nodes at most
#pragma unroll
              for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                  float& y = v[4 * e + 2 * r + t];
                  y = (bad >> (8 * e + t)) & 1 ? CUDART_NAN_F : y;
                  y = (bits >> (8 * e + t)) & 1 ? y : -CUDART_INF_F;
                  if (H == 2) v[32 * (H - 1) + 4 * e + 2 * r + t] = -CUDART_INF_F;
                }
            }
          } else if (end < 64 * H) {
#pragma unroll
            for (int e = 0; e < 8 * H; ++e)
#pragma unroll
              for (int t = 0; t < 2; ++t)
                if (8 * e + col + t >= end) v[4 * e + t] = v[4 * e + 2 + t] = -CUDART_INF_F;
          }
          float e_of[2 * H] = {};                          // Q8: the exponents of the groups of 32 keys
          [[maybe_unused]] const uint32_t exps = base + L::kOffExp + tb * 32 + h0 * 8;
          if constexpr (Q8) {
#pragma unroll
            for (int c = 0; c < 2 * H; ++c) e_of[c] = lds_f(exps + c * 4);
          }
          float top[2];                                    // in the units of m (the scales are positive)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int c = 0; c < 2 * H; ++c) {
              const float* w = &v[16 * c + 2 * r];
              float t = max3(fmaxf(w[0], w[1]), w[4], w[5]);
              t = max3(t, w[8], w[9]);
              t = max3(t, w[12], w[13]);
              if (Q8) t = fmaf(t, q_scale[r], e_of[c]);
              top[r] = c == 0 ? t : fmaxf(top[r], t);
            }
            if (!Q8) top[r] *= scale;
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
          }
          const bool move[2] = {top[0] > m[0] + kMoveBy, top[1] > m[1] + kMoveBy};      // the first key seen too: m is -inf before it
          if (__any_sync(0xffffffffu, move[0] || move[1])) {
            float keep[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              keep[r] = move[r] ? ex2(m[r] - top[r]) : 1.f;                            // 0 the first time
              if (move[r]) m[r] = top[r];
              l[r] *= keep[r];
            }
            if (!first) {                                  // O holds the steps in front: their P V was issued before these scores' product
#pragma unroll 1
              for (uint32_t at = tO + x * 128, end_o = at + 128; at < end_o; at += 16) {
                float ov[8];
                tmem_ld_rows8(ov, at);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e) ov[e] *= keep[(e >> 1) & 1];
                tmem_st_rows8(at, ov);
              }
            }
          }
#pragma unroll
          for (int h = 0; h < H; ++h) {                    // half of the keys are announced when their P is in TMEM
            uint32_t pk[16];
#pragma unroll
            for (int c = 2 * h; c < 2 * h + 2; ++c) {
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const float ref = (m[r] == -CUDART_INF_F ? 0.f : m[r]) - (Q8 ? kShift16 + e_of[c] : 0.f);
                const uint64_t neg2 = pack_f2(-ref, -ref), scale2 = pack_f2(q_scale[r], q_scale[r]);
                uint64_t sum = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int at = 16 * c + 4 * e + 2 * r;
                  float p0, p1;
                  unpack_f2(fma2(pack_f2(v[at], v[at + 1]), scale2, neg2), p0, p1);
                  p0 = ex2(p0);
                  p1 = ex2(p1);
                  sum = add2(sum, pack_f2(p0, p1));
                  pk[8 * (c & 1) + 2 * e + r] = Q8 ? pack_f16(p0, p1) : pack_bf16(p0, p1);
                }
                float s0, s1;
                unpack_f2(sum, s0, s1);
                if (Q8) l[r] = fmaf(s0 + s1, lds_f(exps + 16 + c * 4), l[r]);          // the V rows' exponent is not part of the sum
                else l[r] += s0 + s1;
              }
            }
            tmem_st_pairs(tS + (h0 + h) * 32, pk);
            if (H == 1) {                                  // the other half's weights are the other warp's rows'
#pragma unroll
              for (int e = 0; e < 16; ++e) pk[e] = 0;
              tmem_st_pairs(tS + (1 - h0) * 32, pk);
            }
            tmem_st_wait();
            tc_fence_before();
            arrive(L::P_FULL + 2 * x + (h0 + h));
            if (H == 1) arrive(L::P_FULL + 2 * x + 1 - h0);
          }
        };
        if (half) step(std::integral_constant<int, 1>());
        else step(std::integral_constant<int, 2>());
      }
      if (!ok) break;
      c8 = (c8 + n_cached) & 7;
      o4 = (o4 + n_blocks - n_cached) & 3;
      // ------------------------------------------------------------------ epilogue
      // Two tiles: a slot's warps write their tile. One tile: the warps that have keys of the same queries (of both slots; and both of a
      // lane quarter) know each other's sums, and each writes its share of the columns.
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      }
      const int n = steps_of(x), n_other = steps_of(x ^ 1), q_of[2] = {query0 + (lane >> 2), query0 + (lane >> 2) + 8};
      // weights of the results: slot A's and B's of this warp's half (or all) of the keys, and, `half`, of the other half
      float w[4][2] = {{1.f, 1.f}, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
      if (!two) {
        float2* xchg = reinterpret_cast<float2*>(smem + L::kOffXchg);      // [slot][warp][16]
        if (k8 & 8) ok = wait(L::O_EMPTY, (k8 & 1) ^ 1);   // what the unit before left here has been read
        if (!ok) break;
        if ((lane & 3) < 2)
          xchg[warp * 16 + (lane >> 2) + 8 * (lane & 1)] = lane & 1 ? make_float2(m[1], l[1]) : make_float2(m[0], l[0]);
        arrive(L::XCHG + quarter);
        ok = wait(L::XCHG + quarter, par >> 3);
        par ^= 8;
        if (!ok) break;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float2 ml[4];
          float mm = -CUDART_INF_F;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            ml[i] = i < 2 || half ? xchg[((i & 1) * 8 + ((warp & 7) ^ (i & 2) * 2)) * 16 + (lane >> 2) + 8 * r] : make_float2(-CUDART_INF_F, 0.f);
            mm = fmaxf(mm, ml[i].x);
          }
          const float ref = mm == -CUDART_INF_F ? 0.f : mm;
          l[r] = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i][r] = ex2(ml[i].x - ref);                  // 0 for one that saw no key
            l[r] = fmaf(w[i][r], ml[i].y, l[r]);
          }
          m[r] = mm;
        }
      }
      if (n > 0) ok = wait(L::O_FULL + x, (par >> 1) & 1);
      if (ok && !two && n_other > 0) ok = wait(L::O_FULL + (x ^ 1), (par >> 2) & 1);
      if (!ok) break;
      par ^= (n > 0 ? 2 : 0) | (n_other > 0 ? 4 : 0);
      tc_fence_after();
      if (!idle) {
        const int partial = UNIT(partial_slot), node0 = UNIT(t0) + (two && x ? a.tile_tokens : 0), head = UNIT(head), tok0 = UNIT(tok0);
        const bool split = partial >= 0;
        uint32_t out_row[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          out_row[r] = (uint32_t)((split ? partial : tok0) + node0 + q_of[r] / G) * s.Hq + head * G + q_of[r] % G;
          const float inv = split ? 1.f : l[r] == 0.f ? 0.f : 1.f / l[r];      // no visible key: zeros
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i][r] *= inv;
          if (split && q_of[r] < n_q && (two || (x == 0 && !(half && part))) && (lane & 3) == 0)
            *reinterpret_cast<float2*>(s.part_ml + (size_t)out_row[r] * 2) = make_float2(m[r], l[r]);
        }
        const int c_count = two ? 8 : half ? 2 : 4, c_begin = two ? 0 : half ? (x * 2 + part) * 2 : x * 4;
        const int n_a = two ? n : steps_of(0), n_b = two ? 0 : steps_of(1);
        const uint32_t tO_a = two ? tO + x * 128 : tO;
#pragma unroll 1
        for (int c = c_begin; c < c_begin + c_count; ++c) {                            // sixteen columns at a time
          float ov[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) ov[e] = 0.f;
          auto add = [&](uint32_t at, const float (&by)[2]) {
            float o2[8];
            tmem_ld_rows8(o2, at + c * 16);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 8; ++e) ov[e] = fmaf(o2[e], by[(e >> 1) & 1], ov[e]);
          };
          if (n_a > 0) add(tO_a, w[0]);                    // what a slot without a step holds is no result
          if (n_b > 0) add(tO + 128, w[1]);
          if (half) {
            const uint32_t other = (uint32_t)(part ? -16 : 16) << 16;                  // the other warp's lanes of the quarter
            if (n_a > 0) add(tO + other, w[2]);
            if (n_b > 0) add(tO + other + 128, w[3]);
          }
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            if constexpr (Q8) {                            // V's columns came in the order 0, 2, 1, 3 of each four
              const bool odd = lane & 1;
              const float got = __shfl_xor_sync(0xffffffffu, odd ? ov[e] : ov[e + 1], 1);
              if (odd) ov[e] = got; else ov[e + 1] = got;
            }
            const int r = (e >> 1) & 1;
            if (q_of[r] < n_q) {
              const size_t at = (size_t)out_row[r] * kD + c * 16 + (e >> 2) * 8 + col;
              if (split) *reinterpret_cast<float2*>(s.part_acc + at) = make_float2(ov[e], ov[e + 1]);
              else *reinterpret_cast<uint32_t*>(s.out + at) = pack_bf16(ov[e], ov[e + 1]);
            }
          }
        }
      }
      tc_fence_before();
      arrive(L::O_EMPTY);
      arrive(L::UNIT_EMPTY + (k8 & 3));
      k8 = ((k8 + 1) & 7) | 8;
    }
  } else {
    if (warp < kWarpK) {
      reg_dec<kRegsTransform>();
      // ============================================================== transform
      const int w = warp - kWarpTransform;
      const int half = lane >> 4, ch = lane & 15;            // sixteen lanes per row, 16 bytes each
      int g = 0, raw = 0, n_own = 0;                         // blocks of earlier units; of cached tokens; of nodes
      constexpr int kRaw = Q8 ? L::kRawStages : 1;
      bool ok = true;
      for (int k = 0; ok; ++k) {
        const int ring = k % kUnitRing;                        // the record stays there until the unit is done
        if (!wait(L::UNIT_FULL + ring, (k / kUnitRing) & 1)) break;
        const volatile Unit& u = units[ring];
        if (!u.valid) break;
        if (k > 0 && !(ok = wait(L::Q_EMPTY, (k - 1) & 1))) break;
        // ---- queries
#pragma unroll 1
        for (int tile = 0; tile < (u.cnt_b > 0 ? 2 : 1); ++tile) {
          const int cnt = tile ? u.cnt_b : u.cnt_a;
          const bool twice = u.cnt_b == 0 && cnt * G <= 64;      // see the softmax warps
          const uint16_t* src = s.q + ((size_t)(u.tok0 + u.t0 + tile * a.tile_tokens) * s.Hq + u.head * G) * kD + ch * 8;
          unsigned char* dst = smem + L::kOffQ + tile * kTile;
#pragma unroll 1
          for (int i0 = 0; i0 < 8; i0 += 4) {
            if ((i0 * 16 + w * 2) / G >= cnt) break;   // the rest of the warp's are no queries: whatever the tile holds there stays
            uint4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = (i0 + i) * 16 + w * 2 + half;
              x[i] = make_uint4(0, 0, 0, 0);
              if (r / G < cnt)
                x[i] = *reinterpret_cast<const uint4*>(src + ((r / G) * s.Hq + r % G) * kD);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = (i0 + i) * 16 + w * 2 + half;
              // A query that is not finite becomes one of NaN: it has no softmax, and scores of -inf would count as keys that are not seen.
              if constexpr (Q8) {
                uint32_t most = max_magnitude(x[i]);
#pragma unroll
                for (int sh = 1; sh < 16; sh <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, sh));
                const int e = most == 0 ? 0 : min(max((int)(most >> 7) - 127 - 7, -118), 118);      // largest to 2^7 .. 2^8
                uint2 hi, lo;
                split8(x[i], power(-e), hi, lo);
                if (most >= 0x7f80u) hi = lo = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
                for (int copy = 0; copy < (twice ? 2 : 1); ++copy) {
                  *reinterpret_cast<uint2*>(dst + at8(row_of(r) + 16 * copy, ch)) = hi;
                  *reinterpret_cast<uint2*>(dst + kTile8 + at8(row_of(r) + 16 * copy, ch)) = lo;
                }
                if (ch == 0) reinterpret_cast<float*>(smem + L::kOffQScale)[((k & 1) * NT + tile) * 128 + r] = power(e);
              } else {
                if (__ballot_sync(0xffffffffu, not_finite(x[i])) & (0xffffu << (half * 16))) x[i] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
                *reinterpret_cast<uint4*>(dst + at16(row_of(r), ch)) = x[i];
                if (twice) *reinterpret_cast<uint4*>(dst + at16(row_of(r) + 16, ch)) = x[i];
              }
            }
          }
        }
        fence_proxy_async();
        arrive(L::Q_FULL);
        // ---- key blocks
        const int32_t* table_row = s.table + (size_t)u.table_slot * s.max_pages_per_req + u.p_begin;
        const int n_cached = u.n_cached, n_keys = min(u.ctx - u.p_begin * kPageSize, u.n_pages * kPageSize);
        const int n_blocks = n_cached + u.own;
        for (int j = 0; j < n_blocks; ++j, ++g) {
          const int st = g % L::kVStages;
          const bool own = j == n_cached;
          unsigned char* vt = smem + L::kOffV + st * kTile;
          const int end = own ? u.T : n_keys - j * kBlock;
          if constexpr (Q8) {
            if (!own) {
              if (g >= L::kVStages && !(ok = wait(L::V_EMPTY + st, ((g / L::kVStages) & 1) ^ 1))) break;
              const int tb = raw % kTabStages;
              if (!(ok = wait_both(L::TAB_FULL + tb, (raw / kTabStages) & 1, L::V_LANDED + raw % kRaw, (raw / kRaw) & 1))) break;
              const uint32_t codes = base + L::kOffRaw + raw % kRaw * kTile8;
              const uint16_t* by_row = reinterpret_cast<const uint16_t*>(smem + L::kOffBy) + tb * kBlock;
              // Sixteen codes -> two pieces of eight f16; eight lanes take four pieces' worth of two neighbouring rows, so that their
              // stores fall into different banks.
              uint4 x[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = (w & 3) * 32 + ((w >> 2) * 2 + (i >> 1)) * 8 + (lane >> 3) * 2 + ((lane >> 2) & 1), c = (i & 1) * 4 + (lane & 3);
                x[i] = lds_u4(codes + r * 128 + (((c ^ r) & 7) << 4));
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = (w & 3) * 32 + ((w >> 2) * 2 + (i >> 1)) * 8 + (lane >> 3) * 2 + ((lane >> 2) & 1), c = (i & 1) * 4 + (lane & 3);
                const uint32_t by = by_row[r] * 0x10001u;
                uint4 lo, hi;
                widen4(x[i].x, by, lo.x, lo.y);
                widen4(x[i].y, by, lo.z, lo.w);
                widen4(x[i].z, by, hi.x, hi.y);
                widen4(x[i].w, by, hi.z, hi.w);
                *reinterpret_cast<uint4*>(vt + at16(r, 2 * c)) = lo;
                *reinterpret_cast<uint4*>(vt + at16(r, 2 * c + 1)) = hi;
              }
              arrive(L::RAW_EMPTY + raw % kRaw);
              ++raw;
              fence_proxy_async();
              arrive(L::V_FULL + st);
              continue;
            }
          } else {
            if (!own) {
              if (!(ok = wait(L::V_LANDED + st, (g / L::kVStages) & 1))) break;
              // rows behind the block's last key may hold anything, and 0 * NaN is none
              for (int i = w * 32 + lane; i < (kBlock - end) * 16; i += kTransformWarps * 32) *reinterpret_cast<uint4*>(vt + at16(end + (i >> 4), i & 15)) = make_uint4(0, 0, 0, 0);
              if (end < kBlock) fence_proxy_async();
              arrive(L::V_FULL + st);
              continue;
            }
          }
          // ---- the row's own nodes: sixteen of them for each warp, V for warps 0-3, K for warps 4-7, four loads under way at a time. K does not wait for
          // V's stage: the scores of the nodes are wanted before their V.
          const int kst = g % L::kKStages, tb = kTabStages + (n_own & 1);
          [[maybe_unused]] float* tab = reinterpret_cast<float*>(smem + L::kOffTab) + tb * kBlock;
          const int r0 = (w & 3) * 16;
          const uint16_t* src = (w < 4 ? s.v_new : s.k_new) + ((size_t)u.tok0 * s.Hkv + u.head) * kD + ch * 8;
          auto load4 = [&](int from, uint4 (&x)[4]) {        // two rows at a time
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = from + i * 2 + half;
              x[i] = r < end ? *reinterpret_cast<const uint4*>(src + (size_t)r * s.Hkv * kD) : make_uint4(0, 0, 0, 0);
            }
          };
          uint4 x[4];
          if (w < 4) {
            uint32_t bad = 0, most = 0;
            if constexpr (Q8) {                              // the largest finite element of 32 rows goes to 2^14 .. 2^15: two warps look at them all
#pragma unroll 1
              for (int from = r0 & ~31; from < min((r0 & ~31) + 32, end); from += 8) {
                load4(from, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint32_t odd = __ballot_sync(0xffffffffu, not_finite(x[i]));
                  if (!(odd & (0xffffu << (half * 16)))) most = max(most, max_magnitude(x[i]));
                }
              }
              most = __reduce_max_sync(0xffffffffu, most);
            }
            const int e_v = min(max((int)(most >> 7) - 127 - 14, -kCache8MaxExp), kCache8MaxExp);      // zeros: the smallest there is
            const float down = power(-e_v);
            load4(r0, x);
            if constexpr (Q8) ok = g < L::kVStages || wait(L::V_EMPTY + st, ((g / L::kVStages) & 1) ^ 1);
            else ok = wait(L::V_LANDED + st, (g / L::kVStages) & 1);
            if (!ok) break;
#pragma unroll 1
            for (int from = 0; from < 16; from += 8) {
              if (from > 0) load4(r0 + from, x);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = r0 + from + i * 2 + half;
                const uint32_t odd = __ballot_sync(0xffffffffu, not_finite(x[i]));
                if (odd & (0xffffu << (half * 16))) x[i] = make_uint4(0, 0, 0, 0);       // must not reach the nodes that do not see it; a NaN score for the others
                bad |= (odd & 0xffffu ? 1u : 0u) << (from + i * 2) | (odd >> 16 ? 2u : 0u) << (from + i * 2);
                if constexpr (Q8) {
                  auto lo = [&](uint32_t y) { return __uint_as_float(y << 16) * down; };
                  auto hi = [&](uint32_t y) { return __uint_as_float(y & 0xffff0000u) * down; };
                  x[i] = make_uint4(pack_f16(lo(x[i].x), lo(x[i].y)), pack_f16(hi(x[i].x), hi(x[i].y)), pack_f16(lo(x[i].z), lo(x[i].w)), pack_f16(hi(x[i].z), hi(x[i].w)));
                }
                *reinterpret_cast<uint4*>(vt + at16(r, ch)) = x[i];
                *reinterpret_cast<uint4*>(vt + at16(64 + r, ch)) = make_uint4(0, 0, 0, 0);
              }
            }
            if (lane == 0) {
              reinterpret_cast<uint16_t*>(smem + L::kOffBad + (n_own & 1) * 8)[w] = (uint16_t)bad;
              if (Q8 && (w & 1) == 0) {
                float* e = reinterpret_cast<float*>(smem + L::kOffExp + tb * 32) + (w >> 1);
                e[0] = (float)e_v;
                e[4] = down;
                e[2] = 0.f;
                e[6] = 1.f;
              }
            }
            fence_proxy_async();
            arrive(L::OWN_TAB + (n_own & 1));
          } else {
            load4(r0, x);
            if (!(ok = wait(L::OWN_FREE + (n_own & 3), (n_own >> 2) & 1))) break;
            unsigned char* kt = smem + L::kOffK + kst * L::kKBytes;
#pragma unroll 1
            for (int from = 0; from < 16; from += 8) {
              if (from > 0) load4(r0 + from, x);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int r = r0 + from + i * 2 + half;
                if constexpr (Q8) {
                  uint32_t most = max_magnitude(x[i]);       // over the sixteen lanes of a row
#pragma unroll
                  for (int sh = 1; sh < 16; sh <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, sh));
                  const int e_k = most == 0 ? 0 : min(max((int)(most >> 7) - 127 - 7, -kCache8MaxExp), kCache8MaxExp);
                  uint2 hi, lo;
                  split8(x[i], power(-e_k), hi, lo);
                  *reinterpret_cast<uint2*>(kt + at8(r, ch)) = hi;
                  *reinterpret_cast<uint2*>(kt + at8(64 + r, ch)) = lo;
                  if (ch == 0) tab[tab_at(r)] = most >= 0x7f80u ? CUDART_NAN_F : power(e_k);       // the codes have no infinities
                } else {
                  *reinterpret_cast<uint4*>(kt + at16(r, ch)) = x[i];
                }
              }
            }
            fence_proxy_async();
            arrive(L::OWN_TAB + (n_own & 1));
            arrive(L::K_OWN);
            // V's barrier counts this warp too, not before its stage's last block was multiplied
            if constexpr (Q8) ok = g < L::kVStages || wait(L::V_EMPTY + st, ((g / L::kVStages) & 1) ^ 1);
            else ok = wait(L::V_LANDED + st, (g / L::kVStages) & 1);
            if (!ok) break;
          }
          ++n_own;
          arrive(L::V_FULL + st);
        }
        if (ok) arrive(L::UNIT_EMPTY + ring);
      }
    } else {
      reg_dec<kRegsAux>();
    }
    if (warp == kWarpK || warp == kWarpV) {
      // ============================================================== K and V loaders: a page of a KV head is a copy (bf16: two, 64 columns each)
      const int kv = warp - kWarpK;
      constexpr int kCopies = Q8 ? kBlockPages : 2 * kBlockPages, kCopyBytes = kPageSize * 128;
      const int stages = kv == 0 ? L::kKStages : Q8 ? L::kRawStages : L::kVStages;
      const int landed = kv == 0 ? (int)L::K_FULL : (int)L::V_LANDED, empty = kv == 0 ? (int)L::K_EMPTY : Q8 ? (int)L::RAW_EMPTY : (int)L::V_EMPTY;
      const uint32_t ring = base + (kv == 0 ? L::kOffK : Q8 ? L::kOffRaw : L::kOffV);
      const int stage_bytes = kv == 0 ? L::kKBytes : Q8 ? kTile8 : kTile;
      const int n_tiles = a.n_tiles, n_units = s.n_items * s.Hkv * n_tiles;
      int fetched = -1;                                      // unit that the queue has handed out (K loader)
      int g = 0, n_own = 0;                                  // blocks through this ring; of these of nodes
      bool ok = true;
      for (int k = 0; ok; ++k) {
        if (kv == 0) {
          if (k >= kUnitRing && !(ok = wait(L::UNIT_EMPTY + k % kUnitRing, ((k / kUnitRing) & 1) ^ 1))) break;
          if (lane == 0) {
            Unit u;
            int unit = fetched >= 0 ? fetched : (int)blockIdx.x;
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
        } else if (!wait(L::UNIT_FULL + k % kUnitRing, (k / kUnitRing) & 1)) {
          break;
        }
        const uint32_t rec = base + L::kOffUnits + k % kUnitRing * 64;
        auto field = [&](size_t off) { return lds_i(rec + (uint32_t)off); };
        const int valid = UNIT(valid), n_pages = UNIT(n_pages), n_cached = UNIT(n_cached), own = UNIT(own), head = UNIT(head);
        const int32_t* table_row = s.table + (size_t)UNIT(table_slot) * s.max_pages_per_req + UNIT(p_begin);
        if (kv == 1) arrive(L::UNIT_EMPTY + k % kUnitRing);
        if (!valid) break;
        const int my_page = Q8 ? lane : lane >> 1;
        auto fetch_page = [&](int j) {
          const int p = j * kBlockPages + my_page;
          int page = s.n_pages;
          if (lane < kCopies && p < n_pages) {
            page = table_row[p];
            if ((unsigned)page >= (unsigned)s.n_pages) {
              atomicOr(s.status, TS_DEV_BAD_PAGE);
              page = s.n_pages;                              // out of range on purpose: the copy delivers zeros
            }
          }
          return page;
        };
        int page = fetch_page(0);
        const int n_blocks = n_cached + (kv == 0 || !Q8 ? own : 0);      // the nodes' V in 8-bit steps does not pass the ring of codes
        for (int j = 0; j < n_blocks; ++j, ++g) {
          const int st = g % stages;
          const int page_next = j + 1 < n_cached ? fetch_page(j + 1) : 0;
          if (g >= stages && !(ok = wait(empty + st, ((g / stages) & 1) ^ 1))) break;
          if (j == n_cached) {
            if (lane == 0) {                                 // the transform warps fill the stage
              mbar_arrive(bar(landed + st));
              if (kv == 0) mbar_arrive(bar(L::OWN_FREE + (n_own & 3)));
            }
            ++n_own;
          } else {
            const int n_pg = min(kBlockPages, n_pages - j * kBlockPages);
            if (lane == 0) mbar_expect_tx(bar(landed + st), n_pg * kCopyBytes * (kCopies / kBlockPages));
            __syncwarp();
            if (lane < kCopies && my_page < n_pg) {
              const uint32_t dst = ring + st * stage_bytes + my_page * kCopyBytes + (Q8 ? 0 : (lane & 1) * kHalf);
              tma_load_5d(dst, &tile_map, bar(landed + st), Q8 ? 0 : (lane & 1) * 64, 0, head, kv, page);
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
      int k8 = 0;                                            // units, as the softmax warps count them
      int kst = 0, vst = 0, tst = 0;                         // ring places of the next K block to be multiplied, of the next V block and its tables
      uint32_t par = 0;                                      // parities: bits 0, 1 the rings' phases, 2 blocks of nodes, 3 and 4 steps of the slots
      bool ok = true;
      while (ok) {
        if (!wait(L::UNIT_FULL + (k8 & 3), (k8 >> 2) & 1)) break;
        const uint32_t rec = base + L::kOffUnits + (k8 & 3) * 64;
        // (a reduction: what it gives is known to be the same for all lanes)
        auto field = [&](size_t off) { return (int)__reduce_or_sync(0xffffffffu, (unsigned)lds_i(rec + (uint32_t)off)); };
        const int valid = UNIT(valid), two = UNIT(cnt_b) > 0, n_cached = UNIT(n_cached), n_blocks = n_cached + UNIT(own);
        arrive(L::UNIT_EMPTY + (k8 & 3));
        if (!valid || !(ok = wait(L::Q_FULL, k8 & 1))) break;
        const int n_steps = two ? 2 * n_blocks : n_blocks;
        auto takes_block = [&](int i) { return !two || (i & 1) == 0; };      // the first step of its block
        auto is_own = [&](int i) { return (two ? i >> 1 : i) == n_cached; };
        auto qk = [&](int i) {                               // scores of step i's slot
          const int x = i & 1;
          const uint64_t kd = k_desc + (uint64_t)((kst * L::kKBytes) >> 4), qd = q_desc + (uint64_t)(((two ? x : 0) * kTile) >> 4);
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
          if (!two || x == 1) {
            tc_commit(bar(L::K_EMPTY + kst), issue);
            if (++kst == L::kKStages) {
              kst = 0;
              par ^= 1;
            }
          }
          if (i == n_steps - 1) tc_commit(bar(L::Q_EMPTY), issue);
        };
        auto wait_k = [&](int i) {
          if (takes_block(i)) ok = ok && wait(L::K_FULL + kst, par & 1);
        };
        auto wait_own = [&](int i) {                         // K of the row's own nodes
          if (takes_block(i) && is_own(i)) {
            ok = ok && wait(L::K_OWN, (par >> 2) & 1);
            par ^= 4;
          }
        };
        for (int i = 0; i < 2 && i < n_steps; ++i) {
          wait_k(i);
          wait_own(i);
          tc_fence_after();
          if (ok) qk(i);
        }
        if (k8 & 8) ok = ok && wait(L::O_EMPTY, (k8 & 1) ^ 1);
        for (int i = 0; ok && i < n_steps; ++i) {            // O of the step's slot (+)= P V, then the scores of the slot's next step
          const int x = i & 1;
          // Operands are waited for ahead of P, so that between P and the slot's next scores nothing else is looked at; but for the row's
          // own nodes, whose K and V the transform warps write together once V's stage is free.
          const bool more = i + 2 < n_steps;
          if (takes_block(i)) ok = wait(L::V_FULL + vst, (par >> 1) & 1);
          if (more) wait_k(i + 2);
          if (!ok) break;
          const uint64_t vd = v_desc + (uint64_t)((vst * kTile) >> 4);
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            if (!(ok = wait(L::P_FULL + 2 * x + part, (par >> (3 + x)) & 1))) break;
            tc_fence_after();
#pragma unroll
            for (int kk = part * 4; kk < part * 4 + 4; ++kk)
              mma_ts(tmem + 256 + x * 128, tmem + x * 128 + kk * 8, vd + (uint64_t)((kk * 2048) >> 4), idesc_pv, (i > 1 || kk > 0) ? 1u : 0u, issue);
          }
          if (!ok) break;
          par ^= 8u << x;
          if (!two || x == 1) {
            tc_commit(bar(L::V_EMPTY + vst), issue);
            if (Q8 && (two ? i >> 1 : i) < n_cached) {
              tc_commit(bar(L::TAB_EMPTY + tst), issue);
              tst = (tst + 1) & 3;
            }
            if (++vst == L::kVStages) {
              vst = 0;
              par ^= 2;
            }
          }
          if (!more) {
            tc_commit(bar(L::O_FULL + x), issue);
          } else {
            if (is_own(i + 2)) {
              wait_own(i + 2);
              tc_fence_after();
            }
            if (ok) qk(i + 2);
          }
        }
        k8 = ((k8 + 1) & 7) | 8;
      }
      // no MMA, and no arrival of one, is left behind
      tc_commit(bar(L::DRAIN), issue);
      if (!mbar_wait(bar(L::DRAIN), 0, kDrainCycles) && lane == 0) atomicOr(s.status, TS_DEV_TIMEOUT);
    } else if (Q8 && warp == kWarpTables) {
      // ============================================================== exponents of the cached keys, four of a block's keys per lane
      int c = 0;                                             // blocks of earlier units
      bool ok = true;
      for (int k = 0; ok; ++k) {
        const int ring = k % kUnitRing;
        if (!wait(L::UNIT_FULL + ring, (k / kUnitRing) & 1)) break;
        const uint32_t rec = base + L::kOffUnits + ring * 64;
        auto field = [&](size_t off) { return lds_i(rec + (uint32_t)off); };
        const int valid = UNIT(valid), n_pages = UNIT(n_pages), n_cached = UNIT(n_cached);
        const int n_keys = min(UNIT(ctx) - UNIT(p_begin) * kPageSize, n_pages * kPageSize);
        const int32_t* table_row = s.table + (size_t)UNIT(table_slot) * s.max_pages_per_req + UNIT(p_begin);
        const uint8_t* scales = a.cache.scales + (size_t)UNIT(head) * kPageSize + (lane & 3) * 4;
        arrive(L::UNIT_EMPTY + ring);
        if (!valid) break;
        // loads that depend on each other are a block apart
        int page = -1;
        uint32_t kb = 0, vb = 0;
        auto fetch_page = [&](int j) {
          const int p = j * kBlockPages + (lane >> 2);
          page = p < n_pages ? table_row[p] : -1;
        };
        auto fetch_bytes = [&]() {                           // of the block whose page is known
          kb = vb = 0;
          if ((unsigned)page < (unsigned)s.n_pages) {
            const uint8_t* src = scales + (size_t)page * 2 * s.Hkv * kPageSize;
            kb = *reinterpret_cast<const uint32_t*>(src);
            vb = *reinterpret_cast<const uint32_t*>(src + (size_t)s.Hkv * kPageSize);
          }
        };
        fetch_page(0);
        fetch_bytes();
        fetch_page(1);
        auto table = [&](int j, uint32_t bytes_k, uint32_t bytes_v) {
          // two keys at a time in 16-bit halves: 0 and 2, 1 and 3 of the lane's
          constexpr uint32_t kMin = 127 - kCache8MaxExp, kMax = 127 + kCache8MaxExp;
          const int st = c % kTabStages, left = n_keys - j * kBlock;
          if (left < kBlock) {                               // keys behind the last one: rows of the smallest exponent (their weights are 0)
            const int real = left - lane * 4;
            const uint32_t keep = real >= 4 ? 0xffffffffu : real <= 0 ? 0u : (1u << (8 * real)) - 1;
            bytes_v = (bytes_v & keep) | (kMin * 0x01010101u & ~keep);
          }
          auto clamped = [](uint32_t two) { return __vminu2(__vmaxu2(two & 0x00ff00ffu, kMin * 0x10001u), kMax * 0x10001u); };
          const uint32_t k02 = clamped(bytes_k), k13 = clamped(bytes_k >> 8), v02 = clamped(bytes_v), v13 = clamped(bytes_v >> 8);
          float kp[4] = {__uint_as_float(k02 << 23), __uint_as_float(k13 << 23), __uint_as_float((k02 & 0xff0000u) << 7), __uint_as_float((k13 & 0xff0000u) << 7)};
#pragma unroll
          for (int i = 0; i < 4; ++i)                        // a row with a NaN
            if ((bytes_k >> (8 * i) & 255) == 255 || (bytes_v >> (8 * i) & 255) == 255) kp[i] = CUDART_NAN_F;
          // The V rows of 32 keys are brought to the largest of their exponents: f16 has the range for rows up to 2^22 below it.
          uint32_t top2 = __vmaxu2(v02, v13);
#pragma unroll
          for (int sh = 1; sh < 8; sh <<= 1) top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, sh));
          const int top = max(top2 & 0xffffu, top2 >> 16);
          // 2^(v - top + 8) as f16 (8: see widen4): normal numbers where bit 7 is set here
          const uint32_t x02 = v02 + (0x80u + 22) * 0x10001u - top * 0x10001u, x13 = v13 + (0x80u + 22) * 0x10001u - top * 0x10001u;
          uint32_t by02 = ((x02 & 0x007f007fu) << 10) + 0x04000400u, by13 = ((x13 & 0x007f007fu) << 10) + 0x04000400u;
          if (__any_sync(0xffffffffu, (x02 & x13 & 0x00800080u) != 0x00800080u)) {
            auto pair = [&](uint32_t two) {
              auto one = [&](int v) { return (uint32_t)__half_as_ushort(__float2half_rn(power(v - top + 8))); };
              return one(two & 0xffffu) | one(two >> 16) << 16;
            };
            by02 = pair(v02);
            by13 = pair(v13);
          }
          if (c >= kTabStages && !(ok = wait(L::TAB_EMPTY + st, ((c / kTabStages) & 1) ^ 1))) return;
          float* tab = reinterpret_cast<float*>(smem + L::kOffTab) + st * kBlock;
          *reinterpret_cast<float2*>(tab + tab_at(lane * 4)) = make_float2(kp[0], kp[1]);
          *reinterpret_cast<float2*>(tab + tab_at(lane * 4 + 2)) = make_float2(kp[2], kp[3]);
          *reinterpret_cast<uint2*>(smem + L::kOffBy + (st * kBlock + lane * 4) * 2) = make_uint2(__byte_perm(by02, by13, 0x5410), __byte_perm(by02, by13, 0x7632));
          if ((lane & 7) == 0) {
            float* e = reinterpret_cast<float*>(smem + L::kOffExp + st * 32);
            e[lane >> 3] = (float)(top - 127);
            e[4 + (lane >> 3)] = power(127 - top);
          }
          arrive(L::TAB_FULL + st);
          ++c;
        };
        int j = 0;
        uint32_t bytes_k = 0, bytes_v = 0;
        bool zeros = false;
        for (; ok && j < n_cached; ++j) {
          bytes_k = kb;
          bytes_v = vb;
          fetch_bytes();
          fetch_page(j + 2);
          zeros = __any_sync(0xffffffffu, __vcmpeq4(bytes_v, kCache8ZeroByte * 0x01010101u) != 0);
          if (__builtin_expect(zeros, 0)) break;
          table(j, bytes_k, bytes_v);
        }
        // The rest of a unit from the first block on whose V rows may be zeros, which have the smallest exponent there is. In a loop of its own: with these
        // looks in the loop above, never taken, 37 rows of 8192 keys x 4 nodes took 195 us, not 151 (see the head of this file).
#pragma unroll 1
        for (; ok && j < n_cached; ++j) {
          if (!zeros) {
            bytes_k = kb;
            bytes_v = vb;
            fetch_bytes();
            fetch_page(j + 2);
          }
          zeros = false;
#pragma unroll 1
          for (int i = 0; i < 32; i += 8)
            if ((bytes_v >> i & 255) == kCache8ZeroByte) {   // not of a page that is none: its bytes are 0
              const size_t row = (scales - a.cache.scales) + ((size_t)table_row[j * kBlockPages + (lane >> 2)] * 2 + 1) * s.Hkv * kPageSize + i / 8;
              const uint4* codes = reinterpret_cast<const uint4*>(a.cache.values + row * kD);
              uint32_t some = 0;
#pragma unroll 1
              for (int ch = 0; ch < kD / 16; ++ch) some |= cache8_magnitudes(__ldg(codes + ch));
              if (some == 0) bytes_v ^= (uint32_t)(kCache8ZeroByte ^ (127 - kCache8MaxExp)) << i;
            }
          __syncwarp();
          table(j, bytes_k, bytes_v);
        }
      }
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
