// Log probabilities of given tokens, their ranks, the entropy and the best alternatives of rows of logits (sm_100a).
//
//     y = scale * x,  lse = log sum_j exp y_j,  logprob(t) = y_t - lse,  H = lse - sum_j p_j y_j,
//     rank(t) = number of tokens in front of t in the order (x descending, index ascending); the first n of that order.
//
// One pass over the logits (they are what has to be read; everything else is a few values a row). A row is a thread block's, and a
// block takes row after row; where there are few rows, one is a cluster's of up to eight blocks, which leave their sums in the first one's
// shared memory. A warp of its own copies the row into a ring of 16 KB stages (cp.async.bulk), across the ends of rows, so
// that memory is busy while the other eight warps choose a row's alternatives. Per element a thread adds up e = 2^u and u e, u = scale log2(e) (x - ref)
// up to one rounding of ref's product, which is the same for all logits: H = ln 2 (log2 S - sum u e / S) does not see it, nor what a row's logits
// have in common. The reference is a logit that only moves when one exceeds it by a factor of 2^4 (fp32 has the range); a token that has nearly all
// the probability is the reference, and its u e nothing, so that an entropy near 0 is as exact as its small terms. The thread counts
// what lies in front of the given tokens: bf16 logits two at a time, as pairs of ones that are added up, and no block of 16 bytes whose largest
// logit is behind the token.
//
// Alternatives cost the pass no more than its maximum: every thread keeps the largest logit of its own part of the row and where
// that part first has it. The n best tokens lie in the n parts that come first by (that logit, that place), since each of these
// holds a token at least as far in front as the last part's first one. Of those parts the 16 bytes that hold the first best token are
// read again, the others only where the part's second best such block is not behind the last part's largest either; what is not behind
// that is sorted.
//
// What bounds it: HBM for fp32 logits without given tokens (2000 rows of 100003: 127 us, 6.3 TB/s = 0.98 of a copy; with 20 alternatives 147). For
// bf16 the issue of instructions: an SM's share of HBM is 11 logits a cycle, which is 11 instructions for each; the sums and the maximum take
// about 9, a given token 1.5 more wherever something may be in front of it, the end of a row 7500 a row (1024 x 131072: 59 us for the entropy
// alone, 83 with one and 5 alternatives, 3.2 TB/s; 2000 rows of 32001, whose ends weigh more, 72). One row of 32000: 14 us on
// the device, all of it round trips (cluster launch, copies, two sorts, the cluster's barrier). Tried and dropped: blocks of 16 warps (a row's end
// then idles the SM), sums in packed pairs (moves ate the gain),
// counts as sums of comparison masks (bf16 1 % at most, fp32 a third slower). Five and more given tokens with alternatives spill 10 registers, seldom read.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include <type_traits>

#include "../../include/tokenscale.h"
#include "ts_internal.h"
#include "ts_ptx.h"
#include "ts_tma.h"

namespace ts {
namespace {

namespace cg = cooperative_groups;
constexpr int kThreads = 256, kWarps = kThreads / 32;      // that work on the logits; one more warp copies
constexpr int kBlocksPerSm = 3;          // so that two stream while one chooses its row's alternatives
constexpr int kStageBytes = 16384, kStages = 4, kStageBlocks = kStageBytes / 16, kPerThread = kStageBlocks / kThreads;
constexpr int kCand = 2 * kThreads;      // candidates that are sorted at a time
constexpr int kMaxTop = 32, kMaxGiven = 8, kMaxCluster = 8;
constexpr float kLn2 = 0.6931471805599453f;
// log2: how far a value may exceed the reference of its sum. Any would do for the range; small, so that a likely token's exponent is small and
// rounded little (a token of probability 0.999 18 log2 above the reference was off by 1.3e-6), not 0, so that moves are seldom.
constexpr float kMove = 4.f;
// A reference whose product with c = scale log2(e) is larger than this is a huge one: the product's rounding, by which all weights are off alike, would no
// longer be near 1 (2^-5 log2 here), and from 2^32 on leave fp32. Its weights are 2^((x - ref) c). Rows that are masked throughout, and the like.
constexpr float kHuge = 0x1p20f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
// fp32 numbers as unsigned integers of the same order (-0 as +0)
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// (value, place) as one key: larger is further in front. 0: nothing.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t place) { return (uint64_t)ordered(x) << 32 | (uint32_t)~place; }
__device__ __forceinline__ uint32_t place_of(uint64_t key) { return ~(uint32_t)key; }

// Barrier of the working warps (id 1; 0 is the whole block's).
__device__ __forceinline__ void work_sync() { asm volatile("bar.sync 1, %0;\n" ::"n"(kThreads) : "memory"); }
// The two halves of a cluster's barrier, by all threads of its blocks in turn.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;\n" ::: "memory"); }
// The keys of a warp sorted, largest in lane 0.
__device__ __forceinline__ uint64_t warp_sort(uint64_t k, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
    for (int step = size >> 1; step > 0; step >>= 1) {
      const uint64_t o = __shfl_xor_sync(0xffffffffu, k, step);
      const bool want_max = ((lane & step) == 0) == ((lane & size) == 0);
      k = want_max == (k > o) ? k : o;
    }
  }
  return k;
}
// The 32 largest of two sorted lists, sorted.
__device__ __forceinline__ uint64_t warp_merge(uint64_t a, uint64_t b, int lane) {
  const uint64_t r = __shfl_sync(0xffffffffu, b, 31 - lane);
  uint64_t k = a > r ? a : r;
#pragma unroll
  for (int step = 16; step > 0; step >>= 1) {
    const uint64_t o = __shfl_xor_sync(0xffffffffu, k, step);
    const bool want_max = (lane & step) == 0;
    k = want_max == (k > o) ? k : o;
  }
  return k;
}
// The 32 largest of the warps' sorted lists (one of them each, the first n_lists warps'), left sorted in best[0..31]. All threads call it.
__device__ __forceinline__ void merge_lists(uint64_t k, uint64_t* best, int n_lists, int warp, int lane) {
  work_sync();
  for (int half = kWarps / 2; half > 0; half >>= 1) {
    if (half >= n_lists) continue;                   // the same for all
    if (warp >= half && warp < 2 * half) best[warp * 32 + lane] = k;
    work_sync();
    if (warp < half) k = warp_merge(k, best[(warp + half) * 32 + lane], lane);
    work_sync();
  }
  if (warp == 0) best[lane] = k;
  work_sync();
}
// Stands for -inf, and for what lies below, in the sums of a row whose reference is not huge (a bf16 number): its u is finite, its weight 0.
__device__ __forceinline__ float row_lowest(float to_log2) {
  return -__uint_as_float(__float_as_uint(fminf(0x1p126f, __fdividef(0x1p126f, to_log2))) & 0xffff0000u);
}
struct Stats {                                       // of a part of a row
  float ref, s, t;                                   // a logit to refer to, sum e, sum u e
};
// The factor between weights against two references, as log2. The sums' weights are 2^(x c - fl(ref c)), a huge one's 2^((x - ref) c): so are these.
__device__ __forceinline__ float log2_factor(float from, float to, float to_log2) {
  const float f = __fmul_rn(from, to_log2), t = __fmul_rn(to, to_log2);
  float by = f - t;                                  // -inf: from is, or nothing that counts
  if (__builtin_expect(fabsf(t) > kHuge || (fabsf(f) > kHuge && from != -CUDART_INF_F), 0)) {
    if (fabsf(f) > kHuge && fabsf(t) > kHuge) by = (from - to) * to_log2;
    else if (fabsf(f) > kHuge) by += fabsf(f) < CUDART_INF_F ? fmaf(from, to_log2, -f) : 0.f;
    else by -= fabsf(t) < CUDART_INF_F ? fmaf(to, to_log2, -t) : 0.f;
  }
  return by;
}
__device__ __forceinline__ void move_ref(Stats& a, float ref, float to_log2) {
  const float by = log2_factor(a.ref, ref, to_log2), f = ex2(by);
  // nothing yet, or nothing that counts (ref = -inf before the first number)
  a.t = a.s == 0.f || f == 0.f ? 0.f : f * fmaf(a.s, by, a.t);
  a.s *= f;                                          // a NaN stays
  a.ref = ref;
}
__device__ __forceinline__ Stats join(Stats a, Stats b, float to_log2) {
  const float ref = fmaxf(a.ref, b.ref);
  if (a.ref != ref) move_ref(a, ref, to_log2);
  if (b.ref != ref) move_ref(b, ref, to_log2);
  return Stats{ref, a.s + b.s, a.t + b.t};
}
// Of all N neighbouring lanes of a warp.
template <int N>
__device__ __forceinline__ Stats join_lanes(Stats a, float to_log2) {
  float ref = a.ref;
#pragma unroll
  for (int sh = N / 2; sh > 0; sh >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, sh));
  if (a.ref != ref) move_ref(a, ref, to_log2);
#pragma unroll
  for (int sh = N / 2; sh > 0; sh >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, sh);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, sh);
  }
  return a;
}

struct Args {
  const void* logits;
  long long row_stride;
  const float* scale;
  const int32_t* tokens;
  float *logprob, *entropy, *top_logprob;
  int32_t *rank, *top_token;
  int32_t vocab, n_given, n_top;
};

__device__ __forceinline__ uint64_t pack_f2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack_f2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;\n" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float one_if_ge(float x, float y) {
  float d;
  asm("set.ge.f32.f32 %0, %1, %2;\n" : "=f"(d) : "f"(x), "f"(y));
  return d;
}
// The next number above a finite one or -inf, in the type's bits; above +inf a NaN, which nothing reaches.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ float above(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return __uint_as_float(u == 0x80000000u ? 1u : u >> 31 ? u - 1 : u + 1);
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float largest(const uint4& v) {      // a NaN only where all are
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  // What is below `low` as that number: its weight is 0 all the same, and 0 times its u is no NaN. (A NaN stays one.)
  static __device__ __forceinline__ uint4 not_below(const uint4& v, float low) {
    auto f = [&](uint32_t x) {
      float y;
      asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(y) : "f"(__uint_as_float(x)), "f"(low));
      return __float_as_uint(y);
    };
    return make_uint4(f(v.x), f(v.y), f(v.z), f(v.w));
  }
  static __device__ __forceinline__ float count_ge(const uint4& v, float y) {
    float a, b;
    unpack_f2(add2(pack_f2(one_if_ge(__uint_as_float(v.x), y), one_if_ge(__uint_as_float(v.y), y)),
                   pack_f2(one_if_ge(__uint_as_float(v.z), y), one_if_ge(__uint_as_float(v.w), y))), a, b);
    return a + b;
  }
};
template <>
struct Vec<uint16_t> {                               // bf16 bits
  static constexpr int N = 8;
  static __device__ __forceinline__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ float above(float x) {
    const uint32_t u = __float_as_uint(x + 0.f) >> 16;
    return __uint_as_float((u == 0x8000u ? 1u : u >> 15 ? u - 1 : u + 1) << 16);
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
  static __device__ __forceinline__ float largest(const uint4& v) {
    const __nv_bfloat162 m = __hmax2(__hmax2(pair(v.x), pair(v.y)), __hmax2(pair(v.z), pair(v.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ uint4 not_below(const uint4& v, float low) {      // low is a bf16 number
    const __nv_bfloat162 low2 = __float2bfloat162_rn(low);
    auto f = [&](uint32_t x) {
      const __nv_bfloat162 y = __hmax2_nan(pair(x), low2);
      return *reinterpret_cast<const uint32_t*>(&y);
    };
    return make_uint4(f(v.x), f(v.y), f(v.z), f(v.w));
  }
  static __device__ __forceinline__ float count_ge(const uint4& v, float y) {      // y is a bf16 number
    const __nv_bfloat162 t = __float2bfloat162_rn(y);
    const __nv_bfloat162 n = __hadd2(__hadd2(__hge2(pair(v.x), t), __hge2(pair(v.y), t)), __hadd2(__hge2(pair(v.z), t), __hge2(pair(v.w), t)));
    return __low2float(n) + __high2float(n);
  }
};
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// GIVEN: how many given tokens the loop counts for (at least a.n_given).
template <typename T, int GIVEN, bool TOP>
__global__ void __launch_bounds__(kThreads + 32, kBlocksPerSm) logprobs_kernel(const Args a, const int n_rows) {
  constexpr int N = Vec<T>::N;
  extern __shared__ __align__(128) unsigned char ring[];       // [kStages][kStageBytes]
  __shared__ uint64_t lists[kWarps * 32];
  __shared__ uint64_t cand[kCand];
  __shared__ Stats warp_stats[kWarps], row_stats[kMaxCluster];
  __shared__ int32_t warp_count[kWarps][kMaxGiven];
  __shared__ int32_t row_count[kMaxCluster][kMaxGiven];
  __shared__ uint64_t row_lists[kMaxCluster * 32];
  __shared__ float given_x[kMaxGiven];                         // of the row's given tokens: logit (a NaN for one that is none), index
  __shared__ int32_t given_tok[kMaxGiven];
  __shared__ float seconds[kThreads];                          // see `second`
  __shared__ uint64_t again[kMaxTop];                          // parts that are read again in whole
  __shared__ int32_t n_cand, n_again;
  __shared__ __align__(8) uint64_t full[kStages], empty[kStages];
  cg::cluster_group cluster = cg::this_cluster();
  const int n_parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int first_row = blockIdx.x / n_parts, row_step = gridDim.x / n_parts;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t full0 = smem_u32(full), empty0 = smem_u32(empty);
  pdl_launch_dependents();
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(full0 + 8 * i, 1);
      mbar_init(empty0 + 8 * i, kWarps);
    }
    mbar_init_fence();
  }
  __syncthreads();
  // A block's shared memory may be written by the others once it has started: all say so here, and look before they write. The pass is in between.
  if (n_parts > 1) cluster_arrive();
  pdl_wait();

  // A row as 16-byte blocks of memory: block b holds the tokens b * N - off .. + N - 1, the first and the last one maybe fewer. This thread
  // block's share of those that the row fills: [begin, end); the part-filled ones are the first and the last thread block's.
  struct Row {
    const T* blocks;
    int off, begin, end;
  };
  auto row_of = [&](int row) {
    const T* x0 = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.row_stride;
    Row r;
    r.off = (int)(((uintptr_t)x0 & 15u) / sizeof(T));
    r.blocks = x0 - r.off;
    const int lo = r.off > 0, hi = (a.vocab + r.off) / N, n = max(hi - lo, 0);
    r.begin = lo + (int)((long long)n * part / n_parts);
    r.end = lo + (int)((long long)n * (part + 1) / n_parts);
    return r;
  };

  if (warp == kWarps) {
    // ---------------------------------------------------------------------- copies
    int n = 0;                                                 // stages filled so far
    for (int row = first_row; row < n_rows; row += row_step) {
      const Row r = row_of(row);
      for (int b = r.begin; b < r.end; b += kStageBlocks, ++n) {
        const int st = n % kStages;
        if (n >= kStages && !__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * st, ((n / kStages) & 1) ^ 1))) {
          row = n_rows;                                        // a wait that ran out: nobody takes the stages any more
          break;
        }
        if (lane == 0) {
          const uint32_t bytes = (uint32_t)min(kStageBlocks, r.end - b) * 16;
          mbar_expect_tx(full0 + 8 * st, bytes);
          bulk_load(smem_u32(ring) + st * kStageBytes, r.blocks + (size_t)b * N, bytes, full0 + 8 * st);
        }
        __syncwarp();
      }
    }
    for (int i = max(0, n - kStages); i < n; ++i) mbar_wait(full0 + 8 * (i % kStages), (i / kStages) & 1);      // none is left in flight
    if (n_parts > 1) {
      cluster_wait();
      cluster_arrive();
      cluster_wait();
    }
    return;
  }

  // The given tokens of a row are looked up while the row in front passes: index a row earlier than logit.
  auto tok_of = [&](int row) { return row < n_rows && tid < a.n_given ? a.tokens[(size_t)row * a.n_given + tid] : -1; };
  auto x_of = [&](int row, int tok) {
    return (unsigned)tok < (unsigned)a.vocab ? Vec<T>::load(reinterpret_cast<const T*>(a.logits) + (size_t)row * a.row_stride + tok) : CUDART_NAN_F;
  };
  int tok_now = -1, tok_next = -1;
  float x_now = CUDART_NAN_F;
  if (GIVEN > 0 && tid < a.n_given) {
    tok_now = tok_of(first_row);
    tok_next = tok_of(first_row + row_step);
    x_now = x_of(first_row, tok_now);
  }
  int n = 0;                                                   // stages read so far
  bool dead = false;
  for (int row = first_row; row < n_rows; row += row_step) {
    const Row r = row_of(row);
    const float scale = a.scale ? a.scale[row] : 1.f, to_log2 = scale * 1.4426950408889634f, lowest = row_lowest(to_log2);
    if (GIVEN > 0 && tid < kMaxGiven) {
      given_x[tid] = x_now;
      given_tok[tid] = tok_now;
    }
    if (tid == 0) n_cand = n_again = 0;
    work_sync();
    if (GIVEN > 0 && tid < a.n_given) {                        // these loads fly until the next row
      tok_now = tok_next;
      x_now = x_of(row + row_step, tok_now);
      tok_next = tok_of(row + 2 * row_step);
    }
    // Of a given token: its logit, the next number above (equal logits in front of it count, behind it not), its block. Nothing is in
    // front of a NaN.
    float gx[GIVEN > 0 ? GIVEN : 1], up[GIVEN > 0 ? GIVEN : 1], count[GIVEN > 0 ? GIVEN : 1];
    int gb[GIVEN > 0 ? GIVEN : 1];
#pragma unroll
    for (int j = 0; j < GIVEN; ++j) {
      gx[j] = given_x[j];
      up[j] = Vec<T>::above(gx[j]);
      gb[j] = (given_tok[j] + r.off) / N;
      count[j] = 0.f;
    }

    float ref = -CUDART_INF_F, neg_log2 = 0.f;                 // the reference, and -fl(ref c)
    float sum = 0.f, usum = 0.f;                               // of e and of u e
    float best = CUDART_NAN_F;                                 // this thread's largest logit (a NaN: none yet) and the first block that has it
    int best_block = -1;
    float second = -CUDART_INF_F;                              // the largest of its other blocks'
    auto refer_to = [&](float mx) {                            // the first number too: the reference is -inf before it
      if ((mx - ref) * to_log2 > kMove) {
        const float more = log2_factor(ref, mx, to_log2), f = ex2(more);      // 0 the first time
        usum = f == 0.f ? 0.f : f * fmaf(sum, more, usum);
        sum *= f;
        ref = mx;
        neg_log2 = -__fmul_rn(mx, to_log2);
      }
    };
    // One logit, whatever its size and the reference's.
    auto take_exact = [&](float x) {
      const float u = fabsf(neg_log2) > kHuge ? (x - ref) * to_log2 : fmaf(x, to_log2, neg_log2), e = ex2(u);
      sum += e;
      usum += e == 0.f ? 0.f : e * u;
    };
    // U blocks, kThreads apart. What seldom happens is asked for once for all of them.
    auto take = [&](auto count_tag, const uint4* blocks, int b0) {
      constexpr int U = decltype(count_tag)::value;
      uint4 v[U];
      float mx[U], top = -CUDART_INF_F;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        v[u] = blocks[u * kThreads];
        mx[u] = Vec<T>::largest(v[u]);
        top = fmaxf(top, mx[u]);
        if (TOP) second = fmaxf(second, fminf(fmaxf(best, -CUDART_INF_F), mx[u]));
        if (TOP && !(mx[u] <= best) && mx[u] == mx[u]) {
          best = mx[u];
          best_block = b0 + u * kThreads;
        }
      }
      refer_to(top);
      if (fabsf(neg_log2) > kHuge) {                           // rows of the type's lowest value, and the like
#pragma unroll 1
        for (int i = 0; i < U * N; ++i) take_exact(Vec<T>::load(reinterpret_cast<const T*>(blocks + i / N * kThreads) + i % N));
      } else {
        // Sums of their own first: many small weights are not added one by one to a large one.
        float s0 = 0.f, s1 = 0.f, t0 = 0.f, t1 = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float x[N];
          Vec<T>::unpack(Vec<T>::not_below(v[u], lowest), x);
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const float u0 = fmaf(x[i], to_log2, neg_log2), u1 = fmaf(x[i + 1], to_log2, neg_log2), e0 = ex2(u0), e1 = ex2(u1);
            s0 = u + i == 0 ? e0 : s0 + e0;
            s1 = u + i == 0 ? e1 : s1 + e1;
            t0 = u + i == 0 ? e0 * u0 : fmaf(e0, u0, t0);
            t1 = u + i == 0 ? e1 * u1 : fmaf(e1, u1, t1);
          }
        }
        sum += s0 + s1;
        usum += t0 + t1;
      }
#pragma unroll
      for (int j = 0; j < GIVEN; ++j) {
        if (!(top >= gx[j])) continue;                         // nothing here is in front of the token: most blocks, if it is a likely one
        bool mine = false;
#pragma unroll
        for (int u = 0; u < U; ++u) mine = mine || b0 + u * kThreads == gb[j];
        if (mine) {                                            // index by index, the token's own block is among them
          const int tok = given_tok[j];
#pragma unroll 1
          for (int i = 0; i < U * N; ++i) {
            const float x = Vec<T>::load(reinterpret_cast<const T*>(blocks + i / N * kThreads) + i % N);
            count[j] += x > gx[j] || (x == gx[j] && (b0 + i / N * kThreads) * N - r.off + i % N < tok) ? 1.f : 0.f;
          }
        } else {
#pragma unroll
          for (int u = 0; u < U; ++u) count[j] += Vec<T>::count_ge(v[u], b0 + u * kThreads < gb[j] ? gx[j] : up[j]);
        }
      }
    };
    // One logit of a block that the row fills in part.
    auto take_one = [&](int t) {
      const float x = Vec<T>::load(r.blocks + r.off + t);
      refer_to(x);
      take_exact(x);
#pragma unroll
      for (int j = 0; j < GIVEN; ++j) count[j] += x > gx[j] || (x == gx[j] && t < given_tok[j]) ? 1.f : 0.f;
    };
    // The row's tokens [0, head) and [tail, vocab) lie in such blocks: one thread each.
    const int head = min(a.vocab, r.off > 0 ? N - r.off : 0), tail = max(head, (a.vocab + r.off) / N * N - r.off);
    if (part == 0 && tid < head) take_one(tid);
    if (part == n_parts - 1 && tid >= 32 && tid - 32 < a.vocab - tail) take_one(tail + tid - 32);
    // ---------------------------------------------------------------------- the pass
#pragma unroll 1
    for (int b = r.begin; b < r.end; b += kStageBlocks, ++n) {
      const int st = n % kStages;
      dead = dead || !__all_sync(0xffffffffu, mbar_wait(full0 + 8 * st, (n / kStages) & 1));
      if (!dead) {
        const uint4* blocks = reinterpret_cast<const uint4*>(ring + st * kStageBytes);
        if (r.end - b >= kStageBlocks) {
          take(std::integral_constant<int, kPerThread>(), blocks + tid, b + tid);
        } else {
          for (int i = tid; i < r.end - b; i += kThreads) take(std::integral_constant<int, 1>(), blocks + i, b + i);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty0 + 8 * st);
    }
    Stats st = {ref, sum, usum};
    if (dead) st.s = CUDART_NAN_F;                             // a copy that never came: no result
    // ---------------------------------------------------------------------- sums of the block
    st = join_lanes<32>(st, to_log2);
    if (lane == 0) warp_stats[warp] = st;
#pragma unroll
    for (int j = 0; j < GIVEN; ++j) {                          // a thread's counts are whole numbers below 2^24
      const int sum = __reduce_add_sync(0xffffffffu, (int)count[j]);
      if (lane == 0) warp_count[warp][j] = sum;
    }

    if constexpr (TOP) {
      // -------------------------------------------------------------------- alternatives of the block
      // the parts of the n threads that come first; a part is known by its first block
      seconds[tid] = second;
      merge_lists(warp_sort(best_block < 0 ? 0 : key_of(best, (uint32_t)best_block), lane), lists, kWarps, warp, lane);
      const uint64_t last = lists[a.n_top - 1];                // 0: fewer parts than that hold a number
      const float last_x = last ? from_ordered((uint32_t)(last >> 32)) : -CUDART_INF_F;
      const int last_block = last ? (int)place_of(last) : INT32_MAX;
      const int per_part = (r.end - r.begin + kThreads - 1) / kThreads, n_items = a.n_top * per_part;
      // block `it` of the chosen parts (-1: none)
      auto block_of = [&](const uint64_t* parts, int it) {
        const uint64_t k = parts[it / per_part];
        if (k == 0) return -1;
        const int b = r.begin + ((int)place_of(k) - r.begin) % kThreads + it % per_part * kThreads;
        return b < r.end ? b : -1;
      };
      // key of token t, whose logit is x and lies in block b; 0 where it is none or behind the last part's largest
      auto key_at = [&](float x, int b, int t) -> uint64_t { return x > last_x || (x == last_x && b <= last_block) ? key_of(x, (uint32_t)t) : 0; };
      auto push = [&](uint64_t k) {
        if (k) {
          const int at = atomicAdd(&n_cand, 1);
          if (at < kCand) cand[at] = k;
        }
      };
      if (part == 0 && tid < head) push(key_at(Vec<T>::load(r.blocks + r.off + tid), 0, tid));
      if (part == n_parts - 1 && tid >= 32 && tid - 32 < a.vocab - tail) {
        const int t = tail + tid - 32;
        push(key_at(Vec<T>::load(r.blocks + r.off + t), (t + r.off) / N, t));
      }
      auto push_block = [&](const uint4& v, int b) {
        if (!(Vec<T>::largest(v) >= last_x)) return;
        float x[N];
        Vec<T>::unpack(v, x);
#pragma unroll
        for (int i = 0; i < N; ++i) push(key_at(x[i], b, b * N - r.off + i));
      };
      // A part's first best block, and the others only where another one has something as far in front as the last part.
      if (tid >= 64 && tid - 64 < a.n_top && lists[tid - 64] != 0) {
        const uint64_t k = lists[tid - 64];
        const int b = (int)place_of(k);
        push_block(load16(r.blocks + (size_t)b * N), b);
        const float other = seconds[(b - r.begin) % kThreads];
        // of logits equal to the last part's largest those count that lie no further behind: in the part's blocks behind b, and, where b holds a
        // larger one, in those in front of it
        const int from = from_ordered((uint32_t)(k >> 32)) > other ? r.begin + (b - r.begin) % kThreads : b + kThreads;
        if (other > last_x || (other == last_x && from <= last_block)) again[atomicAdd(&n_again, 1)] = k;
      }
      work_sync();
      for (int it = tid; it < n_again * per_part; it += kThreads) {
        const int b = block_of(again, it);
        if (b >= 0 && b != (int)place_of(again[it / per_part])) push_block(load16(r.blocks + (size_t)b * N), b);
      }
      work_sync();
      const int n_found = n_cand;
      if (n_found <= kCand) {
        const int n_lists = min(kWarps, (n_found + 31) / 32);
        uint64_t k = 0;
        if (warp < n_lists) k = warp_sort(tid < n_found ? cand[tid] : 0, lane);
        if (tid - lane + kThreads < n_found)                   // a second list of the warp's
          k = warp_merge(k, warp_sort(tid + kThreads < n_found ? cand[tid + kThreads] : 0, lane), lane);
        merge_lists(k, lists, n_lists, warp, lane);
      } else {
        // So many only where few parts have the larger share of a row's best tokens: all of these parts' tokens, as many at a time as
        // there are threads, next to the best so far. The tokens of part-filled blocks, 2 N - 2 at most, come last.
        if (tid < 32) cand[tid] = lists[tid];                  // the parts: `lists` is needed
        work_sync();
        uint64_t top32 = 0;                                    // warp 0: the best so far
        const int n_elems = n_items * N;
        for (int e0 = 0; e0 < n_elems + 64; e0 += kThreads) {
          const int e = e0 + tid, odd = e - n_elems;
          uint64_t k = 0;
          if (e < n_elems) {
            const int b = block_of(cand, e / N);
            if (b >= 0) k = key_at(Vec<T>::load(r.blocks + (size_t)b * N + e % N), b, b * N - r.off + e % N);
          } else if (odd < 32 ? part == 0 && odd < head : part == n_parts - 1 && odd - 32 < a.vocab - tail) {
            const int t = odd < 32 ? odd : tail + odd - 32;
            k = key_at(Vec<T>::load(r.blocks + r.off + t), (t + r.off) / N, t);
          }
          merge_lists(warp_sort(k, lane), lists, kWarps, warp, lane);
          if (warp == 0) top32 = warp_merge(top32, lists[lane], lane);
        }
        work_sync();
        if (warp == 0) lists[lane] = top32;
        work_sync();
      }
    }
    work_sync();
    // ---------------------------------------------------------------------- the blocks of the row meet in the first one
    if (n_parts > 1) cluster_wait();                           // the first one has started
    if (warp == 0) {
      const Stats all = join_lanes<kWarps>(lane < kWarps ? warp_stats[lane] : Stats{-CUDART_INF_F, 0.f, 0.f}, to_log2);
      if (lane == 0) *cluster.map_shared_rank(&row_stats[part], 0) = all;
    } else if (warp == 1) {
      if (TOP && n_parts > 1) *cluster.map_shared_rank(&row_lists[part * 32 + lane], 0) = lists[lane];
    } else if (warp == 2 && lane < a.n_given) {
      int sum = 0;
      for (int w = 0; w < kWarps; ++w) sum += warp_count[w][lane];
      *cluster.map_shared_rank(&row_count[part][lane], 0) = sum;
    }
    if (n_parts > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      work_sync();
    }
    if (part != 0) return;                                     // a cluster has one row
    Stats all = row_stats[0];
    for (int p = 1; p < n_parts; ++p) all = join(all, row_stats[p], to_log2);
    // a row without a finite logit has no distribution: every log probability is -inf, the entropy 0
    const bool none = all.s == 0.f;
    // log2 of the sum in two parts, a whole number and what is within a half: a likely token's log probability is the small difference of two
    // numbers as large as the distance from the reference, of which only the second part is rounded. (A NaN stays whole.)
    int sum_exp = 0;
    float sum_part = all.s;
    if (all.s > 0.f && all.s < CUDART_INF_F) {
      const int bits = __float_as_int(all.s) - 0x3f3504f3;       // 2^-1/2
      sum_exp = bits >> 23;
      sum_part = __int_as_float((bits & 0x7fffff) + 0x3f3504f3);
    }
    const float sum_whole = (float)sum_exp, log2_part = log2f(sum_part), log_sum = kLn2 * (sum_whole + log2_part);
    auto logprob = [&](float x) {
      if (none) return -CUDART_INF_F;
      const float ref_log2 = __fmul_rn(all.ref, to_log2);
      if (fabsf(ref_log2) > kHuge || fabsf(x) > 0x1p100f) return fmaf(x - all.ref, scale, -log_sum);
      return kLn2 * ((fmaf(x, to_log2, -ref_log2) - sum_whole) - log2_part);
    };
    if (tid == 0 && a.entropy) {
      const float h = kLn2 * ((sum_whole - all.t / all.s) + log2_part);
      a.entropy[row] = none || h < 0.f ? 0.f : h;              // the roundings of one near 0 may leave it below
    }
    if (tid >= 32 && tid - 32 < a.n_given) {
      const int j = tid - 32;
      const float x = given_x[j];
      a.logprob[(size_t)row * a.n_given + j] = x == x ? logprob(x) : CUDART_NAN_F;
      if (a.rank) {
        int sum = 0;
        for (int p = 0; p < n_parts; ++p) sum += row_count[p][j];
        a.rank[(size_t)row * a.n_given + j] = x == x ? sum : -1;
      }
    }
    if constexpr (TOP) {
      if (n_parts > 1) merge_lists(warp < n_parts ? row_lists[warp * 32 + lane] : 0, lists, n_parts, warp, lane);
      if (tid < a.n_top) {
        const uint64_t k = lists[tid];
        a.top_token[(size_t)row * a.n_top + tid] = k ? (int32_t)place_of(k) : -1;
        a.top_logprob[(size_t)row * a.n_top + tid] = k ? logprob(from_ordered((uint32_t)(k >> 32))) : CUDART_NAN_F;
      }
    }
    work_sync();
  }
}

template <typename T, int GIVEN, bool TOP>
cudaError_t launch_t(const Args& a, int n_rows, int n_parts, int n_sms, cudaStream_t stream) {
  constexpr int smem = kStages * kStageBytes;
  const cudaError_t e = cudaFuncSetAttribute(logprobs_kernel<T, GIVEN, TOP>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  const int at_a_time = kBlocksPerSm * n_sms, blocks = n_parts > 1 || n_rows < at_a_time ? n_rows * n_parts : at_a_time;
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads + 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)n_parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<T, GIVEN, TOP>, a, n_rows);
}
template <typename T, int GIVEN>
cudaError_t launch_g(const Args& a, int n_rows, int n_parts, int n_sms, cudaStream_t stream) {
  return a.n_top > 0 ? launch_t<T, GIVEN, true>(a, n_rows, n_parts, n_sms, stream) : launch_t<T, GIVEN, false>(a, n_rows, n_parts, n_sms, stream);
}
template <typename T>
cudaError_t launch(const Args& a, int n_rows, int n_parts, int n_sms, cudaStream_t stream) {
  if (a.n_given == 0) return launch_g<T, 0>(a, n_rows, n_parts, n_sms, stream);
  if (a.n_given == 1) return launch_g<T, 1>(a, n_rows, n_parts, n_sms, stream);
  if (a.n_given <= 4) return launch_g<T, 4>(a, n_rows, n_parts, n_sms, stream);
  return launch_g<T, kMaxGiven>(a, n_rows, n_parts, n_sms, stream);
}

}  // namespace
}  // namespace ts

extern "C" int ts_token_logprobs(const ts_logprobs* p, void* cuda_stream) {
  if (!p) return TS_ERR_INVALID;
  if (p->n_rows < 0 || p->vocab < 1 || p->row_stride < p->vocab) return TS_ERR_INVALID;
  if (p->n_given < 0 || p->n_given > ts::kMaxGiven || p->n_top < 0 || p->n_top > ts::kMaxTop) return TS_ERR_INVALID;
  if (p->dtype != TS_BF16 && p->dtype != TS_F32) return TS_ERR_UNSUPPORTED;
  if (p->vocab > (1 << 30) || p->n_rows > (1 << 30)) return TS_ERR_UNSUPPORTED;      // the kernel counts both, and a few rows on, in 32 bits
  if (p->n_rows == 0) return TS_OK;
  const uintptr_t elem = p->dtype == TS_BF16 ? 2 : 4;
  if (!p->logits || (uintptr_t)p->logits % elem) return TS_ERR_INVALID;
  if (p->n_given > 0 && (!p->tokens || !p->logprob)) return TS_ERR_INVALID;
  if (p->n_top > 0 && (!p->top_token || !p->top_logprob)) return TS_ERR_INVALID;
  const uintptr_t words = (uintptr_t)p->scale | (uintptr_t)p->tokens | (uintptr_t)p->logprob | (uintptr_t)p->rank | (uintptr_t)p->entropy |
                          (uintptr_t)p->top_logprob | (uintptr_t)p->top_token;
  if (words & 3u) return TS_ERR_INVALID;
  if (cudaSetDevice(p->device) != cudaSuccess) return TS_ERR_CUDA;
  ts::Args a = {p->logits, (long long)p->row_stride, p->scale, p->tokens, p->logprob, p->entropy, p->top_logprob, p->rank, p->top_token, p->vocab,
                p->n_given, p->n_top};
  int n_sms = 0;
  if (cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess) return TS_ERR_CUDA;
  // Few rows: a row is shared, as long as every thread still has a 16-byte block.
  int parts = 1;
  const long long blocks = (long long)p->vocab * (long long)elem / 16;
  while (parts < ts::kMaxCluster && (long long)p->n_rows * parts <= n_sms && blocks / (parts * 2) >= ts::kThreads) parts *= 2;
  if ((long long)p->n_rows * parts > INT32_MAX) return TS_ERR_UNSUPPORTED;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const cudaError_t e = p->dtype == TS_BF16 ? ts::launch<uint16_t>(a, p->n_rows, parts, n_sms, stream)
                                              : ts::launch<float>(a, p->n_rows, parts, n_sms, stream);
  return e == cudaSuccess ? TS_OK : TS_ERR_CUDA;
}
