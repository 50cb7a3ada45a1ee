// Log probabilities of given tokens, their ranks, the entropy and the best alternatives of rows of logits (sm_100a).
//
//     y = scale * x,  lse = log sum_j exp y_j,  logprob(t) = y_t - lse,  H = lse - sum_j p_j y_j,
//     rank(t) = number of tokens in front of t in the order (x descending, index ascending); the first n of that order.
//
// One pass over the logits (they are what has to be read; everything else is a few values a row). A row is a thread block's, or
// a cluster's of up to eight where there are few rows: the blocks leave their sums in the first one's shared memory. Per element
// a thread adds up e^d and (x - ref) e^d, d = scale (x - ref), against a logit ref that only moves when one exceeds it by a factor
// of 2^64 (any reference is exact; fp32 has the range), and counts what lies in front of the given tokens.
//
// Alternatives cost the pass no more than its maximum: every thread keeps the largest logit of its own part of the row and where
// that part first has it. The n best tokens lie in the n parts that come first by (that logit, that place), since each of these
// holds a token at least as far in front as the last part's first one. Only those parts are read again (from L2), and of them only
// what is not behind the last part's largest is sorted.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <math_constants.h>

#include "../../include/tokenscale.h"
#include "ts_internal.h"

namespace ts {
namespace {

namespace cg = cooperative_groups;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxTop = 32, kMaxGiven = 8, kMaxCluster = 8;
constexpr float kMove = 64.f;            // log2: how far a value may exceed the reference of its sum
constexpr float kLowest = -200.f;        // log2 of a weight that is 0 in fp32 anyway (-inf's among them): keeps 0 * inf out of the entropy

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
  __syncthreads();
  for (int half = 8; half > 0; half >>= 1) {
    if (half >= n_lists) continue;                   // the same for all
    if (warp >= half && warp < 2 * half) best[warp * 32 + lane] = k;
    __syncthreads();
    if (warp < half) k = warp_merge(k, best[(warp + half) * 32 + lane], lane);
    __syncthreads();
  }
  if (warp == 0) best[lane] = k;
  __syncthreads();
}
static_assert(kWarps == 16, "the lists of two times eight warps are merged");

struct Stats {                                       // of a part of a row, d = (x - ref) * scale
  float ref, s, t;                                   // a logit to refer to (any is exact), sum e^d, sum (x - ref) e^d
};
__device__ __forceinline__ void move_ref(Stats& a, float ref, float to_log2) {
  const float by = a.ref - ref, f = ex2(by * to_log2);
  if (a.s == 0.f || f == 0.f) {                      // nothing yet, or nothing that counts (ref = -inf before the first number)
    a.t = 0.f;
    a.s = a.s == a.s ? 0.f : a.s;                    // a NaN stays
  } else {
    a.t = f * fmaf(a.s, by, a.t);
    a.s *= f;
  }
  a.ref = ref;
}
__device__ __forceinline__ Stats join(Stats a, Stats b, float to_log2) {
  const float ref = fmaxf(a.ref, b.ref);
  if (a.ref != ref) move_ref(a, ref, to_log2);
  if (b.ref != ref) move_ref(b, ref, to_log2);
  return Stats{ref, a.s + b.s, a.t + b.t};
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

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
};
template <>
struct Vec<uint16_t> {                               // bf16 bits
  static constexpr int N = 8;
  static __device__ __forceinline__ float load(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// GIVEN: how many given tokens the loop counts for (kMaxGiven: any number).
template <typename T, int GIVEN, bool TOP>
__global__ void __launch_bounds__(kThreads, 3) logprobs_kernel(const Args a) {
  constexpr int N = Vec<T>::N, kUnroll = 4;
  __shared__ uint64_t lists[kWarps * 32];
  __shared__ uint64_t cand[kThreads];
  __shared__ Stats warp_stats[kWarps], row_stats[kMaxCluster];
  __shared__ int32_t warp_count[kWarps][kMaxGiven], row_count[kMaxCluster][kMaxGiven];
  __shared__ uint64_t row_lists[kMaxCluster * 32];
  __shared__ int32_t n_cand;
  cg::cluster_group cluster = cg::this_cluster();
  const int n_parts = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int row = blockIdx.x / n_parts;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  pdl_wait();

  const T* x0 = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.row_stride;
  const float scale = a.scale ? a.scale[row] : 1.f, to_log2 = scale * 1.4426950408889634f;
  const float lowest = kLowest / to_log2;
  // The row as 16-byte blocks of memory: block b holds the tokens b * N - off .. + N - 1, the first and last one maybe fewer.
  const int off = (int)(((uintptr_t)x0 & 15u) / sizeof(T));
  const T* blocks = x0 - off;
  const int n_blocks = (a.vocab + off + N - 1) / N;
  const int b_begin = (int)((long long)n_blocks * part / n_parts), b_end = (int)((long long)n_blocks * (part + 1) / n_parts);

  constexpr int kCount = GIVEN;
  const int n_given = GIVEN < kMaxGiven ? GIVEN : a.n_given;
  float given_x[kCount > 0 ? kCount : 1];            // of a given token: its logit, the next number above, its block
  int given_block[kCount > 0 ? kCount : 1], count[kCount > 0 ? kCount : 1];
#pragma unroll
  for (int j = 0; j < kCount; ++j) {
    const int tok = j < n_given ? a.tokens[(size_t)row * n_given + j] : -1;
    const bool real = (unsigned)tok < (unsigned)a.vocab;
    given_x[j] = real ? Vec<T>::load(x0 + tok) : CUDART_NAN_F;   // nothing is in front of a NaN, see below
    given_block[j] = real ? (tok + off) / N : -1;
    count[j] = 0;
  }

  Stats st = {-CUDART_INF_F, 0.f, 0.f};
  float best = -CUDART_INF_F;                        // this thread's largest logit and the first block that has it
  int best_block = -1;
  auto take = [&](const float (&x)[N], int b) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) mx = fmaxf(mx, x[i]);  // a NaN only where all are
    if (TOP && (mx > best || (best_block < 0 && mx == mx))) {
      best = mx;
      best_block = b;
    }
    if ((mx - st.ref) * to_log2 > kMove) move_ref(st, mx, to_log2);       // the first number too: the reference is -inf before it
    const float ref = st.ref == -CUDART_INF_F ? 0.f : st.ref;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = x[i] - ref, e = ex2(d * to_log2);
      st.s += e;
      st.t = fmaf(e, fmaxf(d, lowest), st.t);
    }
#pragma unroll
    for (int j = 0; j < kCount; ++j) {
      if (j >= n_given) break;
      if (b == given_block[j]) {                     // index by index in the token's own block
        const int tok = a.tokens[(size_t)row * n_given + j];
#pragma unroll
        for (int i = 0; i < N; ++i) count[j] += x[i] > given_x[j] || (x[i] == given_x[j] && b * N - off + i < tok);
      } else {
        const bool front = b < given_block[j];       // equal logits count in front of the token
#pragma unroll
        for (int i = 0; i < N; ++i) count[j] += front ? x[i] >= given_x[j] : x[i] > given_x[j];
      }
    }
  };
  // A block that the row fills in part: token by token; what is outside counts as -inf, but for nothing else.
  auto take_partial = [&](int b) {
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      const int t = b * N - off + i;
      if (t < 0 || t >= a.vocab) continue;
      const float x = Vec<T>::load(blocks + (size_t)b * N + i);
      if (TOP && (x > best || (best_block < 0 && x == x))) {
        best = x;
        best_block = b;
      }
      if ((x - st.ref) * to_log2 > kMove) move_ref(st, x, to_log2);
      const float d = x - (st.ref == -CUDART_INF_F ? 0.f : st.ref), e = ex2(d * to_log2);
      st.s += e;
      st.t = fmaf(e, fmaxf(d, lowest), st.t);
#pragma unroll
      for (int j = 0; j < kCount; ++j)
        if (j < n_given) count[j] += x > given_x[j] || (x == given_x[j] && t < a.tokens[(size_t)row * n_given + j]);
    }
  };
  auto whole = [&](int b) { return b * N >= off && (b + 1) * N - off <= a.vocab; };
  // ------------------------------------------------------------------------ the pass
#pragma unroll 1
  for (int b0 = b_begin + tid; b0 < b_end; b0 += kUnroll * kThreads) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int b = b0 + u * kThreads;
      if (b < b_end && whole(b)) v[u] = load16(blocks + (size_t)b * N);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int b = b0 + u * kThreads;
      if (b >= b_end) break;
      if (whole(b)) {
        float x[N];
        Vec<T>::unpack(v[u], x);
        take(x, b);
      } else {
        take_partial(b);
      }
    }
  }
  // ------------------------------------------------------------------------ sums of the block
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) {
    Stats o;
    o.ref = __shfl_xor_sync(0xffffffffu, st.ref, sh);
    o.s = __shfl_xor_sync(0xffffffffu, st.s, sh);
    o.t = __shfl_xor_sync(0xffffffffu, st.t, sh);
    st = join(st, o, to_log2);
  }
#pragma unroll
  for (int j = 0; j < kCount; ++j) {
    if (j >= n_given) break;
    const int sum = __reduce_add_sync(0xffffffffu, count[j]);
    if (lane == 0) warp_count[warp][j] = sum;
  }
  if (lane == 0) warp_stats[warp] = st;
  if (tid == 0) n_cand = 0;

  if constexpr (TOP) {
    // ---------------------------------------------------------------------- alternatives of the block
    // the parts of the n threads that come first; a part is known by its first block
    const uint64_t mine = best_block < 0 ? 0 : key_of(best, (uint32_t)best_block);
    const uint64_t sorted = warp_sort(mine, lane);
    merge_lists(sorted, lists, kWarps, warp, lane);
    const uint64_t last = lists[a.n_top - 1];        // 0: fewer parts than that hold a number
    const float last_x = last ? from_ordered((uint32_t)(last >> 32)) : -CUDART_INF_F;
    const int last_block = last ? (int)place_of(last) : INT32_MAX;
    const int per_part = (b_end - b_begin + kThreads - 1) / kThreads;
    // token i of the block that is item `it`'s: its key, 0 where it is none or behind the last part's largest
    auto block_of = [&](int it) {
      const int p = it / per_part;
      if (p >= a.n_top || lists[p] == 0) return -1;
      const int b = b_begin + ((int)place_of(lists[p]) - b_begin) % kThreads + (it % per_part) * kThreads;
      return b < b_end ? b : -1;
    };
    auto key_at = [&](float x, int b, int i) -> uint64_t {
      const int t = b * N - off + i;
      if (t < 0 || t >= a.vocab || !(x > last_x || (x == last_x && b <= last_block))) return 0;
      return key_of(x, (uint32_t)t);
    };
    const int n_items = a.n_top * per_part;
    for (int it = tid; it < n_items; it += kThreads) {
      const int b = block_of(it);
      if (b < 0) continue;
      float x[N];
      if (whole(b)) {
        Vec<T>::unpack(load16(blocks + (size_t)b * N), x);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int t = b * N - off + i;
          x[i] = t >= 0 && t < a.vocab ? Vec<T>::load(blocks + (size_t)b * N + i) : CUDART_NAN_F;
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint64_t k = key_at(x[i], b, i);
        if (k) {
          const int at = atomicAdd(&n_cand, 1);
          if (at < kThreads) cand[at] = k;
        }
      }
    }
    __syncthreads();
    const int n = n_cand;
    if (n <= kThreads) {
      const int n_lists = (n + 31) / 32;
      uint64_t k = 0;
      if (warp < n_lists) k = warp_sort(tid < n ? cand[tid] : 0, lane);
      merge_lists(k, lists, n_lists, warp, lane);
    } else {
      // So many only where a part has the larger share of a row's best tokens: all of these parts' tokens, as many at a time as
      // there are threads, next to the best so far.
      if (tid < 32) cand[tid] = lists[tid];          // the parts: `lists` is needed
      __syncthreads();
      uint64_t top32 = 0;                            // warp 0: the best so far
      const int n_elems = n_items * N;
      for (int e0 = 0; e0 < n_elems; e0 += kThreads) {
        const int e = e0 + tid, it = e / N, i = e % N;
        uint64_t k = 0;
        const int p = it / per_part;
        if (e < n_elems && p < a.n_top && cand[p] != 0) {
          const int b = b_begin + ((int)place_of(cand[p]) - b_begin) % kThreads + (it % per_part) * kThreads;
          const int t = b * N - off + i;
          if (b < b_end && t >= 0 && t < a.vocab) k = key_at(Vec<T>::load(x0 + t), b, i);
        }
        merge_lists(warp_sort(k, lane), lists, kWarps, warp, lane);
        if (warp == 0) top32 = warp_merge(top32, lists[lane], lane);
      }
      __syncthreads();
      if (warp == 0) lists[lane] = top32;
      __syncthreads();
    }
  }
  __syncthreads();
  // ------------------------------------------------------------------------ the blocks of the row meet in the first one
  if (tid == 0) {
    Stats all = warp_stats[0];
    for (int w = 1; w < kWarps; ++w) all = join(all, warp_stats[w], to_log2);
    *cluster.map_shared_rank(&row_stats[part], 0) = all;
  }
  if (tid < n_given) {
    int sum = 0;
    for (int w = 0; w < kWarps; ++w) sum += warp_count[w][tid];
    *cluster.map_shared_rank(&row_count[part][tid], 0) = sum;
  }
  if (TOP && n_parts > 1 && warp == 1) *cluster.map_shared_rank(&row_lists[part * 32 + lane], 0) = lists[lane];
  if (n_parts > 1) cluster.sync(); else __syncthreads();
  if (part != 0) return;
  Stats all = row_stats[0];
  for (int p = 1; p < n_parts; ++p) all = join(all, row_stats[p], to_log2);
  // a row without a finite logit has no distribution: every log probability is -inf, the entropy 0
  const bool none = all.s == 0.f;
  const float log_sum = logf(all.s);
  auto logprob = [&](float x) { return none ? -CUDART_INF_F : fmaf(x - all.ref, scale, -log_sum); };
  if (tid == 0 && a.entropy) a.entropy[row] = none ? 0.f : fmaf(-scale, all.t / all.s, log_sum);
  if (tid < n_given) {
    const int tok = a.tokens[(size_t)row * n_given + tid];
    const bool real = (unsigned)tok < (unsigned)a.vocab;
    const float x = real ? Vec<T>::load(x0 + tok) : CUDART_NAN_F;
    a.logprob[(size_t)row * n_given + tid] = x == x ? logprob(x) : CUDART_NAN_F;
    if (a.rank) {
      int sum = 0;
      for (int p = 0; p < n_parts; ++p) sum += row_count[p][tid];
      a.rank[(size_t)row * n_given + tid] = x == x ? sum : -1;
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
}

template <typename T, int GIVEN, bool TOP>
cudaError_t launch_t(const Args& a, int n_rows, int n_parts, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n_rows * n_parts));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)n_parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<T, GIVEN, TOP>, a);
}
template <typename T>
cudaError_t launch(const Args& a, int n_rows, int n_parts, cudaStream_t stream) {
  const bool top = a.n_top > 0;
  if (a.n_given == 0) return top ? launch_t<T, 0, true>(a, n_rows, n_parts, stream) : launch_t<T, 0, false>(a, n_rows, n_parts, stream);
  if (a.n_given == 1) return top ? launch_t<T, 1, true>(a, n_rows, n_parts, stream) : launch_t<T, 1, false>(a, n_rows, n_parts, stream);
  return top ? launch_t<T, kMaxGiven, true>(a, n_rows, n_parts, stream) : launch_t<T, kMaxGiven, false>(a, n_rows, n_parts, stream);
}

}  // namespace
}  // namespace ts

extern "C" int ts_token_logprobs(const ts_logprobs* p, void* cuda_stream) {
  if (!p) return TS_ERR_INVALID;
  if (p->n_rows < 0 || p->vocab < 1 || p->row_stride < p->vocab) return TS_ERR_INVALID;
  if (p->n_given < 0 || p->n_given > ts::kMaxGiven || p->n_top < 0 || p->n_top > ts::kMaxTop) return TS_ERR_INVALID;
  if (p->dtype != TS_BF16 && p->dtype != TS_F32) return TS_ERR_UNSUPPORTED;
  if (p->vocab > (1 << 30)) return TS_ERR_UNSUPPORTED;
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
  // Few rows: a row is shared, as long as every thread still has a 16-byte block.
  int parts = 1;
  const long long blocks = (long long)p->vocab * (long long)elem / 16;
  while (parts < ts::kMaxCluster && (long long)p->n_rows * parts * 2 <= 296 && blocks / (parts * 2) >= ts::kThreads) parts *= 2;
  if ((long long)p->n_rows * parts > INT32_MAX) return TS_ERR_UNSUPPORTED;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const cudaError_t e = p->dtype == TS_BF16 ? ts::launch<uint16_t>(a, p->n_rows, parts, stream) : ts::launch<float>(a, p->n_rows, parts, stream);
  return e == cudaSuccess ? TS_OK : TS_ERR_CUDA;
}
