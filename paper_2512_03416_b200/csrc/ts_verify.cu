// Drafted tokens verified against the model's probabilities from given random numbers (sm_100a).
//
// A request's nodes form a tree; row i of the logits is the model's distribution behind node i, p = softmax(scale x), and the children
// of i are the tokens drafted there, drawn from q = softmax(draft_scale d_i) or, without draft logits, given (q = 1 at the token). At node i, with
// r_0 = p, the children are tried in order: child of token t is accepted if u q(t) < r_j(t), and the walk goes on there; else
// r_(j+1) = max(r_j - q, 0) / Z_j, or r_j without t. When none is left a token is drawn from r: the first whose cumulative sum exceeds
// u_sample times the whole. Whatever the draft, what is emitted is distributed as p.
//
// A request is a cluster's of up to eight thread blocks, which share every row in contiguous parts and take all decisions alike, each for
// itself, from sums exchanged through distributed shared memory. A row is read when the walk gets there: the rows of drafts that are not
// reached are never read.
//
// Decisions are those of 64 bits. The sums that a test of a first child needs are taken in fp32, to 2e-6; where u q and r are nearer to each
// other than that could tell, and for what comes behind a rejection (differences of p and q that are nearly alike), the row is summed
// again in 64 bits. The final draw always is: with 100000 tokens, borders of the cumulative sum lie so near to each other that an error of 1e-7
// would draw a neighbour of the token once in a hundred times. Its cumulative sums are kept per strip of the row; one warp then goes through
// the strip that holds the place.
// Sums are added up in a fixed order: equal calls give equal results.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>

#include "../../include/tokenscale.h"
#include "ts_internal.h"

namespace ts {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kTile = 256;               // logits of a warp at a time: eight neighbouring ones per lane
constexpr int kStrips = 512;             // of a block's part of a row
constexpr int kNodes = 64, kMaxCluster = 8;
constexpr int kWords = 767;              // requests of a launch
constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

struct VerifyParams {
  const void *logits, *draft;
  int64_t stride, draft_stride;
  const float *scale, *draft_scale;
  const int32_t *tokens, *parents;
  const float *u_accept, *u_sample;
  int32_t *emitted, *count, *path;
  float* logprob;
  int32_t vocab, cluster;
  int32_t first[kWords + 1];             // of each request's nodes
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ double ld_cluster(uint32_t addr) {
  double v;
  asm volatile("ld.shared::cluster.f64 %0, [%1];\n" : "=d"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;\n" ::: "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }
// Elements of a row from `at` on (at may be negative): -inf outside [0, n). `vec`: address at + row is 16-byte aligned.
__device__ __forceinline__ void load8(const __nv_bfloat16* row, int at, int n, bool vec, float (&x)[8]) {
  if (vec && at >= 0 && at + 8 <= n) {
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(row + at));
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (unsigned)(at + i) < (unsigned)n ? __bfloat162float(row[at + i]) : -CUDART_INF_F;
  }
}
__device__ __forceinline__ void load8(const float* row, int at, int n, bool vec, float (&x)[8]) {
  if (vec && at >= 0 && at + 8 <= n) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 w = __ldg(reinterpret_cast<const float4*>(row + at) + i);
      x[4 * i] = w.x; x[4 * i + 1] = w.y; x[4 * i + 2] = w.z; x[4 * i + 3] = w.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (unsigned)(at + i) < (unsigned)n ? row[at + i] : -CUDART_INF_F;
  }
}

// A distribution's sum: weights 2^((x - max) c). (As x c - max c in one rounding they would overflow for the largest logits.)
struct Sum {
  float max, s;
};
__device__ __forceinline__ float weight(float x, float max, float c) { return ex2((x - max) * c); }
__device__ __forceinline__ void add8(Sum& a, const float (&x)[8], float c) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, x[i]);
  if (m > a.max) {
    a.s *= weight(a.max, m, c);          // of nothing: 2^-inf
    a.max = m;
  }
  if (a.max == -CUDART_INF_F) {          // nothing but -inf and NaN yet
#pragma unroll
    for (int i = 0; i < 8; ++i) a.s += x[i] != x[i] ? x[i] : 0.f;
    return;
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += weight(x[i], a.max, c);
  a.s += s;
}
__device__ __forceinline__ void join(Sum& a, const Sum& b, float c) {
  if (b.max > a.max) {
    a.s = a.s * weight(a.max, b.max, c) + b.s;
    a.max = b.max;
  } else {
    a.s += b.max == -CUDART_INF_F ? b.s : b.s * weight(b.max, a.max, c);
  }
}
__device__ __forceinline__ Sum warp_join(Sum a, float c) {
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) {
    const Sum b = {__shfl_xor_sync(0xffffffffu, a.max, sh), __shfl_xor_sync(0xffffffffu, a.s, sh)};
    // both lanes add the same two in the same order
    const bool lower = !(threadIdx.x & sh);
    Sum lo = lower ? a : b;
    join(lo, lower ? b : a, c);
    a = lo;
  }
  return a;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int sh = 16; sh > 0; sh >>= 1) v += __shfl_xor_sync(0xffffffffu, v, sh);
  return v;
}

// The distribution behind a node in 64 bits.
struct Exact {
  double scale, top, inv, dscale, dtop, dinv;
};

template <typename T, bool DRAFT>
struct Walk {
  const VerifyParams& p;
  const int rank, tid, lane, warp;
  // shared memory
  double* strips;                        // [kStrips]
  double* norm;                          // [kNodes] 1 / Z of the rejections at this node
  int32_t* gone;                         // [kNodes] tokens rejected at this node (no draft)
  double* warps;                         // [kWarps][2]
  double* box;                           // [2][4]: what the blocks exchange, by turns
  int32_t* found;
  int turn = 0;
  const T* row;
  const T* drow;
  int shift, tile0, tile1;               // the row's first 16-byte boundary is `shift` elements in front of it; this block's tiles
  bool dvec;
  int rejected = 0;

  __device__ Walk(const VerifyParams& p_, int rank_) : p(p_), rank(rank_), tid(threadIdx.x), lane(threadIdx.x & 31), warp(threadIdx.x >> 5) {}

  __device__ void at_row(int64_t r) {
    row = static_cast<const T*>(p.logits) + r * p.stride;
    shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    if (DRAFT) {
      drow = static_cast<const T*>(p.draft) + r * p.draft_stride;
      dvec = (int)((reinterpret_cast<uintptr_t>(drow) & 15) / sizeof(T)) == shift;
    }
    const int tiles = (p.vocab + shift + kTile - 1) / kTile;
    tile0 = (int)((int64_t)tiles * rank / p.cluster);
    tile1 = (int)((int64_t)tiles * (rank + 1) / p.cluster);
    rejected = 0;
  }
  __device__ int place(int tile) const { return tile * kTile + lane * 8 - shift; }

  // Sums over the cluster of up to two values per block, by every thread.
  __device__ void total(double a, double b, double& ta, double& tb) {
    a = warp_sum(a);
    b = warp_sum(b);
    __syncthreads();                     // the former use of `warps` is over
    if (lane == 0) {
      warps[2 * warp] = a;
      warps[2 * warp + 1] = b;
    }
    __syncthreads();
    ta = tb = 0.0;
    for (int w = 0; w < kWarps; ++w) {
      ta += warps[2 * w];
      tb += warps[2 * w + 1];
    }
    if (p.cluster == 1) return;
    double* mine = box + turn * 4;
    if (tid == 0) {
      mine[0] = ta;
      mine[1] = tb;
    }
    cluster_sync();
    ta = tb = 0.0;
    for (int r = 0; r < p.cluster; ++r) {
      const uint32_t from = mapa(smem_at(mine), r);
      ta += ld_cluster(from);
      tb += ld_cluster(from + 8);
    }
    turn ^= 1;
  }

  // A part's sum over the block; which: 0 the model's, 1 the draft's, into one turn of the box.
  __device__ Sum whole(Sum a, float c, int which) {
    a = warp_join(a, c);
    float* f = reinterpret_cast<float*>(strips);
    __syncthreads();
    if (lane == 0) {
      f[warp * 2] = a.max;
      f[warp * 2 + 1] = a.s;
    }
    __syncthreads();
    a = Sum{-CUDART_INF_F, 0.f};
    for (int w = 0; w < kWarps; ++w) join(a, Sum{f[w * 2], f[w * 2 + 1]}, c);
    double* mine = box + turn * 4 + which * 2;
    if (p.cluster > 1 && tid == 0) {
      mine[0] = a.max;
      mine[1] = a.s;
    }
    return a;
  }
  __device__ Sum gathered(Sum a, float c, int which) {
    if (p.cluster == 1) return a;
    a = Sum{-CUDART_INF_F, 0.f};
    for (int r = 0; r < p.cluster; ++r) {
      const uint32_t from = mapa(smem_at(box + turn * 4 + which * 2), r);
      join(a, Sum{(float)ld_cluster(from), (float)ld_cluster(from + 8)}, c);
    }
    return a;
  }
  // The row's sums in fp32.
  __device__ void sums(float c, float dc, bool children, Sum& a, Sum& b) {
    const bool both = DRAFT && children;
    a = b = Sum{-CUDART_INF_F, 0.f};
    for (int tile = tile0 + warp; tile < tile1; tile += kWarps) {
      float x[8], y[8];
      load8(row, place(tile), p.vocab, true, x);
      if (both) load8(drow, place(tile), p.vocab, dvec, y);
      add8(a, x, c);
      if (both) add8(b, y, dc);
    }
    a = whole(a, c, 0);
    if (both) b = whole(b, dc, 1);
    if (p.cluster > 1) cluster_sync();
    a = gathered(a, c, 0);
    if (both) b = gathered(b, dc, 1);
    if (p.cluster > 1) turn ^= 1;
  }
  // The same in 64 bits.
  __device__ void exact(Exact& e) {
    double s = 0.0, t = 0.0;
    for (int tile = tile0 + warp; tile < tile1; tile += kWarps) {
      float x[8], y[8];
      load8(row, place(tile), p.vocab, true, x);
      if (DRAFT) load8(drow, place(tile), p.vocab, dvec, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s += exp(fma((double)x[i], e.scale, -e.top));
        if (DRAFT) t += exp(fma((double)y[i], e.dscale, -e.dtop));
      }
    }
    double ts, tt;
    total(s, t, ts, tt);
    e.inv = 1.0 / ts;
    e.dinv = DRAFT ? 1.0 / tt : 0.0;
  }
  // What is left of the probability of a token whose logits are x (the model's) and y (the draft's) behind `rejections`, in units that are the
  // same for all tokens.
  __device__ double left(const Exact& e, float x, float y, int rejections) const {
    double r = exp(fma((double)x, e.scale, -e.top)) * e.inv;
    if (DRAFT && rejections > 0) {
      const double q = exp(fma((double)y, e.dscale, -e.dtop)) * e.dinv;
      for (int i = 0; i < rejections; ++i)
        if (norm[i] > 0.0) r = fmax(r - q, 0.0) * norm[i];
    }
    return r;
  }
  __device__ bool is_gone(int token) const {
    for (int i = 0; i < rejected; ++i)
      if (gone[i] == token) return true;
    return false;
  }
  __device__ void left8(const Exact& e, int tile, double (&w)[8]) const {
    float x[8], y[8];
    const int at = place(tile);
    load8(row, at, p.vocab, true, x);
    if (DRAFT && rejected > 0) load8(drow, at, p.vocab, dvec, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = left(e, x[i], DRAFT ? y[i] : 0.f, rejected);
    if (!DRAFT && rejected > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (is_gone(at + i)) w[i] = 0.0;
    }
  }
  // Z behind one more rejection: norm[rejected] is set, by all.
  __device__ void reject(const Exact& e) {
    double s = 0.0, ts, unused;
    for (int tile = tile0 + warp; tile < tile1; tile += kWarps) {
      float x[8], y[8];
      load8(row, place(tile), p.vocab, true, x);
      load8(drow, place(tile), p.vocab, dvec, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += fmax(left(e, x[i], y[i], rejected) - exp(fma((double)y[i], e.dscale, -e.dtop)) * e.dinv, 0.0);
    }
    total(s, 0.0, ts, unused);
    if (tid == 0) norm[rejected] = ts > 0.0 ? 1.0 / ts : 0.0;
    __syncthreads();
    ++rejected;
  }
  // The token at u of what is left; -1 where nothing is.
  __device__ int draw(const Exact& e, float u) {
    const int tiles = tile1 - tile0, per = max(1, (tiles + kStrips - 1) / kStrips), n = (tiles + per - 1) / per;
    double sum = 0.0;
    __syncthreads();                     // `strips` also holds what sums() exchanged
    for (int s = warp; s < n; s += kWarps) {
      double v = 0.0;
      for (int tile = tile0 + s * per; tile < min(tile1, tile0 + (s + 1) * per); ++tile) {
        double w[8];
        left8(e, tile, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v += w[i];
      }
      v = warp_sum(v);
      if (lane == 0) strips[s] = v;
    }
    __syncthreads();
    for (int s = 0; s < n; ++s) sum += strips[s];          // every thread the same
    double* mine = box + turn * 4;
    double front = 0.0, all = sum;
    int last = 0, holder = -1;           // the last block with anything; the one that holds the place
    if (p.cluster > 1) {
      if (tid == 0) mine[0] = sum;
      cluster_sync();
      all = 0.0;
      for (int r = 0; r < p.cluster; ++r) all += ld_cluster(mapa(smem_at(mine), r));
      const double want = (double)u * all;
      double cum = 0.0;
      for (int r = 0; r < p.cluster; ++r) {
        const double v = ld_cluster(mapa(smem_at(mine), r));
        if (v > 0.0) last = r;
        if (holder < 0 && cum + v > want) {
          holder = r;
          front = cum;
        }
        cum += v;
      }
      turn ^= 1;
    } else {
      holder = 0;
    }
    const bool beyond = holder < 0;      // u not below 1, or a rounding: the last token with anything
    if (beyond) holder = last;
    if (!(all > 0.0) || !(all < CUDART_INF)) return -1;
    if (holder == rank && warp == 0) {
      const double want = beyond ? CUDART_INF : (double)u * all - front;
      // the strip, by all lanes alike
      double cum = 0.0;
      int strip = -1, final = -1;
      double before = 0.0;
      for (int s = 0; s < n; ++s) {
        const double v = strips[s];
        if (v > 0.0) final = s;
        if (strip < 0 && cum + v > want) {
          strip = s;
          before = cum;
        }
        cum += v;
      }
      double place_in = want - before;
      if (strip < 0) {
        strip = final;
        place_in = CUDART_INF;
      }
      int token = -1, some = -1;         // found; the last one with anything
      cum = 0.0;
      for (int tile = tile0 + strip * per; tile < min(tile1, tile0 + (strip + 1) * per) && token < 0; ++tile) {
        double w[8], mine8 = 0.0;
        left8(e, tile, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) mine8 += w[i];
        double upto = mine8;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
          const double o = __shfl_up_sync(0xffffffffu, upto, sh);
          if (lane >= sh) upto += o;
        }
        double c = cum + (upto - mine8);
        int hit = 0x7fffffff, any = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          c += w[i];
          if (w[i] > 0.0) {
            any = place(tile) + i;
            if (c > place_in && hit == 0x7fffffff) hit = any;
          }
        }
        hit = __reduce_min_sync(0xffffffffu, hit);
        any = __reduce_max_sync(0xffffffffu, any);
        if (any >= 0) some = any;
        if (hit != 0x7fffffff) token = hit;
        cum += __shfl_sync(0xffffffffu, upto, 31);
      }
      if (token < 0) token = some;
      if (lane == 0) *found = token;
    }
    if (p.cluster > 1) cluster_sync(); else __syncthreads();
    int token;
    asm volatile("ld.shared::cluster.s32 %0, [%1];\n" : "=r"(token) : "r"(mapa(smem_at(found), holder)));
    return token;
  }
};

template <typename T, bool DRAFT>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyParams p) {
  __shared__ double strips[kStrips], norm[kNodes], warps[kWarps * 2], box[8];
  __shared__ int32_t gone[kNodes], token_of[kNodes], parent_of[kNodes], found;
  __shared__ float chance_of[kNodes];
  const int request = blockIdx.x / p.cluster, rank = blockIdx.x % p.cluster;
  Walk<T, DRAFT> w(p, rank);
  w.strips = strips; w.norm = norm; w.gone = gone; w.warps = warps; w.box = box; w.found = &found;
  const int first = p.first[request], nodes = p.first[request + 1] - first, tid = threadIdx.x;
  pdl_launch_dependents();
  pdl_wait();
  if (tid < nodes) {
    token_of[tid] = p.tokens[first + tid];
    parent_of[tid] = p.parents[first + tid];
    chance_of[tid] = p.u_accept[first + tid];
  }
  __syncthreads();
  if (p.cluster > 1) cluster_sync();     // all blocks of the cluster run: they may be written to and read
  int cur = 0, emitted = 0;
  for (;;) {
    const int64_t r = first + cur;
    const float scale = p.scale ? p.scale[r] : 1.f, dscale = DRAFT && p.draft_scale ? p.draft_scale[r] : 1.f;
    const float c = scale * kLog2e, dc = dscale * kLog2e;
    w.at_row(r);
    bool children = false;               // the draft's row of a node without any is not read
    for (int j = cur + 1; j < nodes; ++j) children = children || (parent_of[j] == cur && (unsigned)token_of[j] < (unsigned)p.vocab);
    Sum a, b;
    w.sums(c, dc, children, a, b);
    bool valid = a.s > 0.f && a.s < CUDART_INF_F;
    if (DRAFT && children) valid = valid && b.s > 0.f && b.s < CUDART_INF_F;
    int chosen = -1, out = -1;
    if (valid) {
      Exact e;
      e.scale = scale; e.top = (double)a.max * scale; e.inv = 1.0;
      e.dscale = dscale; e.dtop = DRAFT && children ? (double)b.max * dscale : 0.0; e.dinv = 0.0;
      bool precise = false;
      float rest = 1.f;                  // no draft: what the rejected tokens leave
      double rest64 = 1.0;
      bool pending = false;              // draft: a rejection whose Z is not summed yet
      for (int j = cur + 1; j < nodes; ++j) {
        if (parent_of[j] != cur) continue;
        const int t = token_of[j];
        if ((unsigned)t >= (unsigned)p.vocab) continue;
        const float u = chance_of[j], x = value(w.row + t), y = DRAFT ? value(w.drow + t) : 0.f;
        if (!DRAFT && w.is_gone(t)) {    // given twice: nothing is left of it
          continue;
        }
        bool accept;
        bool close = precise;
        if (!precise) {
          const float have = weight(x, a.max, c) / a.s;
          const float need = DRAFT ? u * (weight(y, b.max, dc) / b.s) : u * rest;
          accept = need < have;
          close = fabsf(need - have) <= (DRAFT ? 1e-5f * (need + have) : 1e-5f * (1 + w.rejected));
        }
        if (close) {
          if (!precise) {
            w.exact(e);
            precise = true;
            if (!DRAFT)
              for (int i = 0; i < w.rejected; ++i) rest64 -= w.left(e, value(w.row + gone[i]), 0.f, 0);
          }
          if (pending) w.reject(e);
          pending = false;
          const double have = w.left(e, x, y, w.rejected);
          accept = DRAFT ? (double)u * (exp(fma((double)y, e.dscale, -e.dtop)) * e.dinv) < have : (double)u * rest64 < have;
        }
        if (accept) {
          chosen = j;
          out = t;
          break;
        }
        if (DRAFT) {
          if (!precise) w.exact(e);
          precise = pending = true;
        } else {
          rest -= weight(x, a.max, c) / a.s;
          if (precise) rest64 -= w.left(e, x, 0.f, 0);
          __syncthreads();               // the others may still look through the list
          if (tid == 0) gone[w.rejected] = t;
          ++w.rejected;
          __syncthreads();
        }
      }
      if (chosen < 0) {
        if (pending) {                   // its Z is a factor of all that is left: not needed, unless nothing is
          __syncthreads();
          if (tid == 0) norm[w.rejected] = 1.0;
          ++w.rejected;
          __syncthreads();
        }
        out = w.draw(e, p.u_sample[request]);
        if (out < 0 && pending) {        // p = q up to roundings: as if not rejected
          --w.rejected;
          out = w.draw(e, p.u_sample[request]);
        }
      }
    }
    if (rank == 0 && tid == 0) {
      const bool some = out >= 0;
      p.emitted[first + emitted] = out;
      p.path[first + emitted] = first + cur;
      p.logprob[first + emitted] = some ? ((value(w.row + out) - a.max) * c - log2f(a.s)) * kLn2 : CUDART_NAN_F;
    }
    ++emitted;
    if (chosen < 0) break;
    cur = chosen;
  }
  if (rank == 0) {
    if (tid == 0) p.count[request] = emitted;
    for (int i = emitted + tid; i < nodes; i += kThreads) {
      p.emitted[first + i] = p.path[first + i] = -1;
      p.logprob[first + i] = 0.f;
    }
  }
  if (p.cluster > 1) cluster_sync();     // no block leaves while another one reads its sums
}

template <typename T, bool DRAFT>
cudaError_t launch(const VerifyParams& p, int requests, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(requests * p.cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, DRAFT>, p);
}

}  // namespace
}  // namespace ts

extern "C" int ts_verify_tokens(const ts_verify* v, void* cuda_stream) {
  using namespace ts;
  if (!v || v->n_requests < 0 || v->vocab < 1 || v->vocab > 1 << 30 || (v->dtype != TS_BF16 && v->dtype != TS_F32)) return TS_ERR_INVALID;
  if (v->n_requests == 0) return TS_OK;
  if (!v->n_nodes || !v->logits || !v->tokens || !v->parents || !v->u_accept || !v->u_sample || !v->emitted || !v->count || !v->path || !v->logprob)
    return TS_ERR_INVALID;
  const uintptr_t size = v->dtype == TS_BF16 ? 2 : 4;
  if (v->row_stride < v->vocab || (v->draft && v->draft_stride < v->vocab)) return TS_ERR_INVALID;
  if (((uintptr_t)v->logits | (uintptr_t)v->draft) & (size - 1)) return TS_ERR_INVALID;
  if (((uintptr_t)v->tokens | (uintptr_t)v->parents | (uintptr_t)v->u_accept | (uintptr_t)v->u_sample | (uintptr_t)v->scale | (uintptr_t)v->draft_scale |
       (uintptr_t)v->emitted | (uintptr_t)v->count | (uintptr_t)v->path | (uintptr_t)v->logprob) & 3u)
    return TS_ERR_INVALID;
  int64_t n = 0;
  for (int r = 0; r < v->n_requests; ++r) {
    if (v->n_nodes[r] < 1 || v->n_nodes[r] > kNodes) return TS_ERR_INVALID;
    n += v->n_nodes[r];
  }
  if (n > INT32_MAX / 2) return TS_ERR_INVALID;
  int n_sms = 0;
  if (cudaSetDevice(v->device) != cudaSuccess || cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, v->device) != cudaSuccess) return TS_ERR_CUDA;
  VerifyParams p;
  p.logits = v->logits; p.draft = v->draft; p.stride = v->row_stride; p.draft_stride = v->draft_stride;
  p.scale = v->scale; p.draft_scale = v->draft_scale; p.tokens = v->tokens; p.parents = v->parents;
  p.u_accept = v->u_accept; p.emitted = v->emitted; p.path = v->path; p.logprob = v->logprob; p.vocab = v->vocab;
  // as many blocks of a request as run at once, two per SM, each with a few tiles for every warp
  p.cluster = 1;
  while (p.cluster < kMaxCluster && (int64_t)v->n_requests * p.cluster * 2 <= 2 * n_sms && v->vocab / (p.cluster * 2) >= kTile * kWarps / 2) p.cluster *= 2;
  int32_t at = 0;
  for (int r0 = 0; r0 < v->n_requests; r0 += kWords) {
    const int some = std::min(kWords, v->n_requests - r0);
    p.u_sample = v->u_sample + r0;
    p.count = v->count + r0;
    for (int r = 0; r <= some; ++r) {
      p.first[r] = at;
      if (r < some) at += v->n_nodes[r0 + r];
    }
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    const cudaError_t e = v->dtype == TS_BF16 ? (v->draft ? launch<__nv_bfloat16, true>(p, some, stream) : launch<__nv_bfloat16, false>(p, some, stream))
                                              : (v->draft ? launch<float, true>(p, some, stream) : launch<float, false>(p, some, stream));
    if (e != cudaSuccess) return TS_ERR_CUDA;
  }
  return TS_OK;
}
