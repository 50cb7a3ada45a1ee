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
// reached are never read. Exchanges are stores that a barrier in the other block counts: a cluster barrier waits for the copies under way too, 2000 cycles.
//
// Decisions are those of 64 bits. The sums that a test of a first child needs are taken in fp32, to 8.6e-6 at worst (kMargin); where u q and r are nearer to each
// other than that could tell, and for what comes behind a rejection (differences of p and q that are nearly alike), the row is summed
// again in 64 bits. The final draw always is: with 100000 tokens, borders of the cumulative sum lie so near to each other that an error of 1e-7
// would draw a neighbour of the token once in a hundred times. Its cumulative sums are kept per strip of the row; one warp then goes through
// the strip that holds the place.
// Sums are added up in a fixed order: equal calls give equal results.
//
// A launch lasts as long as its longest request. A level of a walk (131072 bf16 logits and the draft's, 64 requests) takes 8 us: some 5 that the row's
// exponentials take an SM's four blocks, the rest joins; a rejection's pass in 64 bits 33, a draw without one 22, finding the token in its strip 2 to 5.
// Measured: 64 chains of 6 nodes 87 to 99 us (library exponentials, one tile at a time: 238), 48 trees of up to 25 nodes over 100003 fp32 logits 135 to 158
// (267), 256 trees of 8 given tokens 110 to 116 (300), one chain of 4 over 32000 20.5, a token each of 64 rows of 131072 28 to 36.
#include <cuda_bf16.h>
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

#include "../../include/tokenscale.h"
#include "ts_internal.h"
#include "ts_ptx.h"
#include "ts_tma.h"

namespace ts {
namespace {

constexpr int kTile = 256;               // logits of a warp at a time: eight neighbouring ones per lane
constexpr int kStrips = 256;             // of a block's part of a row
constexpr int kMostWarps = 16;
constexpr double kNothing = 1e-250;      // what is not more than this is as good as nothing
constexpr int kNodes = 64, kMaxCluster = 8, kValues = 6;
constexpr int kWords = 767;              // requests of a launch
constexpr double kLog2e = 1.4426950408889634;

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

// The distributions behind a node in 64 bits: probability of a logit x e^(x scale - top) inv.
struct Exact {
  double scale, top, inv, dscale, dtop, dinv;
};
// A block's part of a row.
struct Row {
  const void *row, *drow;                // the model's, the draft's
  int32_t vocab, shift;                  // the row's first 16-byte boundary is `shift` logits in front of it
  int32_t from, to;                      // tiles, counted from there
  int32_t dvec;                          // the draft's row has its boundaries at the same places
  int32_t per, n;                        // tiles of a strip, strips
};
__shared__ struct {
  double strips[3][kStrips];
  double part[kMostWarps][kValues];
  double box[2][kMaxCluster][kValues];   // the blocks' values, by turns
  double norm[kNodes];                   // 1 / Z of the rejections at this node
  Exact e;
  Row row;
  int32_t gone[kNodes];                  // tokens rejected at this node (no draft)
  int32_t token[kNodes], child[kNodes], sibling[kNodes];     // child, sibling: a node's first one, the next of the same parent; -1: none
  float chance[kNodes], scale[kNodes], dscale[kNodes];
  float4 sums[2][kMaxCluster];           // the blocks' sums in fp32 (reference, sum of the model; of the draft), by turns
  float4 part32[kMostWarps];
  // The same where all threads have one reference; by turns of their own. Also the warps' parts: where a request has one block, a level has one barrier, and
  // a warp that is through with it may write the next level's while another one still reads.
  float2 even[2][kMaxCluster], part_even[2][kMostWarps];
  uint64_t even_bar[2], box_bar[2];      // barriers of these turns and of box's: a phase each time, of the bytes that all blocks send
  int32_t lost;                          // a block of the cluster has not answered: never, and if it does, the request ends
  int32_t found;
  float c[kNodes], c_rest[kNodes], dc[kNodes], dc_rest[kNodes];
  float ref[kNodes], top[kNodes], sum[kNodes], rest_used[kNodes];      // of the rows walked: the sums (see Sum), the c_rest they were taken with
  int32_t out[kNodes], walked[kNodes];
} sh;

__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};\n" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int32_t v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;\n" ::"r"(addr), "r"(v) : "memory");
}
// Eight bytes into another block's shared memory, counted by a barrier there: neither side needs a fence for what else is under way.
__device__ __forceinline__ void st_async(uint32_t addr, uint32_t bar, float2 v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];\n" ::"r"(addr), "f"(v.x), "f"(v.y), "r"(bar) : "memory");
}
__device__ __forceinline__ void st_async(uint32_t addr, uint32_t bar, double v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.f64 [%0], %1, [%2];\n" ::"r"(addr), "d"(v), "r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;\n" ::: "memory");
}
__device__ __forceinline__ void sync_all(int cluster) {
  if (cluster > 1) cluster_sync(); else __syncthreads();
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ uint32_t bits(const __nv_bfloat16& x) { return *reinterpret_cast<const uint16_t*>(&x); }
__device__ __forceinline__ uint32_t bits(const float& x) { return __float_as_uint(x); }

// N neighbouring logits as they lie in memory, in words.
template <typename T, int N>
struct Raw {
  uint32_t w[N * sizeof(T) / 4];
};
// Those of a row from `at` on (at may be negative): -inf outside [0, n). `vec`: address at + row is a multiple of N logits' bytes, 16 at most.
template <int N, typename T>
__device__ __forceinline__ Raw<T, N> load(const T* row, int at, int n, bool vec) {
  constexpr int kWide = (int)(N * sizeof(T)) / 4;
  Raw<T, N> r;
  if (vec && at >= 0 && at + N <= n) {
    if constexpr (kWide == 2) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(row + at));
      r.w[0] = v.x; r.w[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < kWide / 4; ++i) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(row + at) + i);
        r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
      }
    }
  } else {
    constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80u : 0xff800000u;
    constexpr int kEach = 4 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kWide; ++i) {
      r.w[i] = 0;
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int a = at + i * kEach + k;
        r.w[i] |= ((unsigned)a < (unsigned)n ? bits(row[a]) : kNone) << (16 * k);
      }
    }
  }
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void unpack(const Raw<T, N>& r, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(r.w[i]);
    else x[i] = __uint_as_float(i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
  }
}

// A warp's tiles on their way: every lane copies its own eight logits (and the draft's) into shared memory, kRing tiles ahead of their use, and
// waits for its own copies only. kRing tiles of both rows are 8 KB a warp, 128 KB an SM under way.
template <typename T>
struct Ring {
  static constexpr int kLane = 8 * sizeof(T), kRing = 8192 / (2 * 32 * kLane);
  static constexpr int kBytes = 2 * kRing * 32 * kLane;      // of a warp
  const T *row, *drow;
  int vocab;
  bool both, dvec;
  uint32_t mine;                         // this lane's first slot
  __device__ Ring(const T* r, const T* d, int n, bool b, bool v, unsigned char* all, int warp, int lane)
      : row(r), drow(d), vocab(n), both(b), dvec(v), mine(smem_u32(all) + warp * kBytes + lane * kLane) {}
  __device__ __forceinline__ uint32_t slot(int k, int which) const { return mine + ((k % kRing) * 2 + which) * 32 * kLane; }
  __device__ __forceinline__ void copy(const T* from, uint32_t to) const {
#pragma unroll
    for (int i = 0; i < kLane / 16; ++i) cp_async16(to + 16 * i, from + i * (16 / sizeof(T)), 16);
  }
  __device__ __forceinline__ void by_hand(const T* from, int at, uint32_t to) const {      // the row's ends, rows of another alignment
    const Raw<T, 8> r = load<8>(from, at, vocab, false);
#pragma unroll
    for (int i = 0; i < kLane / 16; ++i)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(to + 16 * i), "r"(r.w[4 * i]), "r"(r.w[4 * i + 1]), "r"(r.w[4 * i + 2]), "r"(r.w[4 * i + 3]) : "memory");
  }
  // The k-th tile that is asked for, logits from `at` on in this lane. Called for every k in turn, `some` false behind the last one.
  __device__ __forceinline__ void ask(int k, int at, bool some) const {
    if (some) {
      if (at >= 0 && at + 8 <= vocab && (!both || dvec)) {
        copy(row + at, slot(k, 0));
        if (both) copy(drow + at, slot(k, 1));
      } else {
        by_hand(row, at, slot(k, 0));
        if (both) by_hand(drow, at, slot(k, 1));
      }
    }
    cp_async_commit();
  }
  __device__ __forceinline__ void get(int k, float (&x)[8], float (&y)[8]) const {
    cp_async_wait<kRing - 1>();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (which && !both) break;
      Raw<T, 8> r;
#pragma unroll
      for (int i = 0; i < kLane / 16; ++i)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(r.w[4 * i]), "=r"(r.w[4 * i + 1]), "=r"(r.w[4 * i + 2]), "=r"(r.w[4 * i + 3]) : "r"(slot(k, which) + 16 * i) : "memory");
      unpack(r, which ? y : x);
    }
  }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int sh_ = 16; sh_ > 0; sh_ >>= 1) v += __shfl_xor_sync(0xffffffffu, v, sh_);
  return v;
}
// Warp 0's n values go to every block of the cluster, as exchange number `turn`; arrived: they all are there.
__device__ __forceinline__ void publish(int n, double (&v)[kValues], int rank, int cluster, int turn, int lane) {
  double* const to = sh.box[turn & 1][rank];
  if (cluster > 1) {
    const uint32_t bar = smem_u32(&sh.box_bar[turn & 1]);
    if (lane == 0) mbar_expect_tx(bar, 8 * n * cluster);
    if (lane < cluster) {
      const uint32_t there = mapa(smem_u32(to), lane), there_bar = mapa(bar, lane);
#pragma unroll
      for (int i = 0; i < kValues; ++i)
        if (i < n) st_async(there + 8 * i, there_bar, v[i]);
    }
  } else if (lane == 0) {
#pragma unroll
    for (int i = 0; i < kValues; ++i)
      if (i < n) to[i] = v[i];
  }
}
__device__ __forceinline__ void arrived(int cluster, int turn) {
  if (cluster > 1 && threadIdx.x < 32 && !mbar_poll(smem_u32(&sh.box_bar[turn & 1]), turn >> 1 & 1)) sh.lost = 1;
  __syncthreads();
}

// ---- sums in fp32
__device__ __forceinline__ float sum8(const float (&v)[8]) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
// Weights 2^(x c - top), top = ref c rounded, the same for all: it is as if ref were another number nearby. Where it would not be (kHuge), top is a
// NaN, and weights are 2^((x - ref) c).
struct Sum {
  float ref, top, s;
};
constexpr float kLarge = 0x1p60f, kHuge = 0x1p20f, kSmall = 0x1p-60f;
// A thread adds up a tile's eight terms by pairs, up to kChain tiles one by one, and these sums in 64 bits, so that what is rounded does not grow with the row. A sum of n
// terms one by one may be off by n 2^-24 of itself, and terms of one size are off in one direction (4096 of them, a thread's share of 2^20 logits: 5.7e-5).
constexpr int kChain = 64;
// How near u q and r (times the sums), relative to both, may be for a test in fp32. One reference for all (2^-24 = 6e-8, ex2 2^-22): a sum's tile, chain, lanes, warps
// and blocks 96 x 6e-8, its exponents up to 64, rounded twice, 2.6e-6, ex2 0.2e-6: 8.6e-6. A single weight, exponents to 126: 5.5e-6. Three products: 0.2e-6. In all
// 1.43e-5. Given tokens: r's own sum of rejected weights adds as much again, which (1 + rejected) covers. Moving references: c is short by up to 2^-23 and differences of
// huge logits are rounded too, exponents to 126 2.4e-5; of a sum, 30 such terms 1.0e-5, moves and joins 1.0e-5, adding 5.6e-6: 5.1e-5 in all.
constexpr float kMargin = 1.5e-5f, kMarginMoving = 6e-5f;
__device__ __forceinline__ float top_of(float ref, float c) {
  const float top = __fmul_rn(ref, c);
  return fabsf(top) < kHuge ? top : CUDART_NAN_F;
}
__device__ __forceinline__ float exponent(float x, const Sum& a, float c, float c_rest) {
  return a.top == a.top ? fmaf(x, c_rest, fmaf(x, c, -a.top)) : (x - a.ref) * c;
}
__device__ __forceinline__ float weight(float x, const Sum& a, float c, float c_rest) { return ex2(exponent(x, a, c, c_rest)); }
// The sum in weights of another reference.
__device__ __forceinline__ float moved(const Sum& a, float ref, float top, float c) {
  if (a.ref == -CUDART_INF_F || a.ref == ref) return a.s;                    // nothing, or a NaN
  return a.s * ex2(a.top == a.top && top == top ? a.top - top : (a.ref - ref) * c);
}
// Where references move, they do so only for a logit whose weight would be more than 2^kAbove: the factor by which a sum then shrinks is rounded, and of
// two or three moves before all that is left of the sum, and of its error, is nothing. (A reference that follows the largest logit at once may move by a
// little with every tile, and the roundings of all these moves would add up.)
constexpr float kAbove = 20.f;
struct Moving {
  float ref, top;
  double s;
};
__device__ __noinline__ Moving add(Moving a, float x0, float x1, float x2, float x3, float x4, float x5, float x6, float x7, float c) {
  const float x[8] = {x0, x1, x2, x3, x4, x5, x6, x7};
  float m = x[0], w[8];
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, x[i]);
  if (a.ref == -CUDART_INF_F ? m > a.ref : (m - a.ref) * c > kAbove) {
    const float top = top_of(m, c);
    a = Moving{m, top, a.s * moved(Sum{a.ref, a.top, 1.f}, m, top, c)};
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = a.ref != -CUDART_INF_F ? weight(x[i], Sum{a.ref, a.top, 0.f}, c, 1e-37f) : x[i] != x[i] ? x[i] : 0.f;
  a.s += sum8(w);
  return a;
}
// Over groups of 2 * WIDEST lanes.
template <int WIDEST>
__device__ __forceinline__ void lanes_sum(Sum& a, float c) {
  float m = a.ref;
#pragma unroll
  for (int s = WIDEST; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
  const float top = top_of(m, c);
  a = Sum{m, top, moved(a, m, top, c)};
#pragma unroll
  for (int s = WIDEST; s > 0; s >>= 1) a.s += __shfl_xor_sync(0xffffffffu, a.s, s);
}

// ---- sums in 64 bits
// e^v in 64 bits for v up to 700: 2^n e^f with n the nearest whole number to v / ln 2, |f| <= ln 2 / 2, e^f by its Taylor series up to f^10, 3e-13
// off. Below e^-690 it stays there (kNothing). Half the operations of a library function that serves all arguments. (With sixteenths of n, a table
// of roots and the series up to f^5, 10 operations instead of 14, a pass takes 1.25 times as long.)
__device__ __forceinline__ double exp64(double v) {
  v = __hiloint2double((int)min((unsigned)__double2hiint(v), 0xc0859000u), __double2loint(v));      // not below -690; -inf neither
  const double magic = 6755399441055744.0;           // 1.5 * 2^52: adding it rounds to whole numbers, which are then its lowest bits
  const double y = fma(v, 1.4426950408889634, magic);
  const double f = fma(y - magic, -0.6931471805599453, v);
  double s = 1.0 / 3628800;
  s = fma(s, f, 1.0 / 362880);
  s = fma(s, f, 1.0 / 40320);
  s = fma(s, f, 1.0 / 5040);
  s = fma(s, f, 1.0 / 720);
  s = fma(s, f, 1.0 / 120);
  s = fma(s, f, 1.0 / 24);
  s = fma(s, f, 1.0 / 6);
  s = fma(s, f, 0.5);
  s = fma(s, f, 1.0);
  s = fma(s, f, 1.0);
  return __hiloint2double(__double2hiint(s) + (int)((unsigned)__double2loint(y) << 20), __double2loint(s));
}
__device__ __forceinline__ double weight64(float x, double scale, double top) { return exp64(fma((double)x, scale, -top)); }
// The sum over the blocks of value i.
__device__ __forceinline__ double total(int i, int cluster, int turn) {
  double v = 0.0;
  for (int r = 0; r < cluster; ++r) v += sh.box[turn & 1][r][i];
  return v;
}
// What is left of the probability of a token whose logits are x (the model's) and y (the draft's) behind the rejections so far.
template <bool DRAFT>
__device__ __noinline__ double left(float x, float y, int rejected) {
  double r = weight64(x, sh.e.scale, sh.e.top) * sh.e.inv;
  if (DRAFT && rejected > 0) {
    const double q = weight64(y, sh.e.dscale, sh.e.dtop) * sh.e.dinv;
    for (int i = 0; i < rejected; ++i)
      if (sh.norm[i] > 0.0) r = fmax(r - q, 0.0) * sh.norm[i];
  }
  return r;
}

// One pass over (a part of) the block's part of the row in 64 bits. The exponentials are the bulk of the work and of the code, which every SM has to
// fetch: all uses but for single tokens are modes of this one loop. A warp has strips from, from + step, ... below to.
//   SUMS    values 0, 1: the sums of e^(x scale - top) of the model and of the draft
//   REST    value 0: what one more rejection leaves
//   STRIPS  what is left, per strip, and value 0: in all
//   FIRST   what the first rejection leaves, with e.inv and e.dinv known to 2^-19 or so: strips and values 3, 4, 5 of max(p - q, 0), and of
//           e^.. of the model and of the draft where that is not 0, by which it is corrected; values 0, 1 as SUMS; value 2: p + q of tokens whose
//           p and q are alike to 2^-18, of which it may not be known which is larger
// Values are published. find, by one warp: the token at `want` of a strip, or the last one there that has anything.
enum { SUMS, REST, STRIPS, FIRST };
template <typename T, bool DRAFT>
__device__ __noinline__ int find(int rejected, int strip, double want) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool both = DRAFT && rejected > 0;
  const T* const row = static_cast<const T*>(sh.row.row);
  const T* const drow = static_cast<const T*>(sh.row.drow);
  const int vocab = sh.row.vocab, first = sh.row.from + strip * sh.row.per, end = min(sh.row.to, first + sh.row.per);
  extern __shared__ __align__(16) unsigned char copies[];
  const Ring<T> ring(row, drow, vocab, both, sh.row.dvec, copies, warp, lane);
  const int base = lane * 8 - sh.row.shift;
  for (int k = 0; k < Ring<T>::kRing; ++k) ring.ask(k, (first + k) * kTile + base, first + k < end);
  double cum = 0.0;
  int some_tile = -1;
  auto given = [&](int token) {          // no such token, or one that is rejected
    bool no = (unsigned)token >= (unsigned)vocab;
    if (!DRAFT)
      for (int k = 0; k < rejected; ++k) no = no || sh.gone[k] == token;
    return no;
  };
#pragma unroll 1
  for (int tile = first, k = 0; tile < end; ++tile, ++k) {
    float x[8], y[8] = {};
    ring.get(k, x, y);
    ring.ask(k + Ring<T>::kRing, (tile + Ring<T>::kRing) * kTile + base, tile + Ring<T>::kRing < end);
    double mine = 0.0;
#pragma unroll 1
    for (int half = 0; half < 8; half += 4) {       // short code: it is gone through a few times, and has to be fetched first
      double r[4], q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r[i] = weight64(half ? x[i + 4] : x[i], sh.e.scale, sh.e.top) * sh.e.inv;
        q[i] = both ? weight64(half ? y[i + 4] : y[i], sh.e.dscale, sh.e.dtop) * sh.e.dinv : 0.0;
      }
      if (both) {
        for (int k = 0; k < rejected; ++k) {
          const double z = sh.norm[k];
          if (z > 0.0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = fmax(r[i] - q[i], 0.0) * z;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) mine += DRAFT || !given(tile * kTile + base + half + i) ? r[i] : 0.0;
    }
    double upto = mine;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const double o = __shfl_up_sync(0xffffffffu, upto, s);
      if (lane >= s) upto += o;
    }
    const uint32_t there = __ballot_sync(0xffffffffu, cum + upto > want && mine > kNothing);
    const bool any = __any_sync(0xffffffffu, mine > kNothing);
    if (there != 0) {                    // in the first of these lanes: lane i < 8 looks at its i-th token
      const int lead = __ffs(there) - 1;
      float xi = 0.f, yi = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float xs = __shfl_sync(0xffffffffu, x[i], lead), ys = __shfl_sync(0xffffffffu, y[i], lead);
        xi = lane == i ? xs : xi;
        yi = lane == i ? ys : yi;
      }
      const int token = tile * kTile + lead * 8 - sh.row.shift + lane;
      const double r = lane >= 8 || given(token) ? 0.0 : left<DRAFT>(xi, yi, rejected);
      double c = r;
#pragma unroll
      for (int s = 1; s < 8; s <<= 1) {
        const double o = __shfl_up_sync(0xffffffffu, c, s);
        if (lane >= s) c += o;
      }
      c += __shfl_sync(0xffffffffu, cum + (upto - mine), lead);
      const uint32_t some = __ballot_sync(0xffffffffu, r > kNothing), hit = __ballot_sync(0xffffffffu, r > kNothing && c > want);
      return __shfl_sync(0xffffffffu, token, hit ? __ffs(hit) - 1 : 31 - __clz(some));
    }
    if (any) some_tile = tile;
    cum += __shfl_sync(0xffffffffu, upto, 31);
  }
  int last = -1;
#pragma unroll 1
  for (int i = 0; i < 8 && some_tile >= 0; ++i) {
    const int token = some_tile * kTile + base + i;
    if (!given(token) && left<DRAFT>(value(row + token), both ? value(drow + token) : 0.f, rejected) > kNothing) last = token;
  }
  return __reduce_max_sync(0xffffffffu, last);
}

template <typename T, bool DRAFT, int WARPS, int MODE>
__device__ __noinline__ void pass(int rejected, int to, int rank, int cluster, int turn) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* const row = static_cast<const T*>(sh.row.row);
  const T* const drow = static_cast<const T*>(sh.row.drow);
  const int vocab = sh.row.vocab, per = sh.row.per, tile0 = sh.row.from, tile1 = sh.row.to, base = lane * 8 - sh.row.shift;
  const bool dvec = sh.row.dvec, both = DRAFT && (MODE != STRIPS || rejected > 0);
  const double scale = sh.e.scale, top = sh.e.top, inv = sh.e.inv, dscale = sh.e.dscale, dtop = sh.e.dtop, dinv = sh.e.dinv;
  extern __shared__ __align__(16) unsigned char copies[];
  const Ring<T> ring(row, drow, vocab, both, dvec, copies, warp, lane);
  // tiles in turn, strip after strip; `ahead` is the one to ask for
  int ahead_strip = warp, ahead = tile0 + warp * per, asked = 0;
  auto ask = [&]() {
    ring.ask(asked++, ahead * kTile + base, ahead_strip < to);
    if (++ahead >= min(tile1, tile0 + (ahead_strip + 1) * per)) {
      ahead_strip += WARPS;
      ahead = tile0 + ahead_strip * per;
    }
  };
#pragma unroll 1
  for (int k = 0; k < Ring<T>::kRing; ++k) ask();
  double v[kValues] = {};
  int k_tile = 0;
#pragma unroll 1
  for (int strip = warp; strip < to; strip += WARPS) {
    const int end = min(tile1, tile0 + (strip + 1) * per);
    double in_strip = 0.0, p_strip = 0.0, q_strip = 0.0;
    int tile = tile0 + strip * per;
    if (MODE == STRIPS && !both) {       // without a rejected token in the strip: sums of weights, short code
      bool plain = true;
      if (!DRAFT)
        for (int k = 0; k < rejected; ++k) plain = plain && (unsigned)(sh.gone[k] + sh.row.shift - tile * kTile) >= (unsigned)((end - tile) * kTile);
      if (plain) {
        double s[2] = {0.0, 0.0};
#pragma unroll 1
        for (; tile < end; ++tile) {
          float x[8], y[8];
          ring.get(k_tile++, x, y);
          ask();
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i & 1] += weight64(x[i], scale, top);
        }
        in_strip = (s[0] + s[1]) * inv;
      }
    }
#pragma unroll 1
    for (; tile < end; ++tile) {
      float x[8], y[8];
      ring.get(k_tile++, x, y);
      ask();
      const int at = tile * kTile + base;
#pragma unroll
      for (int part = 0; part < 8; part += 4) {
        double w[4], q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = weight64(x[part + i], scale, top);
        if (both) {
#pragma unroll
          for (int i = 0; i < 4; ++i) q[i] = weight64(y[part + i], dscale, dtop);
        }
        if (MODE == SUMS || MODE == FIRST) {
          v[0] += (w[0] + w[1]) + (w[2] + w[3]);
          if (both) v[1] += (q[0] + q[1]) + (q[2] + q[3]);
          if (DRAFT && MODE == FIRST) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const double p = w[i] * inv, d = fma(-q[i], dinv, p);
              if ((__double2hiint(d) & 0x7fffffff) + (18 << 20) <= __double2hiint(p)) v[2] += 2.0 * p;
              if (d > 0.0) {
                in_strip += d;
                p_strip += w[i];
                q_strip += q[i];
              }
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] *= inv;
          if (both) {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] *= dinv;
          }
#pragma unroll 1
          for (int k = 0; k < rejected; ++k) {
            if (DRAFT) {
              const double z = sh.norm[k];
              if (z > 0.0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = fmax(w[i] - q[i], 0.0) * z;
              }
            } else {
              const int d = sh.gone[k] - at - part;
              if ((unsigned)d < 4u) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (d == i) w[i] = 0.0;
              }
            }
          }
          if (DRAFT && MODE == REST) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = fmax(w[i] - q[i], 0.0);
          }
          const double sum = (w[0] + w[1]) + (w[2] + w[3]);
          in_strip += sum;
        }
      }
    }
    if (MODE == FIRST) {
      v[3] += in_strip;
      v[4] += p_strip;
      v[5] += q_strip;
      in_strip = warp_sum(in_strip);
      p_strip = warp_sum(p_strip);
      q_strip = warp_sum(q_strip);
      if (lane == 0) {
        sh.strips[0][strip] = in_strip;
        sh.strips[1][strip] = p_strip;
        sh.strips[2][strip] = q_strip;
      }
    } else if (MODE == STRIPS || MODE == REST) {
      v[0] += in_strip;
      in_strip = warp_sum(in_strip);
      if (lane == 0) sh.strips[0][strip] = in_strip;
    }
  }
  constexpr int n = MODE == FIRST ? 6 : MODE == SUMS ? 2 : 1;
#pragma unroll
  for (int i = 0; i < kValues; ++i) {
    if (i < n) {
      v[i] = warp_sum(v[i]);
      if (lane == 0) sh.part[warp][i] = v[i];
    }
  }
  __syncthreads();
  if (warp == 0) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      if (i < n) {
        v[i] = sh.part[lane & (WARPS - 1)][i];
#pragma unroll
        for (int s = WARPS / 2; s > 0; s >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], s);
      }
    }
    publish(n, v, rank, cluster, turn, lane);
  }
  arrived(cluster, turn);
}

// THREADS: 512 where there are few requests, so that what runs of them has the threads of an SM each; else 128, four blocks of which an SM runs (128
// registers): blocks of different requests then pass through their joins and draws at different times.
template <typename T, bool DRAFT, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS) verify_kernel(const __grid_constant__ VerifyParams p) {
  constexpr int kWarps = THREADS / 32;
  extern __shared__ __align__(16) unsigned char copies[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cluster = p.cluster;
  const int request = blockIdx.x / cluster, rank = blockIdx.x % cluster;
  const int first = p.first[request], nodes = p.first[request + 1] - first;
  pdl_launch_dependents();
  pdl_wait();
  if (tid < kNodes) {                    // gone: here, the nodes' parents
    const bool node = tid < nodes;
    const int token = node ? p.tokens[first + tid] : -1, parent = node && tid > 0 ? p.parents[first + tid] : -1;
    sh.token[tid] = token;
    sh.gone[tid] = (unsigned)token < (unsigned)p.vocab && parent >= 0 && parent < tid ? parent : -1;      // -1: passed over
    sh.chance[tid] = node ? p.u_accept[first + tid] : 0.f;
    sh.scale[tid] = node && p.scale ? p.scale[first + tid] : 1.f;
    sh.dscale[tid] = DRAFT && node && p.draft_scale ? p.draft_scale[first + tid] : 1.f;
    // c, rounded down, and what is missing of it, always something (-inf times it stays -inf): left out, all terms of a sum would share an error of 1e-6
    auto split = [](float scale, float& c, float& rest) {
      const double exact = scale * kLog2e;
      c = __double2float_rd(exact * (1.0 - 0x1p-30));
      rest = (float)(exact - c);
    };
    split(sh.scale[tid], sh.c[tid], sh.c_rest[tid]);
    split(sh.dscale[tid], sh.dc[tid], sh.dc_rest[tid]);
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.even_bar[i]), 1);
      mbar_init(smem_u32(&sh.box_bar[i]), 1);
    }
    sh.lost = 0;
    mbar_init_fence();
  }
  __syncthreads();
  if (tid < nodes) {
    int child = -1, sibling = -1;
    const int parent = sh.gone[tid];
    for (int j = nodes - 1; j > tid; --j) {
      if (sh.gone[j] == tid) child = j;
      if (parent >= 0 && sh.gone[j] == parent) sibling = j;
    }
    sh.child[tid] = child;
    sh.sibling[tid] = sibling;
  }
  sync_all(cluster);                     // all blocks of the cluster run: they may be written to
  const int shares = 31 - __clz(cluster);            // log2
  // A node's rows and this block's tiles of them.
  struct Place {
    const T *row, *drow;
    int shift, from, to;
    bool both, dvec;                     // the draft's row of a node without children is not read
  };
  auto place_of = [&](int node) {
    Place s;
    s.row = static_cast<const T*>(p.logits) + (int64_t)(first + node) * p.stride;
    s.drow = DRAFT ? static_cast<const T*>(p.draft) + (int64_t)(first + node) * p.draft_stride : nullptr;
    s.shift = (int)((reinterpret_cast<uintptr_t>(s.row) & 15) / sizeof(T));
    s.dvec = DRAFT && (int)((reinterpret_cast<uintptr_t>(s.drow) & 15) / sizeof(T)) == s.shift;
    s.both = DRAFT && sh.child[node] >= 0;
    const int tiles = (p.vocab + s.shift + kTile - 1) / kTile;
    s.from = tiles * rank >> shares;
    s.to = tiles * (rank + 1) >> shares;
    return s;
  };
  auto ring_of = [&](const Place& s) { return Ring<T>(s.row, s.drow, p.vocab, s.both, s.dvec, copies, warp, lane); };
  auto ask_first = [&](const Place& s) {
    const Ring<T> ring = ring_of(s);
    const int at = (s.from + warp) * kTile + lane * 8 - s.shift;
    int k = 0;
#pragma unroll 1
    for (; k < Ring<T>::kRing && s.from + warp + k * kWarps < s.to; ++k) ring.ask(k, at + k * kWarps * kTile, true);
#pragma unroll 1
    for (; k < Ring<T>::kRing; ++k) cp_async_commit();
  };
  int cur = 0, emitted = 0, turn = 0, joins = 0, moves = 0, asked = -1;    // asked: the node whose first tiles are on their way
  float ref = 0.f, dref = 0.f;           // logits of likely tokens: the last accepted one's, where it was accepted
  for (;;) {
    const float scale = sh.scale[cur], dscale = sh.dscale[cur];
    const float c = sh.c[cur], dc = sh.dc[cur];
    float c_rest = sh.c_rest[cur], dc_rest = sh.dc_rest[cur];
    const Place here = place_of(cur);
    const T *const row = here.row, *const drow = here.drow;
    const int vocab = p.vocab, shift = here.shift, from = here.from, to = here.to;
    const bool both = here.both, dvec = here.dvec;
    if (asked != cur) {
      if (asked >= 0) cp_async_wait<0>();
      ask_first(here);
    }
    asked = -1;
    const int child = sh.child[cur];
    // the first child's logits: asked for before the sums
    const float x0 = child >= 0 ? value(row + sh.token[child]) : 0.f, y0 = both ? value(drow + sh.token[child]) : 0.f;

    // The row's sums in fp32. All threads first take one reference, a logit that may be far from the row's largest but seldom is: then a logit is a
    // product, an exponential and a sum, and sums are joined by adding. Where the whole sum says that it was too far, or no number, once more with
    // references that move.
    if (emitted == 0) {
      ref = child >= 0 ? x0 : value(row);
      dref = y0;
    }
    Sum a = {ref, top_of(ref, c), 0.f}, b = {dref, top_of(dref, dc), 0.f};
    const int base = lane * 8 - shift;
    auto ask_child = [&]() {             // the first child is the likeliest to be next: its tiles fly while this row's sums are joined
      if (child < 0) return;
      ask_first(place_of(child));
      asked = child;
    };
    bool lost = false, moving = false;
    {
      const Ring<T> ring = ring_of(here);
      float s = 0.f, d = 0.f;
      double whole = 0.0, dwhole = 0.0;
      int tile = from + warp;
#pragma unroll 1
      for (int k = 0;;) {
        const int stop = min(to, tile + kChain * kWarps);
#pragma unroll 1
        for (; tile < stop; ++k, tile += kWarps) {
          float x[8], y[8];
          ring.get(k, x, y);
          const int next = tile + Ring<T>::kRing * kWarps;
          ring.ask(k, next * kTile + base, next < to);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = ex2(fmaf(x[i], c_rest, fmaf(x[i], c, -a.top)));
          s += sum8(x);
          if (both) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = ex2(fmaf(y[i], dc_rest, fmaf(y[i], dc, -b.top)));
            d += sum8(y);
          }
        }
        if (tile >= to) break;
        whole += s;
        dwhole += d;
        s = d = 0.f;
      }
      ask_child();
      float sa = (float)(whole + s), sb = (float)(dwhole + d);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        sa += __shfl_xor_sync(0xffffffffu, sa, o);
        sb += __shfl_xor_sync(0xffffffffu, sb, o);
      }
      const int slot = joins & 1;
      if (lane == 0) sh.part_even[slot][warp] = make_float2(sa, sb);
      __syncthreads();
      if (cluster > 1) {
        const uint32_t bar = smem_u32(&sh.even_bar[slot]);
        if (warp == 0) {
          if (lane == 0) mbar_expect_tx(bar, 8 * cluster);
          const float2 mine = sh.part_even[slot][lane & (kWarps - 1)];
          sa = mine.x;
          sb = mine.y;
#pragma unroll
          for (int o = kWarps / 2; o > 0; o >>= 1) {
            sa += __shfl_xor_sync(0xffffffffu, sa, o);
            sb += __shfl_xor_sync(0xffffffffu, sb, o);
          }
          if (lane < cluster) st_async(mapa(smem_u32(&sh.even[slot][rank]), lane), mapa(bar, lane), make_float2(sa, sb));
        }
        if (warp == 0 && !mbar_poll(bar, joins >> 1 & 1)) sh.lost = 1;
        __syncthreads();                 // one warp looks, the others leave it the issue slots
        lost = sh.lost;
        sa = sb = 0.f;
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
          if (r < cluster) {
            sa += sh.even[slot][r].x;
            sb += sh.even[slot][r].y;
          }
        }
      } else {
        sa = sb = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          sa += sh.part_even[slot][w].x;
          sb += sh.part_even[slot][w].y;
        }
      }
      ++joins;
      a.s = sa;
      b.s = both ? sb : 1.f;
    }
    if (__builtin_expect(!lost && !(a.s > 1.f / kLarge && a.s < kLarge && b.s > 1.f / kLarge && b.s < kLarge), 0)) {
      moving = true;
      Moving ma = {-CUDART_INF_F, CUDART_NAN_F, 0.0}, mb = ma;
      c_rest = dc_rest = 1e-37f;         // nothing: references move, the same c everywhere
      cp_async_wait<0>();
      __syncthreads();
      ask_first(here);
      asked = -1;
      const Ring<T> ring = ring_of(here);
#pragma unroll 1
      for (int k = 0, tile = from + warp; tile < to; ++k, tile += kWarps) {
        float x[8], y[8];
        ring.get(k, x, y);
        const int next = tile + Ring<T>::kRing * kWarps;
        ring.ask(k, next * kTile + base, next < to);
        ma = add(ma, x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7], c);
        if (both) mb = add(mb, y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7], dc);
      }
      auto join = [&](const float4& v, auto widest) {
        a = Sum{v.x, top_of(v.x, c), v.y};
        b = Sum{v.z, top_of(v.z, dc), v.w};
        lanes_sum<widest.value>(a, c);
        if (both) lanes_sum<widest.value>(b, dc);
      };
      join(make_float4(ma.ref, (float)ma.s, mb.ref, (float)mb.s), std::integral_constant<int, 16>{});
      if (lane == 0) sh.part32[warp] = make_float4(a.ref, a.s, b.ref, b.s);
      __syncthreads();
      join(sh.part32[lane & (kWarps - 1)], std::integral_constant<int, kWarps / 2>{});
      if (cluster > 1) {
        if (tid < cluster) st_cluster(mapa(smem_u32(&sh.sums[moves][rank]), tid), make_float4(a.ref, a.s, b.ref, b.s));
        cluster_sync();
        join(lane % kMaxCluster < cluster ? sh.sums[moves][lane % kMaxCluster] : make_float4(-CUDART_INF_F, 0.f, -CUDART_INF_F, 0.f),
             std::integral_constant<int, kMaxCluster / 2>{});
        moves ^= 1;
      }
      if (!both) b = Sum{0.f, 0.f, 1.f};
    }
    const bool valid = !lost && a.s > 0.f && a.s < CUDART_INF_F && b.s > 0.f && b.s < CUDART_INF_F;
    int chosen = -1, out = -1;
    if (valid) {
      int n = 0;                         // strips
      bool precise = false;              // sh.e holds sums of 64 bits
      int rejected = 0;
      float rest = 1.f;                  // no draft: what the rejected tokens leave
      double rest64 = 1.0;
      bool pending = false;              // draft: a rejection whose Z is not summed yet
      bool ready = false;
      auto prepare = [&]() {             // what the passes read; e.inv, e.dinv: to 2^-19 or so (a sum's c is rounded)
        if (ready) return;
        ready = true;
        if (asked >= 0) cp_async_wait<0>();          // the passes use the same slots
        asked = -1;
        // strips as short as there is room for, but a few for every warp at most: their sums cost a strip as much as a tile does
        const int per = max(1, max((to - from + kStrips - 1) / kStrips, min(2, (to - from) / (4 * kWarps))));
        n = (to - from + per - 1) / per;
        if (tid == 0) {
          sh.row = Row{row, drow, vocab, shift, from, to, dvec, per, n};
          // the sums are of 2^(x c - top): what rounding ref c has changed them by is known
          auto less = [](const Sum& v, float scale) { return v.top == v.top ? 1.0 - 0.6931471805599453 * ((double)v.top - (double)v.ref * scale * 1.4426950408889634) : 1.0; };
          sh.e = Exact{scale, (double)a.ref * scale, less(a, scale) / a.s, dscale, (double)b.ref * dscale, less(b, dscale) / b.s};
        }
        __syncthreads();
      };
      auto sum64 = [&](auto mode) {      // SUMS or FIRST: the distributions' sums become those of 64 bits
        prepare();
        pass<T, DRAFT, kWarps, mode.value>(rejected, n, rank, cluster, turn);
        if (tid == 0) {
          sh.e.inv = 1.0 / total(0, cluster, turn);
          if (DRAFT) sh.e.dinv = 1.0 / total(1, cluster, turn);
        }
        __syncthreads();
        ++turn;
        precise = true;
      };
      auto reject = [&]() {              // Z of the pending rejection
        if constexpr (DRAFT) pass<T, DRAFT, kWarps, REST>(rejected, n, rank, cluster, turn);
        const double z = total(0, cluster, turn);
        ++turn;
        if (tid == 0) sh.norm[rejected] = z > kNothing ? 1.0 / z : 0.0;
        __syncthreads();
        ++rejected;
        pending = false;
      };
      for (int j = child; j >= 0; j = sh.sibling[j]) {
        const int t = sh.token[j];
        const float u = sh.chance[j], x = j == child ? x0 : value(row + t), y = j == child ? y0 : DRAFT ? value(drow + t) : 0.f;
        bool again = false;              // given twice: nothing is left of it
        if (!DRAFT)
          for (int i = 0; i < rejected; ++i) again = again || sh.gone[i] == t;
        if (again) continue;
        bool accept = false, close = precise || pending;
        if (!close) {
          // p and u q, or p and u times what is left, both times the sums: no divisions. Below kSmall a weight of 2^-126 or less, which counts as 0, may have been one of theirs
          // (its product with a sum, below kLarge, is less than that): where both are, 64 bits decide.
          const float have = DRAFT ? weight(x, a, c, c_rest) * b.s : weight(x, a, c, c_rest);
          const float need = DRAFT ? u * weight(y, b, dc, dc_rest) * a.s : u * rest * a.s;
          accept = need < have;
          const float margin = moving ? kMarginMoving : kMargin;
          close = fabsf(need - have) <= margin * (DRAFT ? need + have : (1 + rejected) * a.s) || (DRAFT && fmaxf(need, have) < kSmall);
        }
        if (close) {
          if (!precise) {
            sum64(std::integral_constant<int, SUMS>{});
            if (!DRAFT)
              for (int i = 0; i < rejected; ++i) rest64 -= weight64(value(row + sh.gone[i]), sh.e.scale, sh.e.top) * sh.e.inv;
          }
          if (pending) reject();
          const double have = left<DRAFT>(x, y, rejected);
          accept = have > kNothing && (DRAFT ? (double)u * (weight64(y, sh.e.dscale, sh.e.dtop) * sh.e.dinv) : (double)u * rest64) < have;
        }
        if (accept) {
          chosen = j;
          out = t;
          ref = x;
          dref = y;
          break;
        }
        if (DRAFT) {
          pending = true;
        } else {
          rest -= weight(x, a, c, c_rest) / a.s;
          if (precise) rest64 -= weight64(x, sh.e.scale, sh.e.top) * sh.e.inv;
          __syncthreads();               // the others may still look through the list
          if (tid == 0) sh.gone[rejected] = t;
          ++rejected;
          __syncthreads();
        }
      }
      if (chosen < 0) {
        const float at = p.u_sample[request];
        // the last rejection's Z is a factor of all that is left: it is not needed, unless nothing is
        prepare();
        const bool one = DRAFT && pending && rejected == 0 && !precise;
        bool done = false;
        double fix_p = 0.0, fix_q = 0.0;
        const double inv = sh.e.inv, dinv = sh.e.dinv;
        if (DRAFT && pending) {
          __syncthreads();
          if (tid == 0) sh.norm[rejected] = 1.0;
          __syncthreads();
        }
        if constexpr (DRAFT) if (one) {
          // One rejection and none before: the sums of 64 bits and what it leaves in one pass. The latter is linear in the sums' reciprocals as long
          // as the corrections change no sign.
          sum64(std::integral_constant<int, FIRST>{});
          --turn;                        // its values are read here
          fix_p = sh.e.inv - inv;
          fix_q = sh.e.dinv - dinv;
          const double off = fmax(fabs(fix_p) * a.s, fabs(fix_q) * b.s);
          done = off < 0x1p-19 && off * total(2, cluster, turn) <= 1e-12 * total(3, cluster, turn);
          if (!done) ++turn;
        } else if (pending && !precise) {
          sum64(std::integral_constant<int, SUMS>{});
        }
        const int all_rejected = rejected + pending;
        for (int tries = 0; tries < 2 && out < 0; ++tries) {
          const int gone = tries ? rejected : all_rejected;          // nothing left: p = q up to roundings, as if not rejected
          if (tries && !pending) break;
          if (!done) pass<T, DRAFT, kWarps, STRIPS>(gone, n, rank, cluster, turn);
          // the blocks' sums; the last block with anything, the one that holds the place
          auto sum_of = [&](int k) {
            const double* v = sh.box[turn & 1][k];
            return done ? fmax(0.0, v[3] + fix_p * v[4] - fix_q * v[5]) : v[0];
          };
          double all = 0.0, front = 0.0, cum = 0.0;
          for (int k = 0; k < cluster; ++k) all += sum_of(k);
          const double want = (double)at * all;
          int holder = -1, last = 0;
          for (int k = 0; k < cluster; ++k) {
            const double v = sum_of(k);
            if (v > kNothing) last = k;
            if (holder < 0 && cum + v > want) {
              holder = k;
              front = cum;
            }
            cum += v;
          }
          ++turn;
          const bool fixed = done;
          done = false;
          if (!(all > kNothing) || !(all < CUDART_INF)) continue;
          const bool beyond = holder < 0;            // u not below 1, or a rounding: the last token with anything
          if (beyond) holder = last;
          if (holder == rank && warp == 0) {
            // the strip: a lane has n / 32 neighbouring ones
            const double here = beyond ? CUDART_INF : want - front;
            const int each = (n + 31) / 32, s0 = min(n, lane * each), s1 = min(n, s0 + each);
            auto strip_of = [&](int s) {
              return fixed ? fmax(0.0, sh.strips[0][s] + fix_p * sh.strips[1][s] - fix_q * sh.strips[2][s]) : sh.strips[0][s];
            };
            double own = 0.0;
            int final = -1;
            for (int s = s0; s < s1; ++s) {
              const double v = strip_of(s);
              own += v;
              if (v > kNothing) final = s;
            }
            double upto = own;
#pragma unroll
            for (int s = 1; s < 32; s <<= 1) {
              const double o = __shfl_up_sync(0xffffffffu, upto, s);
              if (lane >= s) upto += o;
            }
            const uint32_t behind = __ballot_sync(0xffffffffu, upto > here);
            final = __reduce_max_sync(0xffffffffu, final);
            double before = upto - own, place = CUDART_INF;
            int strip = -1;
            const int lead = behind != 0 ? __ffs(behind) - 1 : 0;
            if (behind != 0 && lane == lead) {
              for (int s = s0; s < s1 && strip < 0; ++s) {
                const double v = strip_of(s);
                if (before + v > here) strip = s; else before += v;
              }
              place = here - before;
            }
            strip = __shfl_sync(0xffffffffu, strip, lead);
            place = __shfl_sync(0xffffffffu, place, lead);
            if (strip < 0) {
              strip = final;
              place = CUDART_INF;
            }
            const int token = find<T, DRAFT>(gone, strip, place);
            if (lane < cluster) {
              const uint32_t found = smem_u32(&sh.found);
              st_cluster(cluster > 1 ? mapa(found, lane) : found, token);
            }
          }
          sync_all(cluster);
          out = sh.found;
        }
      }
    }
    if (sh.lost) chosen = out = -1;
    if (rank == 0 && tid == 0) {
      sh.out[emitted] = out;
      sh.walked[emitted] = cur;
      sh.ref[emitted] = a.ref;
      sh.top[emitted] = a.top;
      sh.sum[emitted] = a.s;
      sh.rest_used[emitted] = c_rest;
    }
    ++emitted;
    if (chosen < 0) break;
    cur = chosen;
  }
  if (rank == 0) {
    if (tid == 0) p.count[request] = emitted;
    __syncthreads();
    if (tid < nodes) {
      const int out = tid < emitted ? sh.out[tid] : -1, at = tid < emitted ? sh.walked[tid] : -1;
      p.emitted[first + tid] = out;
      p.path[first + tid] = at >= 0 ? first + at : -1;
      float lp = at >= 0 ? CUDART_NAN_F : 0.f;
      if (out >= 0) {                    // the exponent as it went into the sum: of a token that has nearly all, their roundings cancel
        const Sum a = {sh.ref[tid], sh.top[tid], sh.sum[tid]};
        lp = (float)(exponent(value(place_of(at).row + out), a, sh.c[at], sh.rest_used[tid]) * 0.6931471805599453 - log((double)a.s));
      }
      p.logprob[first + tid] = lp;
    }
  }
  if (cluster > 1) cluster_sync();       // no block leaves while another one may write to it
}

template <typename T, bool DRAFT, int THREADS>
cudaError_t launch_t(const VerifyParams& p, int requests, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(requests * p.cluster));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = THREADS / 32 * Ring<T>::kBytes;
  const cudaError_t e = cudaFuncSetAttribute(verify_kernel<T, DRAFT, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
  if (e != cudaSuccess) return e;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, DRAFT, THREADS>, p);
}
template <typename T, bool DRAFT>
cudaError_t launch(const VerifyParams& p, int requests, bool wide, cudaStream_t stream) {
  return wide ? launch_t<T, DRAFT, 512>(p, requests, stream) : launch_t<T, DRAFT, 128>(p, requests, stream);
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
  // as many blocks of a request as run at once, four of 128 threads per SM or one of 512, each with a few tiles for every warp
  const bool wide = (int64_t)v->n_requests * kMaxCluster <= n_sms;
  p.cluster = 1;
  while (p.cluster < kMaxCluster && (wide || (int64_t)v->n_requests * p.cluster * 2 <= 4 * n_sms) && v->vocab / (p.cluster * 2) >= kTile * (wide ? 4 : 2)) p.cluster *= 2;
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
    const cudaError_t e = v->dtype == TS_BF16 ? (v->draft ? launch<__nv_bfloat16, true>(p, some, wide, stream) : launch<__nv_bfloat16, false>(p, some, wide, stream))
                                              : (v->draft ? launch<float, true>(p, some, wide, stream) : launch<float, false>(p, some, wide, stream));
    if (e != cudaSuccess) return TS_ERR_CUDA;
  }
  return TS_OK;
}
