// Attention for trees of drafted tokens over the paged KV cache (sm_100a): bf16 pages or the 8-bit cache. A row of one node
// is a decode row.
//
// Node i of a row attends its ctx cached tokens and the nodes its mask names:
//     s_j = scale <q_i, k_j>,  p_j = exp(s_j - max s),  out = sum p_j v_j / sum p_j,  0 where no key is visible.
//
// tree_kernel, one CTA of four warps per work unit = (split of a row's keys, KV head, query tile). The warps take the
// unit's pages in turn; each has a ring of page stages of its own that TMA fills (the page id is a coordinate of the copy), and
// keeps its own online softmax; they are added up once at the unit's end. Products are transposed (S^T = K Q^T, O^T = V^T P^T,
// mma.sync m16n8k16 with keys and head_dim as M), so that few queries cost few MMAs: a query tile is 8, 16 or 32 (node, head) pairs.
//
// 8-bit pages: codes are widened to f16 between shared memory and the tensor core (exact). A key's K exponent is part of
// its score's scale. Its V exponent e_j goes into the weight, p'_j = 2^(s_j + e_j - m) with m the running maximum of s_j + e_j, so that
// the largest contribution is always 1, however far the exponents are apart, and the sum takes it out again: l += p'_j 2^-e_j.
// Weights are f16 there, shifted by 2^15: normal numbers down to 2^-29 of the largest. A row's own nodes are not quantised: they
// are laid into shared memory as f16 with a power of two per row, which the same code multiplies (eight significant bits of bf16
// fit f16's eleven; an element below 2^-28 of its row's largest rounds).
//
// What bounds it (37 rows of 8192 keys, 8 KV heads of 128, 4 query heads each): HBM in bf16, one node 1.24 GB in 188 to 194 us, what a copy
// takes; four nodes 203. In 8 bits one node 0.64 GB in 129 us (4.9 TB/s): the instructions that widen the codes and the MMAs that pad 4 queries
// to 8 (59 % of the issue slots, tensor pipe 15 %); from 9 queries on a second and fourth MMA per widened operand, 188 us for four nodes,
// 277 for eight. Tried and dropped: K Q^T in e4m3 against two addends of Q (one node 125, but four 235), codes widened by conversion
// instructions (163), scales by bulk copies instead of cp.async (no difference).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "../../include/tokenscale.h"
#include "ts_ptx.h"
#include "ts_tma.h"
#include "ts_tree.h"

namespace ts {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr long long kDrainCycles = 20000000;     // about 10 ms: limit of the wait for copies in flight after a failure
constexpr float kShift8 = 15.f;                  // log2 of the factor on the f16 weights

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }
// arrives on `bar` when this thread's cp.async copies so far are done
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(bar) : "memory");
}

// Shared-memory images of a page of one KV head. 16-bit elements: [K, V][64-column half][16 rows of 128 bytes], 128-byte swizzle.
template <int D>
__device__ __forceinline__ uint32_t off16(int kv, int r, int c) {       // 16-byte chunk c of row r
  return (uint32_t)(kv * (kPageSize * D * 2) + (c >> 3) * 2048 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}
// Codes: [K, V][16 rows of D bytes], swizzled over the width of a row.
template <int D>
__device__ __forceinline__ uint32_t off8(int kv, int r, int c) {
  if (D == 128) return (uint32_t)(kv * (kPageSize * D) + r * 128 + ((c ^ (r & 7)) << 4));
  return (uint32_t)(kv * (kPageSize * D) + r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

template <int D, int NB, bool Q8>
struct Smem {
  static constexpr int kBlocks = Q8 ? (NB == 1 ? 4 : NB == 2 ? 3 : 2) : 2;      // thread blocks of an SM at a time
  static constexpr int kStages = Q8 ? (NB == 1 ? 3 : NB == 2 ? 4 : 6) : 3;
  static constexpr int kPageBytes = 2 * kPageSize * D * (Q8 ? 1 : 2);
  // a page of the row's own nodes, 16-bit elements, lies over the first stages of a warp that has no copy in flight any more
  static_assert(kStages * kPageBytes >= 2 * kPageSize * D * 2, "no room for a page of nodes");
  static constexpr int kOffScale = kWarps * kStages * kPageBytes;      // [warp][stage][K, V][16 bytes]
  static constexpr int kOffOwnExp = kOffScale + (Q8 ? kWarps * kStages * 32 : 0);   // [warp][K, V][16] bytes
  static constexpr int kOffBar = kOffOwnExp + kWarps * 32;
  static constexpr int kOffFailed = kOffBar + kWarps * kStages * 8;
  static constexpr int kEnd = kOffFailed + 8;
  // afterwards: results of the warps, [warp][query][D + 2]
  static constexpr int bytes() {
    const int merge = kWarps * NB * 8 * (D + 2) * 4;
    return 1024 + (kEnd > merge ? kEnd : merge);
  }
};

template <int D, int NB, bool Q8>
__global__ void __launch_bounds__(kThreads, Smem<D, NB, Q8>::kBlocks)
tree_kernel(const __grid_constant__ StepParams<kInlineWords> params, const __grid_constant__ TreeArgs a,
            const __grid_constant__ CUtensorMap kv_map) {
  using L = Smem<D, NB, Q8>;
  const StepDevice& s = params.s;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* smem = smem_raw + (base - smem_u32(smem_raw));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c = lane & 3;
  const int G = s.Hq / s.Hkv;
  pdl_launch_dependents();
  const uint32_t my_bars = base + L::kOffBar + warp * L::kStages * 8;
  if (lane == 0) {
    for (int i = 0; i < L::kStages; ++i) mbar_init(my_bars + i * 8, Q8 ? 3 : 1);      // Q8: and the two copies of the scales
    mbar_init_fence();
  }
  __syncwarp();
  if (tid == 0) tma_prefetch_desc(&kv_map);
  pdl_wait();

  const int unit = blockIdx.x;
  const int tile = unit % a.n_tiles, head = unit / a.n_tiles % s.Hkv;
  const WorkItem it = s.item(unit / (a.n_tiles * s.Hkv));
  const int T = it.q_count, t0 = tile * a.tile_tokens;
  const int n_tok = min(a.tile_tokens, T - t0);
  if (n_tok <= 0) return;                         // a row of fewer nodes than the longest one
  const int n_q = n_tok * G;                      // queries of the tile: node t0 + q / G, head head * G + q % G
  const int tok0 = s.row_tok0(it.row), ctx = s.row_ctx(it.row), slot = s.row_slot(it.row);
  const int n_cached = (ctx + kPageSize - 1) / kPageSize;
  const int32_t* table_row = s.table + (size_t)slot * s.max_pages_per_req;
  const bool row_ok = (unsigned)slot < (unsigned)s.max_requests && n_cached <= s.max_pages_per_req;
  if (!row_ok && tid == 0) atomicOr(s.status, TS_DEV_BAD_INDEX);
  const int cached_end = row_ok ? min(it.k_end, n_cached) : it.k_begin;   // this unit's pages of cached tokens: [k_begin, cached_end)

  // ---------------------------------------------------------------- this warp's page copies
  const uint32_t ring = base + warp * L::kStages * L::kPageBytes;
  const uint32_t scale_ring = base + L::kOffScale + warp * L::kStages * 32;
  int n_issued = 0, pages = 0;                    // lane i: page id of this warp's page (n_issued & ~31) + i
  bool dead = false;
  auto fill = [&](int n_consumed) {
#pragma unroll 1
    while (n_issued - n_consumed < L::kStages) {
      const int p = it.k_begin + warp + n_issued * kWarps;
      if (p >= cached_end || dead) break;
      if ((n_issued & 31) == 0) {
        const int mine = p + lane * kWarps;
        pages = mine < cached_end ? table_row[mine] : 0;
      }
      int page = __shfl_sync(0xffffffffu, pages, n_issued & 31);
      const bool ok = (unsigned)page < (unsigned)s.n_pages;
      const int st = n_issued % L::kStages;
      const uint32_t bar = my_bars + st * 8, dst = ring + st * L::kPageBytes;
      if (lane == 0) {
        if (!ok) {
          atomicOr(s.status, TS_DEV_BAD_PAGE);
          page = s.n_pages;                       // out of range on purpose: the copy delivers zeros
        }
        fence_proxy_async();
        mbar_expect_tx(bar, L::kPageBytes);
        if constexpr (Q8) tma_load_4d(dst, &kv_map, bar, 0, head * kPageSize, 0, page);
        else tma_load_5d(dst, &kv_map, bar, 0, head * kPageSize, 0, 0, page);
      }
      if constexpr (Q8) {
        // the scales by two lanes' own copies
        if (lane < 2) {
          cp_async16(scale_ring + st * 32 + lane * 16, a.cache.scales + (((size_t)(ok ? page : 0) * 2 + lane) * s.Hkv + head) * kPageSize, 16);
          cp_async_arrive(bar);
        }
      }
      ++n_issued;
    }
  };
  fill(0);

  // ---------------------------------------------------------------- queries
  // B fragments of S^T = K Q^T: lane (g, c) holds query 8 nb + g. bf16: elements 2c, 2c + 1 and 2c + 8, 2c + 9 of each sixteen.
  // Q8: 4c, 4c + 2 and 4c + 1, 4c + 3 (the K fragments come in the same order), as f16 times a power of two per query.
  // A query with an infinity or a NaN becomes one of NaN: it has no softmax, and scores of -inf would count as keys that are not seen.
  uint32_t qf[NB][D / 16][2];
  float q_scale[NB][2];                           // of queries 8 nb + 2c, + 1: scale * log2(e), times what takes the power out again
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int q = nb * 8 + g;
    const bool real = q < n_q;
    const uint16_t* src = s.q + ((size_t)(tok0 + t0 + (real ? q / G : 0)) * s.Hq + head * G + (real ? q % G : 0)) * D;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      if constexpr (Q8) {
        const uint2 v = real ? *reinterpret_cast<const uint2*>(src + ks * 16 + c * 4) : make_uint2(0, 0);
        qf[nb][ks][0] = v.x;
        qf[nb][ks][1] = v.y;
      } else {
        qf[nb][ks][0] = real ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + c * 2) : 0u;
        qf[nb][ks][1] = real ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + c * 2 + 8) : 0u;
      }
    }
    q_scale[nb][0] = q_scale[nb][1] = s.scale_log2;
    uint32_t most = 0;                            // largest magnitude of the query, as bf16 bits
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) most = max(most, max(qf[nb][ks][i] & 0x7fffu, (qf[nb][ks][i] >> 16) & 0x7fffu));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const bool odd = most >= 0x7f80u;
    if constexpr (!Q8) {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        if (odd) qf[nb][ks][0] = qf[nb][ks][1] = 0x7fc07fc0u;
    } else {
      // to 2^8 .. 2^9: products with codes up to 448 and sums over D stay far from fp32's ends
      const int e = most == 0 ? 0 : min(max((int)(most >> 7) - 127 - 8, -118), 118);
      const float down = odd ? CUDART_NAN_F : power(-e);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const uint32_t x = qf[nb][ks][0], y = qf[nb][ks][1];
        qf[nb][ks][0] = pack_f16(__uint_as_float(x << 16) * down, __uint_as_float(y << 16) * down);
        qf[nb][ks][1] = pack_f16(__uint_as_float(x & 0xffff0000u) * down, __uint_as_float(y & 0xffff0000u) * down);
      }
      // the score fragment holds queries 2c and 2c + 1, whose exponents lanes 8c and 8c + 4 have
      q_scale[nb][0] *= power(__shfl_sync(0xffffffffu, e, 8 * c));
      q_scale[nb][1] *= power(__shfl_sync(0xffffffffu, e, 8 * c + 4));
    }
  }

  float m[NB][2], l[NB][2], o[D / 16][NB][4];     // running maximum (log2) and sum of queries 8 nb + 2c, + 1; O^T
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb][0] = m[nb][1] = -CUDART_INF_F;
    l[nb][0] = l[nb][1] = 0.f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d][nb][0] = o[d][nb][1] = o[d][nb][2] = o[d][nb][3] = 0.f;
  }

  // ---------------------------------------------------------------- one page of sixteen keys
  // CODES: e4m3 image, else 16-bit elements. `see(nb, i, key)`: may query 8 nb + 2c + i see key `key` (0..15) of the page.
  // exps: the K and V exponent bytes of the page (Q8). bad: keys whose score is a NaN.
  auto page_step = [&](auto codes_tag, uint32_t img, const uint8_t* exps, auto&& see, uint32_t bad = 0) {
    constexpr bool CODES = decltype(codes_tag)::value;
    float sc[NB][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sc[nb][0] = sc[nb][1] = sc[nb][2] = sc[nb][3] = 0.f;
    const int lr = (lane & 7) + ((lane >> 3) & 1) * 8, lc = lane >> 4;      // ldmatrix: row and chunk this lane addresses
    if constexpr (CODES) {
#pragma unroll
      for (int ch = 0; ch < D / 16; ch += 2) {
        uint32_t r[4];
        ldmatrix_x4(r, img + off8<D>(0, lr, ch + lc));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t af[4];
          cache8_widen(r[2 * i], af[0], af[2]);
          cache8_widen(r[2 * i + 1], af[1], af[3]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_f16(sc[nb], af, qf[nb][ch + i][0], qf[nb][ch + i][1]);
        }
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t af[4];
        ldmatrix_x4(af, img + off16<D>(0, lr, ks * 2 + lc));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          if constexpr (Q8) mma_f16(sc[nb], af, qf[nb][ks][0], qf[nb][ks][1]);
          else mma_bf16(sc[nb], af, qf[nb][ks][0], qf[nb][ks][1]);
        }
      }
    }
    // scores of keys g (sc[..][0, 1]) and g + 8 (sc[..][2, 3])
    [[maybe_unused]] float ks0 = 1.f, ks1 = 1.f, ve0 = 0.f, ve1 = 0.f;
    float out0 = 1.f, out1 = 1.f;
    if constexpr (Q8) {
      // 2^8: see cache8_widen
      ks0 = 256.f * cache8_power(exps[g]);
      ks1 = 256.f * cache8_power(exps[g + 8]);
      const uint8_t b0 = exps[16 + g], b1 = exps[16 + g + 8];
      int e0 = cache8_exp_of(b0) + 8, e1 = cache8_exp_of(b1) + 8;
      if constexpr (CODES) {
        if (__any_sync(0xffffffffu, b0 == kCache8ZeroByte || b1 == kCache8ZeroByte)) {      // rows of zeros: the smallest exponent there is
          constexpr int CH = D / 16;
#pragma unroll 1
          for (int i = 0; i < CH / 2; ++i) {             // 32 / CH rows at a time
            const int r = i * (32 / CH) + lane / CH;
            const uint4 v = *reinterpret_cast<const uint4*>(smem + (img - base) + off8<D>(1, r, lane % CH));
            const uint32_t some = __ballot_sync(0xffffffffu, cache8_magnitudes(v) != 0);
            auto zeros = [&](int row) { return row / (32 / CH) == i && (some >> (row % (32 / CH) * CH) & ((1u << CH) - 1)) == 0; };
            if (b0 == kCache8ZeroByte && zeros(g)) e0 = 8 - kCache8MaxExp;
            if (b1 == kCache8ZeroByte && zeros(g + 8)) e1 = 8 - kCache8MaxExp;
          }
        }
      }
      ve0 = b0 == 255 ? CUDART_NAN_F : (float)e0;
      ve1 = b1 == 255 ? CUDART_NAN_F : (float)e1;
      out0 = power(-e0);
      out1 = power(-e1);
    }
    bool higher = false;
    float top[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x0 = sc[nb][i] * q_scale[nb][i], x1 = sc[nb][2 + i] * q_scale[nb][i];
        if constexpr (Q8) {
          x0 = fmaf(x0, ks0, ve0);
          x1 = fmaf(x1, ks1, ve1);
        }
        if constexpr (!CODES) {
          if ((bad >> g) & 1) x0 = CUDART_NAN_F;
          if ((bad >> (g + 8)) & 1) x1 = CUDART_NAN_F;
        }
        sc[nb][i] = see(nb, i, g) ? x0 : -CUDART_INF_F;
        sc[nb][2 + i] = see(nb, i, g + 8) ? x1 : -CUDART_INF_F;
        top[nb][i] = fmaxf(sc[nb][i], sc[nb][2 + i]);
        higher = higher || top[nb][i] > m[nb][i];
      }
    if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float t = top[nb][i];
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
          if (t > m[nb][i]) {                       // the same for all lanes that hold this query
            const float keep = ex2(m[nb][i] - t);   // 0 for the first key (m = -inf)
            m[nb][i] = t;
            l[nb][i] *= keep;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              o[d][nb][i] *= keep;
              o[d][nb][2 + i] *= keep;
            }
          }
        }
    }
    uint32_t pb[NB][2];                             // P^T as B fragments: queries down, keys across
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // no key seen so far: every score is -inf, and so must be the weight's exponent
        const float ref = (m[nb][i] == -CUDART_INF_F ? 0.f : m[nb][i]) - (Q8 ? kShift8 : 0.f);
        p[i] = ex2(sc[nb][i] - ref);
        p[2 + i] = ex2(sc[nb][2 + i] - ref);
        l[nb][i] = fmaf(p[i], out0, fmaf(p[2 + i], out1, l[nb][i]));
      }
      if constexpr (Q8) {
        pb[nb][0] = movmatrix_t(pack_f16(p[0], p[1]));
        pb[nb][1] = movmatrix_t(pack_f16(p[2], p[3]));
      } else {
        pb[nb][0] = movmatrix_t(pack_bf16(p[0], p[1]));
        pb[nb][1] = movmatrix_t(pack_bf16(p[2], p[3]));
      }
    }
    // O^T += V^T P^T, sixteen head_dim elements at a time
    if constexpr (CODES) {
      // a transposed 8 x 8 block of 16-bit units is eight pairs of elements of two keys: rows d = 2g of the product (0-7 of the fragment) come
      // from the even bytes, 2g + 1 (8-15) from the odd ones
#pragma unroll
      for (int ch = 0; ch < D / 16; ch += 2) {
        uint32_t r[4];
        ldmatrix_x4_trans(r, img + off8<D>(1, lr, ch + lc));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t af[4];
          cache8_widen(r[2 * i], af[0], af[1]);
          cache8_widen(r[2 * i + 1], af[2], af[3]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_f16(o[ch + i][nb], af, pb[nb][0], pb[nb][1]);
        }
      }
    } else {
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        // matrices: (keys 0-7, first 8 elements), (0-7, second 8), (8-15, first), (8-15, second)
        uint32_t af[4];
        const int key = (lane & 7) + (lane >> 4) * 8, chunk = d * 2 + ((lane >> 3) & 1);
        ldmatrix_x4_trans(af, img + off16<D>(1, key, chunk));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          if constexpr (Q8) mma_f16(o[d][nb], af, pb[nb][0], pb[nb][1]);
          else mma_bf16(o[d][nb], af, pb[nb][0], pb[nb][1]);
        }
      }
    }
  };

  // ---------------------------------------------------------------- cached tokens
  int n_done = 0;
#pragma unroll 1
  for (;; ++n_done) {
    const int p = it.k_begin + warp + n_done * kWarps;
    if (p >= cached_end) break;
    const int st = n_done % L::kStages;
    if (!__all_sync(0xffffffffu, mbar_wait(my_bars + st * 8, (n_done / L::kStages) & 1, s.wait_cycles))) {
      dead = true;
      break;
    }
    const uint32_t img = ring + st * L::kPageBytes;
    const int valid = ctx - p * kPageSize;          // keys of this page that hold a token
    if (valid < kPageSize) {
      // the V rows behind the last token may hold anything, and 0 * NaN is none: clear them
      for (int i = lane; i < (kPageSize - valid) * (L::kPageBytes / 512); i += 32) {
        const int per = L::kPageBytes / 512, r = valid + i / per, ch = i % per;     // 16-byte chunks of a row
        const uint32_t at = Q8 ? off8<D>(1, r, ch) : off16<D>(1, r, ch);
        *reinterpret_cast<uint4*>(smem + (img - base) + at) = make_uint4(0, 0, 0, 0);
      }
      __syncwarp();
    }
    const uint8_t* exps = smem + L::kOffScale + (warp * L::kStages + st) * 32;
    if (valid >= kPageSize)
      page_step(std::integral_constant<bool, Q8>(), img, exps, [](int, int, int) { return true; });
    else
      page_step(std::integral_constant<bool, Q8>(), img, exps, [&](int, int, int key) { return key < valid; });
    __syncwarp();
    fill(n_done + 1);
  }
  if (dead) {
    if (lane == 0) atomicOr(s.status, TS_DEV_TIMEOUT);
    for (int i = n_done; i < n_issued; ++i) mbar_wait(my_bars + i % L::kStages * 8, (i / L::kStages) & 1, kDrainCycles);
  }

  // ---------------------------------------------------------------- the row's own nodes
  const uint32_t own = ring;
  uint8_t* own_exp = smem + L::kOffOwnExp + warp * 32;
#pragma unroll 1
  for (int p = max(it.k_begin, n_cached); p < it.k_end; ++p) {
    if ((p - it.k_begin) % kWarps != warp) continue;
    const int j0 = (p - n_cached) * kPageSize, valid = min(kPageSize, T - j0);
    constexpr int CH = D / 8;                       // 16-byte chunks of a row
    // A V row that is not finite must not reach the nodes that do not see it (0 * NaN): it becomes zeros, and a NaN score for
    // those that do.
    uint32_t bad = 0;                               // bit r: row r is one
    __syncwarp();
#pragma unroll 1
    for (int kv = 0; kv < 2; ++kv) {
      const uint16_t* src = (kv ? s.v_new : s.k_new) + ((size_t)(tok0 + j0) * s.Hkv + head) * D;
#pragma unroll
      for (int i0 = 0; i0 < kPageSize * CH; i0 += 32) {
        const int r = (i0 + lane) / CH, ch = (i0 + lane) % CH;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (r < valid) w = *reinterpret_cast<const uint4*>(src + (size_t)r * s.Hkv * D + ch * 8);
        if (kv) {
          auto odd = [](uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; };
          const uint32_t lanes = __ballot_sync(0xffffffffu, odd(w.x) || odd(w.y) || odd(w.z) || odd(w.w));
          constexpr uint32_t kRow = (uint32_t)((1ull << CH) - 1);
#pragma unroll
          for (int i = 0; i < 32 / CH; ++i)
            if (lanes & (kRow << (i * CH))) bad |= 1u << (i0 / CH + i);
          if ((bad >> r) & 1) w = make_uint4(0, 0, 0, 0);
        }
        if constexpr (Q8) {
          uint32_t x[4] = {w.x, w.y, w.z, w.w}, most = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) most = max(most, max(x[i] & 0x7fffu, (x[i] >> 16) & 0x7fffu));
#pragma unroll
          for (int sh = 1; sh < CH; sh <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, sh));
          // largest element to 2^14 .. 2^15 (f16 ends at 65504)
          const int e = min(max((int)(most >> 7) - 127 - 14, 8 - kCache8MaxExp), 8 + kCache8MaxExp);      // zeros: the smallest there is
          const float down = power(-e);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = pack_f16(__uint_as_float(x[i] << 16) * down, __uint_as_float(x[i] & 0xffff0000u) * down);
          // as of codes; a K row that is not finite is one of NaN, as in the tcgen05 kernel, whose codes have no infinities
          if (ch == 0) own_exp[kv * 16 + r] = most >= 0x7f80u ? 255 : (uint8_t)(e - 8 + 127);
          // in the order that codes come in: of each sixteen elements the even ones first
          const uint32_t at0 = own - base + off16<D>(kv, r, ch & ~1) + (ch & 1) * 8, at1 = own - base + off16<D>(kv, r, ch | 1) + (ch & 1) * 8;
          *reinterpret_cast<uint2*>(smem + at0) = make_uint2(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410));
          *reinterpret_cast<uint2*>(smem + at1) = make_uint2(__byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632));
        } else {
          *reinterpret_cast<uint4*>(smem + (own - base) + off16<D>(kv, r, ch)) = w;
        }
      }
    }
    __syncwarp();
    uint64_t bits[NB][2];                           // the nodes of this page that queries 8 nb + 2c, + 1 see
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int q = nb * 8 + 2 * c + i, node = t0 + (q < n_q ? q / G : 0);
        bits[nb][i] = a.mask ? a.mask[tok0 + node] >> j0 : ((2ull << node) - 1) >> j0;
      }
    page_step(std::false_type(), own, own_exp, [&](int nb, int i, int key) { return key < valid && ((bits[nb][i] >> key) & 1); }, bad);
    __syncwarp();
  }

  // ---------------------------------------------------------------- sum over the warps
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[nb][i] += __shfl_xor_sync(0xffffffffu, l[nb][i], 4);
      l[nb][i] += __shfl_xor_sync(0xffffffffu, l[nb][i], 8);
      l[nb][i] += __shfl_xor_sync(0xffffffffu, l[nb][i], 16);
    }
  __syncthreads();                                  // the stages are free: no copy of any warp is in flight
  float* res = reinterpret_cast<float*>(smem);      // [warp][query][D + 2]: O, maximum, sum
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float* mine = res + ((size_t)warp * NB * 8 + nb * 8 + 2 * c + i) * (D + 2);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        mine[d * 16 + (Q8 ? 2 * g : g)] = o[d][nb][i];
        mine[d * 16 + (Q8 ? 2 * g + 1 : g + 8)] = o[d][nb][2 + i];
      }
      if (g == 0) {
        mine[D] = m[nb][i];
        mine[D + 1] = l[nb][i];
      }
    }
  __syncthreads();
  for (int i = tid; i < n_q * (D / 2); i += kThreads) {
    const int q = i / (D / 2), d = i % (D / 2) * 2;
    const float* first = res + (size_t)q * (D + 2);
    constexpr int stride = NB * 8 * (D + 2);
    float mm = -CUDART_INF_F, ll = 0.f, x0 = 0.f, x1 = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, first[w * stride + D]);
    const float ref = mm == -CUDART_INF_F ? 0.f : mm;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2(first[w * stride + D] - ref);    // 0 for a warp that saw no key
      ll += f * first[w * stride + D + 1];
      x0 += f * first[w * stride + d];
      x1 += f * first[w * stride + d + 1];
    }
    const int node = t0 + q / G, hd = head * G + q % G;
    if (it.partial_slot < 0) {
      const float inv = ll == 0.f ? 0.f : 1.f / ll;         // no visible key: zeros
      *reinterpret_cast<uint32_t*>(s.out + ((size_t)(tok0 + node) * s.Hq + hd) * D + d) = pack_bf16(x0 * inv, x1 * inv);
    } else {
      const size_t ph = (size_t)(it.partial_slot + node) * s.Hq + hd;
      *reinterpret_cast<float2*>(s.part_acc + ph * D + d) = make_float2(x0, x1);
      if (d == 0) *reinterpret_cast<float2*>(s.part_ml + ph * 2) = make_float2(mm, ll);
    }
  }
}

// Merge of the splits of a row's nodes: a warp per (node, head), D / 32 elements a lane, eight splits' loads in flight. Bound by its round trips:
// 12 pages' worth of a unit in the host's rule for pieces (about 3 us behind one row of 32768 keys x 64 nodes, whose partials stay in L2).
template <int D>
__global__ void __launch_bounds__(256)
tree_combine_kernel(const __grid_constant__ StepParams<kInlineWords> params) {
  const StepDevice& s = params.s;
  constexpr int E = D / 32;
  pdl_launch_dependents();
  pdl_wait();
  const CombineItem ci = s.combine(blockIdx.y);
  const int T = ci.reserved, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pair = blockIdx.x * 8 + warp;
  if (pair >= T * s.Hq) return;
  const int node = pair / s.Hq, h = pair % s.Hq;
  const size_t first = (size_t)(ci.first_partial + node) * s.Hq + h, step = (size_t)T * s.Hq;
  float m = -CUDART_INF_F, l = 0.f, acc[E] = {};
  for (int b = 0; b < ci.n_splits; b += 8) {
    float2 ml[8];
    float x[8][E];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool on = b + j < ci.n_splits;
      ml[j] = on ? __ldcg(reinterpret_cast<const float2*>(s.part_ml) + first + (b + j) * step) : make_float2(-CUDART_INF_F, 0.f);
      const float* src = s.part_acc + (first + (b + j) * step) * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 v = on ? __ldcg(reinterpret_cast<const float2*>(src + e)) : make_float2(0.f, 0.f);
        x[j][e] = v.x;
        x[j][e + 1] = v.y;
      }
    }
    float mn = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) mn = fmaxf(mn, ml[j].x);
    const float ref = mn == -CUDART_INF_F ? 0.f : mn;       // nothing seen so far: all weights are 2^-inf
    const float keep = ex2(m - ref);
    l *= keep;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= keep;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float w = ex2(ml[j].x - ref);
      l = fmaf(w, ml[j].y, l);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(w, x[j][e], acc[e]);
    }
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint32_t* dst = reinterpret_cast<uint32_t*>(s.out + ((size_t)(ci.token + node) * s.Hq + h) * D + lane * E);
#pragma unroll
  for (int e = 0; e < E; e += 2) dst[e / 2] = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
}

template <int D, int NB, bool Q8>
cudaError_t launch_t(const StepDevice& s, const TreeArgs& a, const CUtensorMap& kv_map, cudaStream_t stream) {
  constexpr int smem = Smem<D, NB, Q8>::bytes();
  cudaError_t e = cudaFuncSetAttribute(tree_kernel<D, NB, Q8>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  StepParams<kInlineWords> params;
  fill_params(s, &params);
  return launch_pdl(tree_kernel<D, NB, Q8>, dim3((unsigned)(s.n_items * s.Hkv * a.n_tiles)), dim3(kThreads), smem, stream, params, a, kv_map);
}
template <int D, bool Q8>
cudaError_t launch_d(const StepDevice& s, const TreeArgs& a, const CUtensorMap& kv_map, cudaStream_t stream) {
  const int queries = a.tile_tokens * (s.Hq / s.Hkv);
  if (queries <= 8) return launch_t<D, 1, Q8>(s, a, kv_map, stream);
  if (queries <= 16) return launch_t<D, 2, Q8>(s, a, kv_map, stream);
  if constexpr (D == 128 && !Q8) return cudaErrorInvalidValue;      // more than kTreeTcQueries queries: on tcgen05
  else return launch_t<D, 4, Q8>(s, a, kv_map, stream);
}

}  // namespace

int tree_tile_tokens(int G, int nodes) {
  const int most = 32 / G;
  return nodes < most ? nodes : most;
}
int tree_blocks_per_sm(int queries, bool q8) {
  if (!q8) return Smem<128, 1, false>::kBlocks;
  return queries <= 8 ? Smem<128, 1, true>::kBlocks : queries <= 16 ? Smem<128, 2, true>::kBlocks : Smem<128, 4, true>::kBlocks;
}

cudaError_t launch_tree(const StepDevice& s, const TreeArgs& a, const CUtensorMap& kv_map, cudaStream_t stream) {
  if (s.n_items <= 0) return cudaSuccess;
  if (a.cache.values) return s.D == 128 ? launch_d<128, true>(s, a, kv_map, stream) : launch_d<64, true>(s, a, kv_map, stream);
  return s.D == 128 ? launch_d<128, false>(s, a, kv_map, stream) : launch_d<64, false>(s, a, kv_map, stream);
}

cudaError_t launch_tree_combine(const StepDevice& s, int max_nodes, cudaStream_t stream) {
  if (s.n_combines <= 0) return cudaSuccess;
  StepParams<kInlineWords> params;
  fill_params(s, &params);
  const dim3 grid((max_nodes * s.Hq + 7) / 8, s.n_combines);
  return s.D == 128 ? launch_pdl(tree_combine_kernel<128>, grid, dim3(256), 0, stream, params)
                    : launch_pdl(tree_combine_kernel<64>, grid, dim3(256), 0, stream, params);
}

}  // namespace ts
