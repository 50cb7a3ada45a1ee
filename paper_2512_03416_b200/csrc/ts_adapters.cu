// Low-rank adapters of the requests of a step (sm_100a), first half: u = scale_a * x . A_a^T of every token whose request has
// an adapter a, rounded to bf16 and laid out as the GEMM kernels read it (AdapterTiles): an entry per tile of tokens and adapter,
// zeros in the rows of other adapters' tokens. The second half, u . B_a^T, is part of the projection itself (ts_gemm.cu).
//
// A thread block takes up to 16 tokens of an entry and one granule (16, 32 or 64) of the rank: 16 x width sums over K with mma.sync
// (m16n8k16, fp32), eight warps and, where there are few of these, a cluster of up to eight blocks sharing K. Nothing is staged:
// a sum over K may take its elements in any order as long as x and A agree, so a lane loads 16 bytes of a row of x and of the rows of A
// and these are the operands of two MMAs. In a decode batch a block reads A_a (its only user), so that the launch is bound by the bytes of the
// adapters in use; in a prompt's chunk x and A come from L2, each A once per 16 tokens.
// The partial sums are added up in a fixed order (warps, then blocks): equal calls give equal bits.
#include <cuda_bf16.h>

#include <algorithm>
#include <new>

#include "../../include/tokenscale.h"
#include "ts_internal.h"
#include "ts_ptx.h"

namespace ts {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kGroup = 16;                      // tokens of a thread block
constexpr int kMaxCluster = 8;

template <int W>
struct DownParams {
  AdapterDown d;
  int32_t words[W];
};

__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;\n" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(addr));
  return v;
}

// WIDTH: ranks of a granule. U: steps of 32 of K whose loads a warp has in flight.
template <int WIDTH, int U, int W>
__global__ void __launch_bounds__(kThreads) adapter_down_kernel(const __grid_constant__ DownParams<W> p, const int split) {
  constexpr int NT = WIDTH / 8;
  __shared__ float part[kWarps][kGroup][WIDTH + 2];
  __shared__ float sums[kGroup * WIDTH];
  __shared__ int16_t member[kGroup];            // places in the tile of the block's tokens
  const AdapterDown& d = p.d;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  const int32_t* entry_adapter = p.words + d.o_adapter;
  const int32_t* item_first = p.words + d.o_item;
  const int item = blockIdx.x / split, rank_of = blockIdx.x % split;   // the cluster's blocks are consecutive
  const int c = item % d.granules, group_at = item / d.granules;
  int e = 0;                                    // the entry: last one whose first group is <= group_at
  for (int hi = d.n_entries; hi - e > 1;) {
    const int mid = (e + hi) >> 1;
    if (item_first[mid] <= group_at) e = mid; else hi = mid;
  }
  const int group = group_at - item_first[e];
  const int adapter = entry_adapter[e], t0 = p.words[d.o_tile + e] * d.rows;
  // this thread's place in the tile: its number among the entry's tokens, or -1
  int mine = -1, count = 0;
  for (int s = p.words[d.o_seg_first + e]; s < p.words[d.o_seg_first + e + 1]; ++s) {
    const int from = p.words[d.o_seg + s] & 0xffff, len = p.words[d.o_seg + s] >> 16;
    if (tid >= from && tid < from + len) mine = count + tid - from;
    count += len;
  }
  if (mine >= group * kGroup && mine < (group + 1) * kGroup) member[mine - group * kGroup] = (int16_t)tid;
  const int n = min(kGroup, count - group * kGroup);
  __syncthreads();
  pdl_wait();                                   // x comes from the launch in front; the one before may still read u and the plan
  if (blockIdx.x == 0)
    for (int i = tid; i <= d.n_tiles + d.n_entries; i += kThreads) d.plan[i] = p.words[i];
  uint16_t* const u = d.u + (size_t)(e * d.granules + c) * d.rows * WIDTH;
  if (group == 0 && rank_of == 0 && mine < 0 && tid < d.rows) {
#pragma unroll
    for (int i = 0; i < WIDTH / 8; ++i) reinterpret_cast<uint4*>(u + (size_t)tid * WIDTH)[i] = make_uint4(0, 0, 0, 0);
  }

  const int g = lane >> 2, t = lane & 3;
  const int chunks = (d.K + 31) / 32, first = chunks * rank_of / split, end = chunks * (rank_of + 1) / split;
  const uint16_t* x0 = d.x + (size_t)(t0 + (g < n ? member[g] : 0)) * d.K;
  const uint16_t* x1 = d.x + (size_t)(t0 + (g + 8 < n ? member[g + 8] : 0)) * d.K;
  const uint16_t* a0 = d.a + ((size_t)adapter * d.rank + c * WIDTH + g) * d.K;
  const int ranks = d.rank - c * WIDTH - g;     // row j * 8 of a0 is there where j * 8 < ranks
  float acc[NT][4] = {};
  for (int ch = first + warp; ch < end; ch += kWarps * U) {
    uint4 xa[U][2], w[U][NT];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int k = (ch + i * kWarps) * 32 + t * 8;
      const bool in = ch + i * kWarps < end && k < d.K;
      xa[i][0] = xa[i][1] = make_uint4(0, 0, 0, 0);
      if (in && g < n) xa[i][0] = *reinterpret_cast<const uint4*>(x0 + k);
      if (in && g + 8 < n) xa[i][1] = *reinterpret_cast<const uint4*>(x1 + k);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        w[i][j] = make_uint4(0, 0, 0, 0);
        if (in && j * 8 < ranks) w[i][j] = *reinterpret_cast<const uint4*>(a0 + (size_t)(j * 8) * d.K + k);
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const uint32_t lo[4] = {xa[i][0].x, xa[i][1].x, xa[i][0].y, xa[i][1].y}, hi[4] = {xa[i][0].z, xa[i][1].z, xa[i][0].w, xa[i][1].w};
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        mma_bf16(acc[j], lo, w[i][j].x, w[i][j].y);
        mma_bf16(acc[j], hi, w[i][j].z, w[i][j].w);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    *reinterpret_cast<float2*>(&part[warp][g][j * 8 + 2 * t]) = make_float2(acc[j][0], acc[j][1]);
    *reinterpret_cast<float2*>(&part[warp][g + 8][j * 8 + 2 * t]) = make_float2(acc[j][2], acc[j][3]);
  }
  __syncthreads();
  for (int i = tid; i < kGroup * WIDTH; i += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += part[w][i / WIDTH][i % WIDTH];
    sums[i] = v;
  }
  const float scale = d.scale ? d.scale[adapter] : 1.f;
  if (split > 1) cluster_sync(); else __syncthreads();
  const uint32_t at = smem_u32(sums);
  for (int i = (rank_of * kThreads + tid) * 2; i < n * WIDTH; i += split * kThreads * 2) {
    float lo = 0.f, hi = 0.f;
    for (int r = 0; r < split; ++r) {
      const uint32_t from = split > 1 ? mapa(at, r) : at;
      lo += ld_cluster(from + i * 4);
      hi += ld_cluster(from + i * 4 + 4);
    }
    *reinterpret_cast<uint32_t*>(u + (size_t)member[i / WIDTH] * WIDTH + i % WIDTH) = pack_bf16(lo * scale, hi * scale);
  }
  if (split > 1) cluster_sync();                // no block leaves while another one reads its sums
}

template <int WIDTH, int U, int W>
cudaError_t launch_w(const AdapterDown& d, const int32_t* words, int n_words, int items, int split, cudaStream_t stream) {
  DownParams<W> p;
  p.d = d;
  std::memcpy(p.words, words, sizeof(int32_t) * (size_t)n_words);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * split));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, adapter_down_kernel<WIDTH, U, W>, p, split);
}
template <int WIDTH, int U>
cudaError_t launch_t(const AdapterDown& d, const int32_t* words, int n_words, int items, int split, cudaStream_t stream) {
  return n_words <= kInlineWords ? launch_w<WIDTH, U, kInlineWords>(d, words, n_words, items, split, stream)
                                 : launch_w<WIDTH, U, kAdapterWords>(d, words, n_words, items, split, stream);
}

}  // namespace

bool plan_adapters(int M, int rows, int n_rows, const int32_t* row_tokens, const int32_t* row_adapter, int n_adapters, AdapterPlan* out) try {
  struct Run { int entry, from, len; };
  std::vector<int32_t> tile_first{0}, adapter, tile, groups{0}, seg_first{0}, segs;
  std::vector<Run> runs;                        // of the current tile
  std::vector<int32_t> entry_of((size_t)n_adapters, -1);
  int r = 0, left = n_rows > 0 ? row_tokens[0] : 0;
  for (int t0 = 0; t0 < M; t0 += rows) {
    const int first = (int)adapter.size();
    runs.clear();
    for (int at = 0, n = std::min(rows, M - t0); at < n;) {
      while (left == 0) left = row_tokens[++r];
      const int len = std::min(left, n - at), a = row_adapter[r];
      if (a >= 0) {
        if (entry_of[a] < first) {
          entry_of[a] = (int)adapter.size();
          adapter.push_back(a);
          tile.push_back(t0 / rows);
        }
        if (!runs.empty() && runs.back().entry == entry_of[a] && runs.back().from + runs.back().len == at) runs.back().len += len;
        else runs.push_back({entry_of[a], at, len});
      }
      at += len;
      left -= len;
    }
    std::stable_sort(runs.begin(), runs.end(), [](const Run& x, const Run& y) { return x.entry < y.entry; });
    size_t i = 0;
    for (int e = first; e < (int)adapter.size(); ++e) {
      int tokens = 0;
      for (; i < runs.size() && runs[i].entry == e; ++i) {
        segs.push_back(runs[i].from | runs[i].len << 16);
        tokens += runs[i].len;
      }
      seg_first.push_back((int32_t)segs.size());
      groups.push_back(groups.back() + (tokens + kGroup - 1) / kGroup);
    }
    tile_first.push_back((int32_t)adapter.size());
  }
  out->n_tiles = (int)tile_first.size() - 1;
  out->n_entries = (int)adapter.size();
  out->n_groups = groups.back();
  out->words.clear();
  auto put = [&](const std::vector<int32_t>& v) {
    const uint32_t at = (uint32_t)out->words.size();
    out->words.insert(out->words.end(), v.begin(), v.end());
    return at;
  };
  put(tile_first);
  out->o_adapter = put(adapter);
  out->o_tile = put(tile);
  out->o_item = put(groups);
  out->o_seg_first = put(seg_first);
  out->o_seg = put(segs);
  return out->words.size() <= (size_t)kAdapterWords;
} catch (const std::bad_alloc&) {
  return false;
}

cudaError_t launch_adapter_down(AdapterDown d, const AdapterPlan& plan, int width, int n_sms, cudaStream_t stream) {
  if (plan.n_entries == 0) return cudaSuccess;
  d.n_tiles = plan.n_tiles;
  d.n_entries = plan.n_entries;
  d.granules = (d.rank + width - 1) / width;
  d.o_adapter = plan.o_adapter; d.o_tile = plan.o_tile; d.o_item = plan.o_item; d.o_seg_first = plan.o_seg_first; d.o_seg = plan.o_seg;
  const int items = plan.n_groups * d.granules;
  // two blocks per SM, each with a step of 32 of K for every warp at least
  const int split = std::max(1, std::min({kMaxCluster, 2 * n_sms / items, (d.K + 32 * kWarps - 1) / (32 * kWarps)}));
  const int n = (int)plan.words.size();
  switch (width) {
    case 16: return launch_t<16, 4>(d, plan.words.data(), n, items, split, stream);
    case 32: return launch_t<32, 4>(d, plan.words.data(), n, items, split, stream);
    default: return launch_t<64, 2>(d, plan.words.data(), n, items, split, stream);
  }
}

}  // namespace ts
