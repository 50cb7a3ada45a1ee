// Low-rank adapters of the requests of a step (sm_100a), first half: u = scale_a * x . A_a^T of every token whose request has
// an adapter a, rounded to bf16 and laid out as the GEMM kernels read it (AdapterTiles): an entry per tile of tokens and adapter,
// zeros in the rows of other adapters' tokens. The second half, u . B_a^T, is part of the projection itself (ts_gemm.cu).
//
// A thread block takes up to 16 or 64 tokens of an entry and one granule (16, 32 or 64) of the rank, and, where there are few of these blocks, a cluster
// of up to eight shares K. Rows of x (gathered) and of A go through a ring of stages in shared memory by 16-byte asynchronous copies to
// mma.sync (m16n8k16, fp32); a warp has 16 tokens, or a share of each stage's K. In a decode batch a block reads A_a (its only
// user), so that the launch is bound by the bytes of the adapters in use; in a prompt's chunk x and A come from L2, each A once per 64 tokens.
// The launch runs next to the product behind it, whose main loop does not need u: a block is small enough (128 threads, 56 KB) to share an SM
// with one of the product's, and there is one per SM where that is enough. Blocks of 256 threads with 64 to 96 KB of copies under way take less
// by themselves, but the product waited for them: both together 29.5 and 70.5 us where these took 27 and 62.4.
//
// Measured, this launch alone / the product without adapters / both together, us: 64 tokens, 64 adapters of rank 16, K = 4096, N = 6144: 7.6 / 15.8 / 23.3;
// 192 tokens, 48 adapters of rank 32, K = N = 8192: 12.2 / 41.4 / 58.4; 2112 tokens, 16 adapters of rank 64, K = 4096, N = 28672: 22.8 / 321 / 363;
// 2319 tokens, 5 adapters of rank 24, K = 14336, N = 4096: 34.2 / 213 / 236.
// u is rounded to bf16 because that is what the product multiplies: off by 2^-9 of itself, next to a result that is rounded to bf16 as well. In two bf16 parts, both multiplied with the
// same B, it would be as exact as in fp32 at 24.6 / 63.2 / 441 us for the first three (22.8 / 61.6 / 420 with one part, host included).
// The partial sums are added up in a fixed order (warps, then blocks): equal calls give equal bits.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <new>

#include "../../include/tokenscale.h"
#include "ts_internal.h"
#include "ts_ptx.h"

namespace ts {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kRingBytes = 56 * 1024;           // next to 162 KB of a GEMM kernel's stages
constexpr int kGroup = 64;                      // most tokens of a thread block
constexpr int kMaxCluster = 8;

template <int W>
struct DownParams {
  AdapterDown d;
  int32_t words[W];
};
static_assert(sizeof(DownParams<kAdapterWords>) + sizeof(int) <= 32764, "what a launch's parameters may take");

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

// WIDTH: ranks of a granule. MT: sixteens of tokens of a block.
template <int WIDTH, int MT>
struct Down {
  static constexpr int kTokens = 16 * MT, kParts = kWarps / MT;      // of a stage's K, a warp each
  static constexpr int kDepth = MT == 1 && WIDTH < 64 ? 128 : 64;     // K of a stage
  static constexpr int kChunks = kDepth / 8;                         // of 16 bytes in a row
  static constexpr int kStageBytes = (kTokens + WIDTH) * kDepth * 2;
  static constexpr int kStages = kRingBytes / kStageBytes < 8 ? kRingBytes / kStageBytes : 8;
  static constexpr int kSteps = kDepth / 16 / kParts;                // sixteens of K of a warp and stage
  static constexpr int kPartBytes = kParts * kTokens * (WIDTH + 2) * 4;
  static constexpr int kBytes = kStages * kStageBytes > kPartBytes ? kStages * kStageBytes : kPartBytes;
  static_assert(kStages >= 2 && kSteps >= 1, "a stage is read while another one is filled");
  // Place of a 16-byte chunk of a row, such that eight rows' chunks lie in different banks.
  static __device__ __forceinline__ uint32_t place(int stage, int row, int chunk) {
    return (uint32_t)(stage % kStages * kStageBytes + row * kDepth * 2 + ((chunk ^ (row & 7)) << 4));
  }
};

template <int WIDTH, int MT, int W>
__global__ void __launch_bounds__(kThreads, 5) adapter_down_kernel(const __grid_constant__ DownParams<W> p, const int split) {
  using D = Down<WIDTH, MT>;
  constexpr int NT = WIDTH / 8, kTokens = D::kTokens, kPitch = WIDTH + 2;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int32_t token_of[kTokens], entry_of[kTokens];   // the block's tokens and their entries
  float* const part = reinterpret_cast<float*>(smem);      // [kParts][kTokens][kPitch], when the stages are done with
  const AdapterDown& d = p.d;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t* const words = p.words;
  const int item = blockIdx.x / split, rank_of = blockIdx.x % split;   // the cluster's blocks are consecutive
  const int c = item % d.granules, group = item / d.granules;
  const uint32_t what = (uint32_t)words[d.o_item + 2 * group], where = (uint32_t)words[d.o_item + 2 * group + 1];
  const int adapter = what & 0xffff, n = what >> 16;                   // tokens of the group
  const uint32_t base = smem_u32(smem);
  const int stages = (d.K + D::kDepth - 1) / D::kDepth, first = stages * rank_of / split, end = stages * (rank_of + 1) / split;
  const uint16_t* const a = d.a + ((size_t)adapter * d.rank + c * WIDTH) * d.K;
  const int ranks = min(WIDTH, d.rank - c * WIDTH);
  // 16-byte chunks of a stage's rows of A, or of x; what is not there is zero
  auto copy_a = [&](int stage) {
#pragma unroll
    for (int i = tid; i < WIDTH * D::kChunks; i += kThreads) {
      const int row = i / D::kChunks, ch = i % D::kChunks, k = stage * D::kDepth + ch * 8;
      const bool in = row < ranks && k < d.K;
      cp_async16(base + D::place(stage, kTokens + row, ch), in ? a + (size_t)row * d.K + k : a, in ? 16 : 0);
    }
  };
  // The rows of A go to L2 while the launch in front ends: a hint only, nothing is read before the wait.
  if (tid < ranks) {
    const int k0 = first * D::kDepth, ahead = min(min(end, first + D::kStages) * D::kDepth, d.K) - k0;
    if (ahead > 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(a + (size_t)tid * d.K + k0), "r"(ahead * 2) : "memory");
  }

  for (int got = 0, run = where & 0xffff, skip = where >> 16; got < n; ++run, skip = 0) {      // the group's tokens
    const uint32_t place = (uint32_t)words[d.o_run + 2 * run];
    const int t0 = place & 0xffff, len = min((int)(place >> 16) - skip, n - got), e = words[d.o_run + 2 * run + 1];
    for (int k = tid; k < len; k += kThreads) {
      token_of[got + k] = t0 + skip + k;
      entry_of[got + k] = e;
    }
    got += len;
  }
  __syncthreads();
  pdl_wait();                                   // x comes from the launch in front; the one before may still read u and the plan
  // The product behind this launch may start: what was before is done, which is all that its main loop reads.
  pdl_launch_dependents();
  auto copy_x = [&](int stage) {
#pragma unroll
    for (int i = tid; i < kTokens * D::kChunks; i += kThreads) {
      const int row = i / D::kChunks, ch = i % D::kChunks, k = stage * D::kDepth + ch * 8;
      const bool in = row < n && k < d.K;
      cp_async16(base + D::place(stage, row, ch), in ? d.x + (size_t)token_of[row] * d.K + k : d.x, in ? 16 : 0);
    }
  };
#pragma unroll 1
  for (int s = first; s < first + D::kStages; ++s) {
    if (s < end) {
      copy_a(s);
      copy_x(s);
    }
    cp_async_commit();                          // a group per stage, the last ones empty
  }
  if (blockIdx.x == 0 && d.plan)
    for (int i = tid; i <= d.n_tiles + d.n_entries; i += kThreads) d.plan[i] = words[i];
  auto u_of = [&](int entry, int granule) { return reinterpret_cast<char*>(d.u + (size_t)(entry * d.granules + granule) * d.rows * WIDTH); };
  for (int i = blockIdx.x; i < d.n_entries * d.granules; i += gridDim.x) {      // the rows of other adapters' tokens
    const int e = i / d.granules;
    char* const u = u_of(e, i % d.granules);
    for (int row = tid; row < d.rows; row += kThreads) {
      bool member = false;
      for (int s = words[d.o_seg_first + e]; s < words[d.o_seg_first + e + 1]; ++s) {
        const int k = row - (words[d.o_seg + s] & 0xffff);
        member = member || (k >= 0 && k < words[d.o_seg + s] >> 16);
      }
      if (member) continue;
#pragma unroll
      for (int k = 0; k < WIDTH / 8; ++k) *reinterpret_cast<uint4*>(u + granule_place(WIDTH, row, k)) = make_uint4(0, 0, 0, 0);
    }
  }

  const int g = lane >> 2, t = lane & 3, mt = warp % MT, kp = warp / MT;
  float acc[NT][4] = {};
#pragma unroll 1
  for (int s = first; s < end; ++s) {
    cp_async_wait<D::kStages - 1>();
    __syncthreads();                            // the stage is there
    if (mt * 16 < n) {
#pragma unroll
      for (int i = 0; i < D::kSteps; ++i) {
        const int ch = (kp * D::kSteps + i) * 2;
        uint32_t xa[4];
        ldmatrix_x4(xa, base + D::place(s, mt * 16 + (lane & 15), ch + (lane >> 4)));
#pragma unroll
        for (int j = 0; j < NT; j += 2) {       // sixteen rows of A: lanes 0-7, 8-15 the halves of K of the first eight, 16-31 of the others
          uint32_t w[4];
          ldmatrix_x4(w, base + D::place(s, kTokens + j * 8 + (lane & 7) + (lane >> 4) * 8, ch + (lane >> 3 & 1)));
          mma_bf16(acc[j], xa, w[0], w[1]);
          mma_bf16(acc[j + 1], xa, w[2], w[3]);
        }
      }
    }
    __syncthreads();                            // and read
    if (s + D::kStages < end) {
      copy_a(s + D::kStages);
      copy_x(s + D::kStages);
    }
    cp_async_commit();
  }
  cp_async_wait<0>();
  __syncthreads();                              // the sums take the stages' place
  auto at = [&](int k, int row, int col) { return (k * kTokens + row) * kPitch + col; };
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    *reinterpret_cast<float2*>(part + at(kp, mt * 16 + g, j * 8 + 2 * t)) = make_float2(acc[j][0], acc[j][1]);
    *reinterpret_cast<float2*>(part + at(kp, mt * 16 + g + 8, j * 8 + 2 * t)) = make_float2(acc[j][2], acc[j][3]);
  }
  __syncthreads();
  for (int i = tid; i < n * WIDTH; i += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < D::kParts; ++k) v += part[at(k, i / WIDTH, i % WIDTH)];
    part[at(0, i / WIDTH, i % WIDTH)] = v;      // this thread's alone
  }
  const float scale = d.scale ? d.scale[adapter] : 1.f;
  if (split > 1) cluster_sync(); else __syncthreads();
  for (int i = (rank_of * kThreads + tid) * 2; i < n * WIDTH; i += split * kThreads * 2) {
    float lo[kMaxCluster], hi[kMaxCluster];
    const uint32_t own = smem_u32(part + at(0, i / WIDTH, i % WIDTH));
#pragma unroll
    for (int r = 0; r < kMaxCluster; ++r) {      // all loads fly at once
      lo[r] = hi[r] = 0.f;
      if (r < split) {
        const uint32_t from = split > 1 ? mapa(own, r) : own;
        lo[r] = ld_cluster(from);
        hi[r] = ld_cluster(from + 4);
      }
    }
#pragma unroll
    for (int r = 1; r < kMaxCluster; ++r) {
      lo[0] += lo[r];
      hi[0] += hi[r];
    }
    const int col = i % WIDTH, entry = entry_of[i / WIDTH], row = token_of[i / WIDTH] % d.tile;
    *reinterpret_cast<uint32_t*>(u_of(entry, c) + granule_place(WIDTH, row, col / 8) + (col % 8) * 2) = pack_bf16(lo[0] * scale, hi[0] * scale);
  }
  if (split > 1) cluster_sync();                // no block leaves while another one reads its sums
}

// One thread per 16 bytes of the packed form.
__global__ void __launch_bounds__(256) adapter_pack_kernel(const uint16_t* __restrict__ b, char* __restrict__ out, int N, int rank, int width, int granules,
                                                                int blocks, int apart, size_t chunks) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const int per_row = width / 8, chunk = (int)(i % per_row), r = (int)(i / per_row % 128);
  const size_t image = i / per_row / 128;       // (adapter, granule, block)
  const int block = (int)(image % blocks), c = (int)(image / blocks % granules);
  const size_t adapter = image / blocks / granules;
  int row = block * 128 + r;
  if (apart > 0) {                              // sixteen rows and the sixteen `apart` behind them, in turn
    const int span = 2 * apart, first = block * 128 / span * span, s = block * 128 % span / 32 + r / 32;
    row = first + (r / 16 % 2) * apart + s * 16 + r % 16;
  }
  uint32_t v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t word = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int col = c * width + chunk * 8 + k * 2 + h;
      if (row < N && col < rank) word |= (uint32_t)b[(adapter * N + row) * rank + col] << (16 * h);
    }
    v[k] = word;
  }
  *reinterpret_cast<uint4*>(out + image * 128 * width * 2 + granule_place(width, r, chunk)) = make_uint4(v[0], v[1], v[2], v[3]);
}

template <int WIDTH, int MT, int W>
cudaError_t launch_w(const AdapterDown& d, const int32_t* words, int n_words, int items, int split, cudaStream_t stream) {
  DownParams<W> p;
  p.d = d;
  std::memcpy(p.words, words, sizeof(int32_t) * (size_t)n_words);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(items * split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Down<WIDTH, MT>::kBytes;
  static std::atomic<uint64_t> ready{0};        // devices on which these are set
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(ready.load(std::memory_order_acquire) >> device & 1)) {
    // the SM's memory divided as the product behind this launch needs it: it cannot be divided anew while a block runs
    e = cudaFuncSetAttribute(adapter_down_kernel<WIDTH, MT, W>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(adapter_down_kernel<WIDTH, MT, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
    if (e != cudaSuccess) return e;
    if (device < 64) ready.fetch_or(1ull << device, std::memory_order_release);
  }
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, adapter_down_kernel<WIDTH, MT, W>, p, split);
}
template <int WIDTH>
cudaError_t launch_t(const AdapterDown& d, const AdapterPlan& plan, int items, int split, cudaStream_t stream) {
  const int n = (int)plan.words.size();
  const int32_t* words = plan.words.data();
  if (plan.group == 16)
    return n <= kInlineWords ? launch_w<WIDTH, 1, kInlineWords>(d, words, n, items, split, stream)
                             : launch_w<WIDTH, 1, kAdapterWords>(d, words, n, items, split, stream);
  return n <= kInlineWords ? launch_w<WIDTH, 4, kInlineWords>(d, words, n, items, split, stream)
                           : launch_w<WIDTH, 4, kAdapterWords>(d, words, n, items, split, stream);
}

}  // namespace

bool plan_adapters(int M, int rows, int n_rows, const int32_t* row_tokens, const int32_t* row_adapter, int n_adapters, AdapterPlan* out) try {
  struct Run { int entry, from, len; };
  std::vector<int32_t> tile_first{0}, adapter, seg_first{0}, segs;
  std::vector<Run> runs;                        // of the current tile
  std::vector<int32_t> entry_of((size_t)n_adapters, -1);
  struct Part { int32_t adapter, token, len, entry; };
  std::vector<Part> parts;                      // all tiles' runs
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
      for (; i < runs.size() && runs[i].entry == e; ++i) {
        parts.push_back({adapter[e], t0 + runs[i].from, runs[i].len, e});
        segs.push_back(runs[i].from | runs[i].len << 16);
      }
      seg_first.push_back((int32_t)segs.size());
    }
    tile_first.push_back((int32_t)adapter.size());
  }
  std::stable_sort(parts.begin(), parts.end(), [](const Part& x, const Part& y) { return x.adapter < y.adapter; });
  int64_t all = 0;
  int used = 0;
  for (size_t i = 0; i < parts.size(); ++i) {
    all += parts[i].len;
    used += i == 0 || parts[i].adapter != parts[i - 1].adapter;
  }
  std::vector<int32_t> items, run;
  auto lay_out = [&](int group) {
    items.clear();
    run.clear();
    int room = 0;                               // left in the last item
    for (size_t i = 0; i < parts.size(); ++i) {
      if (i > 0 && parts[i].adapter != parts[i - 1].adapter) room = 0;
      for (int skip = 0; skip < parts[i].len;) {
        if (room == 0) {
          items.push_back(parts[i].adapter);
          items.push_back((int32_t)i | skip << 16);
          room = group;
        }
        const int take = std::min(room, parts[i].len - skip);
        items[items.size() - 2] += take << 16;
        skip += take;
        room -= take;
      }
      run.push_back(parts[i].token | parts[i].len << 16);
      run.push_back(parts[i].entry);
    }
    out->group = group;
    return tile_first.size() + adapter.size() + seg_first.size() + segs.size() + items.size() + run.size();
  };
  // Blocks of 64 tokens where an adapter has more than 16 on average: each A is then read once per 64, but no warps share a stage's K. Also where the words run out:
  // an adapter's last block may have one token, and of 16 tokens there are up to four times as many before it.
  if (all > 16 * (int64_t)used || lay_out(16) > (size_t)kAdapterWords) lay_out(kGroup);
  out->n_tiles = (int)tile_first.size() - 1;
  out->n_entries = (int)adapter.size();
  out->n_groups = (int)items.size() / 2;
  out->words.clear();
  auto put = [&](const std::vector<int32_t>& v) {
    const uint32_t at = (uint32_t)out->words.size();
    out->words.insert(out->words.end(), v.begin(), v.end());
    return at;
  };
  put(tile_first);
  out->o_adapter = put(adapter);
  out->o_seg_first = put(seg_first);
  out->o_seg = put(segs);
  out->o_item = put(items);
  out->o_run = put(run);
  return out->words.size() <= (size_t)kAdapterWords;
} catch (const std::bad_alloc&) {
  return false;
}

cudaError_t launch_adapter_down(AdapterDown d, const AdapterPlan& plan, int tile, int width, int n_sms, cudaStream_t stream) {
  if (plan.n_entries == 0) return cudaSuccess;
  d.n_tiles = plan.n_tiles;
  d.n_entries = plan.n_entries;
  d.granules = (d.rank + width - 1) / width;
  d.tile = tile;
  d.o_seg_first = plan.o_seg_first; d.o_seg = plan.o_seg; d.o_item = plan.o_item; d.o_run = plan.o_run;
  const int items = plan.n_groups * d.granules;
  // a block per SM, each with a few stages at least
  const int split = std::max(1, std::min({kMaxCluster, n_sms / items, (d.K + 255) / 256}));
  switch (width) {
    case 16: return launch_t<16>(d, plan, items, split, stream);
    case 32: return launch_t<32>(d, plan, items, split, stream);
    default: return launch_t<64>(d, plan, items, split, stream);
  }
}

cudaError_t launch_adapter_pack(const uint16_t* b, uint16_t* out, int n_adapters, int N, int rank, int width, int apart, cudaStream_t stream) {
  const int granules = (rank + width - 1) / width, blocks = (N + 127) / 128;
  const size_t chunks = (size_t)n_adapters * granules * blocks * 128 * (width / 8);
  adapter_pack_kernel<<<(unsigned)((chunks + 255) / 256), 256, 0, stream>>>(b, (char*)out, N, rank, width, granules, blocks, apart, chunks);
  return cudaGetLastError();
}

}  // namespace ts
