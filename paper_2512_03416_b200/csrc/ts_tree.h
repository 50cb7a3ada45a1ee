// Attention for trees of drafted tokens: what the host hands to the kernels (ts_tree.cu).
#pragma once
#include "ts_cache8.h"
#include "ts_internal.h"

namespace ts {

constexpr int kTreeNodes = 64;         // most nodes of a row: their masks are 64-bit words

// A work item covers the pages [k_begin, k_end) of a row's key list: first the ceil(ctx / 16) pages of cached tokens, then
// the row's own nodes, sixteen at a time. q_count = nodes of the row; a split item's partial of node i is slot partial_slot + i.
// A CombineItem is a row: `token` its first one, `reserved` its nodes, splits `reserved` slots apart.
struct TreeArgs {
  const uint64_t* mask;                // bit j of word i of a row: node i sees node j; null: nodes see those in front and themselves
  Cache8 cache;                        // values null: the bf16 pool
  int32_t tile_tokens, n_tiles;        // query tiles of a row: nodes of one, and how many the longest row has
};
// kv_map: the pool's or the 8-bit cache's pages, box = K and V of one (page, KV head).
cudaError_t launch_tree(const StepDevice& s, const TreeArgs& a, const CUtensorMap& kv_map, cudaStream_t stream);
// The same on tcgen05 (head_dim 128): query tiles of up to 128 / G nodes, a.n_tiles units of tiles_per_unit (1 or 2) of them per row and
// KV head. A row's own nodes are in one item. map: box = 16 slots of K or V of a (page, KV head), 128 bytes of each.
cudaError_t launch_tree_tc(const StepDevice& s, const TreeArgs& a, int tiles_per_unit, const CUtensorMap& map, int n_sms, cudaStream_t stream);
cudaError_t launch_tree_combine(const StepDevice& s, int max_nodes, cudaStream_t stream);
// Nodes of a query tile of the streaming kernel for rows of up to `nodes` nodes.
int tree_tile_tokens(int G, int nodes);
// Its thread blocks that an SM runs at a time, for tiles of `queries` (node, head) pairs.
int tree_blocks_per_sm(int queries, bool q8);

// The cache written and read back (ts_cache.cu): s.k_new, s.v_new are the step's tensors; `source`: see ts_cache_append.
cudaError_t launch_cache_append(const StepDevice& s, const Cache8& cache, const int32_t* source, int n_source, cudaStream_t stream);
cudaError_t launch_cache_read(const StepDevice& s, const Cache8& cache, cudaStream_t stream);

}  // namespace ts
