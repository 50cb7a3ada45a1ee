// Host side of the decoder layer around the attention step: RMSNorm, fused QKV projection with
// rotary embedding, ts_mixed_step, output projection, gated MLP. The public ABI is documented in
// include/tokenscale.h.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/tokenscale.h"
#include "ts_internal.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int kPosRing = 4;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                             const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                             CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// 2-D view of a K-major bf16 matrix [rows][k]: box = 64 of K (128 bytes, the swizzle span) x box_rows rows.
bool make_operand_map(void* encode_fn, const void* ptr, int64_t rows, int64_t k, CUtensorMap* out, int box_rows = 128) {
  const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)k * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return ((EncodeFn)encode_fn)(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// 5-D view of weights whose rows belong together in twos, `apart` rows from one another, in blocks of 2 * apart:
// (K, sixteen rows, the two, sixteens of the block's half, block). Box = 64 of K x 128 rows: four times sixteen
// rows and the sixteen that belong to them, in turn.
bool make_paired_map(void* encode_fn, const void* ptr, int64_t rows, int64_t k, int apart, CUtensorMap* out) {
  const cuuint64_t row = (cuuint64_t)k * 2;
  const cuuint64_t dims[5] = {(cuuint64_t)k, 16, 2, (cuuint64_t)apart / 16, (cuuint64_t)rows / (2 * apart)};
  const cuuint64_t strides[4] = {row, row * apart, row * 16, row * 2 * apart};
  const cuuint32_t box[5] = {64, 16, 2, 4, 1};
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return ((EncodeFn)encode_fn)(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(ptr), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// An activation matrix as the projections read it: boxes of 128 rows, and of 8, 16 .. 128 rows for the pair kernel.
struct Activations {
  CUtensorMap full, pair[16];
};
bool make_activation_maps(void* encode_fn, const void* ptr, int64_t rows, int64_t k, Activations* out) {
  bool ok = make_operand_map(encode_fn, ptr, rows, k, &out->full);
  for (int i = 0; i < 16; ++i) ok = ok && make_operand_map(encode_fn, ptr, rows, k, &out->pair[i], 8 * (i + 1));
  return ok;
}

// ---- low-rank adapters
constexpr int kMaxRank = 256, kMaxAdapters = 65536;
constexpr int kMaxAdapterRows = 1024, kMaxAdapterTokens = 32768, kManyAdapterRows = 512, kManyAdapterTokens = 8192;
// Their plan fits kAdapterWords: of r rows in T tiles (of 128 tokens or, with more tokens each, a pair's) there are at most r + T - 1 segments with 5 words each, T + 2
// words for the tiles, and 2 words for each group, of which there are, in groups of 64, at most one per adapter and one per 64 tokens that are not an
// adapter's first. 1024 rows of 8192 tokens: 66 + 5 * 1087 + 2 * (1024 + 112) = 7773; 512 rows of 32768: 258 + 5 * 767 + 2 * (512 + 504) = 6125.
bool adapter_size_ok(int64_t tokens, int64_t rows) {
  return rows <= kMaxAdapterRows && tokens <= kMaxAdapterTokens && (rows <= kManyAdapterRows || tokens <= kManyAdapterTokens);
}
int granule_width(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }
int padded_rank(int rank) { return (rank + granule_width(rank) - 1) / granule_width(rank) * granule_width(rank); }
// Either side of the adapters' part of a product: runs of 128 values, boxes of `runs` of them.
bool make_runs_map(void* encode_fn, const void* ptr, int64_t values, int runs, CUtensorMap* out) {
  const cuuint64_t dims[2] = {128, (cuuint64_t)(values / 128)}, strides[1] = {256};
  const cuuint32_t box[2] = {128, (cuuint32_t)runs}, estr[2] = {1, 1};
  return ((EncodeFn)encode_fn)(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
int64_t packed_values(int64_t n_adapters, int64_t N, int rank) { return n_adapters * padded_rank(rank) * ((N + 127) / 128 * 128); }
bool make_b_map(void* encode_fn, const void* packed, const ts_adapters* ad, int64_t N, CUtensorMap* out) {
  return make_runs_map(encode_fn, packed, packed_values(ad->n_adapters, N, ad->rank), granule_width(ad->rank), out);
}
bool adapters_ok(const ts_adapters* ad) {
  return ad->n_adapters > 0 && ad->n_adapters <= kMaxAdapters && ad->rank > 0 && ad->rank <= kMaxRank && ad->rank % 8 == 0 && ad->a && ad->b &&
         !((uintptr_t)ad->a & 15u) && !(((uintptr_t)ad->b | (uintptr_t)ad->b_pair) & 127u) && !((uintptr_t)ad->scale & 3u);
}
// Bytes for the plan's device words and for u, for tiles of any size: of M tokens of n_rows rows, entries of tiles of nt tokens are no more than
// rows + tiles, than tiles * adapters, and than tokens.
size_t adapter_plan_bytes(int64_t M, int64_t n_rows) { return align_up((size_t)(2 * (M / 16 + 2) + n_rows + 2) * sizeof(int32_t)); }
size_t adapter_bytes(int64_t M, int64_t n_rows, int64_t n_adapters, int rank) {
  const int64_t rows = std::min(std::min(M * 256, n_rows * 256 + M + 256), (M + 256) * n_adapters);
  return adapter_plan_bytes(M, n_rows) + align_up((size_t)rows * padded_rank(rank) * 2);
}
// Rows of a tile as the adapters' part has them: all that a kernel's tile holds, or of a single tile what its tokens need.
int entry_rows(const ts::GemmPlan& plan, int M) { return plan.pair_tokens > 0 ? plan.pair_tokens : std::min(128, (M + 15) / 16 * 16); }
// Tokens of a tile
int entry_tile(const ts::GemmPlan& plan, int M) { return plan.pair_tokens > 0 ? entry_rows(plan, M) : 128; }
void fill_tiles(const ts::AdapterPlan& plan, int rank, int rows, int64_t N, const int32_t* words, ts::AdapterTiles* out) {
  const int width = granule_width(rank), n = plan.n_tiles + 1 + plan.n_entries;
  out->plan = words;
  out->n_tiles = plan.n_tiles; out->width = width; out->granules = padded_rank(rank) / width; out->rows = rows;
  out->blocks = (int32_t)((N + 127) / 128);
  out->n_inline = n <= ts::kInlineTiles ? n : 0;
  std::memcpy(out->words, plan.words.data(), sizeof(int32_t) * (size_t)out->n_inline);
}
bool adapter_rows_ok(int32_t n_rows, const int32_t* row_tokens, const int32_t* row_adapter, int32_t n_adapters, int64_t M) {
  int64_t n = 0;
  for (int r = 0; r < n_rows; ++r) {
    if (row_tokens[r] < 1 || row_adapter[r] < -1 || row_adapter[r] >= n_adapters) return false;
    n += row_tokens[r];
  }
  return n == M;
}
// How a product with adapters is laid out: planned for the K that the adapters of a tile of 256 tokens add on average.
ts::GemmPlan adapter_gemm_plan(ts::GemmArgs g, int n_sms, int rank, int n_rows, const int32_t* row_adapter, int n_adapters) {
  const int tiles = (g.M + 255) / 256, k_blocks = (g.K + 63) / 64;
  int runs = 0;
  for (int r = 0; r < n_rows; ++r) runs += row_adapter[r] >= 0 && (r == 0 || row_adapter[r] != row_adapter[r - 1]);
  const int per_tile = std::min(n_adapters, (runs + tiles - 1) / tiles);
  const ts::GemmPlan without = ts::gemm_plan(g, n_sms);
  g.K = (k_blocks + (per_tile * padded_rank(rank) + 63) / 64) * 64;
  const ts::GemmPlan plan = ts::gemm_plan(g, n_sms);
  return plan.split > k_blocks ? without : plan;           // every block of a cluster has K blocks also in a tile without adapters
}

struct LayerLayout {
  size_t off_table, off_pos, off_h, off_q, off_k, off_v, off_attn, off_y, off_z, total;
};

bool layer_shape_ok(const ts_config* c, const ts_layer_config* l) {
  if (!c || !l) return false;
  if (c->head_dim != 128) return false;                        // the fused rotary epilogue pairs columns i, i + 64
  if (l->hidden <= 0 || l->hidden % 64 || l->intermediate <= 0 || l->intermediate % 128) return false;
  if (l->max_position <= 0) return false;
  return true;
}

void layer_layout(const ts_config* c, const ts_layer_config* l, int max_tokens, LayerLayout* L) {
  const size_t T = (size_t)max_tokens;
  size_t off = 0;
  L->off_table = off; off += align_up((size_t)l->max_position * 64 * sizeof(float2));
  L->off_pos = off; off += align_up(kPosRing * T * sizeof(int32_t));
  L->off_h = off; off += align_up(T * l->hidden * 2);                       // normalised input of a projection (h, then h2)
  L->off_q = off; off += align_up(T * c->n_q_heads * c->head_dim * 2);
  L->off_k = off; off += align_up(T * c->n_kv_heads * c->head_dim * 2);
  L->off_v = off; off += align_up(T * c->n_kv_heads * c->head_dim * 2);
  L->off_attn = off; off += align_up(T * c->n_q_heads * c->head_dim * 2);
  L->off_y = off; off += align_up(T * l->hidden * 2);
  L->off_z = off; off += align_up(T * l->intermediate * 2);
  L->total = off;
}

}  // namespace

// A projection's adapters as the layer uses them.
struct LayerAdapters {
  ts_adapters a = {};                          // n_adapters 0: none
  CUtensorMap b, b_pair, u[16];                // u[i]: boxes of 8 (i + 1) tokens of width granule_width(a.rank)
};

struct ts_layer {
  ts_ctx* ctx = nullptr;
  ts_layer_config cfg;
  ts::CtxView view;
  LayerLayout L;
  int max_tokens = 0;
  float eps = 0.f, theta = 0.f;
  CUtensorMap w_qkv, w_o, w_gu, w_down;        // weights
  CUtensorMap w_qkv_pair, w_gu_pair;           // rotary pairs, gates and ups together
  Activations a_h, a_attn, a_z;                // in the workspace
  void* pos_host[kPosRing] = {};
  cudaEvent_t pos_ev[kPosRing] = {};
  bool pos_busy[kPosRing] = {};
  int pos_next = 0;
  int last_cuda_error = 0;
  LayerAdapters adapters[4];                   // qkv, o, gate_up, down
  int32_t n_adapters = 0;                      // 0: none attached
  char* adapter_ws = nullptr;
  size_t adapter_plan = 0, adapter_total = 0;  // bytes in front of u, and in all
};

namespace {
int lfail(ts_layer* l, cudaError_t e) {
  l->last_cuda_error = (int)e;
  return TS_ERR_CUDA;
}
#define TSL_CUDA(l, call)                              \
  do {                                                 \
    cudaError_t e__ = (call);                          \
    if (e__ != cudaSuccess) return lfail((l), e__);    \
  } while (0)
}  // namespace

extern "C" {

size_t ts_layer_workspace_bytes(const ts_config* cfg, const ts_layer_config* layer) {
  if (!layer_shape_ok(cfg, layer) || cfg->chunk_size <= 0) return 0;
  LayerLayout L;
  layer_layout(cfg, layer, cfg->chunk_size, &L);
  return L.total;
}

int ts_pack_gate_up(const void* w_gate, const void* w_up, void* w_gate_up, int32_t intermediate, int32_t hidden,
                    void* cuda_stream) {
  if (!w_gate || !w_up || !w_gate_up || intermediate <= 0 || intermediate % 128 || hidden <= 0 || hidden % 8)
    return TS_ERR_INVALID;
  const cudaError_t e = ts::launch_pack_gate_up((const uint16_t*)w_gate, (const uint16_t*)w_up, (uint16_t*)w_gate_up,
                                                intermediate, hidden, (cudaStream_t)cuda_stream);
  return e == cudaSuccess ? TS_OK : TS_ERR_CUDA;
}

int ts_layer_create(ts_ctx* ctx, const ts_layer_config* cfg, void* cuda_stream, ts_layer** out) {
  if (!out) return TS_ERR_INVALID;
  *out = nullptr;
  if (!ctx || !cfg) return TS_ERR_INVALID;
  ts::CtxView view;
  int rc = ts::ctx_view(ctx, (cudaStream_t)cuda_stream, &view);
  if (rc != TS_OK) return rc;
  if (!layer_shape_ok(view.cfg, cfg)) return TS_ERR_UNSUPPORTED;
  if (view.cfg->chunk_size <= 0) return TS_ERR_INVALID;        // the activations are sized by the chunk size
  if (!cfg->w_norm1 || !cfg->w_qkv || !cfg->w_o || !cfg->w_norm2 || !cfg->w_gate_up || !cfg->w_down || !cfg->workspace)
    return TS_ERR_INVALID;
  if (((uintptr_t)cfg->workspace & (kAlign - 1)) || ((uintptr_t)cfg->w_qkv | (uintptr_t)cfg->w_o | (uintptr_t)cfg->w_gate_up |
                                                     (uintptr_t)cfg->w_down | (uintptr_t)cfg->w_norm1 | (uintptr_t)cfg->w_norm2) & 15u)
    return TS_ERR_INVALID;
  ts_layer* l = new (std::nothrow) ts_layer();
  if (!l) return TS_ERR_INVALID;
  l->ctx = ctx;
  l->cfg = *cfg;
  l->view = view;
  l->max_tokens = view.max_tokens;
  layer_layout(view.cfg, cfg, l->max_tokens, &l->L);
  if (cfg->workspace_bytes < l->L.total) {
    delete l;
    return TS_ERR_WORKSPACE;
  }
  l->eps = cfg->rms_eps > 0.f ? cfg->rms_eps : 1e-5f;
  l->theta = cfg->rope_theta > 0.f ? cfg->rope_theta : 500000.f;
  const ts_config* c = view.cfg;
  const int64_t qd = (int64_t)c->n_q_heads * c->head_dim, kvd = (int64_t)c->n_kv_heads * c->head_dim;
  char* ws = (char*)cfg->workspace;
  bool ok = make_operand_map(view.encode_fn, cfg->w_qkv, qd + 2 * kvd, cfg->hidden, &l->w_qkv) &&
            make_operand_map(view.encode_fn, cfg->w_o, cfg->hidden, qd, &l->w_o) &&
            make_operand_map(view.encode_fn, cfg->w_gate_up, 2 * (int64_t)cfg->intermediate, cfg->hidden, &l->w_gu) &&
            make_operand_map(view.encode_fn, cfg->w_down, cfg->hidden, cfg->intermediate, &l->w_down) &&
            make_paired_map(view.encode_fn, cfg->w_qkv, qd + 2 * kvd, cfg->hidden, 64, &l->w_qkv_pair) &&
            make_paired_map(view.encode_fn, cfg->w_gate_up, 2 * (int64_t)cfg->intermediate, cfg->hidden, 128, &l->w_gu_pair) &&
            make_activation_maps(view.encode_fn, ws + l->L.off_h, l->max_tokens, cfg->hidden, &l->a_h) &&
            make_activation_maps(view.encode_fn, ws + l->L.off_attn, l->max_tokens, qd, &l->a_attn) &&
            make_activation_maps(view.encode_fn, ws + l->L.off_z, l->max_tokens, cfg->intermediate, &l->a_z);
  if (!ok) {
    delete l;
    return TS_ERR_CUDA;
  }
  for (int i = 0; i < kPosRing; ++i) {
    if (cudaHostAlloc(&l->pos_host[i], (size_t)l->max_tokens * sizeof(int32_t), cudaHostAllocDefault) != cudaSuccess ||
        cudaEventCreateWithFlags(&l->pos_ev[i], cudaEventDisableTiming) != cudaSuccess) {
      ts_layer_destroy(l);
      return TS_ERR_CUDA;
    }
  }
  if (ts::launch_rope_table((float2*)(ws + l->L.off_table), cfg->max_position, l->theta, (cudaStream_t)cuda_stream) != cudaSuccess) {
    ts_layer_destroy(l);
    return TS_ERR_CUDA;
  }
  *out = l;
  return TS_OK;
}

int ts_layer_destroy(ts_layer* l) {
  if (!l) return TS_ERR_INVALID;
  for (int i = 0; i < kPosRing; ++i) {
    if (l->pos_busy[i]) cudaEventSynchronize(l->pos_ev[i]);
    if (l->pos_ev[i]) cudaEventDestroy(l->pos_ev[i]);
    if (l->pos_host[i]) cudaFreeHost(l->pos_host[i]);
  }
  delete l;
  return TS_OK;
}

size_t ts_layer_adapters_workspace_bytes(const ts_config* cfg, const ts_layer_adapters* ad) {
  if (!cfg || !ad || cfg->chunk_size <= 0 || cfg->max_requests <= 0) return 0;
  size_t total = 0;
  for (const ts_adapters* a : {ad->qkv, ad->o, ad->gate_up, ad->down}) {
    if (!a) continue;
    if (a->rank <= 0 || a->rank > kMaxRank || a->rank % 8 || a->n_adapters <= 0 || a->n_adapters > kMaxAdapters) return 0;
    total = std::max(total, adapter_bytes(std::min(cfg->chunk_size, kMaxAdapterTokens), std::min(cfg->max_requests, kMaxAdapterRows), a->n_adapters, a->rank));
  }
  return total;
}

int ts_layer_attach_adapters(ts_layer* l, const ts_layer_adapters* ad) {
  if (!l || !ad) return TS_ERR_INVALID;
  const ts_adapters* all[4] = {ad->qkv, ad->o, ad->gate_up, ad->down};
  int32_t n_adapters = 0;
  for (const ts_adapters* a : all) {
    if (!a) continue;
    if (!adapters_ok(a) || (n_adapters && a->n_adapters != n_adapters)) return TS_ERR_INVALID;
    n_adapters = a->n_adapters;
  }
  const bool paired[4] = {true, false, true, false};       // the pair kernel has these weights' rows in another order
  for (int i = 0; i < 4; ++i)
    if (all[i] && paired[i] && !all[i]->b_pair) return TS_ERR_INVALID;
  LayerAdapters made[4];
  size_t total = 0, plan = 0;
  const ts_config* c = l->view.cfg;
  if (n_adapters) {
    total = ts_layer_adapters_workspace_bytes(c, ad);
    if (total == 0) return TS_ERR_UNSUPPORTED;
    if (!ad->workspace || ((uintptr_t)ad->workspace & (kAlign - 1))) return TS_ERR_INVALID;
    if (ad->workspace_bytes < total) return TS_ERR_WORKSPACE;
    plan = adapter_plan_bytes(std::min(c->chunk_size, kMaxAdapterTokens), std::min(c->max_requests, kMaxAdapterRows));
    const char* u = (const char*)ad->workspace + plan;
    const int64_t qd = (int64_t)c->n_q_heads * c->head_dim, kvd = (int64_t)c->n_kv_heads * c->head_dim;
    const int64_t out[4] = {qd + 2 * kvd, l->cfg.hidden, 2 * (int64_t)l->cfg.intermediate, l->cfg.hidden};
    TSL_CUDA(l, cudaSetDevice(c->device));
    for (int i = 0; i < 4; ++i) {
      if (!all[i]) continue;
      made[i].a = *all[i];
      const int width = granule_width(all[i]->rank);
      bool ok = make_b_map(l->view.encode_fn, all[i]->b, all[i], out[i], &made[i].b) &&
                make_b_map(l->view.encode_fn, paired[i] ? all[i]->b_pair : all[i]->b, all[i], out[i], &made[i].b_pair);
      for (int k = 0; k < 16; ++k) ok = ok && make_runs_map(l->view.encode_fn, u, (int64_t)(total - plan) / 2, 8 * (k + 1) * width / 128, &made[i].u[k]);
      if (!ok) return lfail(l, cudaErrorInvalidValue);
    }
  }
  for (int i = 0; i < 4; ++i) l->adapters[i] = made[i];
  l->n_adapters = n_adapters;
  l->adapter_ws = n_adapters ? (char*)ad->workspace : nullptr;
  l->adapter_plan = plan;
  l->adapter_total = total;
  return TS_OK;
}

int ts_layer_step(ts_layer* l, const ts_step* st, const void* x_in, void* x_out, void* cuda_stream) {
  return ts_layer_step_adapted(l, st, nullptr, x_in, x_out, cuda_stream);
}

int ts_layer_step_adapted(ts_layer* l, const ts_step* st, const int32_t* row_adapter, const void* x_in, void* x_out, void* cuda_stream) {
  if (!l || !st) return TS_ERR_INVALID;
  if (st->n_rows == 0) return TS_OK;
  if (!x_in || !x_out || (((uintptr_t)x_in | (uintptr_t)x_out) & 15u)) return TS_ERR_INVALID;
  // the step's own checks first (host only): a step that would be refused must launch nothing
  int32_t n_items = 0;
  int rc = ts_plan_step(l->ctx, st, nullptr, 0, &n_items);
  if (rc != TS_OK) return rc;
  int64_t n = 0;
  for (int r = 0; r < st->n_rows; ++r) {
    if ((int64_t)st->ctx_len[r] + st->q_len[r] > l->cfg.max_position) return TS_ERR_INVALID;   // beyond the rotary table
    n += st->q_len[r];
  }
  if (n > l->max_tokens) return TS_ERR_BUDGET;
  bool adapted = false;
  if (row_adapter) {
    if (!adapter_rows_ok(st->n_rows, st->q_len, row_adapter, l->n_adapters, n)) return TS_ERR_INVALID;
    for (int r = 0; r < st->n_rows; ++r) adapted = adapted || row_adapter[r] >= 0;
    if (adapted && !adapter_size_ok(n, st->n_rows)) return TS_ERR_UNSUPPORTED;
  }
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  const ts_config* c = l->view.cfg;
  TSL_CUDA(l, cudaSetDevice(c->device));
  const int N = (int)n, hidden = l->cfg.hidden, inter = l->cfg.intermediate;
  const int qd = c->n_q_heads * c->head_dim, kvd = c->n_kv_heads * c->head_dim;
  // How the projections with adapters are laid out, and for which tiles of tokens: all of it in front of the first launch too.
  ts::GemmPlan planned[4] = {};
  ts::AdapterPlan tile_plans[4];
  int tile_of[4], which_plan[4] = {}, n_tile_plans = 0;
  for (int i = 0; adapted && i < 4; ++i) {
    const ts_adapters& ad = l->adapters[i].a;
    if (!ad.n_adapters) continue;
    const int out_of[4] = {qd + 2 * kvd, hidden, 2 * inter, hidden}, in_of[4] = {hidden, qd, hidden, inter};
    const int epi_of[4] = {ts::GEMM_EPI_ROPE, ts::GEMM_EPI_STORE, ts::GEMM_EPI_SILU_MUL, ts::GEMM_EPI_STORE};
    ts::GemmArgs g;
    std::memset(&g, 0, sizeof g);
    g.M = N; g.N = out_of[i]; g.K = in_of[i]; g.epi = epi_of[i];
    planned[i] = adapter_gemm_plan(g, l->view.n_sms, ad.rank, st->n_rows, row_adapter, l->n_adapters);
    const int tile = entry_tile(planned[i], N);
    int& k = which_plan[i];
    while (k < n_tile_plans && tile_of[k] != tile) ++k;
    if (k == n_tile_plans) {
      if (!ts::plan_adapters(N, tile, st->n_rows, st->q_len, row_adapter, l->n_adapters, &tile_plans[k])) return TS_ERR_UNSUPPORTED;
      tile_of[n_tile_plans++] = tile;
    }
    const size_t u_bytes = (size_t)tile_plans[k].n_entries * entry_rows(planned[i], N) * padded_rank(ad.rank) * 2;
    if (l->adapter_plan + u_bytes > l->adapter_total) return TS_ERR_WORKSPACE;             // never: adapter_bytes is enough
  }
  char* ws = (char*)l->cfg.workspace;
  // positions of the new tokens (row r's token i sits at ctx_len[r] + i): written by the first RMSNorm
  // launch from row arrays in its parameters, or, for more rows than those hold, uploaded
  int32_t* pos_dev = (int32_t*)(ws + l->L.off_pos);
  const bool pos_inline = st->n_rows <= ts::kPosRows;
  ts::PosRows<true> pr;
  if (pos_inline) {
    pr.pos = pos_dev;
    pr.n_rows = st->n_rows;
    int32_t at = 0;
    for (int r = 0; r < st->n_rows; ++r) {
      pr.tok0[r] = at;
      pr.ctx[r] = st->ctx_len[r];
      at += st->q_len[r];
    }
  } else {
    const int slot = l->pos_next;
    l->pos_next = (l->pos_next + 1) % kPosRing;
    if (l->pos_busy[slot]) {
      TSL_CUDA(l, cudaEventSynchronize(l->pos_ev[slot]));
      l->pos_busy[slot] = false;
    }
    int32_t* ph = (int32_t*)l->pos_host[slot];
    int64_t at = 0;
    for (int r = 0; r < st->n_rows; ++r)
      for (int i = 0; i < st->q_len[r]; ++i) ph[at++] = st->ctx_len[r] + i;
    pos_dev += (size_t)slot * l->max_tokens;
    TSL_CUDA(l, cudaMemcpyAsync(pos_dev, ph, (size_t)n * sizeof(int32_t), cudaMemcpyHostToDevice, stream));
    TSL_CUDA(l, cudaEventRecord(l->pos_ev[slot], stream));
    l->pos_busy[slot] = true;
  }

  uint16_t* h = (uint16_t*)(ws + l->L.off_h);
  uint16_t* q = (uint16_t*)(ws + l->L.off_q);
  uint16_t* k = (uint16_t*)(ws + l->L.off_k);
  uint16_t* v = (uint16_t*)(ws + l->L.off_v);
  uint16_t* attn = (uint16_t*)(ws + l->L.off_attn);
  uint16_t* y = (uint16_t*)(ws + l->L.off_y);
  uint16_t* z = (uint16_t*)(ws + l->L.off_z);
  ts::GemmArgs g;
  std::memset(&g, 0, sizeof g);
  g.status = l->view.status;
  g.wait_cycles = l->view.wait_cycles;
  g.M = N;
  ts::AdapterTiles at;
  auto project = [&](const Activations& x, const CUtensorMap& w, const CUtensorMap& w_pair, int which, const uint16_t* in) {
    const LayerAdapters& ad = l->adapters[which];
    ts::GemmPlan plan = {};
    ts::GemmMaps maps = {&x.full, nullptr, &w, &w_pair, nullptr, nullptr, nullptr};
    if (adapted && ad.a.n_adapters) {
      plan = planned[which];
      const ts::AdapterPlan& tiles = tile_plans[which_plan[which]];
      const int rows = entry_rows(plan, N);
      int32_t* words = (int32_t*)l->adapter_ws;
      fill_tiles(tiles, ad.a.rank, rows, g.N, words, &at);
      const ts::AdapterDown down = {in, (const uint16_t*)ad.a.a, ad.a.scale, (uint16_t*)(l->adapter_ws + l->adapter_plan), at.n_inline ? nullptr : words,
                                    g.K, ad.a.rank, rows};
      const cudaError_t e = ts::launch_adapter_down(down, tiles, entry_tile(plan, N), at.width, l->view.n_sms, stream);
      if (e != cudaSuccess) return e;
      maps.adapters = &at;
      maps.b = plan.pair_tokens > 0 ? &ad.b_pair : &ad.b;
      maps.u = &ad.u[(plan.pair_tokens > 0 ? rows / 2 : rows) / 8 - 1];
    } else {
      plan = ts::gemm_plan(g, l->view.n_sms);
    }
    if (plan.pair_tokens > 0) maps.x_pair = &x.pair[plan.pair_tokens / 16 - 1];
    return ts::launch_gemm(g, maps, plan, l->view.n_sms, stream);
  };

  // h = rmsnorm(x); (q, k, v) = rope(h . W_qkv^T)
  if (pos_inline)
    TSL_CUDA(l, ts::launch_rmsnorm_pos((const uint16_t*)x_in, (const uint16_t*)l->cfg.w_norm1, h, N, hidden, l->eps, pr, stream));
  else
    TSL_CUDA(l, ts::launch_rmsnorm((const uint16_t*)x_in, (const uint16_t*)l->cfg.w_norm1, h, N, hidden, l->eps, stream));
  g.N = qd + 2 * kvd; g.K = hidden; g.epi = ts::GEMM_EPI_ROPE; g.B = (const uint16_t*)l->cfg.w_qkv;
  g.C = q; g.C2 = k; g.C3 = v; g.q_cols = qd; g.kv_cols = kvd; g.pos = pos_dev;
  g.rope_table = (const float2*)(ws + l->L.off_table);
  TSL_CUDA(l, project(l->a_h, l->w_qkv, l->w_qkv_pair, 0, h));
  // attention over the paged KV cache, with the append of the new K/V
  ts_step inner = *st;
  inner.q = q; inner.k_new = k; inner.v_new = v; inner.out = attn;
  rc = ts_mixed_step(l->ctx, &inner, cuda_stream);
  if (rc != TS_OK) return rc;
  // y = x + attn . W_o^T
  g.N = hidden; g.K = qd; g.epi = ts::GEMM_EPI_STORE; g.B = (const uint16_t*)l->cfg.w_o; g.C = y; g.R = (const uint16_t*)x_in; g.ldc = hidden;
  TSL_CUDA(l, project(l->a_attn, l->w_o, l->w_o, 1, attn));
  // h2 = rmsnorm(y); z = silu(h2 . W_gate^T) * (h2 . W_up^T)
  TSL_CUDA(l, ts::launch_rmsnorm(y, (const uint16_t*)l->cfg.w_norm2, h, N, hidden, l->eps, stream));
  g.N = 2 * inter; g.K = hidden; g.epi = ts::GEMM_EPI_SILU_MUL; g.B = (const uint16_t*)l->cfg.w_gate_up; g.C = z; g.R = nullptr; g.ldc = inter;
  TSL_CUDA(l, project(l->a_h, l->w_gu, l->w_gu_pair, 2, h));
  // out = y + z . W_down^T
  g.N = hidden; g.K = inter; g.epi = ts::GEMM_EPI_STORE; g.B = (const uint16_t*)l->cfg.w_down; g.C = (uint16_t*)x_out; g.R = y; g.ldc = hidden;
  TSL_CUDA(l, project(l->a_z, l->w_down, l->w_down, 3, z));
  return TS_OK;
}

int ts_gemm_bf16(int32_t device, int32_t M, int32_t N, int32_t K, const void* A, const void* B, const void* R, void* C,
                 int32_t tile_m, int32_t* device_status, void* cuda_stream) {
  if (M < 0 || N <= 0 || K <= 0 || (N % 8) || (K % 8)) return TS_ERR_INVALID;
  if (M == 0) return TS_OK;
  if (!A || !B || !C || !device_status) return TS_ERR_INVALID;
  if (((uintptr_t)A | (uintptr_t)B | (uintptr_t)C | (uintptr_t)R) & 15u) return TS_ERR_INVALID;
  if (tile_m != 0 && tile_m != 128 && tile_m != 256) return TS_ERR_INVALID;
  if (cudaSetDevice(device) != cudaSuccess) return TS_ERR_CUDA;
  void* encode_fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &encode_fn, cudaEnableDefault, &qres) != cudaSuccess || !encode_fn)
    return TS_ERR_CUDA;
  int n_sms = 0;
  if (cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return TS_ERR_CUDA;
  ts::GemmArgs g;
  std::memset(&g, 0, sizeof g);
  g.M = M; g.N = N; g.K = K; g.epi = ts::GEMM_EPI_STORE; g.B = (const uint16_t*)B;
  g.C = (uint16_t*)C; g.R = (const uint16_t*)R; g.ldc = N;
  g.status = device_status;
  g.wait_cycles = ts::kWaitCycles;
  const ts::GemmPlan plan = tile_m ? ts::GemmPlan{tile_m, 0, tile_m == 256 ? ts::pair_tokens(M, (M + 255) / 256) : 0} : ts::gemm_plan(g, n_sms);
  CUtensorMap x, x_pair, w;
  if (!make_operand_map(encode_fn, A, M, K, &x) || !make_operand_map(encode_fn, B, N, K, &w) ||
      (plan.pair_tokens > 0 && !make_operand_map(encode_fn, A, M, K, &x_pair, plan.pair_tokens / 2)))
    return TS_ERR_CUDA;
  return ts::launch_gemm(g, ts::GemmMaps{&x, &x_pair, &w, &w, nullptr, nullptr, nullptr}, plan, n_sms, (cudaStream_t)cuda_stream) == cudaSuccess ? TS_OK : TS_ERR_CUDA;
}

size_t ts_adapter_workspace_bytes(int32_t n_tokens, int32_t n_rows, int32_t n_adapters, int32_t rank) {
  if (n_tokens <= 0 || n_rows <= 0 || !adapter_size_ok(n_tokens, n_rows) || n_adapters <= 0 || n_adapters > kMaxAdapters ||
      rank <= 0 || rank > kMaxRank || rank % 8)
    return 0;
  return adapter_bytes(n_tokens, n_rows, n_adapters, rank);
}

int ts_adapter_project(int32_t device, int32_t M, int32_t N, int32_t K, const void* x, const void* W, const void* R, void* C,
                       const ts_adapters* ad, int32_t n_rows, const int32_t* row_tokens, const int32_t* row_adapter, void* workspace,
                       size_t workspace_bytes, int32_t tile_m, int32_t* device_status, void* cuda_stream) {
  if (M < 0 || N <= 0 || K <= 0 || (N % 8) || (K % 8) || !ad || n_rows < 0) return TS_ERR_INVALID;
  if (!adapters_ok(ad)) return TS_ERR_INVALID;
  if (M == 0) return n_rows == 0 ? TS_OK : TS_ERR_INVALID;
  if (!x || !W || !C || !device_status || !row_tokens || !row_adapter || !workspace) return TS_ERR_INVALID;
  if (((uintptr_t)x | (uintptr_t)W | (uintptr_t)C | (uintptr_t)R) & 15u || ((uintptr_t)workspace & (kAlign - 1))) return TS_ERR_INVALID;
  if (tile_m != 0 && tile_m != 128 && tile_m != 256) return TS_ERR_INVALID;
  if (!adapter_size_ok(M, n_rows)) return TS_ERR_UNSUPPORTED;
  if (!adapter_rows_ok(n_rows, row_tokens, row_adapter, ad->n_adapters, M)) return TS_ERR_INVALID;
  bool adapted = false;
  for (int r = 0; r < n_rows; ++r) adapted = adapted || row_adapter[r] >= 0;
  if (!adapted) return ts_gemm_bf16(device, M, N, K, x, W, R, C, tile_m, device_status, cuda_stream);
  if (workspace_bytes < adapter_bytes(M, n_rows, ad->n_adapters, ad->rank)) return TS_ERR_WORKSPACE;
  if (cudaSetDevice(device) != cudaSuccess) return TS_ERR_CUDA;
  static std::atomic<void*> encode{nullptr};               // the driver's function: looked up once
  void* encode_fn = encode.load(std::memory_order_relaxed);
  cudaDriverEntryPointQueryResult qres;
  if (!encode_fn) {
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &encode_fn, cudaEnableDefault, &qres) != cudaSuccess || !encode_fn) return TS_ERR_CUDA;
    encode.store(encode_fn, std::memory_order_relaxed);
  }
  int n_sms = 0;
  if (cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return TS_ERR_CUDA;
  ts::GemmArgs g;
  std::memset(&g, 0, sizeof g);
  g.M = M; g.N = N; g.K = K; g.epi = ts::GEMM_EPI_STORE; g.B = (const uint16_t*)W;
  g.C = (uint16_t*)C; g.R = (const uint16_t*)R; g.ldc = N;
  g.status = device_status;
  g.wait_cycles = ts::kWaitCycles;
  const ts::GemmPlan plan = tile_m ? ts::GemmPlan{tile_m, 0, tile_m == 256 ? ts::pair_tokens(M, (M + 255) / 256) : 0}
                                   : adapter_gemm_plan(g, n_sms, ad->rank, n_rows, row_adapter, ad->n_adapters);
  const bool pair = plan.pair_tokens > 0;
  const int rows = entry_rows(plan, M);
  ts::AdapterPlan tiles;
  if (!ts::plan_adapters(M, entry_tile(plan, M), n_rows, row_tokens, row_adapter, ad->n_adapters, &tiles)) return TS_ERR_UNSUPPORTED;
  const size_t plan_bytes = adapter_plan_bytes(M, n_rows);
  int32_t* words = (int32_t*)workspace;
  uint16_t* u = (uint16_t*)((char*)workspace + plan_bytes);
  ts::AdapterTiles at;
  fill_tiles(tiles, ad->rank, rows, N, words, &at);
  const int64_t values = (int64_t)tiles.n_entries * rows * padded_rank(ad->rank);
  if (plan_bytes + (size_t)values * 2 > workspace_bytes) return TS_ERR_WORKSPACE;
  CUtensorMap mx, mw, mu, mb;                              // the maps of the plan's kernel only
  if (!make_operand_map(encode_fn, x, M, K, &mx, pair ? rows / 2 : 128) || !make_operand_map(encode_fn, W, N, K, &mw) ||
      !make_runs_map(encode_fn, u, values, (pair ? rows / 2 : rows) * at.width / 128, &mu) || !make_b_map(encode_fn, ad->b, ad, N, &mb))
    return TS_ERR_CUDA;
  const ts::AdapterDown down = {(const uint16_t*)x, (const uint16_t*)ad->a, ad->scale, u, at.n_inline ? nullptr : words, K, ad->rank, rows};
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (ts::launch_adapter_down(down, tiles, entry_tile(plan, M), at.width, n_sms, stream) != cudaSuccess) return TS_ERR_CUDA;
  const ts::GemmMaps maps = {&mx, &mx, &mw, &mw, &mu, &mb, &at};
  return ts::launch_gemm(g, maps, plan, n_sms, stream) == cudaSuccess ? TS_OK : TS_ERR_CUDA;
}

size_t ts_adapter_packed_bytes(int32_t n_adapters, int32_t N, int32_t rank) {
  if (n_adapters <= 0 || n_adapters > kMaxAdapters || N <= 0 || rank <= 0 || rank > kMaxRank || rank % 8) return 0;
  return (size_t)packed_values(n_adapters, N, rank) * 2;
}

int ts_adapter_pack(const void* b, int32_t n_adapters, int32_t N, int32_t rank, int32_t order, void* packed, void* cuda_stream) {
  const size_t bytes = ts_adapter_packed_bytes(n_adapters, N, rank);
  if (bytes == 0 || !b || !packed || ((uintptr_t)b & 1u) || ((uintptr_t)packed & 127u) || order < TS_ROWS_PLAIN || order > TS_ROWS_GATE_UP) return TS_ERR_INVALID;
  const int apart = order == TS_ROWS_QKV ? 64 : order == TS_ROWS_GATE_UP ? 128 : 0;
  if (apart && N % (2 * apart)) return TS_ERR_INVALID;
  if (bytes / 16 / 256 > 0x7fffffffu) return TS_ERR_UNSUPPORTED;
  return ts::launch_adapter_pack((const uint16_t*)b, (uint16_t*)packed, n_adapters, N, rank, granule_width(rank), apart, (cudaStream_t)cuda_stream) == cudaSuccess
             ? TS_OK : TS_ERR_CUDA;
}

int ts_adapter_plan(int32_t M, int32_t tile_tokens, int32_t n_rows, const int32_t* row_tokens, const int32_t* row_adapter, int32_t n_adapters,
                    int32_t* n_entries, int32_t* n_groups, int32_t* group_tokens, int32_t* n_words) {
  if (M <= 0 || n_rows <= 0 || !row_tokens || !row_adapter || n_adapters <= 0 || n_adapters > kMaxAdapters || !n_entries || !n_groups || !group_tokens || !n_words)
    return TS_ERR_INVALID;
  if (tile_tokens < 16 || tile_tokens > 256 || tile_tokens % 16 || !adapter_rows_ok(n_rows, row_tokens, row_adapter, n_adapters, M)) return TS_ERR_INVALID;
  if (!adapter_size_ok(M, n_rows)) return TS_ERR_UNSUPPORTED;
  ts::AdapterPlan plan;
  if (!ts::plan_adapters(M, tile_tokens, n_rows, row_tokens, row_adapter, n_adapters, &plan)) return TS_ERR_UNSUPPORTED;
  *n_entries = plan.n_entries;
  *n_groups = plan.n_groups;
  *group_tokens = plan.group;
  *n_words = (int32_t)plan.words.size();
  return TS_OK;
}

int ts_gemm_plan(int32_t device, int32_t M, int32_t N, int32_t K, int32_t epilogue, int32_t* tile_m, int32_t* split,
                 int32_t* pair_tokens) {
  if (M <= 0 || N <= 0 || K <= 0 || epilogue < ts::GEMM_EPI_STORE || epilogue > ts::GEMM_EPI_SILU_MUL || !tile_m || !split ||
      !pair_tokens)
    return TS_ERR_INVALID;
  int n_sms = 0;
  if (cudaSetDevice(device) != cudaSuccess || cudaDeviceGetAttribute(&n_sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
    return TS_ERR_CUDA;
  ts::GemmArgs g;
  std::memset(&g, 0, sizeof g);
  g.M = M; g.N = N; g.K = K; g.epi = epilogue;
  const ts::GemmPlan plan = ts::gemm_plan(g, n_sms);
  *tile_m = plan.tile_m;
  *split = plan.split;
  *pair_tokens = plan.pair_tokens;
  return TS_OK;
}

int ts_layer_last_cuda_error(const ts_layer* l) { return l ? l->last_cuda_error : 0; }

}  // extern "C"
