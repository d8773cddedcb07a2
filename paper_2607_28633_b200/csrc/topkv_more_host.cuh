// Host side of the calls that stand around the decode side's attention: new tokens on their way into the
// cache, shared prefixes, chosen pages. Included by topkv.cu behind topkv_decode_host.cuh, whose checks
// and launches it shares.
#pragma once
#include "topkv_append.cuh"
#include "topkv_choose.cuh"
#include "topkv_prefix.cuh"

namespace {

inline bool mult8p(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }
constexpr int64_t kFarStride = 1ll << 40;  // no stride is longer: sums of a few stay within 64 bits

// Whether [rows][heads] vectors of `bytes` at these strides do not overlap.
bool apart(int64_t rows, int64_t heads, int64_t row, int64_t head, int64_t bytes) {
  const __int128 R = rows, H = heads, sr = row, sh = head;
  const bool heads_in = (H == 1 || sh >= bytes) && (R <= 1 || sr >= (H - 1) * sh + bytes);
  const bool rows_in = (R <= 1 || sr >= bytes) && (H == 1 || sh >= (R - 1) * sr + bytes);
  return heads_in || rows_in;
}
int check_strides(std::initializer_list<int64_t> strides) {
  for (const int64_t s : strides)
    if (s < 0 || s > kFarStride) return TOPKV_ERR_INVALID_ARG;
  for (const int64_t s : strides)
    if (!mult16(s)) return TOPKV_ERR_ALIGNMENT;
  return TOPKV_OK;
}

// launch_pdl with clusters of `ctas` CTAs.
template <typename... K, typename... P>
cudaError_t launch_cluster(void (*kernel)(K...), unsigned ctas, dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const P&... params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, params...);
}

// ---- new tokens ---------------------------------------------------------------------------------
int check_new_tokens(const topkv_layout* lo, const topkv_batch* b, const topkv_new_tokens* n) {
  Resolved rs;
  int st = check_layout(lo, &rs);
  if (st != TOPKV_OK) return st;
  st = check_tables_batch(lo, b);
  if (st != TOPKV_OK) return st;
  if (b->window_tokens != 0) return TOPKV_ERR_INVALID_ARG;
  if (n == nullptr || n->struct_size != sizeof(topkv_new_tokens)) return TOPKV_ERR_INVALID_ARG;
  if (n->cache_type < TOPKV_TYPE_BF16 || n->cache_type > TOPKV_TYPE_E4M3) return TOPKV_ERR_INVALID_ARG;
  if (n->io_type != TOPKV_TYPE_BF16 && n->io_type != TOPKV_TYPE_FP16) return TOPKV_ERR_INVALID_ARG;
  const bool narrow = n->cache_type == TOPKV_TYPE_E4M3;
  if (!narrow && (n->io_type != n->cache_type || n->k_scale != 1.f || n->v_scale != 1.f)) return TOPKV_ERR_INVALID_ARG;
  for (const float s : {n->k_scale, n->v_scale})
    if (!std::isfinite(s) || s == 0.f || !std::isfinite(1.f / s)) return TOPKV_ERR_INVALID_ARG;
  if (lo->elem_bytes != (narrow ? 1u : 2u) || lo->head_dim % 8 != 0 || lo->head_dim > 2048) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (n->num_rows < 0 || n->num_rows > 0x7fffffffll || n->num_q_heads > 65535) return TOPKV_ERR_INVALID_ARG;
  if (lo->num_kv_heads > 65535) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (n->cu_tokens == nullptr && n->num_rows < b->num_requests) return TOPKV_ERR_INVALID_ARG;
  st = check_strides({n->k_row_stride, n->k_head_stride, n->q_row_stride, n->q_head_stride, n->q_out_row_stride, n->q_out_head_stride});
  if (st == TOPKV_OK && lo->kv_factor == 2) st = check_strides({n->v_row_stride, n->v_head_stride});
  if (st != TOPKV_OK) return st;
  if (!mult8p(n->cu_tokens) || !mult4p(n->positions)) return TOPKV_ERR_ALIGNMENT;
  if (n->num_q_heads > 0 && !apart(n->num_rows, n->num_q_heads, n->q_out_row_stride, n->q_out_head_stride, 2ll * lo->head_dim))
    return TOPKV_ERR_INVALID_ARG;
  if (const topkv_rotary* t = n->rotary) {
    if (t->struct_size != sizeof(topkv_rotary) || t->reserved != 0) return TOPKV_ERR_INVALID_ARG;
    if (t->style != TOPKV_ROTARY_HALVES && t->style != TOPKV_ROTARY_PAIRS) return TOPKV_ERR_INVALID_ARG;
    if (t->count % 2 != 0 || t->count > lo->head_dim || t->first > lo->head_dim - t->count || !std::isfinite(t->scale))
      return TOPKV_ERR_INVALID_ARG;
    if (t->count > 0 && t->turns == nullptr) return TOPKV_ERR_INVALID_ARG;
    if (!mult8p(t->turns)) return TOPKV_ERR_ALIGNMENT;
  }
  return TOPKV_OK;
}

template <bool BF16, bool E8>
int launch_append(const AppendParams& p, bool chunks, dim3 grid, cudaStream_t s) {
  const dim3 block(kAppendThreads);
  return launched(!chunks ? launch_pdl(topkv_append_kernel<BF16, E8, kByElements>, grid, block, 0, s, p)
                  : p.pairs ? launch_pdl(topkv_append_kernel<BF16, E8, kByNeighbours>, grid, block, 0, s, p)
                            : launch_pdl(topkv_append_kernel<BF16, E8, kByHalves>, grid, block, 0, s, p), 1);
}

// ---- shared prefixes ------------------------------------------------------------------------------
struct SharedPlan {
  AttendPlan attend;      // of the tokens behind the prefixes
  int tiles, tokens;      // of the prefix kernel's shape
  int64_t own_rows, rows; // rows of parts: of the tokens behind the prefixes, of the prefixes
  int64_t bytes;
};
std::atomic<int64_t> g_sharing_bytes{TOPKV_DEFAULT_SHARING_BYTES};
int64_t aligned16(int64_t x) { return (x + 15) / 16 * 16; }

int check_shared(const topkv_layout* lo, const topkv_batch* b, const topkv_attention* at, SharedPlan* plan) {
  const int st = check_attention(lo, b, at, &plan->attend);
  if (st != TOPKV_OK) return st;
  if (lo->kv_factor != 2) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (b->window_tokens != 0 || at->sink_tokens != 0) return TOPKV_ERR_INVALID_ARG;
  const AttendPlan& a = plan->attend;
  plan->tiles = lo->head_dim <= 128 ? 2 : 1;
  plan->tokens = lo->head_dim <= 128 ? 128 : 64;
  const int64_t R = b->num_requests, q_rows = (int64_t)at->num_q_heads * R;
  // the line on which all units lie, tiles long, is counted in 32 bits
  const __int128 units = q_rows / (kPrefixRows * plan->tiles) + lo->num_kv_heads * (R / 2 + 1);
  const __int128 line = units * plan->tiles * (((int64_t)b->max_pages_per_req * lo->page_tokens) / plan->tokens + 1);
  if (line > 0x7fffffff) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  plan->own_rows = (R + (a.uncut ? 0 : a.teams)) * a.units * a.rows;
  plan->rows = plan->tiles * (q_rows + (int64_t)kPrefixCtas * kPrefixRows);
  plan->bytes = R == 0 ? 0
                       : R * 16 + (int64_t)sizeof(PrefixHeader) + R * (int64_t)sizeof(PrefixGroup) + aligned16((plan->own_rows + plan->rows) * 8) +
                             (plan->own_rows + plan->rows) * a.dv * 4;
  plan->bytes = (plan->bytes + 255) / 256 * 256;
  return TOPKV_OK;
}

// Tensor map of a layer's keys and values, [page][plane][head][token][column], for boxes of p->box tokens: x 64
// columns in the swizzled order of the operands, or whole rows of 8-bit values as they lie. Box 0 where there is
// none: pieces of 8 to `tokens` tokens that never straddle a page need page sizes that are multiples of 8.
CUtensorMap prefix_map(AttendParams* p, uint32_t type, int tokens) {
  CUtensorMap map = {};
  p->box = 0;
  const bool narrow = type == TOPKV_TYPE_E4M3;
  const int box = std::min(tokens, p->P & -p->P);
  const int64_t head = p->H > 1 ? p->S_head : 16;
  if (box < 8 || (!narrow && p->D < 64) || p->num_pages > 0x7ffffff0ll) return map;
  for (const int64_t s : {p->S_page, p->S_kv, p->S_tok, head})
    if (s <= 0 || s >= (1ll << 40) || !mult16(s)) return map;
  const EncodeTiled encode = encode_tiled();
  if (encode == nullptr) return map;
  const cuuint64_t dims[5] = {(cuuint64_t)p->D, (cuuint64_t)p->P, (cuuint64_t)p->H, 2, (cuuint64_t)p->num_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)p->S_tok, (cuuint64_t)head, (cuuint64_t)p->S_kv, (cuuint64_t)p->S_page};
  const cuuint32_t sizes[5] = {narrow ? (cuuint32_t)p->D : 64, (cuuint32_t)box, 1, 1, 1}, steps[5] = {1, 1, 1, 1, 1};
  const CUresult r = encode(&map, narrow                     ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                                  : type == TOPKV_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                            : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5,
                            const_cast<uint8_t*>(p->pool), dims, strides, sizes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            narrow ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r == CUDA_SUCCESS) p->box = box;
  return map;
}

template <int DP, int TYPE>
int launch_prefix(PrefixParams p, cudaStream_t s) {
  using S = PrefixShape<DP, TYPE>;
  static std::atomic<uint64_t> done{0};
  const int st = raise_smem(topkv_prefix_kernel<DP, TYPE>, S::kSmem, &done);
  if (st != TOPKV_OK) return st;
  const CUtensorMap map = prefix_map(&p.a, TYPE, S::kTokens);
  return launched(launch_pdl(topkv_prefix_kernel<DP, TYPE>, dim3(kPrefixCtas), dim3(S::kThreads), S::kSmem, s, p, map), 1);
}
template <int TYPE>
int launch_prefix_dim(const PrefixParams& p, cudaStream_t s) {
  if (p.a.D <= 64) return launch_prefix<64, TYPE>(p, s);
  if (p.a.D <= 128) return launch_prefix<128, TYPE>(p, s);
  return launch_prefix<256, TYPE>(p, s);
}

// ---- chosen pages -----------------------------------------------------------------------------------
constexpr uint32_t kChooseMaxHeads = 128;     // query heads per KV head: they are held in shared memory
constexpr int64_t kChooseMaxKeys = kGatherKeys;  // pages whose keys a CTA's are
struct ChoosePlan {
  AttendPlan attend;
  int ctas;          // of a cluster
  bool gather;       // its first CTA has all keys
  int64_t cap;       // keys of a CTA at most
  int64_t key_bytes; // of the workspace, where shared memory does not hold the keys
  int pitch, smem;
};
int choose_columns(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : 256; }

int check_choice(const topkv_layout* lo, const topkv_batch* b, const topkv_attention* at, const topkv_page_choice* c, ChoosePlan* plan) {
  if (c == nullptr || c->struct_size != sizeof(topkv_page_choice)) return TOPKV_ERR_INVALID_ARG;
  if (c->budget == 0 || c->budget > 0x7ffff000u || c->last_pages == 0 || c->first_pages > 0x7fffffffu || c->last_pages > 0x7fffffffu)
    return TOPKV_ERR_INVALID_ARG;
  const int st = check_attention(lo, b, at, &plan->attend, c->budget);
  if (st != TOPKV_OK) return st;
  if (lo->kv_factor != 2) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (b->window_tokens != 0 || at->sink_tokens != 0 || !(at->k_scale > 0.f)) return TOPKV_ERR_INVALID_ARG;
  const uint32_t G = at->num_q_heads / lo->num_kv_heads;
  if (G > kChooseMaxHeads) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  const int64_t units = (int64_t)b->num_requests * lo->num_kv_heads;
  if (units * kChooseCluster > 0x7fffffffll) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (!mult16p(c->bounds) || !mult4p(c->steps) || !mult4p(c->chosen)) return TOPKV_ERR_ALIGNMENT;
  // Two CTAs per SM are wanted, but none with fewer than 256 pages.
  plan->ctas = 1;
  while (plan->ctas < kChooseCluster && units * plan->ctas < 2 * 148 && b->max_pages_per_req / plan->ctas > 256) plan->ctas *= 2;
  plan->gather = b->max_pages_per_req <= kGatherKeys;
  plan->cap = plan->gather ? b->max_pages_per_req : (b->max_pages_per_req + plan->ctas - 1) / plan->ctas + 8;
  const bool inside = plan->cap <= kChooseMaxKeys;
  plan->key_bytes = inside ? 0 : units * b->max_pages_per_req * 4;
  plan->pitch = choose_columns((int)lo->head_dim) * 2 + 16;
  plan->smem = (int)G * (plan->pitch + 4) + (inside ? (int)plan->cap * 4 : 0);
  return TOPKV_OK;
}

template <int DP, bool BF16, bool GATHER>
int launch_choose2(const ChooseParams& p, const ChoosePlan& plan, int64_t units, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  constexpr int kMost = (int)kChooseMaxHeads * (DP * 2 + 20) + (int)kChooseMaxKeys * 4;
  static_assert(kMost + (int)sizeof(ChooseShared) <= kSmemBudget, "queries and keys fit a CTA");
  const int st = raise_smem(topkv_choose_pages_kernel<DP, BF16, GATHER>, kMost, &done);
  if (st != TOPKV_OK) return st;
  return launched(launch_cluster(topkv_choose_pages_kernel<DP, BF16, GATHER>, plan.ctas, dim3((unsigned)(units * plan.ctas)),
                                 dim3(kChooseThreads), plan.smem, s, p), 1);
}
template <int DP>
int launch_choose(const ChooseParams& p, const ChoosePlan& plan, int64_t units, bool bf16, cudaStream_t s) {
  if (plan.gather) return bf16 ? launch_choose2<DP, true, true>(p, plan, units, s) : launch_choose2<DP, false, true>(p, plan, units, s);
  return bf16 ? launch_choose2<DP, true, false>(p, plan, units, s) : launch_choose2<DP, false, false>(p, plan, units, s);
}

int check_choice_workspace(const void* ws, int64_t bytes, int64_t needed) {
  if (needed == 0) return TOPKV_OK;
  if (ws == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(ws)) return TOPKV_ERR_ALIGNMENT;
  return bytes < needed ? TOPKV_ERR_CAPACITY : TOPKV_OK;
}

}  // namespace

extern "C" {

int topkv_bound_pages_layer(int layer, const void* pool, const topkv_layout* layout, const topkv_batch* batch,
                            uint32_t cache_type, int8_t* d_bounds, float* d_steps, topkv_stream_t stream) {
  Resolved rs;
  int st = check_layout(layout, &rs);
  if (st == TOPKV_OK) st = check_tables_batch(layout, batch);
  if (st != TOPKV_OK) return st;
  if (cache_type < TOPKV_TYPE_BF16 || cache_type > TOPKV_TYPE_E4M3) return TOPKV_ERR_INVALID_ARG;
  const bool narrow = cache_type == TOPKV_TYPE_E4M3;
  if (layout->kv_factor != 2 || layout->elem_bytes != (narrow ? 1u : 2u) || layout->head_dim > 256 ||
      !mult16((int64_t)layout->head_dim * layout->elem_bytes))
    return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (layer < 0 || (uint32_t)layer >= layout->num_layers) return TOPKV_ERR_LAYER_RANGE;
  if (layout->num_kv_heads > 1 && !mult16(layout->pool_head_stride)) return TOPKV_ERR_ALIGNMENT;
  if (pool == nullptr || d_bounds == nullptr || d_steps == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(pool) || !mult16p(d_bounds) || !mult4p(d_steps)) return TOPKV_ERR_ALIGNMENT;
  if (batch->num_requests == 0 || batch->max_pages_per_req == 0) return TOPKV_OK;
  BoundParams p = {};
  p.pool = static_cast<const uint8_t*>(pool) + (int64_t)layer * layout->pool_layer_stride;
  p.bt = batch->block_table;
  p.sl = batch->seq_lens;
  p.bounds = d_bounds;
  p.steps = d_steps;
  p.S_page = layout->pool_page_stride;
  p.S_tok = layout->page_tokens > 1 ? layout->pool_token_stride : 0;
  p.S_head = layout->num_kv_heads > 1 ? layout->pool_head_stride : 0;
  p.num_pages = layout->num_pool_pages;
  p.maxp = batch->max_pages_per_req;
  p.P = (int)layout->page_tokens;
  p.H = layout->num_kv_heads;
  p.D = (int)layout->head_dim;
  p.window = batch->window_tokens;
  p.columns = (uint32_t)p.maxp;
  if (p.window > 0) p.columns = (uint32_t)std::min<int64_t>(p.maxp, ((int64_t)p.window + p.P - 2) / p.P + 1);
  const int64_t items = (int64_t)batch->num_requests * p.columns * p.H;
  if (items > 0x7fffffffll) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  p.items = (uint32_t)items;
  const int64_t ctas = (items + kBoundThreads / 32 - 1) / (kBoundThreads / 32);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const dim3 grid((unsigned)ctas), block(kBoundThreads);
  return launched(cache_type == TOPKV_TYPE_BF16   ? launch_pdl(topkv_bound_pages_kernel<kBf16>, grid, block, 0, s, p)
                  : cache_type == TOPKV_TYPE_FP16 ? launch_pdl(topkv_bound_pages_kernel<kFp16>, grid, block, 0, s, p)
                                                  : launch_pdl(topkv_bound_pages_kernel<kE4m3>, grid, block, 0, s, p), 1);
}

int64_t topkv_page_choice_workspace_bytes(const topkv_layout* layout, const topkv_batch* batch,
                                          const topkv_attention* attention, const topkv_page_choice* choice) {
  ChoosePlan plan;
  const int st = check_choice(layout, batch, attention, choice, &plan);
  return st != TOPKV_OK ? st : std::max(plan.attend.bytes, (plan.key_bytes + 255) / 256 * 256);
}

int topkv_choose_pages_layer(const topkv_layout* layout, const topkv_batch* batch, const topkv_attention* attention,
                             const topkv_page_choice* choice, const void* d_q, void* d_workspace, int64_t workspace_bytes,
                             topkv_stream_t stream) {
  ChoosePlan plan;
  int st = check_choice(layout, batch, attention, choice, &plan);
  if (st != TOPKV_OK) return st;
  if (attention->scale < 0.f) return TOPKV_ERR_INVALID_ARG;  // the pages with the smallest products would count
  if (d_q == nullptr || choice->bounds == nullptr || choice->steps == nullptr || choice->chosen == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(d_q)) return TOPKV_ERR_ALIGNMENT;
  st = check_choice_workspace(d_workspace, workspace_bytes, plan.key_bytes);
  if (st != TOPKV_OK) return st;
  if (batch->num_requests == 0) return TOPKV_OK;
  ChooseParams p = {};
  p.bt = batch->block_table;
  p.sl = batch->seq_lens;
  p.q = static_cast<const uint8_t*>(d_q);
  p.bounds = choice->bounds;
  p.steps = choice->steps;
  p.chosen = choice->chosen;
  p.keys = plan.key_bytes > 0 ? static_cast<uint32_t*>(d_workspace) : nullptr;
  p.q_req = attention->q_request_stride;
  p.q_head = attention->q_head_stride;
  p.num_pages = layout->num_pool_pages;
  p.maxp = batch->max_pages_per_req;
  p.P = (int)layout->page_tokens;
  p.H = (int)layout->num_kv_heads;
  p.G = (int)(attention->num_q_heads / layout->num_kv_heads);
  p.D = (int)layout->head_dim;
  p.budget = (int)choice->budget;
  p.firsts = (int)choice->first_pages;
  p.lasts = (int)choice->last_pages;
  p.pitch = plan.pitch;
  const int64_t units = (int64_t)batch->num_requests * p.H;
  const bool bf16 = attention->io_type == TOPKV_TYPE_BF16;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (p.D <= 64) return launch_choose<64>(p, plan, units, bf16, s);
  if (p.D <= 128) return launch_choose<128>(p, plan, units, bf16, s);
  return launch_choose<256>(p, plan, units, bf16, s);
}

int topkv_attend_pages_layer(int layer, const void* pool, const topkv_layout* layout, const topkv_batch* batch,
                             const topkv_attention* attention, const topkv_page_choice* choice, const void* d_q, void* d_out,
                             void* d_workspace, int64_t workspace_bytes, topkv_stream_t stream) {
  ChoosePlan plan;
  int st = check_choice(layout, batch, attention, choice, &plan);
  if (st != TOPKV_OK) return st;
  st = check_attend_pointers(layer, layout, pool, d_q, d_out, d_workspace, workspace_bytes, plan.attend.bytes);
  if (st != TOPKV_OK) return st;
  if (choice->chosen == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (batch->num_requests == 0) return TOPKV_OK;
  AttendParams p = attend_params(layer, pool, layout, batch, attention, plan.attend, d_q, d_out);
  p.chosen = choice->chosen;
  p.budget = (int)choice->budget;
  return attend_and_join<kChosenPages>(p, plan.attend, false, attention->cache_type, d_workspace, reinterpret_cast<cudaStream_t>(stream));
}

int topkv_plan_prefixes(const topkv_layout* layout, const topkv_batch* batch, int32_t min_tokens, int32_t* d_plan,
                        topkv_stream_t stream) {
  Resolved rs;
  const int st = check_pages(layout, batch, &rs);
  if (st != TOPKV_OK) return st;
  if (min_tokens < 0) return TOPKV_ERR_INVALID_ARG;
  if (batch->num_requests == 0) return TOPKV_OK;
  if (d_plan == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult4p(d_plan)) return TOPKV_ERR_ALIGNMENT;
  if ((int64_t)batch->num_requests * TOPKV_PLAN_ROWS > 0x7fffffffll) return TOPKV_ERR_INVALID_ARG;
  PrefixPlanParams p;
  p.bt = batch->block_table;
  p.sl = batch->seq_lens;
  p.plan = d_plan;
  p.num_pages = layout->num_pool_pages;
  p.R = batch->num_requests;
  p.maxp = batch->max_pages_per_req;
  p.P = (int)layout->page_tokens;
  p.min_tokens = min_tokens;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const dim3 grid((unsigned)((p.R + kPrefixPlanThreads / 32 - 1) / (kPrefixPlanThreads / 32)));
  if (p.R <= kPrefixPlanRows) return launched(launch_cluster(topkv_plan_cluster_kernel, grid.x, grid, dim3(kPrefixPlanThreads), 0, s, p), 1);
  const int first = launched(launch_pdl(topkv_plan_leaders_kernel, grid, dim3(kPrefixPlanThreads), 0, s, p), 1);
  if (first != TOPKV_OK) return first;
  return launched(launch_pdl(topkv_plan_groups_kernel, grid, dim3(kPrefixPlanThreads), 0, s, p), 1);
}

int64_t topkv_set_sharing_bytes(int64_t bytes) {
  return bytes < 0 ? TOPKV_ERR_INVALID_ARG : g_sharing_bytes.exchange(bytes, std::memory_order_relaxed);
}

int64_t topkv_attend_shared_workspace_bytes(const topkv_layout* layout, const topkv_batch* batch,
                                            const topkv_attention* attention) {
  SharedPlan plan;
  const int st = check_shared(layout, batch, attention, &plan);
  return st != TOPKV_OK ? st : plan.bytes;
}

int topkv_attend_shared_layer(int layer, const void* pool, const topkv_layout* layout, const topkv_batch* batch,
                              const topkv_attention* attention, const int32_t* d_plan, const void* d_q, void* d_out,
                              void* d_workspace, int64_t workspace_bytes, topkv_stream_t stream) {
  SharedPlan plan;
  int st = check_shared(layout, batch, attention, &plan);
  if (st != TOPKV_OK) return st;
  st = check_attend_pointers(layer, layout, pool, d_q, d_out, d_workspace, workspace_bytes, plan.bytes);
  if (st != TOPKV_OK) return st;
  if (batch->num_requests == 0) return TOPKV_OK;
  if (d_plan == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult4p(d_plan)) return TOPKV_ERR_ALIGNMENT;
  if ((int64_t)batch->num_requests * TOPKV_PLAN_ROWS > 0x7fffffffll) return TOPKV_ERR_INVALID_ARG;
  PrefixParams p = {};
  p.a = attend_params(layer, pool, layout, batch, attention, plan.attend, d_q, d_out);
  p.a.plan = d_plan;
  // Whether a group's tokens are formed once. 8 KV heads of 128, both ways after other work has been through L2,
  // once / by each request: 16-bit, 40 pairs of 4,096 tokens 170 / 236 us, 40 fours of 1,024 105 / 118, 20 pairs of 1,024
  // 60 / 51, eight of 8,192 42 / 55: worth it from 8 MB on. 8-bit tokens are converted tile by tile, at a rate that does
  // not depend on the rows: 40 pairs of 4,096 197 / 152, 40 fours of 1,024 118 / 101, 8 eights of 4,096 79 / 122, 8
  // sixteens of 1,024 76 / 87, as if two more members had to read them.
  const int64_t least = g_sharing_bytes.load(std::memory_order_relaxed);
  const int64_t token_bytes = 2ll * p.a.H * p.a.D * (int64_t)layout->elem_bytes;
  p.a.least_saved = least / token_bytes + (least % token_bytes != 0);  // rounded up: at least that many bytes
  p.a.spent = layout->elem_bytes == 1 && least > 0 ? 3 : 1;
  p.tiles = plan.tiles;
  p.tokens = plan.tokens;
  uint8_t* w = static_cast<uint8_t*>(d_workspace);
  auto part = [&](int64_t bytes) {
    uint8_t* at = w;
    w += aligned16(bytes);
    return at;
  };
  const int64_t R = p.a.R;
  p.a.joins = reinterpret_cast<int4*>(part(R * 16));
  p.a.by_request = 1;
  p.header = reinterpret_cast<PrefixHeader*>(part(sizeof(PrefixHeader)));
  p.groups = reinterpret_cast<PrefixGroup*>(part(R * (int64_t)sizeof(PrefixGroup)));
  p.a.ml = reinterpret_cast<float2*>(part((plan.own_rows + plan.rows) * 8));
  p.ml = p.a.ml + plan.own_rows;
  p.a.part = reinterpret_cast<float*>(w);
  p.part = p.a.part + plan.own_rows * p.a.Dv;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const uint32_t type = attention->cache_type;
  st = type == TOPKV_TYPE_BF16 ? launch_prefix_dim<kBf16>(p, s) : type == TOPKV_TYPE_FP16 ? launch_prefix_dim<kFp16>(p, s) : launch_prefix_dim<kE4m3>(p, s);
  if (st != TOPKV_OK) return st;
  st = launch_attend_type<kBehindPrefix>(p.a, type, plan.attend.units, s);
  if (st != TOPKV_OK) return st;
  const int64_t ctas = R * plan.attend.units;
  const unsigned z = (unsigned)std::max<int64_t>((plan.attend.rows + kJoinRows - 1) / kJoinRows, std::min<int64_t>(plan.attend.rows, 4 * 148 / ctas));
  return launched(launch_pdl(topkv_prefix_join_kernel, dim3((unsigned)R, plan.attend.units, z), dim3(kPrefixJoinThreads), 0, s, p), 1);
}

int topkv_append_layer(int layer, void* pool, const topkv_layout* layout, const topkv_batch* batch,
                       const topkv_new_tokens* tokens, const void* d_k, const void* d_v, const void* d_q,
                       void* d_q_out, topkv_stream_t stream) {
  const int st = check_new_tokens(layout, batch, tokens);
  if (st != TOPKV_OK) return st;
  if (layer < 0 || (uint32_t)layer >= layout->num_layers) return TOPKV_ERR_LAYER_RANGE;
  const bool values = layout->kv_factor == 2, queries = tokens->num_q_heads > 0;
  if (tokens->num_rows == 0) return TOPKV_OK;  // tensors without rows may have no address
  if (pool == nullptr || d_k == nullptr || (values && d_v == nullptr) || (queries && (d_q == nullptr || d_q_out == nullptr)))
    return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(pool) || !mult16p(d_k) || (values && !mult16p(d_v)) || (queries && (!mult16p(d_q) || !mult16p(d_q_out))))
    return TOPKV_ERR_ALIGNMENT;
  if (queries && d_q == d_q_out && (tokens->q_row_stride != tokens->q_out_row_stride || tokens->q_head_stride != tokens->q_out_head_stride))
    return TOPKV_ERR_INVALID_ARG;
  if (batch->num_requests == 0 || batch->max_pages_per_req == 0) return TOPKV_OK;
  AppendParams p = {};
  p.pool = static_cast<uint8_t*>(pool) + (int64_t)layer * layout->pool_layer_stride;
  p.bt = batch->block_table;
  p.sl = batch->seq_lens;
  p.cu = tokens->cu_tokens;
  p.positions = tokens->positions;
  const void* in[3] = {d_q, d_k, d_v};
  const int64_t row[3] = {tokens->q_row_stride, tokens->k_row_stride, tokens->v_row_stride};
  const int64_t head[3] = {tokens->q_head_stride, tokens->k_head_stride, tokens->v_head_stride};
  for (int i = 0; i < 3; ++i) {
    p.in[i] = static_cast<const uint8_t*>(in[i]);
    p.in_row[i] = row[i];
    p.in_head[i] = head[i];
  }
  p.q_out = static_cast<uint8_t*>(d_q_out);
  p.out_row = tokens->q_out_row_stride;
  p.out_head = tokens->q_out_head_stride;
  p.S_page = layout->pool_page_stride;
  p.S_kv = values ? layout->pool_kv_stride : 0;
  p.S_tok = layout->page_tokens > 1 ? layout->pool_token_stride : 0;
  p.S_head = layout->num_kv_heads > 1 ? layout->pool_head_stride : 0;
  p.num_pages = layout->num_pool_pages;
  // rows behind the last request's are spare: without offsets there is one row per request
  p.num_rows = tokens->cu_tokens == nullptr ? batch->num_requests : tokens->num_rows;
  p.R = batch->num_requests;
  p.maxp = batch->max_pages_per_req;
  p.P = (int)layout->page_tokens;
  p.Hq = (int)tokens->num_q_heads;
  p.H = (int)layout->num_kv_heads;
  p.rows = p.Hq + p.H * (values ? 2 : 1);
  p.D = (int)layout->head_dim;
  const float scales[2] = {tokens->k_scale, tokens->v_scale};
  for (int i = 0; i < 2; ++i) {
    int exponent;
    const bool exact = std::fabs(std::frexp(scales[i], &exponent)) == 0.5f;  // a power of two
    p.stored[i] = exact ? 0.f : scales[i];
    p.inv[i] = 1.f / scales[i];
    if (!exact && !std::isnormal(p.inv[i])) p.inv[i] = 0.f;  // has lost bits: products of zero are all looked at
  }
  if (const topkv_rotary* t = tokens->rotary) {
    p.first = (int)t->first;
    p.half = (int)t->count / 2;
    p.pairs = t->style == TOPKV_ROTARY_PAIRS;
    p.turns = t->turns;
    p.scale = t->scale;
  }
  const bool chunks = p.first % 8 == 0 && (p.pairs ? 2 * p.half : p.half) % 8 == 0;
  // A CTA has a few tokens, or a share of a token's heads. All take about as long, so they are cut such that the rounds of
  // 4 x 148, which are on the GPU at a time, come out short: a CTA costs half a pass (two rows a thread) to begin. With 128
  // heads of 576: 64 tokens in 576 CTAs 5.5 us, in 1,216 8.2; 256 tokens in 512 CTAs 18.8 us, in 1,280 21.6, in 768 22.0; 600
  // tokens in 3,600 41.6, in 600 53. With 80 rows of 128: 1,000 tokens two a CTA 11.6 us, one 13.8, four 13.1; 2,000 four a
  // CTA 19.1, one 24.1. More than eight are slower (13,312 tokens 61 us, sixteen a CTA 67).
  constexpr int kResident = 4 * 148;
  const int most = std::min(8, p.half > 0 ? kAppendPairs / p.half : 8);
  const int items = chunks ? (p.pairs ? p.half / 4 : p.half / 8) + p.D / 8 - p.half / 4 : p.D - p.half;
  const double passes = (double)p.rows * items / (2 * kAppendThreads);
  const int64_t shares = std::min<int64_t>(65535, (int64_t)std::ceil(passes));
  double least = std::numeric_limits<double>::infinity();
  int64_t ctas = 0, y = 1;
  auto weigh = [&](int tokens, int64_t parts) {
    const int64_t n = (p.num_rows + tokens - 1) / tokens, rounds = (n * parts + kResident - 1) / kResident;
    const double cost = rounds * (0.5 + passes * tokens / parts);
    if (cost >= least) return;
    least = cost;
    p.tokens = tokens;
    ctas = n;
    y = parts;
  };
  for (int t = 1; t <= most; ++t) weigh(t, 1);
  for (int64_t k = 2; k <= std::min<int64_t>(shares, 8); ++k) weigh(1, k);
  if (p.num_rows < kResident) weigh(1, std::min(shares, kResident / p.num_rows));
  const dim3 grid((unsigned)ctas, (unsigned)y);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const bool bf16 = tokens->io_type == TOPKV_TYPE_BF16, narrow = tokens->cache_type == TOPKV_TYPE_E4M3;
  if (bf16) return narrow ? launch_append<true, true>(p, chunks, grid, s) : launch_append<true, false>(p, chunks, grid, s);
  return narrow ? launch_append<false, true>(p, chunks, grid, s) : launch_append<false, false>(p, chunks, grid, s);
}

}  // extern "C"
