// Host side of the decode side's entry points: attention over the paged cache and the page
// operators. Included by topkv.cu, whose argument checks, launch counter and error state it shares.
#pragma once
#include "topkv_attend.cuh"
#include "topkv_latent.cuh"
#include "topkv_pages.cuh"

namespace {

inline bool mult4p(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

// The parts of a batch that these calls use: unlike the copies they need no prefix sums, so any
// number of requests is fine without cu_seq_lens.
int check_tables_batch(const topkv_layout* lo, const topkv_batch* b) {
  if (lo->page_tokens > 0x7fffffffu) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (b == nullptr || b->struct_size != sizeof(topkv_batch) ||
      (b->flags & ~(uint32_t)(TOPKV_FLAG_OVERLAP_PREVIOUS | TOPKV_FLAG_TABLES_SETTLED)) != 0)
    return TOPKV_ERR_INVALID_ARG;
  if (b->num_requests < 0 || b->max_pages_per_req < 0 || b->total_tokens < -1 || b->window_tokens < 0 ||
      b->reserved != 0)
    return TOPKV_ERR_INVALID_ARG;
  if (b->num_requests > 0) {
    if (b->seq_lens == nullptr || (b->max_pages_per_req > 0 && b->block_table == nullptr))
      return TOPKV_ERR_INVALID_ARG;
    if (!mult4p(b->seq_lens) || !mult4p(b->block_table)) return TOPKV_ERR_ALIGNMENT;
    if ((int64_t)b->num_requests * b->max_pages_per_req > 0x7fffffffll) return TOPKV_ERR_INVALID_ARG;
    if ((int64_t)b->max_pages_per_req * lo->page_tokens > 0x7fffffffll) return TOPKV_ERR_INVALID_ARG;
  }
  return TOPKV_OK;
}

int launched(cudaError_t e, int kernels) {
  if (e != cudaSuccess) {
    cudaGetLastError();
    return cuda_fail(e);
  }
  g_launches.fetch_add(kernels, std::memory_order_relaxed);
  return TOPKV_OK;
}

// The dynamic shared memory of a kernel is raised once per device.
template <typename K>
int raise_smem(K kernel, int bytes, std::atomic<uint64_t>* done) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= 64) return TOPKV_ERR_INVALID_ARG;
  if (done->load(std::memory_order_acquire) >> dev & 1) return TOPKV_OK;
  const cudaError_t a = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (a != cudaSuccess) {
    cudaGetLastError();
    return cuda_fail(a);
  }
  done->fetch_or(1ull << dev, std::memory_order_release);
  return TOPKV_OK;
}

// ---- attention ----------------------------------------------------------------------------------

struct AttendPlan {
  int units;        // CTAs per team
  int row_tile;     // query heads per CTA
  int rows;         // rows of a partial result
  int dv;
  int teams;
  int joins;        // join records: one per request or per team, whichever are fewer
  bool uncut;
  bool narrow;      // a warp per request
  int64_t bytes;    // of the workspace
};

int check_attention(const topkv_layout* lo, const topkv_batch* b, const topkv_attention* at, AttendPlan* plan) {
  Resolved rs;
  int st = check_layout(lo, &rs);
  if (st != TOPKV_OK) return st;
  st = check_tables_batch(lo, b);
  if (st != TOPKV_OK) return st;
  if (at == nullptr || at->struct_size != sizeof(topkv_attention) || at->reserved != 0) return TOPKV_ERR_INVALID_ARG;
  if (at->cache_type < TOPKV_TYPE_BF16 || at->cache_type > TOPKV_TYPE_E4M3) return TOPKV_ERR_INVALID_ARG;
  const bool narrow = at->cache_type == TOPKV_TYPE_E4M3;
  if (at->io_type != TOPKV_TYPE_BF16 && at->io_type != TOPKV_TYPE_FP16) return TOPKV_ERR_INVALID_ARG;
  if (!narrow && at->io_type != at->cache_type) return TOPKV_ERR_INVALID_ARG;
  if (at->num_q_heads == 0 || at->num_q_heads > 65535 || at->num_q_heads % lo->num_kv_heads != 0)
    return TOPKV_ERR_INVALID_ARG;
  if (at->sink_tokens > 0x7fffffffu) return TOPKV_ERR_INVALID_ARG;
  if (!std::isfinite(at->scale) || !std::isfinite(at->k_scale) || !std::isfinite(at->v_scale)) return TOPKV_ERR_INVALID_ARG;
  if (!narrow && (at->k_scale != 1.f || at->v_scale != 1.f)) return TOPKV_ERR_INVALID_ARG;
  if (lo->elem_bytes != (narrow ? 1u : 2u)) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  const int D = (int)lo->head_dim;
  const int64_t head_bytes = (int64_t)D * lo->elem_bytes;
  if (!mult16(head_bytes)) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (lo->kv_factor == 2) {
    if (D > 256) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
    if (at->value_dim != 0 && at->value_dim != lo->head_dim) return TOPKV_ERR_INVALID_ARG;
    if (lo->num_kv_heads > 1 && !mult16(lo->pool_head_stride)) return TOPKV_ERR_ALIGNMENT;
    plan->dv = D;
  } else {
    if (lo->num_kv_heads != 1 || narrow || D > kLatentMaxD) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
    if (at->value_dim == 0 || at->value_dim > lo->head_dim || at->value_dim % 16 != 0) return TOPKV_ERR_INVALID_ARG;
    if (at->value_dim > (uint32_t)kLatentMaxDv) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
    plan->dv = (int)at->value_dim;
  }
  const int64_t q_row = 2ll * D, o_row = 2ll * plan->dv;
  if (at->q_request_stride < 0 || at->q_head_stride < 0 || at->out_request_stride < 0 || at->out_head_stride < 0)
    return TOPKV_ERR_INVALID_ARG;
  if (!mult16(at->q_request_stride) || !mult16(at->q_head_stride) || !mult16(at->out_request_stride) ||
      !mult16(at->out_head_stride) || !mult16(q_row) || !mult4p(at->lse))
    return TOPKV_ERR_ALIGNMENT;
  // rows of out must not overlap: heads inside a request, or requests inside a head
  const int64_t far = 1ll << 40;
  const __int128 R = b->num_requests, Hq = at->num_q_heads, sr = at->out_request_stride, sh = at->out_head_stride;
  if (sh > far || sr > far || at->q_request_stride > far || at->q_head_stride > far) return TOPKV_ERR_INVALID_ARG;
  const bool heads_in = (Hq == 1 || sh >= o_row) && (R <= 1 || sr >= (Hq - 1) * sh + o_row);
  const bool requests_in = (R <= 1 || sr >= o_row) && (Hq == 1 || sh >= (R - 1) * sr + o_row);
  if (!heads_in && !requests_in) return TOPKV_ERR_INVALID_ARG;

  // How the work is shared out. A request can have at most `most` visible tokens.
  const int G = (int)(at->num_q_heads / lo->num_kv_heads);
  // query heads per CTA: latent rows take 16, 32 or 64 as columns of one product, whichever holds
  // them all, so that few heads do not pay for empty columns
  plan->row_tile = lo->kv_factor == 2 ? kAttendRows : G <= 16 ? 16 : G <= 32 ? 32 : 64;
  const int gtiles = (G + plan->row_tile - 1) / plan->row_tile;
  plan->units = (int)lo->num_kv_heads * gtiles;
  plan->rows = std::min(G, plan->row_tile);
  if (plan->units > 65535) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  int64_t most = (int64_t)b->max_pages_per_req * lo->page_tokens;
  if (most > 0x7ffff000ll) return TOPKV_ERR_INVALID_ARG;  // token numbers a few tiles further still fit an int
  if (b->window_tokens > 0) most = std::min(most, (int64_t)b->window_tokens + at->sink_tokens);
  if (b->total_tokens >= 0) most = std::min(most, b->total_tokens);
  const int64_t tiles = (most + kTileTokens - 1) / kTileTokens;
  const int64_t resident = lo->kv_factor == 1 ? 148 : 148 * attend_ctas_per_sm(D, (int)at->cache_type) - 4;
  int64_t teams = std::max<int64_t>(1, resident / plan->units);
  // units that do not divide the resident CTAs would leave some of them idle: two rounds then
  if (teams * plan->units * 8 < resident * 7) teams = std::max<int64_t>(1, 2 * resident / plan->units);
  teams = std::min<int64_t>(teams, kJoinParts);
  teams = std::min(teams, std::max<int64_t>(1, b->num_requests) * std::max<int64_t>(1, tiles));
  plan->uncut = tiles <= kUncutTiles || (teams == 1 && b->num_requests == 1);
  // Many more short requests than CTAs at a time: a warp each, so that no warp waits for another and
  // there are fewer rounds. 8 KV heads of 64, 132 visible tokens: 256 requests 26 -> 20 us, 160 the same,
  // 96 from 13 to 15; of 128, up to 200 tokens: 192 requests 29 -> 25, 128 from 22 to 23, up to 60
  // tokens: 128 requests 15 -> 13.
  plan->narrow = plan->uncut && lo->kv_factor == 2 &&
                 (int64_t)b->num_requests * plan->units > resident * (tiles <= 1 ? 1 : 3);
  plan->teams = !plan->uncut ? (int)teams : plan->narrow ? (b->num_requests + kAttendWarps - 1) / kAttendWarps : b->num_requests;
  plan->bytes = 0;
  if (!plan->uncut && b->num_requests > 0) {
    const int64_t slots = 2ll * plan->teams * plan->units * plan->rows;
    if (slots * plan->dv > 0x7fffffffll) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
    plan->joins = std::min(plan->teams, b->num_requests);
    plan->bytes = (int64_t)plan->joins * 16 + slots * 8 + slots * plan->dv * 4;
    plan->bytes = (plan->bytes + 255) / 256 * 256;
  }
  return TOPKV_OK;
}

template <int DP, int TYPE>
int launch_attend(const AttendParams& p, int units, cudaStream_t s) {
  using S = AttendShape<DP, TYPE>;
  static std::atomic<uint64_t> done{0};
  const int st = raise_smem(topkv_attend_kernel<DP, TYPE>, S::kSmem, &done);
  if (st != TOPKV_OK) return st;
  return launched(launch_pdl(topkv_attend_kernel<DP, TYPE>, dim3(p.teams, units), dim3(kAttendThreads), S::kSmem, s, p), 1);
}
template <int TYPE>
int launch_attend_dim(const AttendParams& p, int units, cudaStream_t s) {
  if (p.D <= 64) return launch_attend<64, TYPE>(p, units, s);
  if (p.D <= 128) return launch_attend<128, TYPE>(p, units, s);
  return launch_attend<256, TYPE>(p, units, s);
}

// Tensor map of one layer's rows, [page][token][column], for boxes of p->box tokens x 64 columns in the
// swizzled order of the operands. Pieces of 8 to 64 tokens that never straddle a page: the page size
// must be a multiple of 8 and tiles must begin at multiples of 8 tokens, so windowed layers, whose
// first token is anywhere, do without (box 0), as does a layout that a tensor map cannot describe.
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    if (e != cudaSuccess) cudaGetLastError();
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(f) : nullptr;
  }();
  return fn;
}
CUtensorMap latent_map(AttendParams* p) {
  CUtensorMap map = {};
  p->box = 0;
  const int box = std::min(kLatentTile, p->P & -p->P);
  const int64_t tok = p->P > 1 ? p->S_tok : 16;
  if (p->window > 0 || box < 8 || p->S_page >= (1ll << 40) || tok >= (1ll << 40) || p->num_pages > 0x7fffffffll) return map;
  const EncodeTiled encode = encode_tiled();
  if (encode == nullptr) return map;
  const cuuint64_t dims[3] = {(cuuint64_t)p->D, (cuuint64_t)p->P, (cuuint64_t)p->num_pages};
  const cuuint64_t strides[2] = {(cuuint64_t)tok, (cuuint64_t)p->S_page};
  const cuuint32_t sizes[3] = {64, (cuuint32_t)box, 1}, steps[3] = {1, 1, 1};
  const CUresult r = encode(&map, p->io_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                            const_cast<uint8_t*>(p->pool), dims, strides, sizes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r == CUDA_SUCCESS) p->box = box;
  return map;
}

// ... and of the queries, [request][head][column], for boxes of one request's heads_per_box heads.
CUtensorMap query_map(AttendParams* p, int heads_per_box) {
  CUtensorMap map = {};
  p->q_box = 0;
  if ((p->G > 1 && p->q_head < 2ll * p->D) || p->q_head >= (1ll << 40) || p->q_req >= (1ll << 40)) return map;
  const EncodeTiled encode = encode_tiled();
  if (encode == nullptr) return map;
  const bool shared = p->q_req == 0;  // one query for all requests
  const cuuint64_t dims[3] = {(cuuint64_t)p->D, (cuuint64_t)p->G, (cuuint64_t)(shared ? 1 : p->R)};
  const cuuint64_t strides[2] = {(cuuint64_t)(p->G > 1 ? p->q_head : 16), (cuuint64_t)(shared ? 16 : p->q_req)};
  const cuuint32_t sizes[3] = {64, (cuuint32_t)heads_per_box, 1}, steps[3] = {1, 1, 1};
  const CUresult r = encode(&map, p->io_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                            const_cast<uint8_t*>(p->q), dims, strides, sizes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r == CUDA_SUCCESS) p->q_box = 1;
  return map;
}

template <int N, bool BF16>
int launch_latent2(AttendParams p, int units, cudaStream_t s) {
  static std::atomic<uint64_t> done{0};
  const int st = raise_smem(topkv_latent_kernel<N, BF16>, (int)latent_smem(N, kLatentMaxD, kLatentMaxDv).total, &done);
  if (st != TOPKV_OK) return st;
  const CUtensorMap map = latent_map(&p), q_map = query_map(&p, N);
  return launched(launch_pdl(topkv_latent_kernel<N, BF16>, dim3(p.teams, units), dim3(kLatentThreads),
                             latent_smem(N, p.D, p.Dv).total, s, p, map, q_map), 1);
}
template <bool BF16>
int launch_latent(const AttendParams& p, int units, cudaStream_t s) {
  if (p.row_tile == 16) return launch_latent2<16, BF16>(p, units, s);
  if (p.row_tile == 32) return launch_latent2<32, BF16>(p, units, s);
  return launch_latent2<64, BF16>(p, units, s);
}
static_assert(latent_smem(64, kLatentMaxD, kLatentMaxDv).total <= kSmemBudget, "the largest layout fits a CTA");

// ---- page operators -------------------------------------------------------------------------------
int check_pages(const topkv_layout* lo, const topkv_batch* b, Resolved* rs) {
  int st = check_layout(lo, rs);
  if (st != TOPKV_OK) return st;
  st = check_tables_batch(lo, b);
  if (st != TOPKV_OK) return st;
  if (b->window_tokens != 0) return TOPKV_ERR_INVALID_ARG;
  if (lo->num_pool_pages > 0x7ffffff0ll) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  return TOPKV_OK;
}

int check_page_tables(const topkv_batch* b, const topkv_page_tables* t) {
  if (t == nullptr || t->struct_size != sizeof(topkv_page_tables) || t->reserved != 0) return TOPKV_ERR_INVALID_ARG;
  if (t->ref_counts == nullptr || t->ref_counts_out == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (b->num_requests > 0 && (t->seq_lens_out == nullptr || (b->max_pages_per_req > 0 && t->block_table_out == nullptr)))
    return TOPKV_ERR_INVALID_ARG;
  if (!mult4p(t->ref_counts) || !mult4p(t->ref_counts_out) || !mult4p(t->seq_lens_out) || !mult4p(t->block_table_out))
    return TOPKV_ERR_ALIGNMENT;
  return TOPKV_OK;
}

int64_t page_workspace_ints(const topkv_layout* lo, const topkv_batch* b, int64_t forks) {
  const int64_t N = lo->num_pool_pages, R = b->num_requests;
  const int64_t fork = 4 * forks + R + forks;     // records, claims, free pages
  const int64_t extend = R + 1 + N;               // prefix sums, free pages
  const int64_t compact = N + 2 * (N / 2 + 1) + 1;  // codes, holes, movers, number of moves
  return std::max(fork, std::max(extend, compact));
}

int check_page_workspace(const topkv_layout* lo, const topkv_batch* b, int64_t forks, const void* ws, int64_t bytes) {
  if (ws == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(ws)) return TOPKV_ERR_ALIGNMENT;
  return bytes < 4 * page_workspace_ints(lo, b, forks) ? TOPKV_ERR_CAPACITY : TOPKV_OK;
}

PageTables page_tables(const topkv_layout* lo, const topkv_batch* b, const topkv_page_tables* t) {
  return PageTables{t->block_table_out, t->seq_lens_out, t->ref_counts_out, b->num_requests, b->max_pages_per_req,
                    (int)lo->page_tokens, (int)lo->num_pool_pages};
}

// The copy that brings the tables into the out arrays, where the operator then works in place.
TablesCopyParams tables_copy(const topkv_layout* lo, const topkv_batch* b, const topkv_page_tables* t, int64_t* most) {
  TablesCopyParams p = {};
  p.src[0] = b->block_table;
  p.src[1] = b->seq_lens;
  p.src[2] = t->ref_counts;
  p.dst[0] = t->block_table_out;
  p.dst[1] = t->seq_lens_out;
  p.dst[2] = t->ref_counts_out;
  p.n[0] = (int64_t)b->num_requests * b->max_pages_per_req;
  p.n[1] = b->num_requests;
  p.n[2] = lo->num_pool_pages;
  *most = 0;
  for (int i = 0; i < 3; ++i) {
    if (p.src[i] == p.dst[i]) p.n[i] = 0;
    *most = std::max(*most, p.n[i]);
  }
  return p;
}
unsigned copy_ctas(int64_t most, int threads) { return (unsigned)std::min<int64_t>((most + threads - 1) / threads, 2 * 148); }
int copy_tables(const topkv_layout* lo, const topkv_batch* b, const topkv_page_tables* t, cudaStream_t s) {
  int64_t most;
  const TablesCopyParams p = tables_copy(lo, b, t, &most);
  if (most == 0) return TOPKV_OK;
  return launched(launch_pdl(topkv_tables_copy_kernel, dim3(copy_ctas(most, 256)), dim3(256), 0, s, p), 1);
}

// Small tables (128 KiB: what one CTA copies in the time of a launch, 2 us) are left to the operator's own
// kernel, larger ones copied by a launch before it.
int copy_or_pass(const topkv_layout* lo, const topkv_batch* b, const topkv_page_tables* t, TablesCopyParams* pass, cudaStream_t s) {
  int64_t most;
  *pass = tables_copy(lo, b, t, &most);
  if (pass->n[0] + pass->n[1] + pass->n[2] <= 32768) return TOPKV_OK;
  *pass = TablesCopyParams{};
  return copy_tables(lo, b, t, s);
}

// How the contents of a page are moved; *vec = bytes per access.
PageGeom page_geometry(int first_layer, int num_layers, void* pool, const topkv_layout* lo, const Resolved& rs, int* vec) {
  PageGeom g;
  g.pool = static_cast<uint8_t*>(pool) + (int64_t)first_layer * lo->pool_layer_stride;
  g.F = (int)lo->kv_factor;
  g.U = rs.U;
  g.P = (int)lo->page_tokens;
  g.layers = num_layers;
  g.S_layer = lo->pool_layer_stride;
  g.S_page = lo->pool_page_stride;
  g.S_kv = g.F > 1 ? lo->pool_kv_stride : 0;
  g.S_tok = g.P > 1 ? lo->pool_token_stride : rs.unit_bytes;
  g.S_unit = g.U > 1 ? lo->pool_head_stride : 0;
  g.unit_bytes = rs.unit_bytes;
  g.linear = g.S_tok == rs.unit_bytes;
  // equal parts of about 64 KiB (a page of 72 KiB stays whole: as 56 + 16 KiB its copy took 20 % longer)
  const int64_t page_bytes = g.P * g.F * rs.row_bytes;
  const int64_t parts = std::min<int64_t>(g.P, std::max<int64_t>(1, (page_bytes + kSpanTargetBytes / 2) / kSpanTargetBytes));
  g.tps = (int)((g.P + parts - 1) / parts);
  g.cpp = (g.P + g.tps - 1) / g.tps;
  const uintptr_t m = reinterpret_cast<uintptr_t>(g.pool) | (uintptr_t)g.S_layer | (uintptr_t)g.S_page |
                      (uintptr_t)g.S_kv | (uintptr_t)g.S_tok | (uintptr_t)g.S_unit | (uintptr_t)g.unit_bytes;
  *vec = (m & 31) == 0 ? 32 : 16;
  return g;
}

constexpr int kMoveCtas = 3 * 148;  // resident CTAs of the kernels that move pages

}  // namespace

extern "C" {

int64_t topkv_attend_workspace_bytes(const topkv_layout* layout, const topkv_batch* batch,
                                     const topkv_attention* attention) {
  AttendPlan plan;
  const int st = check_attention(layout, batch, attention, &plan);
  return st != TOPKV_OK ? st : plan.bytes;
}

int topkv_attend_layer(int layer, const void* pool, const topkv_layout* layout, const topkv_batch* batch,
                       const topkv_attention* attention, const void* d_q, void* d_out, void* d_workspace,
                       int64_t workspace_bytes, topkv_stream_t stream) {
  AttendPlan plan;
  int st = check_attention(layout, batch, attention, &plan);
  if (st != TOPKV_OK) return st;
  if (layer < 0 || (uint32_t)layer >= layout->num_layers) return TOPKV_ERR_LAYER_RANGE;
  if (pool == nullptr || d_q == nullptr || d_out == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(pool) || !mult16p(d_q) || !mult16p(d_out)) return TOPKV_ERR_ALIGNMENT;
  if (plan.bytes > 0) {
    if (d_workspace == nullptr) return TOPKV_ERR_INVALID_ARG;
    if (!mult16p(d_workspace)) return TOPKV_ERR_ALIGNMENT;
    if (workspace_bytes < plan.bytes) return TOPKV_ERR_CAPACITY;
  }
  if (batch->num_requests == 0) return TOPKV_OK;
  AttendParams p = {};
  p.pool = static_cast<const uint8_t*>(pool) + (int64_t)layer * layout->pool_layer_stride;
  p.bt = batch->block_table;
  p.sl = batch->seq_lens;
  p.q = static_cast<const uint8_t*>(d_q);
  p.out = static_cast<uint8_t*>(d_out);
  p.lse = attention->lse;
  p.S_page = layout->pool_page_stride;
  p.S_kv = layout->kv_factor > 1 ? layout->pool_kv_stride : 0;
  p.S_tok = layout->page_tokens > 1 ? layout->pool_token_stride : 0;
  p.S_head = layout->num_kv_heads > 1 ? layout->pool_head_stride : 0;
  p.q_req = attention->q_request_stride;
  p.q_head = attention->q_head_stride;
  p.o_req = attention->out_request_stride;
  p.o_head = attention->out_head_stride;
  p.num_pages = layout->num_pool_pages;
  p.R = batch->num_requests;
  p.maxp = batch->max_pages_per_req;
  p.P = (int)layout->page_tokens;
  p.page_shift = (p.P & (p.P - 1)) == 0 ? __builtin_ctz((unsigned)p.P) : -1;
  p.H = (int)layout->num_kv_heads;
  p.G = (int)(attention->num_q_heads / layout->num_kv_heads);
  p.gtiles = plan.units / p.H;
  p.D = (int)layout->head_dim;
  p.Dv = plan.dv;
  p.window = batch->window_tokens;
  p.sinks = (int)attention->sink_tokens;
  p.qk_scale = attention->scale * attention->k_scale * kLog2e;
  p.v_scale = attention->v_scale;
  p.io_bf16 = attention->io_type == TOPKV_TYPE_BF16;
  p.teams = plan.teams;
  p.uncut = plan.uncut;
  p.narrow = plan.narrow;
  // Beginning with a request and writing its result takes a latent CTA, alone on its SM, about as long as
  // three tiles (32 requests of 1,024 to 8,192 tokens, 128 heads: 77.6 us without, 75.2 with); of
  // grouped-head CTAs others on the SM use that time (1 tile more made no difference)
  p.start_cost = layout->kv_factor == 1 ? 3 : 0;
  p.late_wait = (batch->flags & TOPKV_FLAG_TABLES_SETTLED) ? 1 : 0;
  p.rows = plan.rows;
  p.row_tile = plan.row_tile;
  if (!plan.uncut) {
    uint8_t* w = static_cast<uint8_t*>(d_workspace);
    const int64_t slots = 2ll * plan.teams * plan.units * plan.rows;
    p.joins = reinterpret_cast<int4*>(w);
    p.by_request = plan.joins == p.R;
    w += (int64_t)plan.joins * 16;
    p.ml = reinterpret_cast<float2*>(w);
    p.part = reinterpret_cast<float*>(w + slots * 8);
  }
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (layout->kv_factor == 1)
    st = p.io_bf16 ? launch_latent<true>(p, plan.units, s) : launch_latent<false>(p, plan.units, s);
  else if (attention->cache_type == TOPKV_TYPE_BF16)
    st = launch_attend_dim<kBf16>(p, plan.units, s);
  else if (attention->cache_type == TOPKV_TYPE_FP16)
    st = launch_attend_dim<kFp16>(p, plan.units, s);
  else
    st = launch_attend_dim<kE4m3>(p, plan.units, s);
  if (st != TOPKV_OK || plan.uncut || plan.teams < 2) return st;
  // about eight CTAs per SM for the requests that can be cut
  const int64_t cuts = (int64_t)plan.joins * plan.units;
  const unsigned z = (unsigned)std::max((plan.rows + kJoinRows - 1) / kJoinRows, (int)std::min<int64_t>(plan.rows, 8 * 148 / cuts));
  return launched(launch_pdl(topkv_attend_join_kernel, dim3(plan.joins, plan.units, z), dim3(kJoinThreads), 0, s, p), 1);
}

int64_t topkv_page_workspace_bytes(const topkv_layout* layout, const topkv_batch* batch, int32_t num_forks) {
  Resolved rs;
  const int st = check_pages(layout, batch, &rs);
  if (st != TOPKV_OK) return st;
  if (num_forks < 0) return TOPKV_ERR_INVALID_ARG;
  return 4 * page_workspace_ints(layout, batch, num_forks);
}

int topkv_extend_requests(const topkv_layout* layout, const topkv_batch* batch, const topkv_page_tables* tables,
                          const int32_t* d_new_tokens, void* d_workspace, int64_t workspace_bytes,
                          topkv_stream_t stream) {
  Resolved rs;
  int st = check_pages(layout, batch, &rs);
  if (st == TOPKV_OK) st = check_page_tables(batch, tables);
  if (st != TOPKV_OK) return st;
  if (batch->num_requests == 0 || batch->max_pages_per_req == 0) return TOPKV_OK;
  if (d_new_tokens == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult4p(d_new_tokens)) return TOPKV_ERR_ALIGNMENT;
  st = check_page_workspace(layout, batch, 0, d_workspace, workspace_bytes);
  if (st != TOPKV_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  ExtendParams p;
  st = copy_or_pass(layout, batch, tables, &p.copy, s);
  if (st != TOPKV_OK) return st;
  p.t = page_tables(layout, batch, tables);
  p.add = d_new_tokens;
  p.prefix = static_cast<int32_t*>(d_workspace);
  p.list = p.prefix + p.t.R + 1;
  return launched(launch_pdl(topkv_extend_kernel, dim3(1), dim3(kPlanThreads), 0, s, p), 1);
}

int topkv_fork_requests(void* pool, const topkv_layout* layout, const topkv_batch* batch,
                        const topkv_page_tables* tables, const int32_t* d_parents, const int32_t* d_children,
                        int32_t num_forks, void* d_workspace, int64_t workspace_bytes, topkv_stream_t stream) {
  Resolved rs;
  int st = check_pages(layout, batch, &rs);
  if (st == TOPKV_OK) st = check_page_tables(batch, tables);
  if (st != TOPKV_OK) return st;
  if (pool == nullptr || num_forks < 0) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(pool)) return TOPKV_ERR_ALIGNMENT;
  if (batch->num_requests == 0 || batch->max_pages_per_req == 0) return TOPKV_OK;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (num_forks > 0) {
    if (d_parents == nullptr || d_children == nullptr) return TOPKV_ERR_INVALID_ARG;
    if (!mult4p(d_parents) || !mult4p(d_children)) return TOPKV_ERR_ALIGNMENT;
    st = check_page_workspace(layout, batch, num_forks, d_workspace, workspace_bytes);
    if (st != TOPKV_OK) return st;
  }
  int vec;
  ForkParams p;
  p.g = page_geometry(0, (int)layout->num_layers, pool, layout, rs, &vec);
  if ((int64_t)p.g.layers * p.g.cpp > 65534) {  // one CTA per page then
    p.g.tps = p.g.P;
    p.g.cpp = 1;
    if (p.g.layers > 65534) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  }
  if (num_forks == 0) return copy_tables(layout, batch, tables, s);
  int64_t most;
  p.copy = tables_copy(layout, batch, tables, &most);
  p.t = page_tables(layout, batch, tables);
  p.parents = d_parents;
  p.children = d_children;
  p.n = num_forks;
  p.rec = static_cast<ForkRecord*>(d_workspace);
  p.claim = reinterpret_cast<int32_t*>(p.rec + num_forks);
  p.list = p.claim + p.t.R;
  st = launched(launch_pdl(topkv_fork_plan_kernel, dim3(1 + copy_ctas(most, kPlanThreads)), dim3(kPlanThreads), 0, s, p), 1);
  if (st != TOPKV_OK) return st;
  const dim3 grid((unsigned)num_forks, (unsigned)(1 + p.g.layers * p.g.cpp));
  return launched(vec == 32 ? launch_pdl(topkv_fork_apply_kernel<32>, grid, dim3(kMoveThreads), 0, s, p)
                            : launch_pdl(topkv_fork_apply_kernel<16>, grid, dim3(kMoveThreads), 0, s, p), 1);
}

int topkv_free_requests(const topkv_layout* layout, const topkv_batch* batch, const topkv_page_tables* tables,
                        const int32_t* d_rows, int32_t num_rows, topkv_stream_t stream) {
  Resolved rs;
  int st = check_pages(layout, batch, &rs);
  if (st == TOPKV_OK) st = check_page_tables(batch, tables);
  if (st != TOPKV_OK) return st;
  if (num_rows < 0 || (num_rows > 0 && d_rows == nullptr)) return TOPKV_ERR_INVALID_ARG;
  if (!mult4p(d_rows)) return TOPKV_ERR_ALIGNMENT;
  if (batch->num_requests == 0 || batch->max_pages_per_req == 0) return TOPKV_OK;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (num_rows == 0) return copy_tables(layout, batch, tables, s);
  FreeParams p;
  st = copy_or_pass(layout, batch, tables, &p.copy, s);
  if (st != TOPKV_OK) return st;
  p.t = page_tables(layout, batch, tables);
  p.rows = d_rows;
  p.n = num_rows;
  // one CTA if it has the tables to copy or little to do, else 32 rows each
  const bool passed = p.copy.n[0] + p.copy.n[1] + p.copy.n[2] > 0;
  const unsigned ctas = passed ? 1 : (unsigned)std::min<int64_t>(((int64_t)num_rows + 31) / 32, 2 * 148);
  return launched(launch_pdl(topkv_free_kernel, dim3(ctas), dim3(kPlanThreads), 0, s, p), 1);
}

int topkv_compact_pages(void* pool, const topkv_layout* layout, const topkv_batch* batch,
                        const topkv_page_tables* tables, int32_t* d_num_used, int32_t* d_page_map,
                        void* d_workspace, int64_t workspace_bytes, topkv_stream_t stream) {
  Resolved rs;
  int st = check_pages(layout, batch, &rs);
  if (st == TOPKV_OK) st = check_page_tables(batch, tables);
  if (st != TOPKV_OK) return st;
  if (pool == nullptr || d_num_used == nullptr || d_page_map == nullptr) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(pool) || !mult4p(d_num_used) || !mult4p(d_page_map)) return TOPKV_ERR_ALIGNMENT;
  st = check_page_workspace(layout, batch, 0, d_workspace, workspace_bytes);
  if (st != TOPKV_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  int vec;
  const PageGeom g = page_geometry(0, (int)layout->num_layers, pool, layout, rs, &vec);
  CompactParams p;
  int64_t most;
  p.copy = tables_copy(layout, batch, tables, &most);
  p.t = page_tables(layout, batch, tables);
  const int64_t N = p.t.num_pages;
  p.code = static_cast<int32_t*>(d_workspace);
  p.holes = p.code + N;
  p.movers = p.holes + N / 2 + 1;
  p.moves = p.movers + N / 2 + 1;
  p.num_used = d_num_used;
  p.map = d_page_map;
  const int block = kPlanThreads * kPlanPages;
  p.blocks = (int)((N + block - 1) / block);
  st = launched(launch_pdl(topkv_compact_plan_kernel, dim3(p.blocks + copy_ctas(most, kPlanThreads)), dim3(kPlanThreads), 0, s, p), 1);
  if (st != TOPKV_OK) return st;
  return launched(vec == 32 ? launch_pdl(topkv_compact_apply_kernel<32>, dim3(kMoveCtas), dim3(kMoveThreads), 0, s, p, g)
                            : launch_pdl(topkv_compact_apply_kernel<16>, dim3(kMoveCtas), dim3(kMoveThreads), 0, s, p, g), 1);
}

int topkv_copy_pages(int first_layer, int num_layers, void* pool, const topkv_layout* layout,
                     const int32_t* d_src_pages, const int32_t* d_dst_pages, int32_t num_pages, topkv_stream_t stream) {
  Resolved rs;
  const int st = check_layout(layout, &rs);
  if (st != TOPKV_OK) return st;
  if (layout->num_pool_pages > 0x7ffffff0ll || layout->page_tokens > 0x7fffffffu) return TOPKV_ERR_UNSUPPORTED_LAYOUT;
  if (first_layer < 0 || num_layers < 0 || (int64_t)first_layer + num_layers > (int64_t)layout->num_layers)
    return TOPKV_ERR_LAYER_RANGE;
  if (pool == nullptr || num_pages < 0) return TOPKV_ERR_INVALID_ARG;
  if (num_pages > 0 && (d_src_pages == nullptr || d_dst_pages == nullptr)) return TOPKV_ERR_INVALID_ARG;
  if (!mult16p(pool) || !mult4p(d_src_pages) || !mult4p(d_dst_pages)) return TOPKV_ERR_ALIGNMENT;
  if (num_pages == 0 || num_layers == 0) return TOPKV_OK;
  int vec;
  MoveParams p;
  p.g = page_geometry(first_layer, num_layers, pool, layout, rs, &vec);
  p.src = d_src_pages;
  p.dst = d_dst_pages;
  p.n = num_pages;
  p.num_pages = (int)layout->num_pool_pages;
  const int64_t items = p.n * p.g.layers * p.g.cpp;
  const dim3 grid((unsigned)std::min<int64_t>(items, 0x7fffffffll));  // one CTA per part
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return launched(vec == 32 ? launch_pdl(topkv_page_move_kernel<32>, grid, dim3(kMoveThreads), 0, s, p)
                            : launch_pdl(topkv_page_move_kernel<16>, grid, dim3(kMoveThreads), 0, s, p), 1);
}

}  // extern "C"
