// C-ABI layer of libpkv: attention of prompts, and of decode steps over pools with a scale for each block and KV head.
#include "pkv_host.h"

using namespace pkv;

namespace {

constexpr int64_t kMaxTokens = ((int64_t)1 << 24) - 1;

bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
bool good_scale(float x) { return x > 0.f && x < __builtin_inff(); }

bool meet(const void* p, uint64_t bytes, const void* q, uint64_t more) {
  const uint64_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
  return x < y + more && y < x + bytes;
}
uint64_t pool_bytes(const pkv_attn_shape* sh, int kv_fp8) {
  return (uint64_t)sh->num_pool_blocks * sh->num_kv_heads * sh->block_size * sh->head_dim * (kv_fp8 ? 1 : 2);
}
uint64_t scales_bytes(const pkv_attn_shape* sh) { return (uint64_t)sh->num_pool_blocks * scale_row_bytes(sh->num_kv_heads); }

int check_prompt(const pkv_attn_shape* shape, int64_t tokens, Geometry* g, PromptPlan* plan, size_t* workspace) {
  const int rc = check_shape(shape, g);
  if (rc != PKV_OK) return rc;
  if (tokens < 0 || tokens > kMaxTokens || g->max_ctx > kMaxTiledContext) return PKV_ERR_SHAPE;
  *workspace = 0;
  if (tokens == 0 || shape->num_seqs == 0) return PKV_OK;
  *plan = prompt_plan(tokens, shape->num_seqs, shape->num_kv_heads, g->G, shape->head_dim, g->max_ctx);
  // a launch has fewer than 2^32 lanes in a dimension
  if (plan->slots * shape->num_kv_heads * plan->threads > UINT32_MAX) return PKV_ERR_SHAPE;
  if (plan->pieces > 1) *workspace = (size_t)plan->pieces * tokens * shape->num_q_heads * (shape->head_dim + 2) * sizeof(float);
  return PKV_OK;
}

int attend_prompt(const void* q, const void* k_pool, const void* v_pool, const uint8_t* k_scales, const uint8_t* v_scales,
                  const int32_t* block_tables, const int32_t* context_lens, const int32_t* token_starts, int64_t tokens, float scale, int kv_fp8,
                  float k_scale, float v_scale, void* out, const pkv_attn_shape* shape, void* workspace, size_t workspace_bytes_given,
                  void* stream) {
  Geometry g;
  PromptPlan plan;
  size_t need;
  const int rc = check_prompt(shape, tokens, &g, &plan, &need);
  if (rc != PKV_OK) return rc;
  if (!good_scale(k_scale) || !good_scale(v_scale)) return PKV_ERR_SHAPE;
  if (!token_starts && tokens != shape->num_seqs) return PKV_ERR_SHAPE;
  if (tokens == 0 || shape->num_seqs == 0) return PKV_OK;
  if (!q || !k_pool || !v_pool || !block_tables || !context_lens || !out) return PKV_ERR_NULL;
  if (kv_fp8 == kBlkPools && (!k_scales || !v_scales)) return PKV_ERR_NULL;
  if (misaligned16(q) || misaligned16(k_pool) || misaligned16(v_pool) || misaligned16(out) || misaligned16(k_scales) || misaligned16(v_scales) ||
      misaligned4(block_tables) || misaligned4(context_lens) || misaligned4(token_starts))
    return PKV_ERR_ALIGN;
  if (need) {
    if (!workspace || workspace_bytes_given < need) return PKV_ERR_WORKSPACE;
    if (misaligned16(workspace)) return PKV_ERR_ALIGN;
  }
  // rows are written while others are read
  const uint64_t rows = (uint64_t)tokens * shape->num_q_heads * shape->head_dim * 2, pool = pool_bytes(shape, kv_fp8);
  if ((out != q && meet(out, rows, q, rows)) || meet(out, rows, k_pool, pool) || meet(out, rows, v_pool, pool) ||
      (kv_fp8 == kBlkPools && (meet(out, rows, k_scales, scales_bytes(shape)) || meet(out, rows, v_scales, scales_bytes(shape)))) ||
      meet(out, rows, block_tables, (uint64_t)shape->num_seqs * shape->max_blocks_per_seq * 4) ||
      meet(out, rows, context_lens, (uint64_t)shape->num_seqs * 4) ||
      (token_starts && meet(out, rows, token_starts, ((uint64_t)shape->num_seqs + 1) * 4)))
    return PKV_ERR_SHAPE;
  PromptLaunch a;
  a.q = static_cast<const uint16_t*>(q);
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.k_scales = k_scales;
  a.v_scales = v_scales;
  a.block_tables = block_tables;
  a.context_lens = context_lens;
  a.token_starts = token_starts;
  a.out = static_cast<uint16_t*>(out);
  a.parts = static_cast<float*>(workspace);
  a.stats = a.parts + (need ? (int64_t)plan.pieces * tokens * shape->num_q_heads * shape->head_dim : 0);
  a.id_faults = g_id_faults;
  a.scale_log2e = scale * k_scale * 1.4426950408889634f;
  a.out_scale = v_scale;
  a.kv_fp8 = kv_fp8;
  a.T = (int)tokens;
  a.S = shape->num_seqs;
  a.Hq = shape->num_q_heads;
  a.Hkv = shape->num_kv_heads;
  a.G = g.G;
  a.D = shape->head_dim;
  a.MAXB = shape->max_blocks_per_seq;
  a.log_block = __builtin_ctz(shape->block_size);
  a.max_ctx = g.max_ctx;
  a.NB = (int)shape->num_pool_blocks;
  a.piece = plan.piece;
  a.pieces = plan.pieces;
  a.ordered = plan.ordered && token_starts;
  return launch_status(launch_prompt(a, plan, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int pkv_fp8blk_scale_bytes(const pkv_attn_shape* shape, size_t* out_bytes) {
  if (!out_bytes) return PKV_ERR_NULL;
  Geometry g;
  const int rc = check_shape(shape, &g);
  if (rc != PKV_OK) return rc;
  *out_bytes = scale_row_bytes(shape->num_kv_heads);
  return PKV_OK;
}

int paged_decode_attn_fp8blk(const void* q, const void* k_pool, const void* v_pool, const uint8_t* k_scales, const uint8_t* v_scales,
                             const int32_t* block_tables, const int32_t* context_lens, float scale, void* out, const pkv_attn_shape* shape,
                             void* workspace, size_t workspace_bytes_given, void* stream) {
  AttnLaunch a;
  bool empty = false;
  int rc = prepare_attn(block_tables, context_lens, scale, kBlkPools, nullptr, shape, workspace, workspace_bytes_given, &a, &empty);
  if (rc != PKV_OK || empty) return rc;
  rc = check_layer_pointers(q, k_pool, v_pool, out);
  if (rc != PKV_OK) return rc;
  if (!k_scales || !v_scales) return PKV_ERR_NULL;
  if (misaligned16(k_scales) || misaligned16(v_scales)) return PKV_ERR_ALIGN;
  if (meet(out, row_bytes(a), k_scales, scales_bytes(shape)) || meet(out, row_bytes(a), v_scales, scales_bytes(shape))) return PKV_ERR_SHAPE;
  return launch_layer(a, layer_of(q, k_pool, v_pool, out), static_cast<hipStream_t>(stream),
                      [=](const AttnLaunch& launch, const AttnLayers*, hipStream_t st) { return launch_attn_blk(launch, k_scales, v_scales, st); });
}

int pkv_prompt_workspace_bytes(const pkv_attn_shape* shape, int64_t num_tokens, size_t* out_bytes) {
  if (!out_bytes) return PKV_ERR_NULL;
  Geometry g;
  PromptPlan plan;
  return check_prompt(shape, num_tokens, &g, &plan, out_bytes);
}

int paged_prompt_attn(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables, const int32_t* context_lens,
                      const int32_t* token_starts, int64_t num_tokens, float scale, void* out, const pkv_attn_shape* shape, void* workspace,
                      size_t workspace_bytes_given, void* stream) {
  return attend_prompt(q, k_pool, v_pool, nullptr, nullptr, block_tables, context_lens, token_starts, num_tokens, scale, 0, 1.f, 1.f, out, shape,
                       workspace, workspace_bytes_given, stream);
}

int paged_prompt_attn_fp8kv(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables, const int32_t* context_lens,
                            const int32_t* token_starts, int64_t num_tokens, float scale, float k_scale, float v_scale, void* out,
                            const pkv_attn_shape* shape, void* workspace, size_t workspace_bytes_given, void* stream) {
  return attend_prompt(q, k_pool, v_pool, nullptr, nullptr, block_tables, context_lens, token_starts, num_tokens, scale, 1, k_scale, v_scale, out,
                       shape, workspace, workspace_bytes_given, stream);
}

int paged_prompt_attn_fp8blk(const void* q, const void* k_pool, const void* v_pool, const uint8_t* k_scales, const uint8_t* v_scales,
                             const int32_t* block_tables, const int32_t* context_lens, const int32_t* token_starts, int64_t num_tokens,
                             float scale, void* out, const pkv_attn_shape* shape, void* workspace, size_t workspace_bytes_given, void* stream) {
  return attend_prompt(q, k_pool, v_pool, k_scales, v_scales, block_tables, context_lens, token_starts, num_tokens, scale, kBlkPools, 1.f, 1.f, out,
                       shape, workspace, workspace_bytes_given, stream);
}

}  // extern "C"
