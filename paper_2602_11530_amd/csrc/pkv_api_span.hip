// C-ABI layer of libpkv: attention of requests that see part of their context, and over pools held in 4 bits.
#include "pkv_host.h"

using namespace pkv;

namespace {

// One layer's attention; window and sinks nullptr: over all of a request's context.
int attend(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables, const int32_t* context_lens, float scale,
           int kv_fp8, float k_scale, float v_scale, const int32_t* window, const int32_t* sinks, void* out, const pkv_attn_shape* shape,
           void* workspace, size_t workspace_bytes_given, void* stream) {
  Geometry g;
  int rc = check_shape(shape, &g);
  if (rc != PKV_OK) return rc;
  if (!(k_scale > 0.f) || !(v_scale > 0.f) || !(k_scale < __builtin_inff()) || !(v_scale < __builtin_inff())) return PKV_ERR_SHAPE;
  Span given = {0, 0};
  if (window) {
    if (*window < 0 || *sinks < 0) return PKV_ERR_SHAPE;
    given = {*window, *sinks};
  }
  const Span span = {given.window < g.max_ctx ? given.window : g.max_ctx, given.sinks < g.max_ctx ? given.sinks : g.max_ctx};   // no request is longer
  const Span* seen = window ? &span : nullptr;
  AttnLaunch a;
  bool empty = false;
  rc = prepare_attn(block_tables, context_lens, scale, kv_fp8, window ? &given : nullptr, shape, workspace, workspace_bytes_given, &a, &empty);
  if (rc != PKV_OK || empty) return rc;
  rc = check_layer_pointers(q, k_pool, v_pool, out);
  if (rc != PKV_OK) return rc;
  a.scale_log2e = scale * k_scale * 1.4426950408889634f;
  a.out_scale = v_scale;
  return launch_layer(a, layer_of(q, k_pool, v_pool, out), static_cast<hipStream_t>(stream),
                      [seen](const AttnLaunch& launch, const AttnLayers*, hipStream_t st) { return launch_attn_span(launch, seen, st); });
}

}  // namespace

extern "C" {

int pkv_fp4_block_bytes(const pkv_attn_shape* shape, size_t* out_bytes) {
  if (!out_bytes) return PKV_ERR_NULL;
  Geometry g;
  const int rc = check_shape(shape, &g);
  if (rc != PKV_OK) return rc;
  *out_bytes = (size_t)shape->num_kv_heads * (shape->block_size / kBlockTokens) * fp4_tile_bytes(shape->head_dim);
  return PKV_OK;
}

int paged_decode_attn_window(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables,
                             const int32_t* context_lens, float scale, int32_t window, int32_t sinks, void* out,
                             const pkv_attn_shape* shape, void* workspace, size_t workspace_bytes_given, void* stream) {
  return attend(q, k_pool, v_pool, block_tables, context_lens, scale, 0, 1.f, 1.f, &window, &sinks, out, shape, workspace,
                workspace_bytes_given, stream);
}

int paged_decode_attn_window_fp8kv(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables,
                                   const int32_t* context_lens, float scale, float k_scale, float v_scale, int32_t window,
                                   int32_t sinks, void* out, const pkv_attn_shape* shape, void* workspace,
                                   size_t workspace_bytes_given, void* stream) {
  return attend(q, k_pool, v_pool, block_tables, context_lens, scale, 1, k_scale, v_scale, &window, &sinks, out, shape, workspace,
                workspace_bytes_given, stream);
}

int paged_decode_attn_window_fp4kv(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables,
                                   const int32_t* context_lens, float scale, int32_t window, int32_t sinks, void* out,
                                   const pkv_attn_shape* shape, void* workspace, size_t workspace_bytes_given, void* stream) {
  return attend(q, k_pool, v_pool, block_tables, context_lens, scale, kFp4Pools, 1.f, 1.f, &window, &sinks, out, shape, workspace,
                workspace_bytes_given, stream);
}

int paged_decode_attn_fp4kv(const void* q, const void* k_pool, const void* v_pool, const int32_t* block_tables,
                            const int32_t* context_lens, float scale, void* out, const pkv_attn_shape* shape, void* workspace,
                            size_t workspace_bytes_given, void* stream) {
  return attend(q, k_pool, v_pool, block_tables, context_lens, scale, kFp4Pools, 1.f, 1.f, nullptr, nullptr, out, shape, workspace,
                workspace_bytes_given, stream);
}

}  // extern "C"
