// C-ABI layer of libpkv: new tokens normalised, rotated and appended, and the append to pools held in 4 bits.
#include "pkv_host.h"

using namespace pkv;

namespace {

bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

// Rows of `tokens` tokens, `width` elements each and `stride` apart, as a range of addresses.
struct Range {
  uint64_t from, to;
};
Range rows_at(const void* p, int64_t tokens, int64_t stride, int64_t width) {
  const uint64_t from = reinterpret_cast<uintptr_t>(p);
  return {from, from + ((uint64_t)(tokens - 1) * (uint64_t)stride + (uint64_t)width) * 2};
}
bool meet(const Range& x, const Range& y) { return x.from < y.to && y.from < x.to; }

// Quotients that are not beyond the format's range nor round to zero in it, and their remainders, are normal numbers.
float inverse_of(float scale) { return scale >= 0x1p-60f && scale <= 0x1p60f ? 1.f / scale : 0.f; }

constexpr int64_t kMaxTokens = ((int64_t)1 << 24) - 1;   // a workgroup of 256 lanes for each in one dimension of a launch
constexpr int64_t kMaxStride = (int64_t)1 << 31;

int rope_append(const void* q, const void* k, const void* v, const void* q_norm, const void* k_norm, const float* cos_sin, void* q_out,
                void* k_pool, void* v_pool, const int32_t* block_tables, const int32_t* context_lens, const int32_t* token_starts, int kv_fp8,
                float k_scale, float v_scale, const pkv_rope_shape* rope, const pkv_attn_shape* shape, void* stream) {
  if (!rope) return PKV_ERR_NULL;
  Geometry g;
  const int rc = check_shape(shape, &g);
  if (rc != PKV_OK) return rc;
  if (!(k_scale > 0.f) || !(v_scale > 0.f) || !(k_scale < __builtin_inff()) || !(v_scale < __builtin_inff())) return PKV_ERR_SHAPE;
  const int D = shape->head_dim, R = rope->rotary_dim;
  const int64_t T = rope->num_tokens, q_row = (int64_t)shape->num_q_heads * D, kv_row = (int64_t)shape->num_kv_heads * D;
  if (T < 0 || T > kMaxTokens) return PKV_ERR_SHAPE;
  if (R < 0 || R > D || R % 16 != 0) return PKV_ERR_SHAPE;
  if (rope->interleaved != 0 && rope->interleaved != 1) return PKV_ERR_SHAPE;
  if (!(rope->norm_eps >= 0.f) || !(rope->norm_eps < __builtin_inff())) return PKV_ERR_SHAPE;
  if (R > 0 && rope->num_positions < g.max_ctx) return PKV_ERR_SHAPE;
  const int64_t strides[3] = {rope->q_stride ? rope->q_stride : q_row, rope->k_stride ? rope->k_stride : kv_row,
                              rope->v_stride ? rope->v_stride : kv_row};
  if (strides[0] < q_row || strides[1] < kv_row || strides[2] < kv_row) return PKV_ERR_SHAPE;
  for (const int64_t s : strides) {
    if (s > kMaxStride) return PKV_ERR_SHAPE;
    if (s % 8 != 0) return PKV_ERR_ALIGN;
  }
  if (!token_starts && T != shape->num_seqs) return PKV_ERR_SHAPE;
  if (T == 0 || shape->num_seqs == 0) return PKV_OK;
  if (!q || !k || !v || !q_out || !k_pool || !v_pool || !block_tables || !context_lens || (R > 0 && !cos_sin)) return PKV_ERR_NULL;
  if (misaligned16(q) || misaligned16(k) || misaligned16(v) || misaligned16(q_out) || misaligned16(k_pool) || misaligned16(v_pool) ||
      misaligned16(q_norm) || misaligned16(k_norm) || misaligned16(cos_sin) || misaligned4(block_tables) || misaligned4(context_lens) ||
      misaligned4(token_starts))
    return PKV_ERR_ALIGN;
  // a row of q is read by the lanes that write it, so it may be written in place; no other row may be written before it is read
  const Range out = rows_at(q_out, T, q_row, q_row);
  const bool in_place = q_out == q && strides[0] == q_row;
  if ((!in_place && meet(out, rows_at(q, T, strides[0], q_row))) || meet(out, rows_at(k, T, strides[1], kv_row)) ||
      meet(out, rows_at(v, T, strides[2], kv_row)))
    return PKV_ERR_SHAPE;
  RopeLaunch a;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q_stride = strides[0];
  a.k_stride = strides[1];
  a.v_stride = strides[2];
  a.q_norm = static_cast<const uint16_t*>(q_norm);
  a.k_norm = static_cast<const uint16_t*>(k_norm);
  a.cos_sin = cos_sin;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.block_tables = block_tables;
  a.context_lens = context_lens;
  a.token_starts = token_starts;
  a.id_faults = g_id_faults;
  a.eps = rope->norm_eps;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.k_inverse = inverse_of(k_scale);
  a.v_inverse = inverse_of(v_scale);
  a.kv_fp8 = kv_fp8;
  a.T = (int)T;
  a.S = shape->num_seqs;
  a.Hq = shape->num_q_heads;
  a.Hkv = shape->num_kv_heads;
  a.D = D;
  a.R = R;
  a.interleaved = rope->interleaved;
  a.MAXB = shape->max_blocks_per_seq;
  a.log_block = __builtin_ctz(shape->block_size);
  a.max_ctx = g.max_ctx;
  a.NB = (int)shape->num_pool_blocks;
  return launch_status(launch_kv_rope(a, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int kv_rope_append(const void* q, const void* k, const void* v, const void* q_norm, const void* k_norm, const float* cos_sin, void* q_out,
                   void* k_pool, void* v_pool, const int32_t* block_tables, const int32_t* context_lens, const int32_t* token_starts,
                   const pkv_rope_shape* rope, const pkv_attn_shape* shape, void* stream) {
  return rope_append(q, k, v, q_norm, k_norm, cos_sin, q_out, k_pool, v_pool, block_tables, context_lens, token_starts, 0, 1.f, 1.f, rope,
                     shape, stream);
}

int kv_rope_append_fp8(const void* q, const void* k, const void* v, const void* q_norm, const void* k_norm, const float* cos_sin, void* q_out,
                       void* k_pool, void* v_pool, const int32_t* block_tables, const int32_t* context_lens, const int32_t* token_starts,
                       float k_scale, float v_scale, const pkv_rope_shape* rope, const pkv_attn_shape* shape, void* stream) {
  return rope_append(q, k, v, q_norm, k_norm, cos_sin, q_out, k_pool, v_pool, block_tables, context_lens, token_starts, 1, k_scale, v_scale,
                     rope, shape, stream);
}

int kv_rope_append_fp4(const void* q, const void* k, const void* v, const void* q_norm, const void* k_norm, const float* cos_sin, void* q_out,
                       void* k_pool, void* v_pool, const int32_t* block_tables, const int32_t* context_lens, const int32_t* token_starts,
                       const pkv_rope_shape* rope, const pkv_attn_shape* shape, void* stream) {
  return rope_append(q, k, v, q_norm, k_norm, cos_sin, q_out, k_pool, v_pool, block_tables, context_lens, token_starts, kFp4Pools, 1.f, 1.f,
                     rope, shape, stream);
}

int kv_append_fp4(const void* k_new, const void* v_new, void* k_pool, void* v_pool, const int32_t* block_tables, const int32_t* context_lens,
                  const pkv_attn_shape* shape, void* stream) {
  Geometry g;
  const int rc = check_shape(shape, &g);
  if (rc != PKV_OK) return rc;
  if (shape->num_seqs == 0) return PKV_OK;
  if (!k_new || !v_new || !k_pool || !v_pool || !block_tables || !context_lens) return PKV_ERR_NULL;
  if (misaligned16(k_new) || misaligned16(v_new) || misaligned16(k_pool) || misaligned16(v_pool) || misaligned4(block_tables) ||
      misaligned4(context_lens))
    return PKV_ERR_ALIGN;
  RopeLaunch a = {};   // no queries, no weights, nothing rotated
  a.k = static_cast<const uint16_t*>(k_new);
  a.v = static_cast<const uint16_t*>(v_new);
  a.k_stride = a.v_stride = (int64_t)shape->num_kv_heads * shape->head_dim;
  a.k_pool = k_pool;
  a.v_pool = v_pool;
  a.block_tables = block_tables;
  a.context_lens = context_lens;
  a.id_faults = g_id_faults;
  a.kv_fp8 = kFp4Pools;
  a.T = a.S = shape->num_seqs;
  a.Hkv = shape->num_kv_heads;
  a.D = shape->head_dim;
  a.MAXB = shape->max_blocks_per_seq;
  a.log_block = __builtin_ctz(shape->block_size);
  a.max_ctx = g.max_ctx;
  a.NB = (int)shape->num_pool_blocks;
  return launch_status(launch_kv_rope(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
