// What the entry points share: argument checks (all of them before any launch, so they can be exercised without a GPU), launch geometry,
// statuses.
#pragma once

#include "../../include/pkv.h"

#include "fp4.h"
#include "pkv_kernels.h"

namespace pkv {

inline thread_local hipError_t g_last_launch_error = hipSuccess;
inline thread_local int32_t* g_id_faults = nullptr;   // see pkv_set_id_fault_counter

inline bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Library's partition choice when the caller leaves it open.  With the stream
// decomposition a partition only bounds how many tokens one partial result may
// stand for before it is folded into its segment's record, so the largest value
// is the cheapest.
constexpr int kDefaultPartition = kMaxPartition;

// Query heads.  Keeps every size product far inside 64 bits.
constexpr int kMaxHeads = 16384;

struct Geometry {
  int G, P, max_ctx;
  int64_t slots;   // records that the workspace has room for
};

// A record for every (wavefront, request, KV head) that meet, at most, as wavefronts' own records would need.  Workgroups leave far
// fewer; the rest takes those of further layers of a launch, or rows (launch_layer).
inline int64_t record_slots(int S, int Hkv) { return (int64_t)Hkv * S + kStreamWaves; }

// Longest context of the calls for prompts and of appends with block scales, whose device code numbers positions some tiles behind a context's end.
constexpr int kMaxTiledContext = INT32_MAX - 4096;

inline int check_shape(const pkv_attn_shape* sh, Geometry* g) {
  if (!sh) return PKV_ERR_NULL;
  if (sh->num_seqs < 0 || sh->num_seqs > kMaxSeqs) return PKV_ERR_SHAPE;
  if (sh->num_q_heads <= 0 || sh->num_kv_heads <= 0 || sh->num_q_heads > kMaxHeads)
    return PKV_ERR_SHAPE;
  const int D = sh->head_dim;
  if (D != 64 && D != 128 && D != 256) return PKV_ERR_SHAPE;
  const int B = sh->block_size;
  if (B != 16 && B != 32 && B != kMaxBlockSize) return PKV_ERR_SHAPE;
  if (sh->num_q_heads % sh->num_kv_heads != 0) return PKV_ERR_SHAPE;
  const int G = sh->num_q_heads / sh->num_kv_heads;
  if (G > kMaxGroup) return PKV_ERR_SHAPE;
  // a wavefront keeps two whole records (G rows of D floats) in its share of LDS
  if (D == 256 && G > 8) return PKV_ERR_SHAPE;
  if (sh->max_blocks_per_seq <= 0) return PKV_ERR_SHAPE;
  if ((int64_t)sh->max_blocks_per_seq * B > INT32_MAX) return PKV_ERR_SHAPE;
  const int cap = sh->max_blocks_per_seq * B;
  if (sh->max_context_len < 0 || sh->max_context_len > cap) return PKV_ERR_SHAPE;
  const int max_ctx = sh->max_context_len ? sh->max_context_len : cap;
  int P = sh->partition_size;
  if (P < 0) return PKV_ERR_SHAPE;
  if (P == 0) P = kDefaultPartition;
  if (P % B != 0 || P < B || P > kMaxPartition) return PKV_ERR_SHAPE;
  // 4 KiB slabs (16 tokens of one KV head) are numbered in 32 bits on the device
  if (sh->num_pool_blocks < 1 ||
      sh->num_pool_blocks > INT32_MAX / ((int64_t)sh->num_kv_heads * (B / kBlockTokens)))
    return PKV_ERR_SHAPE;
  // stream positions, slots and rows are 32-bit on the device
  const int64_t max_blocks = (max_ctx + kBlockTokens - 1) / kBlockTokens;
  if ((int64_t)sh->num_kv_heads * sh->num_seqs * max_blocks > INT32_MAX) return PKV_ERR_SHAPE;
  if ((int64_t)sh->num_seqs * sh->num_q_heads > INT32_MAX) return PKV_ERR_SHAPE;
  g->G = G;
  g->P = P;
  g->max_ctx = max_ctx;
  g->slots = record_slots(sh->num_seqs, sh->num_kv_heads);
  return PKV_OK;
}

// Workspace: the partial records, then room for a prefix array, which nothing uses but which is part of the size that callers know.
inline size_t workspace_bytes(const pkv_attn_shape* sh, const Geometry& g) {
  if (sh->num_seqs == 0) return 0;
  const size_t records = (size_t)g.slots * record_floats(g.G, sh->head_dim) * sizeof(float);
  return records + (((size_t)(sh->num_seqs + 1) * sizeof(int32_t) + 15) & ~(size_t)15);
}

inline int launch_status(hipError_t e) {
  if (e == hipSuccess) return PKV_OK;
  g_last_launch_error = e;
  return PKV_ERR_LAUNCH;
}

// Validation shared by the single-layer and the multi-layer call; fills the
// launch descriptor except for the per-layer pointers.  `given`: window and sinks of requests that see part of their context, as the caller has
// them, else nullptr.
inline int prepare_attn(const int32_t* block_tables, const int32_t* context_lens, float scale, int kv_fp8,
                        const Span* given, const pkv_attn_shape* shape, void* workspace, size_t workspace_bytes_given,
                        AttnLaunch* a, bool* empty) {
  Geometry g;
  const int rc = check_shape(shape, &g);
  if (rc != PKV_OK) return rc;
  *empty = shape->num_seqs == 0;
  if (*empty) return PKV_OK;
  if (!block_tables || !context_lens) return PKV_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(block_tables) & 3u) || (reinterpret_cast<uintptr_t>(context_lens) & 3u))
    return PKV_ERR_ALIGN;
  const size_t need = workspace_bytes(shape, g);
  if (need) {
    if (!workspace || workspace_bytes_given < need) return PKV_ERR_WORKSPACE;
    if (misaligned16(workspace)) return PKV_ERR_ALIGN;
  }
  a->block_tables = block_tables;
  a->context_lens = context_lens;
  a->S = shape->num_seqs;
  a->Hq = shape->num_q_heads;
  a->Hkv = shape->num_kv_heads;
  a->G = g.G;
  a->D = shape->head_dim;
  a->waves = kLayerGroups * group_waves(shape->head_dim);
  const int group = group_waves(shape->head_dim);
  const int64_t segments = (int64_t)a->S * a->Hkv;
  const int64_t max_blocks = given ? given->most_units(g.max_ctx) : (g.max_ctx + kBlockTokens - 1) / kBlockTokens;
  a->short_blocks = kv_fp8 == kFp4Pools ? short_segment_fp4(a->D) : short_segment(segments, a->D, kv_fp8);
  a->leaves_records = 1;
  const bool bounded = given && given->most_units() <= a->short_blocks;
  if (cut_by_segment(segments, a->D, bounded, kv_fp8 == kFp4Pools) && max_blocks <= a->short_blocks) {
    // Cut along its segments, a workgroup for each.  Nothing is left in the workspace, and the layers of such
    // a launch may be more than it has room for.
    a->leaves_records = 0;
    a->waves = (int)segments * group;
  }
  a->id_faults = g_id_faults;
  a->MAXB = shape->max_blocks_per_seq;
  a->upb = shape->block_size / kBlockTokens;
  a->P = g.P;
  a->max_ctx = g.max_ctx;
  a->NB = (int)shape->num_pool_blocks;
  a->scale_log2e = scale * 1.4426950408889634f;
  a->out_scale = 1.f;
  a->kv_fp8 = kv_fp8;
  a->ws_rec = static_cast<float*>(workspace);
  a->ws_words = a->ws_rec + (int64_t)kRecordsBeforeWords * record_floats(a->G, a->D);
  a->layer_ws_floats = layer_ws_floats(g.G, a->D);
  return PKV_OK;
}

inline int check_layer_pointers(const void* q, const void* k_pool, const void* v_pool, const void* out) {
  if (!q || !k_pool || !v_pool || !out) return PKV_ERR_NULL;
  if (misaligned16(q) || misaligned16(k_pool) || misaligned16(v_pool) || misaligned16(out))
    return PKV_ERR_ALIGN;
  return PKV_OK;
}

inline AttnLayer layer_of(const void* q, const void* k_pool, const void* v_pool, void* out) {
  return AttnLayer{static_cast<const uint16_t*>(q), k_pool, v_pool, static_cast<uint16_t*>(out)};
}

// The launches for the layer of `a`, or for `layers`; `stream_pass`: its launch.
template <typename StreamPass>
int launch_attn(const AttnLaunch& a, const AttnLayers* layers, hipStream_t st, StreamPass stream_pass) {
  hipError_t e = stream_pass(a, layers, st);
  if (e == hipSuccess && a.leaves_records) e = launch_attn_reduce(a, layers, st);
  if (e != hipSuccess) return launch_status(e);
  return PKV_OK;
}

inline uint64_t row_bytes(const AttnLaunch& a) { return (uint64_t)a.S * a.Hq * a.D * 2; }

// Does layer x's output overlap these bytes?
inline bool overlaps(const AttnLaunch& a, const AttnLayer& x, const void* p, uint64_t bytes) {
  const uint64_t out = reinterpret_cast<uintptr_t>(x.out), at = reinterpret_cast<uintptr_t>(p);
  return out < at + bytes && at < out + row_bytes(a);
}

inline bool overlaps_pools(const AttnLaunch& a, const AttnLayer& x, const AttnLayer& y) {
  const uint64_t tile = a.kv_fp8 == kFp4Pools ? fp4_tile_bytes(a.D) : kBlockTokens * a.D * (a.kv_fp8 ? 1 : 2);
  const uint64_t pool = (uint64_t)a.NB * a.Hkv * a.upb * tile;
  return overlaps(a, x, y.k_pool, pool) || overlaps(a, x, y.v_pool, pool);
}

// Does what layer x writes overlap what layer y reads or writes?  Then they cannot share a launch.
inline bool writes_into(const AttnLaunch& a, const AttnLayer& x, const AttnLayer& y) {
  return overlaps(a, x, y.q, row_bytes(a)) || overlaps(a, x, y.out, row_bytes(a)) || overlaps_pools(a, x, y);
}

// Does a layer write into its own inputs?  The stream pass stores rows while others are still being read, which
// is right where the output is q itself: a segment's rows of q are read by those who write them.
inline bool writes_own_input(const AttnLaunch& a, const AttnLayer& x) {
  return (x.out != x.q && overlaps(a, x, x.q, row_bytes(a))) || overlaps_pools(a, x, x) ||
         overlaps(a, x, a.block_tables, (uint64_t)a.S * a.MAXB * 4) || overlaps(a, x, a.context_lens, (uint64_t)a.S * 4);
}

// One layer.  Where it writes into its own inputs the rows are kept at the end of the workspace's room for records until all
// is read: a layer's records and words leave three quarters of it.
template <typename StreamPass>
int launch_layer(AttnLaunch a, const AttnLayer& layer, hipStream_t st, StreamPass stream_pass) {
  a.layer = layer;
  if (!writes_own_input(a, layer)) return launch_attn(a, nullptr, st, stream_pass);
  a.layer.out = reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(a.ws_rec + record_slots(a.S, a.Hkv) * record_floats(a.G, a.D)) - row_bytes(a));
  const int rc = launch_attn(a, nullptr, st, stream_pass);
  if (rc != PKV_OK) return rc;
  return launch_status(launch_copy(a.layer.out, layer.out, row_bytes(a), st));
}

}  // namespace pkv
